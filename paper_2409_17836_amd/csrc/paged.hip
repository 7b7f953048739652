// The paged key/value cache: appending with the rotation on the way, and
// attention over it for ragged batches, with or without a prefix that all of
// them share.
//
// Cache of one layer: two pools of pages, keys and values, bf16 [n_pages, Hkv,
// page, hd].  A page of a head is a row of groups of 32 tokens, each in the
// order in which the lanes of the 16x16x32 matrix instruction take it:
//   key   (t, d): ((t/16) (hd/32) + d/32) 512 + ((t%16) + 16 ((d%32)/8)) 8 + d%8
//   value (t, d): (d/16) 512 + ((d%16) + 16 ((t%16)/4)) 8 + 4 (t/16) + t%4
// so a lane's 16 bytes are its operand, a wave's load is 1 KB of consecutive
// memory, and the value order is the one in which the scores come out of the
// first product: the probabilities are the second product's operand where they
// are.  32 tokens are the depth of one instruction, and so the smallest page.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "async_lds.h"
#include "common.h"
#include "paged.h"

namespace lmgc {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kGroup = 32;

// ----------------------------------------------------------- ragged batches
// The last of B sequences whose first place is at most `at` (0 if none is), by
// all lanes of a wave: 64 probes a round, places rising with the sequence.
template <class F>
__device__ inline int last_at_most(int B, int64_t at, F place) {
  const int lane = threadIdx.x & 63;
  int lo = 0, n = B;
  while (n > 1) {
    const int step = (n + 63) / 64;
    const bool le = lane * step < n && place(lo + lane * step) <= at;
    const int c = max(1, (int)__popcll(__ballot(le)));
    lo += (c - 1) * step;
    n = min(step, n - (c - 1) * step);
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

// Rows row .. row + T - 1, len tokens before them.  Rows outside [0, n), a
// length outside the pages and rows behind their end are none of it.
struct Seq {
  int row, T, len;
};
__device__ inline Seq sequence(const Ragged& r, int b, int limit) {
  const int r0 = r.starts[b], r1 = r.starts[b + 1], len = r.lens[b], tokens = r.max_pages * r.page;
  const bool ok = r0 >= 0 && r1 >= r0 && r1 <= r.n && len >= 0 && len < tokens;
  return {r0, ok ? min(min(r1 - r0, limit), tokens - len) : 0, len};
}

// The last sequence that begins at or before a row, for each lane of a wave and its
// own row: the lanes hold 64 of the first rows and look them up in one another's
// registers, for look-ups in memory would wait one for the other.
__device__ inline int sequence_of(const Ragged& r, int row) {
  const int lane = threadIdx.x & 63, step = (r.B + 63) / 64;
  const int first = lane * step < r.B ? r.starts[lane * step] : INT32_MAX;
  int b = 0;
  for (int h = 32; h; h >>= 1) b += __shfl(first, b + h) <= row ? h : 0;
  b *= step;
  for (int n = min(step, r.B - b); n > 1;) {
    const int h = n / 2;
    const bool right = r.starts[b + h] <= row;
    b += right ? h : 0;
    n = right ? n - h : h;
  }
  return b;
}

// A lane's row's position; -1 if it is no token.
__device__ inline int position_of(const Ragged& r, int row, int limit) {
  const Seq s = sequence(r, sequence_of(r, row), limit);
  const int t = row - s.row;
  return t >= 0 && t < s.T ? s.len + t : -1;
}

// First number of a head's group of 32 tokens on a page.
__device__ inline int64_t group_at(const Ragged& r, int page, int Hkv, int h, int j, int hd) {
  return (((int64_t)page * Hkv + h) * r.page + ((j & (r.page - 1)) & ~(kGroup - 1))) * hd;
}

// ------------------------------------------------------------------ append
// Grid: (Hkv, places), 256 threads: a group of 32 tokens of one sequence's cache
// and one key/value head, with the query heads that read it.  Place starts[b] /
// 32 + 2 b + i is group i of sequence b's new tokens (so no sequence's places
// run into the next one's, wherever its groups begin).
//
// A thread has the two runs of 8 dims of 8 pairs of one token, so their cos and
// sin are read once for the key and the queries.  Keys go out as they are in a
// group, 16 bytes a lane; values meet in LDS, whose 16-byte slots are permuted so
// that the 64 halves of a store fall on all banks.
//
// It is bound by memory: 4 x 4096 rows of 32 and 32 heads of 128, bf16, 790 MB, take
// 158 us (5.0 TB/s; a copy 5.15), without the queries 105.  Number by number (not FAST)
// 786, and 644 where rot is 100.  With 4 places of 16 tokens to a wave, so half lines
// to a load, it was 180, with the heads in the grid's slower dimension 206,
// with non-temporal loads 207.
template <class T>
struct Eight;  // 8 dims of a row
template <>
struct Eight<float> {
  f32x4 v[2];
  __device__ inline float get(int i) const { return v[i >> 2][i & 3]; }
};
template <>
struct Eight<uint16_t> {
  u32x4 v[1];
  __device__ inline float get(int i) const {
    return __builtin_bit_cast(float, i & 1 ? v[0][i >> 1] & 0xffff0000u : v[0][i >> 1] << 16);
  }
};
__device__ inline float load1(const float* p) { return *p; }
__device__ inline float load1(const uint16_t* p) { return bf16_to_f32(*p); }

template <class T>
__device__ inline Eight<T> load8(const T* p) {
  Eight<T> e;
#pragma unroll
  for (int i = 0; i < (int)(sizeof(e.v) / 16); i++) e.v[i] = reinterpret_cast<const decltype(e.v[0] + 0)*>(p)[i];
  return e;
}
__device__ inline u32x4 pack8(const float* y) {
  u32x4 w;
#pragma unroll
  for (int i = 0; i < 4; i++) w[i] = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)y[2 * i], (__bf16)y[2 * i + 1]});
  return w;
}

constexpr int kPlaces = 32768;  // in one plane of the grid

// FAST: rot a multiple of 16 and every run of 8 dims aligned to 16 bytes.
template <class T, int HD, bool FAST>
__global__ __launch_bounds__(256) void paged_append_kernel(AppendArgs a) {
  constexpr int U = HD / 16;          // places of 16 dims in a token
  constexpr int NH = 256 / (32 * U);  // heads side by side
  __shared__ u32x4 sv[HD * 4];        // a group of values
  const Ragged& r = a.r;
  const int64_t at_place = (int64_t)blockIdx.z * kPlaces + blockIdx.y;
  const int b = last_at_most(r.B, at_place, [&](int i) { return (int64_t)r.starts[i] / kGroup + 2 * (int64_t)i; });
  Seq q = sequence(r, b, INT32_MAX);
  if (a.table) q.T = (int)min((int64_t)q.T, max((int64_t)0, a.n_pos - q.len));
  if (q.T <= 0) return;
  const int64_t place = at_place - (q.row / kGroup + 2 * (int64_t)b);
  if (place < 0) return;
  const int64_t t0 = q.len / kGroup * (int64_t)kGroup + place * kGroup;  // the group's first token
  if (t0 >= q.len + (int64_t)q.T) return;
  const int kvh = blockIdx.x, G = a.q ? a.Hq / a.Hkv : 0, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int lo = (int)max((int64_t)0, q.len - t0), hi = (int)min((int64_t)kGroup, q.len + (int64_t)q.T - t0);
  const int page = r.pages[(int64_t)b * r.max_pages + (t0 >> __builtin_ctz(r.page))];
  const bool there = page >= 0 && page < r.n_pages;
  const int64_t at = there ? group_at(r, page, a.Hkv, kvh, (int)t0, HD) : 0;
  // token and place of the thread: the places of a token side by side, so that a load
  // has whole lines of a row
  const int t = U == 8 ? 8 * wave + (lane >> 3) : 16 * (wave & 1) + (lane >> 2), unit = lane % U, h0 = U == 8 ? 0 : wave >> 1;
  const bool mine = t >= lo && t < hi;
  const int64_t row = q.row + (t0 - q.len) + t;  // (only where it is mine)
  const int half = a.rot / 2, nrot = a.table ? a.rot / 16 : 0;
  const bool rotates = FAST && unit < nrot, split = a.layout == LMGC_ROPE_HALF;
  // the thread's two runs
  const int d0 = rotates && split ? 8 * unit : 16 * unit, d1 = rotates && split ? d0 + half : d0 + 8;
  const float2* tab = reinterpret_cast<const float2*>(a.table) + (t0 + t) * half;
  float c[8], s[8];
  if (FAST && rotates && mine) {
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      const f32x4 w = *reinterpret_cast<const f32x4*>(tab + 8 * unit + i);
      c[i] = w[0], s[i] = w[1], c[i + 1] = w[2], s[i + 1] = w[3];
    }
  }
  // the thread's 16 numbers of a row: as they are, then rotated, as bf16
  struct Pair {
    Eight<T> u, v;
  };
  auto load = [&](const T* p) __attribute__((always_inline)) { return Pair{load8(p + d0), load8(p + d1)}; };
  auto rotated = [&](const Pair& w, u32x4& y0, u32x4& y1) __attribute__((always_inline)) {
    float y[16];
#pragma unroll
    for (int i = 0; i < 8; i++) {
      y[i] = w.u.get(i);
      y[8 + i] = w.v.get(i);
    }
    if (rotates) {
      if (split) {
#pragma unroll
        for (int i = 0; i < 8; i++) {
          const float m = y[i], n = y[8 + i];
          y[i] = turn_first(m, n, c[i], s[i]);
          y[8 + i] = turn_second(m, n, c[i], s[i]);
        }
      } else {
#pragma unroll
        for (int i = 0; i < 8; i++) {
          const float m = y[2 * i], n = y[2 * i + 1];
          y[2 * i] = turn_first(m, n, c[i], s[i]);
          y[2 * i + 1] = turn_second(m, n, c[i], s[i]);
        }
      }
    }
    y0 = pack8(y);
    y1 = pack8(y + 8);
  };
  // the same number by number, wherever they are
  auto rotated_slowly = [&](const T* p, u32x4& y0, u32x4& y1) __attribute__((always_inline)) {
    float y[16];
    for (int i = 0; i < 16; i++) {
      const int d = d0 + i;
      float v = load1(p + d);
      if (a.table && d < a.rot) {
        const bool second = split ? d >= half : d & 1;
        const int k = split ? (second ? d - half : d) : d >> 1, e = split ? (second ? d - half : d + half) : d ^ 1;
        const float other = load1(p + e);
        v = second ? turn_second(other, v, tab[k].x, tab[k].y) : turn_first(v, other, tab[k].x, tab[k].y);
      }
      y[i] = v;
    }
    y0 = pack8(y);
    y1 = pack8(y + 8);
  };
  const T* krow = static_cast<const T*>(a.k) + row * a.ldk + kvh * HD;
  const T* vrow = static_cast<const T*>(a.v) + row * a.ldv + kvh * HD;
  const T* qrow = static_cast<const T*>(a.q) + row * a.ldq + (int64_t)kvh * G * HD;
  const bool keys = mine && h0 == 0;  // (with heads side by side the first of them has the keys and values)
  // values: 8 dims of each half
  const int dv0 = 8 * unit, dv1 = dv0 + HD / 2;
  // everything that is there from the start is asked for before anything is used
  Pair kw{}, qw{};
  Eight<T> v0{}, v1{};
  if (FAST) {
    if (keys) {
      kw = load(krow);
      v0 = load8(vrow + dv0);
      v1 = load8(vrow + dv1);
    }
    if (mine && h0 < G) qw = load(qrow + h0 * HD);
  }
  u32x4 y0, y1;
  if (keys && there) {
    if (FAST) rotated(kw, y0, y1);
    else rotated_slowly(krow, y0, y1);
    auto put = [&](int d, u32x4 w) __attribute__((always_inline)) {
      *reinterpret_cast<u32x4*>(a.kc + at + ((t >> 4) * (HD / 32) + (d >> 5)) * 512 + ((t & 15) + 16 * ((d & 31) >> 3)) * 8) = w;
    };
    put(d0, y0);
    put(d1, y1);
  }
  // values: slot (d, 4 tokens) holds tokens 4 k .. + 3 of both halves
  auto slot = [](int s) __attribute__((always_inline)) { return s ^ (((s >> 4 & 3) ^ (s >> 7 & 1) << 1) | (s >> 6 & 1) << 2); };
  if (keys && there) {
    uint16_t* words = reinterpret_cast<uint16_t*>(sv);
#pragma unroll
    for (int k = 0; k < 2; k++) {
      const int d = k ? dv1 : dv0;
      float y[8];
#pragma unroll
      for (int i = 0; i < 8; i++) y[i] = FAST ? (k ? v1 : v0).get(i) : load1(vrow + d + i);
      const u32x4 w = pack8(y);
#pragma unroll
      for (int i = 0; i < 8; i++)
        words[slot(((d + i) >> 4) * 64 + ((d + i) & 15) + 16 * ((t & 15) >> 2)) * 8 + 4 * (t >> 4) + (t & 3)] =
            (uint16_t)(w[i >> 1] >> (16 * (i & 1)));
    }
  }
  if (mine) {
    for (int h = h0; h < G; h += NH) {
      const Pair w = qw;
      if (FAST && h + NH < G) qw = load(qrow + (h + NH) * HD);
      if (FAST) rotated(w, y0, y1);
      else rotated_slowly(qrow + h * HD, y0, y1);
      uint16_t* o = a.q_out + row * a.ldqo + ((int64_t)kvh * G + h) * HD;
      if (FAST) {
        *reinterpret_cast<u32x4*>(o + d0) = y0;
        *reinterpret_cast<u32x4*>(o + d1) = y1;
      } else {
        for (int i = 0; i < 8; i++) {
          o[d0 + i] = (uint16_t)(y0[i >> 1] >> (16 * (i & 1)));
          o[d1 + i] = (uint16_t)(y1[i >> 1] >> (16 * (i & 1)));
        }
      }
    }
  }
  if (!there) return;
  __syncthreads();
  for (int i = tid; i < HD * 4; i += 256) {
    const int k = 4 * (i >> 4 & 3);  // tokens k .. + 3 and 16 + k .. + 3
    uint16_t* o = a.vc + at + (int64_t)i * 8;
    const u32x4 w = sv[slot(i)];
    if (lo <= k && 16 + k + 4 <= hi) {
      *reinterpret_cast<u32x4*>(o) = w;
    } else {
#pragma unroll
      for (int e = 0; e < 8; e++) {
        const int tok = 16 * (e >> 2) + k + (e & 3);
        if (tok >= lo && tok < hi) o[e] = (uint16_t)(w[e >> 1] >> (16 * (e & 1)));
      }
    }
  }
}

// --------------------------------------------------------------- attention
// Keys that a query at position pos sees: j <= pos and, with a window, j >
// pos - window or j < sinks.
struct Mask {
  int window, sinks;
  __device__ inline int low(int pos) const { return window ? pos - window : -1; }  // the last key before the window
  __device__ inline bool sees(int pos, int low, int j) const { return (j <= pos) & ((j > low) | (j < sinks)); }
  // whether any query at positions p0 .. p1 may see a key of [j0, j1)
  __device__ inline bool any(int p0, int p1, int j0, int j1) const {
    return j0 <= p1 && (window == 0 || j1 - 1 > p0 - window || j0 < sinks);
  }
  // whether every query at positions p0 .. p1 sees every key of [j0, j1)
  __device__ inline bool all(int p0, int p1, int j0, int j1) const {
    return j1 - 1 <= p0 && (window == 0 || j0 > p1 - window || j1 <= sinks);
  }
  // the tokens of the group at j0 that some query at positions p0 .. p1 sees, a bit each
  __device__ inline uint32_t seen(int p0, int p1, int j0) const {
    auto first = [](int n) __attribute__((always_inline)) { return n >= kGroup ? ~0u : (1u << max(n, 0)) - 1; };
    return first(p1 + 1 - j0) & (~first(max(low(p0), -1) + 1 - j0) | first(sinks - j0));
  }
};

// The keys that a sequence's new tokens see, with those between the sinks and
// the window (whole groups that none sees) and those before `cut` left out:
// place v of `total` is key real(v).
struct Span {
  int cut, hole, gap, total;
  __device__ inline int real(int v) const { return cut + v + (cut + v >= hole ? gap : 0); }
};
__device__ inline Span span_of(const Seq& q, const Mask& m, int cut) {
  const int end = q.len + q.T, down = ~(kGroup - 1);
  Span s{cut, cut, 0, max(0, end - cut)};
  if (m.window) {
    s.hole = max(cut, (min(m.sinks, end) + kGroup - 1) & down);
    s.gap = max(0, (max(0, q.len - m.window + 1) & down) - s.hole);
    s.total = max(0, end - cut - s.gap);
  }
  return s;
}

// How the length is split: at most `most` parts of a whole number of `unit`
// tokens, `least` at least, by the sequence's own length.
struct Splits {
  int most, least, unit;
  __device__ inline int chunk(int total) const { return max(least, ((total + most - 1) / most + unit - 1) / unit * unit); }
};

// Buffer over n bytes (stride 0, word 3 of gfx9).
__device__ inline __amdgpu_buffer_rsrc_t buffer(const uint16_t* p, int bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t*>(p), (short)0, bytes, 0x00020000);
}

// A score where bit `at` of `seen` is set, else -inf.
__device__ inline float hide(float s, uint32_t seen, int at) {
  const int t = (int)(seen << (31 - at)) >> 31;
  return __builtin_bit_cast(float, (__builtin_bit_cast(int, s) & t) | ((int)0xff800000 & ~t));
}

// The words of a lane's 8 values (tokens 4 g .. + 3 of both halves of a group)
// with only those of `tokens`, a bit each.
__device__ inline u32x4 words_of(uint32_t tokens, int g) {
  u32x4 w;
#pragma unroll
  for (int e = 0; e < 4; e++) {
    const uint32_t two = tokens >> (16 * (e >> 1) + 2 * (e & 1)) >> (4 * g) & 3;
    w[e] = (two & 1 ? 0xffffu : 0u) | (two & 2 ? 0xffff0000u : 0u);
  }
  return w;
}

// Masked values.  A probability of zero times a NaN or an infinity is NaN.  The
// values of tokens that no query sees (all but `seen`), which may be anything,
// are cleared before the product.  What some queries see and others do not is
// numbers as a rule: the products are taken as they are, and only where a result
// comes out as none the wave does its columns again, this way:
// O^T += V^T P^T for a group of keys, tokens with a value that is not finite left
// to products of their own, which only the columns that see them take.  value(i):
// a lane's operand of dims 16 i ..; pf, pos: of the lane's columns; o: their
// results.
template <int ND, int NT, class Value>
__device__ inline void add_masked_values(Value value, const bf16x8 (&pf)[NT], f32x4 (&o)[NT][ND], const Mask& mask, uint32_t seen,
                                         const int (&pos)[NT], int j0) {
  const int g = (threadIdx.x & 63) >> 4;
  u32x4 keep = words_of(seen, g);
  uint32_t odd = 0;  // a bit for each half word of the lane
#pragma unroll
  for (int i = 0; i < ND; i++) {
    if (i % 2 == 0) __builtin_amdgcn_sched_barrier(0);  // (side by side they take more registers than there are)
    const u32x4 v = value(i) & keep;
#pragma unroll
    for (int e = 0; e < 4; e++)
      odd |= ((v[e] & 0x7f80u) == 0x7f80u ? 1u << (2 * e) : 0u) | ((v[e] & 0x7f800000u) == 0x7f800000u ? 2u << (2 * e) : 0u);
  }
  uint32_t bad = 0;
  if (__ballot(odd != 0)) {
#pragma unroll
    for (int e = 0; e < 8; e++) {
      const uint64_t lanes = __ballot(odd >> e & 1);
#pragma unroll
      for (int k = 0; k < 4; k++) bad |= lanes >> (16 * k) & 0xffff ? 1u << (16 * (e >> 2) + 4 * k + (e & 3)) : 0u;
    }
    keep = words_of(seen & ~bad, g);
  }
#pragma unroll
  for (int i = 0; i < ND; i++) {
    if (i % 2 == 0) __builtin_amdgcn_sched_barrier(0);
    const bf16x8 v = __builtin_bit_cast(bf16x8, value(i) & keep);
#pragma unroll
    for (int y = 0; y < NT; y++) o[y][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, pf[y], o[y][i], 0, 0, 0);
  }
  for (; bad; bad &= bad - 1) {
    const int j = __builtin_ctz(bad);
    keep = words_of(1u << j, g);
#pragma unroll
    for (int i = 0; i < ND; i++) {
      __builtin_amdgcn_sched_barrier(0);
      const bf16x8 v = __builtin_bit_cast(bf16x8, value(i) & keep);
#pragma unroll
      for (int y = 0; y < NT; y++) {
        const f32x4 x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, pf[y], f32x4{}, 0, 0, 0);
        if (mask.sees(pos[y], mask.low(pos[y]), j0 + j)) o[y][i] += x;
      }
    }
  }
}

// Sums of values near bf16's largest pass float32 where their mean does not.  So the
// columns whose results are no numbers the second time either get a third one, with
// their references kLift above the largest score: 2^24 probabilities of 2^8 / 2^kLift
// each are less than one.  Joins weigh their large sums, of four waves or up to 128
// parts, against kWaveLift or kJoinLift above the largest reference (little enough for
// bf16's smallest normal values to keep 11 bits).
constexpr float kLift = 34.f, kWaveLift = 3.f, kJoinLift = 8.f;

// Zeros for the queries of columns that are no token's, which may hold anything: no
// number there would have the wave do all its columns again.
template <int NT, int KQ>
__device__ inline void clear_no_tokens(bf16x8 (&qf)[NT][KQ], const int (&pos)[NT]) {
#pragma unroll
  for (int y = 0; y < NT; y++)
#pragma unroll
    for (int x = 0; x < KQ; x++)
      if (pos[y] < 0) qf[y][x] = bf16x8{};
}

// The running softmax of a wave's 16 NT columns.
template <int HD, int NT>
struct Columns {
  static constexpr int KQ = HD / 32, ND = HD / 16;
  float m[NT];
  f32x4 l[NT], o[NT][ND];  // row sums (four times), O^T: 4 dims of 16 each
  // Groups v, v + step, .. of the span up to v1: S^T = K Q^T, an online softmax,
  // O^T += V^T P^T.  EXACT: where masked values may be no numbers; the references lie
  // `lift` above the largest scores.
  template <bool EXACT>
  __device__ inline void walk(const bf16x8 (&qf)[NT][KQ], const uint16_t* kc, const uint16_t* vc, const Ragged& r, const int32_t* pages, int Hkv,
                              int kvh, const Span& span, int v, int v1, int step, int p0, int p1, const int (&pos)[NT], const Mask& mask,
                              float sl2, const float (&lift)[NT]) {
    const int lane = threadIdx.x & 63, g = lane >> 4;
#pragma unroll
    for (int y = 0; y < NT; y++) {
      m[y] = -INFINITY;
      l[y] = f32x4{};
#pragma unroll
      for (int i = 0; i < ND; i++) o[y][i] = f32x4{};
    }
    const __bf16 one = (__bf16)1.0f;
    const bf16x8 ones = {one, one, one, one, one, one, one, one};
    int held = -1;
    for (int it = 0; v < v1; v += step, it++) {
      // a lane holds the page of each of the wave's next 64 groups
      if ((it & 63) == 0) {
        const int64_t mine = v + (int64_t)lane * step;
        held = mine < v1 ? pages[span.real((int)mine) >> __builtin_ctz(r.page)] : -1;
      }
      const int page = __builtin_amdgcn_readlane(held, it & 63), j0 = span.real(v);
      if (page < 0 || page >= r.n_pages || !mask.any(p0, p1, j0, j0 + kGroup)) continue;
      const int64_t at = group_at(r, page, Hkv, kvh, j0, HD);
      const __amdgpu_buffer_rsrc_t kb = buffer(kc + at, kGroup * HD * 2), vb = buffer(vc + at, kGroup * HD * 2);
      u32x4 kr[2 * KQ], vr[ND];
#pragma unroll
      for (int i = 0; i < 2 * KQ; i++) kr[i] = __builtin_amdgcn_raw_buffer_load_b128(kb, lane * 16, i * 1024, 0);
#pragma unroll
      for (int i = 0; i < ND; i++) vr[i] = __builtin_amdgcn_raw_buffer_load_b128(vb, lane * 16, i * 1024, 0);
      const bool whole = mask.all(p0, p1, j0, j0 + kGroup);
      bf16x8 pf[NT];
#pragma unroll
      for (int y = 0; y < NT; y++) {
        f32x4 s[2] = {};
#pragma unroll
        for (int i = 0; i < 2; i++)
#pragma unroll
          for (int x = 0; x < KQ; x++)
            s[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kr[i * KQ + x]), qf[y][x], s[i], 0, 0, 0);
        if (!whole) {
          const uint32_t seen = mask.seen(pos[y], pos[y], j0) >> (4 * g);
#pragma unroll
          for (int i = 0; i < 2; i++)
#pragma unroll
            for (int e = 0; e < 4; e++) s[i][e] = hide(s[i][e], seen, 16 * i + e);
        }
        float mx = -INFINITY;
#pragma unroll
        for (int i = 0; i < 2; i++)
#pragma unroll
          for (int e = 0; e < 4; e++) mx = fmaxf(mx, s[i][e]);  // (drops a NaN; it comes back through the exponential)
        mx = fmaxf(mx, __shfl_xor(mx, 16));
        mx = fmaxf(mx, __shfl_xor(mx, 32)) * sl2;
        if (EXACT) mx += lift[y];
        if (mx > m[y]) {
          const float a = __builtin_amdgcn_exp2f(m[y] - mx);
          l[y] *= a;
#pragma unroll
          for (int i = 0; i < ND; i++) o[y][i] *= a;
          m[y] = mx;
        }
        const float sub = m[y] == -INFINITY ? 0.f : -m[y];
        // rounded to bf16 for the second product; the sum is of the rounded values
#pragma unroll
        for (int i = 0; i < 2; i++)
#pragma unroll
          for (int e = 0; e < 4; e++) pf[y][4 * i + e] = (__bf16)__builtin_amdgcn_exp2f(fmaf(s[i][e], sl2, sub));
        l[y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, pf[y], l[y], 0, 0, 0);
      }
      const uint32_t seen = mask.seen(p0, p1, j0);
      if (EXACT) {
        add_masked_values([&](int i) __attribute__((always_inline)) { return vr[i]; }, pf, o, mask, seen, pos, j0);
      } else {
        if (seen != ~0u) {
          const u32x4 keep = words_of(seen, g);
#pragma unroll
          for (int i = 0; i < ND; i++) vr[i] &= keep;
        }
#pragma unroll
        for (int i = 0; i < ND; i++)
#pragma unroll
          for (int y = 0; y < NT; y++)
            o[y][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vr[i]), pf[y], o[y][i], 0, 0, 0);
      }
    }
  }
  // The lanes that have a number of a column's result that is none: then what a
  // masked value was may have come in, or a sum have passed float32.
  __device__ inline uint64_t odd(int y) const {
    float x = 0.f;
#pragma unroll
    for (int i = 0; i < ND; i++)
#pragma unroll
      for (int e = 0; e < 4; e++) x = fmaf(o[y][i][e], 0.f, x);
    return __ballot(!(x == 0.f));
  }
  // Whether there are any; lift: what their columns' references are to be raised by.
  __device__ inline bool odd(float (&lift)[NT], float by) const {
    uint64_t any = 0;
#pragma unroll
    for (int y = 0; y < NT; y++) {
      const uint64_t lanes = odd(y);
      lift[y] = lanes >> (threadIdx.x & 15) & 0x1000100010001 ? by : 0.f;
      any |= lanes;
    }
    return any != 0;
  }
};

// ---- few columns
// Columns: column c = t G + i of a (sequence, key/value head) is query head
// kvh G + i of its new token t; for the prefix, of row t of the batch.
//
// Grid: (tiles of 16 NT columns x splits, Hkv, B), 256 threads.  Wave w takes
// groups w, w + 4, .. of its split: S^T = K Q^T, so lane (col, g) holds the
// scores of its column and tokens 16 i + 4 g + r of a group, an online softmax,
// O^T += V^T P^T.  The waves' parts meet in LDS.
//
// For single tokens it is bound by the cache's bytes: 8 sequences of up to 4095, 32 heads
// of 128, 520 MB, in 91 us (5.7 TB/s), and 5 for the join; of 64, 260 MB, 52 in all.  Twelve waves a CU, each
// with a group of 16 KB under way, hide the loads' way; parts of 64 KB a wave keep
// what is left for the join small.
constexpr int kWaves = 4;

struct AttnPlan {
  int64_t cols;          // of the longest sequence, at most
  int few, few_short;    // columns of a sequence that the form for few takes, and of one whose keys are one part
  int columns;           // how many of them there are at most
  int places;            // partial results of a sequence's columns in one head, at most
  int by_row;            // whether these lie row by row or, where that is less, sequence by sequence
  Splits split;          // of the form for few columns
  Splits prompt;         // of the form for many
  int many, joined;      // whether the form for many is needed; whether it leaves partial results
  int cut;               // tokens that all share, computed for the batch
  int pre, pre_chunk;    // splits of these
  float *po, *prompt_o, *pre_o;      // partial results, and maxima and sums
  float2 *pml, *prompt_ml, *pre_ml;
  // The first partial result of column c of sequence b and a head of so many with so many
  // keys; at: its row and query head.
  __device__ inline int64_t own(int b, int Hkv, int kvh, int c, int total, int64_t at) const {
    return by_row ? at * split.most : ((int64_t)b * Hkv + kvh) * places + c * (total <= split.least ? 1 : split.most);
  }
  // Whether a sequence of so many columns and keys has few.
  __device__ inline bool is_few(int cols, int total) const { return cols <= few || (cols <= few_short && total <= split.least); }
};

template <int HD, int NT, bool PREFIX>
__global__ __launch_bounds__(kWaves * 64, NT > 1 ? 2 : HD == 64 ? 4 : 3) void attn_paged_split_kernel(
    const uint16_t* __restrict__ q, int64_t ldq, const uint16_t* __restrict__ kc, const uint16_t* __restrict__ vc, Ragged r, int max_new,
    int Hkv, int G, AttnPlan plan, Mask mask, float sl2, uint16_t* __restrict__ out) {
  constexpr int KQ = HD / 32, ND = HD / 16, NW = kWaves, TILE = 16 * NT;
  __shared__ float so[NW][16][HD + 4];
  __shared__ float sm[NW][16], sl[NW][16];
  const int tid = threadIdx.x, lane = tid & 63, col = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int kvh = blockIdx.y, b = PREFIX ? 0 : blockIdx.z;
  // the tiles that a sequence of any length may have, all their splits; then those of sequences in one part
  const int all = PREFIX ? plan.pre : plan.split.most, of_any = PREFIX ? INT32_MAX : plan.few / TILE * all, bx = blockIdx.x;
  const int tile = bx < of_any ? bx / all : plan.few / TILE + bx - of_any, split = bx < of_any ? bx % all : 0, c0 = tile * TILE;
  Seq sq{0, r.n, 0};
  if (!PREFIX) sq = sequence(r, b, max_new);
  const int cols = sq.T * G, ncol = min(TILE, cols - c0);
  if (ncol <= 0) return;
  const Span span = PREFIX ? Span{0, 0, 0, plan.cut} : span_of(sq, mask, plan.cut);
  if (!PREFIX && !plan.is_few(cols, span.total)) return;
  // the lane's columns (past the last: the last one's again), their positions
  int pos[NT], p0, p1;
  if (PREFIX) {
    p0 = INT32_MAX;
    p1 = -1;
#pragma unroll
    for (int y = 0; y < NT; y++) {
      pos[y] = position_of(r, (c0 + min(16 * y + col, ncol - 1)) / G, max_new);
      p0 = min(p0, pos[y] < 0 ? INT32_MAX : pos[y]);
      p1 = max(p1, pos[y]);
    }
    for (int o = 8; o; o >>= 1) {
      p0 = min(p0, __shfl_xor(p0, o));
      p1 = max(p1, __shfl_xor(p1, o));
    }
    p0 = __builtin_amdgcn_readfirstlane(p0);
    p1 = __builtin_amdgcn_readfirstlane(p1);
  } else {
#pragma unroll
    for (int y = 0; y < NT; y++) pos[y] = sq.len + (c0 + min(16 * y + col, ncol - 1)) / G;
    p0 = sq.len + c0 / G;
    p1 = sq.len + (c0 + ncol - 1) / G;
  }
  const int chunk = PREFIX ? plan.pre_chunk : plan.split.chunk(span.total);
  const int v0 = split * chunk, v1 = min(span.total, v0 + chunk);
  if (v0 >= v1) return;
  const bool only = !PREFIX && plan.cut == 0 && span.total <= chunk;  // the only split writes the result
  const uint16_t* qrow = q + sq.row * ldq + (int64_t)kvh * G * HD + 8 * g;
  bf16x8 qf[NT][KQ];
#pragma unroll
  for (int y = 0; y < NT; y++) {
    const int c = c0 + min(16 * y + col, ncol - 1), t = c / G;
#pragma unroll
    for (int x = 0; x < KQ; x++) qf[y][x] = *reinterpret_cast<const bf16x8*>(qrow + t * ldq + (c - t * G) * HD + 32 * x);
  }
  if (PREFIX) clear_no_tokens(qf, pos);
  Columns<HD, NT> x;
  const int32_t* pages = r.pages + (int64_t)b * r.max_pages;
  float lift[NT] = {};
  x.template walk<false>(qf, kc, vc, r, pages, Hkv, kvh, span, v0 + wave * kGroup, v1, NW * kGroup, p0, p1, pos, mask, sl2, lift);
  for (int again = 0; again < 2 && x.odd(lift, again ? kLift : 0.f); again++)
    x.template walk<true>(qf, kc, vc, r, pages, Hkv, kvh, span, v0 + wave * kGroup, v1, NW * kGroup, p0, p1, pos, mask, sl2, lift);
  // HD / (4 NW) dims of a column to a thread
  constexpr int DT = HD / (4 * NW);
  typedef float f32xd __attribute__((ext_vector_type(DT)));
#pragma unroll
  for (int y = 0; y < NT; y++) {
    if (y) __syncthreads();
    if (g == 0) {
      sm[wave][col] = x.m[y];
      sl[wave][col] = x.l[y][0];
    }
#pragma unroll
    for (int i = 0; i < ND; i++) *reinterpret_cast<f32x4*>(&so[wave][col][16 * i + 4 * g]) = x.o[y][i];
    __syncthreads();
    const int oc = tid / (4 * NW), d0 = tid % (4 * NW) * DT, c = c0 + 16 * y + oc;
    if (16 * y + oc >= ncol) continue;
    float M = sm[0][oc];
#pragma unroll
    for (int w = 1; w < NW; w++) M = fmaxf(M, sm[w][oc]);
    M += kWaveLift;
    float L = 0.f;
    f32xd acc = {};
#pragma unroll
    for (int w = 0; w < NW; w++) {
      // waves without a token they see (m = -inf, l = 0) count for nothing
      const float mw = sm[w][oc], lw = sl[w][oc], a = mw == -INFINITY && lw == 0.f ? 0.f : __builtin_amdgcn_exp2f(mw - M);
      L += a * lw;
      acc += a * *reinterpret_cast<const f32xd*>(&so[w][oc][d0]);
    }
    const int t = c / G, hq = kvh * G + c - t * G;
    if (only) {
      const float inv = 1.0f / (L == 0.f ? 1.0f : L);
      if (L == 0.f) acc = f32xd{};  // no weight, nothing of the values
      uint32_t* op = reinterpret_cast<uint32_t*>(out + ((int64_t)(sq.row + t) * Hkv * G + hq) * HD + d0);
#pragma unroll
      for (int e = 0; e < DT / 2; e++)
        op[e] = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)(acc[2 * e] * inv), (__bf16)(acc[2 * e + 1] * inv)});
    } else {
      const int64_t row = (int64_t)(sq.row + t) * Hkv * G + hq, at = (PREFIX ? row * plan.pre : plan.own(b, Hkv, kvh, c, span.total, row)) + split;
      *reinterpret_cast<f32xd*>((PREFIX ? plan.pre_o : plan.po) + at * HD + d0) = acc;
      if (d0 == 0) (PREFIX ? plan.pre_ml : plan.pml)[at] = make_float2(M, L);
    }
  }
}

// ---- many columns
// A workgroup of eight waves takes 256 columns of one (sequence, key/value
// head), or of the batch, each wave 32, and walks the keys 64 at a time.  Keys
// and values come straight to LDS, kAhead steps ahead, in the order of the
// matrix operands; the products read a lane's 16 bytes in a row.
//
// A step has two phases: one for the vector unit (maxima, exponentials; and the
// loads are asked for), one for the matrix unit (the step's values, the next step's
// scores).  The waves of a SIMD, w and w + 4, are a phase apart, so that the
// units work side by side: all waves meet once a step, waves 0 to 3 before their
// first phase, waves 4 to 7 between the two.  So in stretch t, behind the t-th
// barrier, the former have both phases of step t, the latter the second of step t -
// 1 and then the first of step t, and what is read is values t and keys t + 1
// (bundle t) and those before them.  A bundle's place in the ring is free again two
// stretches behind its own, so bundle t + kRing - 2 is asked for in stretch t; and
// before a barrier each wave waits for its own part of the bundle that is read next.
//
// Two prompts of 3001 rows behind 1000 tokens, 32 on 8 heads of 128: 226 us (1.06
// PFLOP/s; another card 244), where the products alone take 203 and all but them
// 171.  With two barriers a step and all waves in one phase 242, 32 x 32 x 16
// products 260, loads beside the products instead of the exponentials 264 (249).
constexpr int kTileCols = 256;
constexpr int kStep = 2 * kGroup;
constexpr int kRing = 4, kAhead = kRing - 2;
constexpr int kReads = 4;          // operands read ahead of their products
constexpr int kNowhere = 1 << 30;  // where no query sees a key

template <int HD, bool PREFIX>
__global__ __launch_bounds__(512, 2) void attn_paged_prompt_kernel(
    const uint16_t* __restrict__ q, int64_t ldq, const uint16_t* __restrict__ kc, const uint16_t* __restrict__ vc, Ragged r, int max_new,
    int Hkv, int G, AttnPlan plan, Mask mask, float sl2, int nslot, int by_turns, int nsplit, uint16_t* __restrict__ out) {
  constexpr int ND = HD / 16, KQ = HD / 32;  // dim tiles; 32-dim steps of a score
  constexpr int PIECES = HD / 16;            // KB of a group of keys (or values)
  constexpr int LOADS = 2 * PIECES / 8;      // KB of a step's keys (or values) to a wave
  __shared__ u32x4 sk[kRing][2 * PIECES * 64], sv[kRing][2 * PIECES * 64];
  // heads fastest: with a multiple of eight heads all tiles of a head run on one
  // XCD and share its L2
  const int kvh = blockIdx.x % Hkv, rest = blockIdx.x / Hkv, split = rest % nsplit, slot = rest / nsplit;
  const int tid = threadIdx.x, lane = tid & 63, col = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  int b = 0, c0 = slot * kTileCols;
  Seq sq{0, r.n, 0};
  if (!PREFIX) {
    int64_t tile;
    if (by_turns) {
      // the sequences' last tiles, the longest, then those before them, ..
      b = slot % r.B;
      sq = sequence(r, b, max_new);
      tile = ((int64_t)sq.T * G + kTileCols - 1) / kTileCols - 1 - slot / r.B;
    } else {
      // place starts[b] G / 256 + b + i is tile i of sequence b
      const int64_t place = nslot - 1 - slot;
      b = last_at_most(r.B, place, [&](int i) { return (int64_t)r.starts[i] * G / kTileCols + i; });
      sq = sequence(r, b, max_new);
      tile = place - ((int64_t)sq.row * G / kTileCols + b);
    }
    if (sq.T <= 0 || tile < 0 || tile * kTileCols >= (int64_t)sq.T * G) return;
    c0 = (int)tile * kTileCols;
  }
  const int ncol = min(kTileCols, sq.T * G - c0);
  if (ncol <= 0) return;
  const Span span = PREFIX ? Span{0, min(plan.cut, (min(mask.sinks, plan.cut) + kGroup - 1) & ~(kGroup - 1)), 0, plan.cut} : span_of(sq, mask, plan.cut);
  if (!PREFIX && plan.is_few(sq.T * G, span.total)) return;
  // the wave's columns (past the last: the last one's again), their positions
  const int w0 = min(c0 + wave * 32, c0 + ncol - 1), w1 = min(c0 + wave * 32 + 31, c0 + ncol - 1);
  const bool works = wave * 32 < ncol;
  int pos[2], p0, p1, q0, q1;  // p0, p1: of the tile's columns, q0, q1: of the wave's
  if (PREFIX) {
    __shared__ int ends[2][8];
    q0 = INT32_MAX;
    q1 = -1;
#pragma unroll
    for (int y = 0; y < 2; y++) {
      pos[y] = position_of(r, min(w0 + 16 * y + col, w1) / G, max_new);
      q0 = min(q0, pos[y] < 0 ? INT32_MAX : pos[y]);
      q1 = max(q1, pos[y]);
    }
    for (int o = 8; o; o >>= 1) {
      q0 = min(q0, __shfl_xor(q0, o));
      q1 = max(q1, __shfl_xor(q1, o));
    }
    q0 = __builtin_amdgcn_readfirstlane(q0);
    q1 = __builtin_amdgcn_readfirstlane(q1);
    ends[0][wave] = q0;
    ends[1][wave] = q1;
    __syncthreads();
    p0 = INT32_MAX;
    p1 = -1;
    for (int w = 0; w < 8; w++) {
      p0 = min(p0, ends[0][w]);
      p1 = max(p1, ends[1][w]);
    }
    p0 = __builtin_amdgcn_readfirstlane(p0);
    p1 = __builtin_amdgcn_readfirstlane(p1);
  } else {
#pragma unroll
    for (int y = 0; y < 2; y++) pos[y] = sq.len + min(w0 + 16 * y + col, w1) / G;
    p0 = sq.len + c0 / G;
    p1 = sq.len + (c0 + ncol - 1) / G;
    q0 = sq.len + w0 / G;
    q1 = sq.len + w1 / G;
  }
  const int chunk = PREFIX ? plan.pre_chunk : plan.prompt.chunk(span.total);
  // the split's places of the span, without those behind the tile's last query
  const int v0 = split * chunk, vend = min(span.total, v0 + chunk);
  if (v0 >= vend) return;
  const int v1 = min(vend, max(v0, p1 + 1 - span.cut - (p1 >= span.hole ? min(span.gap, p1 - span.hole) : 0)));
  const bool only = !PREFIX && plan.cut == 0 && span.total <= chunk;  // the only split writes the result
  bf16x8 qf[2][KQ];
#pragma unroll
  for (int y = 0; y < 2; y++) {
    const int c = min(w0 + 16 * y + col, w1), t = c / G;
    const uint16_t* qp = q + (sq.row + (int64_t)t) * ldq + ((int64_t)kvh * G + c - t * G) * HD + 8 * g;
#pragma unroll
    for (int x = 0; x < KQ; x++) qf[y][x] = *reinterpret_cast<const bf16x8*>(qp + 32 * x);
  }
  if (PREFIX) clear_no_tokens(qf, pos);
  keep(qf[0]);
  keep(qf[1]);  // (arrived: a wait for them further on would be one for all loads)
  // Step k is place v0 + 64 k of the span, and `jump` more from step `hole` on:
  // those between the sinks and the tile's window are left out.
  const int hole = max(0, (span.hole - span.cut - v0 + kStep - 1) / kStep);
  const int low = mask.window ? p0 - mask.window + 1 : 0;  // the tile's first key behind the hole
  const int vlow = low >= span.hole + span.gap ? min(low - span.cut - span.gap, vend) : 0, vhole = v0 + hole * kStep;
  const int jump = max(0, vlow - vhole) / kStep * kStep;
  const int steps = v1 <= vhole ? (v1 - v0 + kStep - 1) / kStep : hole + max(0, v1 - vhole - jump + kStep - 1) / kStep;
  const int32_t* pages = r.pages + (int64_t)b * r.max_pages;
  // A lane has one of 64 steps from step `first` on: its two groups' first keys and
  // where they are in a head's part of the pools.  (A page that is not there is page
  // 0 where no query sees it, so that the loads under way stay countable.)  And a
  // bit for each of them: whether every query of the wave sees every key, and
  // whether some key is seen by none of the tile.
  int key[2], first;
  int64_t at[2];
  uint64_t whole, partly;
  auto look = [&](int k0) __attribute__((always_inline)) {
    first = k0;
    const int k = k0 + lane, v = v0 + k * kStep + (k >= hole ? jump : 0);
    bool all = true, none = false;
#pragma unroll
    for (int i = 0; i < 2; i++) {
      const bool in = k < steps && v + i * kGroup < vend;
      key[i] = in ? span.real(v + i * kGroup) : kNowhere;
      const int page = in ? pages[key[i] >> __builtin_ctz(r.page)] : -1;
      const bool there = (uint32_t)page < (uint32_t)r.n_pages;
      at[i] = there ? 2 * ((int64_t)page * (Hkv * r.page * HD) + (key[i] & (r.page - 1)) * HD) : 0;
      key[i] = there ? key[i] : kNowhere;
      all = all && mask.all(q0, q1, key[i], key[i] + kGroup);
      none = none || mask.seen(p0, p1, key[i]) != ~0u;
    }
    whole = __ballot(all);
    partly = __ballot(none);
  };
  // of the i-th group of step k
  auto key_of = [&](int k, int i) __attribute__((always_inline)) { return __builtin_amdgcn_readlane(key[i], k - first); };
  auto at_of = [&](int k, int i) __attribute__((always_inline)) {
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)at[i], k - first), hi = (uint32_t)__builtin_amdgcn_readlane((int)(at[i] >> 32), k - first);
    return (int64_t)((uint64_t)hi << 32 | lo);
  };
  // The wave's pieces of 1 KB of a step: one of each group, or one of one of them.
  constexpr bool kBoth = LOADS == 2;
  const int mine = wave / PIECES, piece = wave % PIECES;  // (mine: 0 where it has one of each)
  const char *kp = reinterpret_cast<const char*>(kc + (int64_t)kvh * r.page * HD + piece * 512);
  const char *vp = reinterpret_cast<const char*>(vc + (int64_t)kvh * r.page * HD + piece * 512);
  const LdsAt lk = lds_at(sk) + wave * 1024, lv = lds_at(sv) + wave * 1024;
  constexpr int kSlot = 2 * PIECES * 1024;
  struct Where {
    int64_t at[LOADS];
  };
  auto where = [&](int k) __attribute__((always_inline)) {
    Where w;
#pragma unroll
    for (int i = 0; i < LOADS; i++) w.at[i] = kBoth ? at_of(k, i) : mine ? at_of(k, 1) : at_of(k, 0);
    return w;
  };
  Columns<HD, 2> cs = {};
  f32x4(&acc)[2][ND] = cs.o;
  f32x4 sc[4][2];   // scores of a step
  bf16x8 pf[2][2];  // its probabilities, by column tile and group
  float(&m)[2] = cs.m;
  m[0] = m[1] = -INFINITY;
  f32x4(&l)[2] = cs.l;  // the product of the probabilities with ones
  const __bf16 one = (__bf16)1.0f;
  const bf16x8 ones = {one, one, one, one, one, one, one, one};
  // (two tiles by turns: a product waits for none of the three before it)
  auto scores = [&](auto key) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 4; i += 2)
#pragma unroll
      for (int x = 0; x < KQ; x++)
#pragma unroll
        for (int e = 0; e < 2; e++) {
          const bf16x8 kf = __builtin_bit_cast(bf16x8, key(i + e, x));
#pragma unroll
          for (int y = 0; y < 2; y++)
            sc[i + e][y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[y][x], x == 0 ? f32x4{} : sc[i + e][y], 0, 0, 0);
        }
  };
  auto held = [&](const u32x4* k) __attribute__((always_inline)) {
    return [=](int i, int x) __attribute__((always_inline)) { return k[(i * KQ + x) * 64 + lane]; };
  };
  auto sums = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int x = 0; x < 2; x++)
#pragma unroll
      for (int y = 0; y < 2; y++) l[y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, pf[y][x], l[y], 0, 0, 0);
  };
  auto add_value = [&](int i, int x, u32x4 w) __attribute__((always_inline)) {
#pragma unroll
    for (int y = 0; y < 2; y++)
      acc[y][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w), pf[y][x], acc[y][i], 0, 0, 0);
  };
  auto add_values = [&](const u32x4* v) __attribute__((always_inline)) {
    sums();
#pragma unroll
    for (int i = 0; i < ND; i += 2)
#pragma unroll
      for (int x = 0; x < 2; x++)
#pragma unroll
        for (int e = 0; e < 2; e++) add_value(i + e, x, v[(x * ND + i + e) * 64 + lane]);
  };
  // Clears, in the wave's part of a step's values, the tokens that no query of the
  // tile sees.
  auto clear = [&](u32x4* v, int k) __attribute__((always_inline)) {
    if (!(partly >> (k - first) & 1)) return;
#pragma unroll
    for (int i = 0; i < LOADS; i++) {
      const uint32_t seen = mask.seen(p0, p1, kBoth ? key_of(k, i) : mine ? key_of(k, 1) : key_of(k, 0));
      v[(wave + 8 * i) * 64 + lane] &= words_of(seen, g);
    }
  };
  // scores to probabilities (lifted: with references `lift` above the scores)
  float lift[2] = {};
  auto soften = [&](int k, auto lifted) __attribute__((always_inline)) {
    if (!(whole >> (k - first) & 1)) {
#pragma unroll
      for (int y = 0; y < 2; y++)
#pragma unroll
        for (int x = 0; x < 2; x++) {
          const uint32_t seen = mask.seen(pos[y], pos[y], key_of(k, x)) >> (4 * g);
#pragma unroll
          for (int i = 0; i < 2; i++)
#pragma unroll
            for (int e = 0; e < 4; e++) sc[2 * x + i][y][e] = hide(sc[2 * x + i][y][e], seen, 16 * i + e);
        }
    }
    float mx[2];
#pragma unroll
    for (int y = 0; y < 2; y++) {
      float x = -INFINITY;
#pragma unroll
      for (int i = 0; i < 4; i++)
#pragma unroll
        for (int e = 0; e < 4; e++) x = fmaxf(x, sc[i][y][e]);
      mx[y] = x * sl2;
      if (decltype(lifted)::value) mx[y] += lift[y];
    }
    // a column's reference moves only when a score passes it by 2^8
    if (__ballot(mx[0] > m[0] + 8.0f || mx[1] > m[1] + 8.0f)) {
#pragma unroll
      for (int y = 0; y < 2; y++) {
        float x = fmaxf(mx[y], __shfl_xor(mx[y], 16));
        x = fmaxf(x, __shfl_xor(x, 32));
        if (x > m[y] + 8.0f) {
          const float a = __builtin_amdgcn_exp2f(m[y] - x);
          l[y] *= a;
#pragma unroll
          for (int i = 0; i < ND; i++) acc[y][i] *= a;
          m[y] = x;
        }
      }
    }
#pragma unroll
    for (int y = 0; y < 2; y++) {
      const float sub = m[y] == -INFINITY ? 0.f : -m[y];
#pragma unroll
      for (int i = 0; i < 4; i++) {
        float p[4];
#pragma unroll
        for (int e = 0; e < 4; e++) p[e] = __builtin_amdgcn_exp2f(fmaf(sc[i][y][e], sl2, sub));
        const bf16x2 lo = {(__bf16)p[0], (__bf16)p[1]}, hi = {(__bf16)p[2], (__bf16)p[3]};
#pragma unroll
        for (int e = 0; e < 2; e++) {
          pf[y][i >> 1][(i & 1) * 4 + e] = lo[e];
          pf[y][i >> 1][(i & 1) * 4 + 2 + e] = hi[e];
        }
      }
    }
  };

  const bool late = wave >= 4;
  look(0);
  Where last = where(0);  // of the keys asked for last: their values are next
  auto fetch = [&](const char* pool, LdsAt to) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < LOADS; i++) load_lds(pool + last.at[i], lane * 16, to + i * (kSlot / 2));
  };
  fetch(kp, lk);
  auto ask = [&](int s) __attribute__((always_inline)) {
    fetch(vp, lv + (s & (kRing - 1)) * kSlot);
    last = where(s + 1);
    fetch(kp, lk + ((s + 1) & (kRing - 1)) * kSlot);
  };
  for (int s = 0; s < kAhead; s++) ask(s);
  wait_loads<(kAhead - 1) * 2 * LOADS>();  // the first keys and bundle 0
  clear(sv[0], 0);
  meet();
  if (works) scores(held(sk[0]));
  for (int k = 0; k < steps; k++) {
    if (k - first == 32) look(k);
    ask(k + kAhead);
    const int ring = k & (kRing - 1), up = (k + 1) & (kRing - 1);  // of the step's values; of the next step's keys
    __builtin_amdgcn_sched_barrier(0);
    if (works) {
      soften(k, std::false_type{});
      // (kept here: the compiler would move the exponentials to their use)
      keep(pf[0]);
      keep(pf[1]);
    }
    __builtin_amdgcn_sched_barrier(0);
    auto next = [&]() __attribute__((always_inline)) {
      wait_loads<(kAhead - 1) * 2 * LOADS>();
      clear(sv[up], k + 1);
      meet();
    };
    if (late) next();
    __builtin_amdgcn_sched_barrier(0);
    if (works) {
      // operands read kReads ahead, two products to a read
      add_values(sv[ring]);
      scores(held(sk[up]));
      __builtin_amdgcn_sched_group_barrier(0x100, kReads, 0);
#pragma unroll
      for (int i = 0; i < 2 + 2 * ND + 4 * KQ; i++) {
        __builtin_amdgcn_sched_group_barrier(0x008, 2, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    if (!late) next();
    __builtin_amdgcn_sched_barrier(0);
  }
  wait_loads<0>();  // no load to LDS outlives the workgroup
  if (!works) return;
  for (int again = 0; again < 2 && cs.odd(lift, again ? kLift : 0.f); again++) {
    // once more, by itself and in the same order
    cs = Columns<HD, 2>{};
    m[0] = m[1] = -INFINITY;
    look(0);
    for (int k = 0; k < steps; k++) {
      if (k - first == 32) look(k);
      auto group = [&](const uint16_t* pool, int i) __attribute__((always_inline)) {
        return reinterpret_cast<const u32x4*>(reinterpret_cast<const char*>(pool + (int64_t)kvh * r.page * HD) + at_of(k, i)) + lane;
      };
      const u32x4* keys[2] = {group(kc, 0), group(kc, 1)};
      scores([&](int i, int x) __attribute__((always_inline)) { return keys[i >> 1][((i & 1) * KQ + x) * 64]; });
      soften(k, std::true_type{});
      sums();
#pragma unroll
      for (int x = 0; x < 2; x++) {
        const bf16x8 p[2] = {pf[0][x], pf[1][x]};
        const u32x4* values = group(vc, x);
        add_masked_values([&](int i) __attribute__((always_inline)) { return values[i * 64]; }, p, acc, mask,
                          mask.seen(q0, q1, key_of(k, x)), pos, key_of(k, x));
      }
    }
  }
#pragma unroll
  for (int y = 0; y < 2; y++) {
    const int c = w0 + 16 * y + col, t = c / G;
    const float L = l[y][0];
    if (c > w1) continue;
    const int64_t row = ((int64_t)sq.row + t) * Hkv * G + (int64_t)kvh * G + c - t * G;
    if (only) {
      const float inv = 1.0f / (L == 0.f ? 1.0f : L);
      if (L == 0.f) {  // no weight, nothing of the values
#pragma unroll
        for (int i = 0; i < ND; i++) acc[y][i] = f32x4{};
      }
      uint16_t* op = out + row * HD + 4 * g;
#pragma unroll
      for (int i = 0; i < ND; i++) {
        uint2 w;
        w.x = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)(acc[y][i][0] * inv), (__bf16)(acc[y][i][1] * inv)});
        w.y = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)(acc[y][i][2] * inv), (__bf16)(acc[y][i][3] * inv)});
        *reinterpret_cast<uint2*>(op + 16 * i) = w;
      }
    } else {
      const int64_t to = row * (PREFIX ? plan.pre : plan.prompt.most) + split;
#pragma unroll
      for (int i = 0; i < ND; i++) *reinterpret_cast<f32x4*>((PREFIX ? plan.pre_o : plan.prompt_o) + to * HD + 16 * i + 4 * g) = acc[y][i];
      if (g == 0) (PREFIX ? plan.pre_ml : plan.prompt_ml)[to] = make_float2(m[y], L);
    }
  }
}

// Joins the parts of a row and head: HD / 4 lanes each, 4 dims to a lane, which takes
// the parts 8 at a time with a running maximum.  ROWS: all rows; else the columns of
// sequences with few of them, where the others are in one part.  A step's statistics and numbers are asked for together.  14400 rows of 64 dims in 5 parts
// take 6.6 us (with a wave to a row 13.5), mostly the way to a row's sequence and back.
template <int HD, bool ROWS>
__global__ __launch_bounds__(256) void attn_paged_join_kernel(Ragged r, int max_new, int Hkv, int G, AttnPlan plan, Mask mask,
                                                              uint16_t* __restrict__ out) {
  constexpr int LANES = HD / 4, NR = 256 / LANES;
  const int own_row = threadIdx.x / LANES, d = threadIdx.x % LANES * 4, Hq = Hkv * G;
  const int per = ROWS ? Hq : plan.columns;
  const int64_t count = ROWS ? (int64_t)r.n * Hq : (int64_t)r.B * Hkv * plan.columns;
  for (int64_t i0 = (int64_t)blockIdx.x * NR; i0 < count; i0 += (int64_t)gridDim.x * NR) {
    // i = i0 + own_row, divided by what is the same for a block and by few
    const int64_t unit0 = i0 / per;
    const int rest = (int)(i0 - unit0 * per) + own_row, more = rest / per, i = rest - more * per;
    int b, t, hq;
    Seq q;
    if (ROWS) {
      const int row = (int)min(unit0 + more, (int64_t)r.n - 1);
      b = sequence_of(r, row);
      q = sequence(r, b, max_new);
      t = row - q.row;
      hq = i;
    } else {
      const uint32_t unit = (uint32_t)min(unit0 + more, (int64_t)r.B * Hkv - 1);
      b = unit / Hkv;
      q = sequence(r, b, max_new);
      t = i / G;
      hq = (int)(unit - (uint32_t)b * Hkv) * G + i - t * G;
    }
    if (i0 + own_row >= count || t < 0 || t >= q.T) continue;
    const Span span = span_of(q, mask, plan.cut);
    const bool few = plan.is_few(q.T * G, span.total);
    if (!ROWS && !few) continue;
    const int kvh = hq / G, chunk = (few ? plan.split : plan.prompt).chunk(span.total), nown = (span.total + chunk - 1) / chunk;
    if (plan.cut == 0 && nown <= 1) continue;  // written by the only split
    const int64_t at = ((int64_t)q.row + t) * Hq + hq, pre = at * plan.pre;
    const int64_t own = few ? plan.own(b, Hkv, kvh, t * G + hq - kvh * G, span.total, at) : at * plan.prompt.most;
    const float* own_o = few ? plan.po : plan.prompt_o;
    const float2* own_ml = few ? plan.pml : plan.prompt_ml;
    // parts: those of the prefix, then the sequence's own; M is kJoinLift above their largest
    const int n = plan.pre + nown;
    float M = -INFINITY, L = 0.f;
    f32x4 acc = {};
    for (int e0 = 0; e0 < n; e0 += 8) {
      float2 ml[8];
      f32x4 x[8];
#pragma unroll
      for (int k = 0; k < 8; k++) {
        const int e = min(e0 + k, n - 1);
        const bool shared = e < plan.pre;
        const int64_t part = shared ? pre + e : own + (e - plan.pre);
        ml[k] = (shared ? plan.pre_ml : own_ml)[part];
        x[k] = *reinterpret_cast<const f32x4*>((shared ? plan.pre_o : own_o) + part * HD + d);
        if (e0 + k >= n) {
          ml[k] = make_float2(-INFINITY, 0.f);
          x[k] = f32x4{};
        }
      }
      float top = ml[0].x;
#pragma unroll
      for (int k = 1; k < 8; k++) top = fmaxf(top, ml[k].x);
      top += kJoinLift;
      if (top > M) {
        const float a = __builtin_amdgcn_exp2f(M - top);  // (0 times what came of a NaN stays one)
        L *= a;
        acc *= a;
        M = top;
      }
#pragma unroll
      for (int k = 0; k < 8; k++) {
        // parts without a token that the query sees (m = -inf, l = 0) count for nothing
        const float w = ml[k].x == -INFINITY && ml[k].y == 0.f ? 0.f : __builtin_amdgcn_exp2f(ml[k].x - M);
        L += w * ml[k].y;
        acc += w * x[k];  // (of no weight too: what is no number there stays none)
      }
    }
    const float inv = 1.0f / (L == 0.f ? 1.0f : L);
    if (L == 0.f) acc = f32x4{};  // no weight, nothing of the values
    typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
    u32x2 y;
#pragma unroll
    for (int e = 0; e < 2; e++) y[e] = f32_to_bf16(acc[2 * e] * inv) | (uint32_t)f32_to_bf16(acc[2 * e + 1] * inv) << 16;
    *reinterpret_cast<u32x2*>(out + at * HD + d) = y;
  }
}

// Tokens that are computed for the batch: whole steps of the form for many.
int cut_of(int B, int shared) { return B > 1 ? shared / kStep * kStep : 0; }

// Columns of a sequence that the form for few takes: of any, and (where max_new allows
// no more, for the launch has to hold the tiles of all) of one whose keys are one part.
// Every 16 columns read all keys, so it is the faster the fewer of either there are,
// and for a sequence by itself: of 8 heads of 128, G = 4, 96 columns over 4000 keys
// take 13.9 us by it and 22.6 by the form for many, those of 8 sequences 48.5 and
// 48.8, 128 columns of 8 sequences 61.0 and 51.9; over 200 keys 256 columns of 8
// sequences 17.0 and 20.1, over 380 22.7 and 22.2, 96 columns over 1000 40.0 and 25.6;
// of 12 heads of 64, 512 columns of 8 sequences over 712 keys 32 and 48.
constexpr int kFew = 64, kFewShort = 512;

// Keys of a part, at least, in the form for many (fewer fill the chip with one prompt,
// more leave less to join with several: 128 rows over 1000 keys take 29.5 us, 26.8
// with 256, 38.1 with 1024; 8 prompts of them over 4000 keys 152, 204 and 123).
constexpr int kLeast = 512;

// Columns of the batch up to which a shared prefix goes to the form for few, with 32
// columns to a workgroup: its four waves wait for less than the eight of the form for
// many, of which each has its own 32 columns.  A step behind 8192 shared tokens, 8
// heads of 128: 32.7 us for 36.6 with 128 columns, 43.0 for 48.5 with 256, 66.5 for
// 64.6 with 512; 12 heads of 64: 30.7 for 33.4 with 64 columns, 46.8 for 44.4 with 128.
constexpr int kFewPre = 256, kPreTile = 32;

// Workgroups for the tiles of many columns of one head and split: as many tiles of
// every sequence as the longest may have, by turns, so that the longest tiles run
// first (of two prompts of 3001 rows the last workgroups end 15 % later the other way
// round); where that were many more than there are, as many as the rows can fill.
struct Tiles {
  int64_t count;
  int by_turns;
};
Tiles tiles_of(int n, int G, int B, int64_t cols) {
  const int64_t places = (int64_t)n * G / kTileCols + B, turns = (cols + kTileCols - 1) / kTileCols * B;
  return turns <= 2 * places ? Tiles{turns, 1} : Tiles{places, 0};
}

AttnPlan plan_of(int n, int B, int Hq, int Hkv, int hd, int max_new, int tokens, int shared, Mask mask, void* ws, int64_t* bytes) {
  // the rules count max_new as it was given, not the batch, for the bits of a sequence
  // are not to depend on the rows of others; sizes count no more than n rows
  const int64_t rule = (int64_t)max_new * (Hq / Hkv), cols = std::min<int64_t>(max_new, n) * (Hq / Hkv);
  AttnPlan p{};
  p.few = kFew;
  p.few_short = rule <= kFewShort ? kFewShort : kFew;
  p.cols = cols;
  p.columns = (int)std::min<int64_t>(cols, p.few_short);
  p.cut = std::min(cut_of(B, shared), tokens);
  const int least = 512 * 128 / hd;  // keys of a part in the form for few, at least
  // most tokens of a sequence's own part: those of its pages, or, with a window, of
  // whole groups around it, its new tokens and the first ones (a step in a window of
  // 512 needs one part, no join and 2.7 us less)
  int own_tokens = std::max(1, tokens - p.cut);
  if (mask.window) own_tokens = (int)std::min<int64_t>(own_tokens, (int64_t)mask.window + mask.sinks + max_new + 2 * kGroup);
  p.split = {std::min(64, (own_tokens + least - 1) / least), least, kWaves * kGroup};
  const int64_t groups = (rule + kTileCols - 1) / kTileCols * Hkv;
  // (split where the tiles of the longest sequence fill less than half of the chip)
  p.prompt = {groups >= 128 ? 1 : (int)std::min<int64_t>({16, 256 / groups, (own_tokens + kLeast - 1) / kLeast}), kLeast, kStep};
  // the prefix in parts that fill the chip (two workgroups of few columns to a CU, one
  // of many), half of kLeast or more each: with 128 columns behind 8192 tokens 17.5 us
  // in 16 parts, 18.4 in 8, 25 in 32
  const int64_t pre_cols = (int64_t)n * (Hq / Hkv), pre_tile = pre_cols <= kFewPre ? kPreTile : kTileCols;
  const int64_t pre_groups = (pre_cols + pre_tile - 1) / pre_tile * Hkv;
  const int parts = (int)std::max<int64_t>(1, std::min<int64_t>(64, (pre_cols <= kFewPre ? 512 : 256) / pre_groups));
  p.pre_chunk = (std::max(kLeast / 2, (p.cut + parts - 1) / parts) + kStep * 2 - 1) / (kStep * 2) * (kStep * 2);
  p.pre = (p.cut + p.pre_chunk - 1) / p.pre_chunk;
  p.places = std::max(std::min(p.columns, kFew) * p.split.most, p.columns);
  // (one chunk of 64 rows beside 63 single tokens, 32 heads of 128, 64 parts: 135 MB by
  // rows, 4.3 GB by sequences; 2 prompts of 3000 rows 6.4 GB and 136 MB)
  const int64_t by_row = (int64_t)n * Hq * p.split.most, by_seq = (int64_t)B * Hkv * p.places;
  p.by_row = by_row < by_seq;
  const int64_t own = p.cut || p.split.most > 1 ? std::min(by_row, by_seq) : 0;
  p.many = cols > kFew && !(rule <= kFewShort && own_tokens <= least);
  p.joined = p.many && (p.cut || p.prompt.most > 1);
  const int64_t many = p.joined ? (int64_t)n * Hq * p.prompt.most : 0;
  const int64_t pre = (int64_t)n * Hq * p.pre;
  p.po = (float*)ws;
  p.prompt_o = p.po + own * hd;
  p.pre_o = p.prompt_o + many * hd;
  p.pml = (float2*)(p.pre_o + pre * hd);
  p.prompt_ml = p.pml + own;
  p.pre_ml = p.prompt_ml + many;
  if (bytes) *bytes = (own + many + pre) * (hd + 2) * 4;
  return p;
}

}  // namespace

int64_t paged_workspace_bytes(int n, int B, int Hq, int Hkv, int hd, int max_new, int tokens, int shared) {
  int64_t bytes;
  plan_of(n, B, Hq, Hkv, hd, max_new, tokens, shared, Mask{0, 0}, nullptr, &bytes);
  return bytes;
}

int64_t paged_workgroups(int n, int B, int Hq, int Hkv, int hd, int max_new, int tokens, int shared, int window, int sinks) {
  const AttnPlan p = plan_of(n, B, Hq, Hkv, hd, max_new, tokens, shared, Mask{window, sinks}, nullptr, nullptr);
  const int64_t pre = p.cut ? ((int64_t)n * (Hq / Hkv) + kTileCols - 1) / kTileCols * p.pre : 0;
  const int64_t own = p.many ? tiles_of(n, Hq / Hkv, B, p.cols).count * p.prompt.most : 0;
  return std::max(own, pre) * Hkv;
}

hipError_t launch_paged_append(const AppendArgs& a, hipStream_t s) {
  const int run = a.dtype == LMGC_DTYPE_BF16 ? 8 : 4;
  auto whole = [&](const void* p, int64_t ld, int n) { return ld % n == 0 && ((uintptr_t)p & 15) == 0; };
  const bool fast = a.rot % 16 == 0 && whole(a.k, a.ldk, run) && whole(a.v, a.ldv, run) &&
                    (!a.q || (whole(a.q, a.ldq, run) && whole(a.q_out, a.ldqo, 8)));
  const int places = a.r.n / kGroup + 2 * a.r.B;
  const dim3 grid(a.Hkv, std::min(places, kPlaces), (places + kPlaces - 1) / kPlaces);
  auto go = [&](auto t, auto h) {
    using T = decltype(t);
    constexpr int HD = decltype(h)::value;
    if (fast) hipLaunchKernelGGL((paged_append_kernel<T, HD, true>), grid, 256, 0, s, a);
    else hipLaunchKernelGGL((paged_append_kernel<T, HD, false>), grid, 256, 0, s, a);
  };
  auto heads = [&](auto t) {
    if (a.hd == 64) go(t, std::integral_constant<int, 64>{});
    else go(t, std::integral_constant<int, 128>{});
  };
  if (a.dtype == LMGC_DTYPE_BF16) heads(uint16_t{});
  else heads(float{});
  return hipGetLastError();
}

hipError_t launch_attention_paged(const PagedAttnArgs& a, hipStream_t s) {
  const Ragged& r = a.r;
  const int G = a.Hq / a.Hkv;
  const Mask mask{a.window, a.sinks};
  const AttnPlan plan = plan_of(r.n, r.B, a.Hq, a.Hkv, a.hd, a.max_new, r.max_pages * r.page, a.shared, mask, a.ws, nullptr);
  const float sl2 = scores_scale(a.scale);
  auto go = [&](auto h) {
    constexpr int HD = decltype(h)::value;
    auto split = [&](auto prefix, auto nt, int64_t blocks, int seqs) {
      hipLaunchKernelGGL((attn_paged_split_kernel<HD, decltype(nt)::value, decltype(prefix)::value>), dim3((unsigned)blocks, a.Hkv, seqs), kWaves * 64, 0, s, a.q, a.ldq, a.kc, a.vc, r,
                         a.max_new, a.Hkv, G, plan, mask, sl2, a.out);
    };
    auto prompt = [&](auto prefix, int64_t slots, int by_turns, int splits) {
      hipLaunchKernelGGL((attn_paged_prompt_kernel<HD, decltype(prefix)::value>), (unsigned)(slots * splits * a.Hkv), 512, 0, s, a.q, a.ldq,
                         a.kc, a.vc, r, a.max_new, a.Hkv, G, plan, mask, sl2, (int)slots, by_turns, splits, a.out);
    };
    if (plan.cut) {
      const int64_t all = (int64_t)r.n * G;
      if (all <= kFewPre) split(std::true_type{}, std::integral_constant<int, kPreTile / 16>{}, (all + kPreTile - 1) / kPreTile * plan.pre, 1);
      else prompt(std::true_type{}, (all + kTileCols - 1) / kTileCols, 0, plan.pre);
    }
    const int tiles = (plan.columns + 15) / 16, of_any = std::min(tiles, kFew / 16);
    split(std::false_type{}, std::integral_constant<int, 1>{}, of_any * plan.split.most + tiles - of_any, r.B);
    if (plan.many) {
      const Tiles t = tiles_of(r.n, G, r.B, plan.cols);
      prompt(std::false_type{}, t.count, t.by_turns, plan.prompt.most);
    }
    auto join = [&](auto rows, int64_t count) {
      hipLaunchKernelGGL((attn_paged_join_kernel<HD, decltype(rows)::value>), (unsigned)std::min<int64_t>((count + 1024 / HD - 1) / (1024 / HD), 1 << 20), 256, 0,
                         s, r, a.max_new, a.Hkv, G, plan, mask, a.out);
    };
    if (plan.cut || plan.joined) join(std::true_type{}, (int64_t)r.n * a.Hq);
    else if (plan.split.most > 1) join(std::false_type{}, (int64_t)r.B * a.Hkv * plan.columns);
  };
  if (a.hd == 64) go(std::integral_constant<int, 64>{});
  else go(std::integral_constant<int, 128>{});
  return hipGetLastError();
}

}  // namespace lmgc
