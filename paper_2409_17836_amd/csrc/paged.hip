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

// First number of a head's group of 32 tokens on a page.
__device__ inline int64_t group_at(const Ragged& r, int page, int Hkv, int h, int j, int hd) {
  return (((int64_t)page * Hkv + h) * r.page + ((j & (r.page - 1)) & ~(kGroup - 1))) * hd;
}

// ------------------------------------------------------------------ append
// Grid: (places, Hkv), 256 threads: a group of 32 tokens of one sequence's cache
// and one key/value head, with the query heads that read it.  Place starts[b] /
// 32 + 2 b + i is group i of sequence b's new tokens (so no sequence's places
// run into the next one's, wherever its groups begin).
//
// A thread has the two runs of 8 dims of 8 pairs of one token, so their cos and
// sin are read once for the key and the queries.  Keys go out as they are in a
// group, 16 bytes a lane; values meet in LDS, whose 16-byte slots are permuted so
// that the 64 halves of a store fall on all banks.
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

// FAST: rot a multiple of 16 and every run of 8 dims aligned to 16 bytes.
template <class T, int HD, bool FAST>
__global__ __launch_bounds__(256) void paged_append_kernel(AppendArgs a) {
  constexpr int U = HD / 16;          // places of 16 dims in a token
  constexpr int NH = 256 / (32 * U);  // heads side by side
  __shared__ u32x4 sv[HD * 4];        // a group of values
  const Ragged& r = a.r;
  const int b = last_at_most(r.B, blockIdx.x, [&](int i) { return (int64_t)r.starts[i] / kGroup + 2 * (int64_t)i; });
  Seq q = sequence(r, b, INT32_MAX);
  if (a.table) q.T = (int)min((int64_t)q.T, max((int64_t)0, a.n_pos - q.len));
  if (q.T <= 0) return;
  const int64_t place = (int64_t)blockIdx.x - (q.row / kGroup + 2 * (int64_t)b);
  if (place < 0) return;
  const int64_t t0 = q.len / kGroup * (int64_t)kGroup + place * kGroup;  // the group's first token
  if (t0 >= q.len + (int64_t)q.T) return;
  const int kvh = blockIdx.y, G = a.q ? a.Hq / a.Hkv : 0, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int lo = (int)max((int64_t)0, q.len - t0), hi = (int)min((int64_t)kGroup, q.len + (int64_t)q.T - t0);
  const int page = r.pages[(int64_t)b * r.max_pages + (t0 >> __builtin_ctz(r.page))];
  const bool there = page >= 0 && page < r.n_pages;
  const int64_t at = there ? group_at(r, page, a.Hkv, kvh, (int)t0, HD) : 0;
  // token and place of the thread: 16 tokens x 4 places to a wave
  const int t = 16 * (wave & 1) + (lane & 15), g = lane >> 4, x = U == 8 ? wave >> 1 : 0, h0 = U == 8 ? 0 : wave >> 1;
  const int unit = 4 * x + g;
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
  // the thread's 16 numbers of a row, rotated, as bf16
  auto rotated = [&](const T* p, u32x4& y0, u32x4& y1) __attribute__((always_inline)) {
    float y[16];
    if (FAST) {
      const Eight<T> u = load8(p + d0), v = load8(p + d1);
#pragma unroll
      for (int i = 0; i < 8; i++) {
        y[i] = u.get(i);
        y[8 + i] = v.get(i);
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
    } else {
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
    }
    y0 = pack8(y);
    y1 = pack8(y + 8);
  };
  if (mine) {
    for (int h = h0; h < 1 + G; h += NH) {
      u32x4 y0, y1;
      if (h == 0) {
        rotated(static_cast<const T*>(a.k) + row * a.ldk + kvh * HD, y0, y1);
        if (there) {
          auto put = [&](int d, u32x4 w) __attribute__((always_inline)) {
            *reinterpret_cast<u32x4*>(a.kc + at + ((t >> 4) * (HD / 32) + (d >> 5)) * 512 + ((t & 15) + 16 * ((d & 31) >> 3)) * 8) = w;
          };
          put(d0, y0);
          put(d1, y1);
        }
      } else {
        const int hq = kvh * G + h - 1;
        rotated(static_cast<const T*>(a.q) + row * a.ldq + (int64_t)hq * HD, y0, y1);
        uint16_t* o = a.q_out + row * a.ldqo + (int64_t)hq * HD;
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
  }
  if (!there) return;
  // values: slot (d, 4 tokens) holds tokens 4 k .. + 3 of both halves
  auto slot = [](int s) __attribute__((always_inline)) { return s ^ ((s >> 4 & 3) | (s >> 6 & 1) << 2); };
  if (mine && h0 == 0) {
    const T* p = static_cast<const T*>(a.v) + row * a.ldv + kvh * HD;
    uint16_t* words = reinterpret_cast<uint16_t*>(sv);
#pragma unroll
    for (int k = 0; k < 2; k++) {
      const int d = 32 * (x + (U / 4) * k) + 8 * g;  // (a run of 64 bytes for the four lanes of a token)
      u32x4 w;
      if (FAST) {
        const Eight<T> e = load8(p + d);
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; i++) y[i] = e.get(i);
        w = pack8(y);
      } else {
        float y[8];
        for (int i = 0; i < 8; i++) y[i] = load1(p + d + i);
        w = pack8(y);
      }
#pragma unroll
      for (int i = 0; i < 8; i++)
        words[slot(((d + i) >> 4) * 64 + ((d + i) & 15) + 16 * ((t & 15) >> 2)) * 8 + 4 * (t >> 4) + (t & 3)] =
            (uint16_t)(w[i >> 1] >> (16 * (i & 1)));
    }
  }
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

__device__ inline bool odd_bf16(uint32_t b) { return (b & 0x7f80u) == 0x7f80u; }  // NaN or infinity

// Values of a group that some, but not all, of a tile's queries see.  A
// probability of zero times a NaN or an infinity is NaN, so the values of tokens
// that no query sees (`seen`), which may be anything, are cleared; and where
// another one is not finite, its products are added here, to the columns that
// see it, and it is cleared too.  vr: a lane's operands (16 dims x 32 tokens
// each); pf, pos, low: of the lane's column; o: its result, 4 dims of 16 each.
template <int ND, int NT>
__device__ inline void clear_values(u32x4 (&vr)[ND], const bf16x8 (&pf)[NT], f32x4 (&o)[NT][ND], const Mask& mask, uint32_t seen,
                                    const int (&pos)[NT], int j0) {
  const int lane = threadIdx.x & 63, g = lane >> 4;
  uint32_t odd = 0;  // a bit for each half word e of the lane
#pragma unroll
  for (int e = 0; e < 4; e++) {
    // tokens 16 (e / 2) + 4 g + 2 (e % 2) and the next
    const uint32_t two = seen >> (16 * (e >> 1) + 2 * (e & 1)) >> (4 * g) & 3;
    const uint32_t keep = (two & 1 ? 0xffffu : 0u) | (two & 2 ? 0xffff0000u : 0u);
#pragma unroll
    for (int i = 0; i < ND; i++) {
      vr[i][e] &= keep;
      odd |= (uint32_t)odd_bf16(vr[i][e]) << (2 * e) | (uint32_t)odd_bf16(vr[i][e] >> 16) << (2 * e + 1);
    }
  }
  if (__ballot(odd != 0) == 0) return;
  for (int j = 0; j < kGroup; j++) {
    const int from = (j & 15) >> 2, e = 2 * (j >> 4) + ((j & 3) >> 1), hi = j & 1;
    if ((__ballot(odd >> (2 * e + hi) & 1) >> (16 * from) & 0xffff) == 0) continue;
    u32x4 w[(ND + 3) / 4];  // the token's values of the lane's dim, 16 i + lane % 16
#pragma unroll
    for (int i = 0; i < ND; i++) {
      const uint32_t x = e == 0 ? vr[i][0] : e == 1 ? vr[i][1] : e == 2 ? vr[i][2] : vr[i][3];
      w[i >> 2][i & 3] = hi ? x & 0xffff0000u : x << 16;
    }
#pragma unroll
    for (int y = 0; y < NT; y++) {
      float p = 0.f;
#pragma unroll
      for (int k = 0; k < 8; k++)
        if (k == 4 * (j >> 4) + (j & 3)) p = (float)pf[y][k];
      p = __shfl(p, 16 * from + (lane & 15));
      const bool sees = mask.sees(pos[y], mask.low(pos[y]), j0 + j);
#pragma unroll
      for (int i = 0; i < ND; i++)
#pragma unroll
        for (int r = 0; r < 4; r++) {
          const float v = __builtin_bit_cast(float, __shfl((int)w[i >> 2][i & 3], 16 * from + 4 * g + r));
          if (sees) o[y][i][r] = fmaf(p, v, o[y][i][r]);
        }
    }
    if (g == from) {
      const uint32_t keep = hi ? 0xffffu : 0xffff0000u;
#pragma unroll
      for (int i = 0; i < ND; i++) {
        if (e == 0) vr[i][0] &= keep;
        if (e == 1) vr[i][1] &= keep;
        if (e == 2) vr[i][2] &= keep;
        if (e == 3) vr[i][3] &= keep;
      }
    }
  }
}

// ---- few columns
// Columns: column c = t G + i of a (sequence, key/value head) is query head
// kvh G + i of its new token t; for the prefix, of row t of the batch.
//
// Grid: (splits, tiles of 16 NT columns x Hkv, B), 512 threads.  Wave w takes
// groups w, w + 8, .. of its split: S^T = K Q^T, so lane (col, g) holds the
// scores of its column and tokens 16 i + 4 g + r of a group, an online softmax,
// O^T += V^T P^T.  The waves' parts meet in LDS.
constexpr int kWaves = 8;

struct AttnPlan {
  int few;               // columns that the form for few takes, at most
  int columns;           // rows of its partial results for a sequence
  Splits split;          // of the form for few columns
  int cut;               // tokens that all share, computed for the batch
  int pre, pre_chunk;    // splits of these
  float *po, *pre_o;     // partial results, and maxima and sums
  float2 *pml, *pre_ml;
};

template <int HD, int NT, bool PREFIX>
__global__ __launch_bounds__(kWaves * 64, NT > 1 ? 2 : HD == 64 ? 6 : 4) void attn_paged_split_kernel(
    const uint16_t* __restrict__ q, int64_t ldq, const uint16_t* __restrict__ kc, const uint16_t* __restrict__ vc, Ragged r, int max_new,
    int Hkv, int G, AttnPlan plan, Mask mask, float sl2, uint16_t* __restrict__ out) {
  constexpr int KQ = HD / 32, ND = HD / 16, NW = kWaves, TILE = 16 * NT;
  __shared__ float so[NW][16][HD + 4];
  __shared__ float sm[NW][16], sl[NW][16];
  const int tid = threadIdx.x, lane = tid & 63, col = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int tile = blockIdx.y / Hkv, kvh = blockIdx.y - tile * Hkv, split = blockIdx.x, b = PREFIX ? 0 : blockIdx.z;
  const int c0 = tile * TILE;
  Seq sq{0, r.n, 0};
  if (!PREFIX) sq = sequence(r, b, max_new);
  const int cols = sq.T * G, ncol = min(TILE, cols - c0);
  if (ncol <= 0 || (!PREFIX && cols > plan.few)) return;
  // the lane's columns (past the last: the last one's again), their positions
  int pos[NT], p0, p1;
  if (PREFIX) {
    p0 = INT32_MAX;
    p1 = -1;
#pragma unroll
    for (int y = 0; y < NT; y++) {
      // the last sequence that begins at or before the row
      const int row = (c0 + min(16 * y + col, ncol - 1)) / G;
      int lo = 0, n = r.B;
      while (n > 1) {
        const int h = n / 2;
        const bool right = r.starts[lo + h] <= row;
        lo += right ? h : 0;
        n = right ? n - h : h;
      }
      const Seq s = sequence(r, lo, max_new);
      const int t = row - s.row;
      pos[y] = t >= 0 && t < s.T ? s.len + t : -1;  // (no token: sees nothing)
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
  const Span span = PREFIX ? Span{0, 0, 0, plan.cut} : span_of(sq, mask, plan.cut);
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
  float m[NT];
  f32x4 l[NT], o[NT][ND];
#pragma unroll
  for (int y = 0; y < NT; y++) {
    m[y] = -INFINITY;
    l[y] = f32x4{};
#pragma unroll
    for (int i = 0; i < ND; i++) o[y][i] = f32x4{};
  }
  const __bf16 one = (__bf16)1.0f;
  const bf16x8 ones = {one, one, one, one, one, one, one, one};
  const int32_t* pages = r.pages + (int64_t)b * r.max_pages;
  int held = -1;
  int it = 0;
  for (int v = v0 + wave * kGroup; v < v1; v += NW * kGroup, it++) {
    // a lane holds the page of each of the wave's next 64 groups
    if ((it & 63) == 0) {
      const int mine = v + lane * (NW * kGroup);
      held = mine < v1 ? pages[span.real(mine) >> __builtin_ctz(r.page)] : -1;
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
        const int low = mask.low(pos[y]);
#pragma unroll
        for (int i = 0; i < 2; i++)
#pragma unroll
          for (int e = 0; e < 4; e++)
            if (!mask.sees(pos[y], low, j0 + 16 * i + 4 * g + e)) s[i][e] = -INFINITY;
      }
      float mx = -INFINITY;
#pragma unroll
      for (int i = 0; i < 2; i++)
#pragma unroll
        for (int e = 0; e < 4; e++) mx = fmaxf(mx, s[i][e]);  // (drops a NaN; it comes back through the exponential)
      mx = fmaxf(mx, __shfl_xor(mx, 16));
      mx = fmaxf(mx, __shfl_xor(mx, 32)) * sl2;
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
    if (!whole) clear_values<ND, NT>(vr, pf, o, mask, mask.seen(p0, p1, j0), pos, j0);
#pragma unroll
    for (int i = 0; i < ND; i++)
#pragma unroll
      for (int y = 0; y < NT; y++)
        o[y][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vr[i]), pf[y], o[y][i], 0, 0, 0);
  }
  // HD / 32 dims of a column to a thread
  typedef float f32xd __attribute__((ext_vector_type(HD / 32)));
#pragma unroll
  for (int y = 0; y < NT; y++) {
    if (y) __syncthreads();
    if (g == 0) {
      sm[wave][col] = m[y];
      sl[wave][col] = l[y][0];
    }
#pragma unroll
    for (int i = 0; i < ND; i++) *reinterpret_cast<f32x4*>(&so[wave][col][16 * i + 4 * g]) = o[y][i];
    __syncthreads();
    const int oc = tid >> 5, d0 = (tid & 31) * (HD / 32), c = c0 + 16 * y + oc;
    if (16 * y + oc >= ncol) continue;
    float M = sm[0][oc];
#pragma unroll
    for (int w = 1; w < NW; w++) M = fmaxf(M, sm[w][oc]);
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
      const float inv = L == 0.f ? 0.f : 1.0f / L;  // (no visible key: zeros)
      uint32_t* op = reinterpret_cast<uint32_t*>(out + ((int64_t)(sq.row + t) * Hkv * G + hq) * HD + d0);
#pragma unroll
      for (int e = 0; e < HD / 64; e++)
        op[e] = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)(acc[2 * e] * inv), (__bf16)(acc[2 * e + 1] * inv)});
    } else {
      const int64_t at = PREFIX ? ((int64_t)t * Hkv * G + hq) * plan.pre + split
                                : (((int64_t)b * Hkv + kvh) * plan.columns + c) * plan.split.most + split;
      *reinterpret_cast<f32xd*>((PREFIX ? plan.pre_o : plan.po) + at * HD + d0) = acc;
      if (d0 == 0) (PREFIX ? plan.pre_ml : plan.pml)[at] = make_float2(M, L);
    }
  }
}

// Joins the parts of a row and head: a wave each, first a lane per part (its
// weight), then HD / 64 dims to a lane.
template <int HD>
__global__ __launch_bounds__(256) void attn_paged_join_kernel(Ragged r, int max_new, int Hkv, int G, AttnPlan plan, Mask mask,
                                                              uint16_t* __restrict__ out) {
  const int lane = threadIdx.x & 63;
  const int64_t at = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int Hq = Hkv * G, row = (int)(at / Hq), hq = (int)(at - (int64_t)row * Hq), kvh = hq / G;
  if (row >= r.n) return;
  const int b = last_at_most(r.B, row, [&](int i) { return (int64_t)r.starts[i]; });
  const Seq q = sequence(r, b, max_new);
  const int t = row - q.row;
  if (t < 0 || t >= q.T) return;
  const Span span = span_of(q, mask, plan.cut);
  const int chunk = plan.split.chunk(span.total), nown = (span.total + chunk - 1) / chunk;
  if (plan.cut == 0 && nown <= 1) return;  // written by the only split
  const int64_t own = (((int64_t)b * Hkv + kvh) * plan.columns + t * G + (hq - kvh * G)) * plan.split.most, pre = at * plan.pre;
  // parts: those of the prefix, then the sequence's own
  const int n = plan.pre + nown;
  float M = -INFINITY, ms[2], ls[2];
#pragma unroll
  for (int k = 0; k < 2; k++) {
    const int i = lane + 64 * k;
    const float2 ml = i < plan.pre ? plan.pre_ml[pre + i] : i < n ? plan.pml[own + i - plan.pre] : make_float2(-INFINITY, 0.f);
    ms[k] = ml.x;
    ls[k] = ml.y;
    M = fmaxf(M, ml.x);
  }
  for (int o = 32; o; o >>= 1) M = fmaxf(M, __shfl_xor(M, o));
  float L = 0.f, a[2];
#pragma unroll
  for (int k = 0; k < 2; k++) {
    // parts without a token that the query sees (m = -inf, l = 0) count for nothing
    a[k] = ms[k] == -INFINITY && ls[k] == 0.f ? 0.f : __builtin_amdgcn_exp2f(ms[k] - M);
    L += a[k] * ls[k];
  }
  for (int o = 32; o; o >>= 1) L += __shfl_xor(L, o);
  typedef float f32xd __attribute__((ext_vector_type(HD / 64)));
  f32xd acc = {};
  for (int i = 0; i < n; i++) {
    const float w = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, i < 64 ? a[0] : a[1]), i & 63));
    const float* p = i < plan.pre ? plan.pre_o + (pre + i) * HD : plan.po + (own + i - plan.pre) * HD;
    acc += w * reinterpret_cast<const f32xd*>(p)[lane];
  }
  const float inv = L == 0.f ? 0.f : 1.0f / L;
  uint16_t* op = out + at * HD + lane * (HD / 64);
#pragma unroll
  for (int i = 0; i < HD / 64; i++) op[i] = f32_to_bf16(acc[i] * inv);
}

// Tokens that are computed for the batch: whole pairs of groups.
int cut_of(int B, int shared) { return B > 1 ? shared / 64 * 64 : 0; }

AttnPlan plan_of(int n, int B, int Hq, int Hkv, int hd, int max_new, int tokens, int shared, void* ws, int64_t* bytes) {
  AttnPlan p{};
  p.few = INT32_MAX;
  p.columns = max_new * (Hq / Hkv);
  p.cut = std::min(cut_of(B, shared), tokens);
  const int least = 256 * 128 / hd * 2;
  p.split.unit = kWaves * kGroup;
  p.split.least = least;
  p.split.most = std::min(64, (tokens + least - 1) / least);
  p.pre_chunk = std::max(least, (p.cut + 63) / 64);
  p.pre_chunk = (p.pre_chunk + p.split.unit - 1) / p.split.unit * p.split.unit;
  p.pre = (p.cut + p.pre_chunk - 1) / p.pre_chunk;
  const int64_t own = p.cut || p.split.most > 1 ? (int64_t)B * Hkv * p.columns * p.split.most : 0, pre = (int64_t)n * Hq * p.pre;
  float* at = (float*)ws;
  p.po = at;
  p.pre_o = p.po + own * hd;
  p.pml = (float2*)(p.pre_o + pre * hd);
  p.pre_ml = p.pml + own;
  if (bytes) *bytes = (own + pre) * (hd + 2) * 4;
  return p;
}

}  // namespace

int64_t paged_workspace_bytes(int n, int B, int Hq, int Hkv, int hd, int max_new, int tokens, int shared) {
  int64_t bytes;
  plan_of(n, B, Hq, Hkv, hd, max_new, tokens, shared, nullptr, &bytes);
  return bytes;
}

int64_t paged_workgroups(int n, int B, int Hq, int Hkv, int hd, int max_new, int tokens, int shared) {
  return ((int64_t)max_new * (Hq / Hkv) + 15) / 16 * Hkv;
}

hipError_t launch_paged_append(const AppendArgs& a, hipStream_t s) {
  const int run = a.dtype == LMGC_DTYPE_BF16 ? 8 : 4;
  auto whole = [&](const void* p, int64_t ld, int n) { return ld % n == 0 && ((uintptr_t)p & 15) == 0; };
  const bool fast = a.rot % 16 == 0 && whole(a.k, a.ldk, run) && whole(a.v, a.ldv, run) &&
                    (!a.q || (whole(a.q, a.ldq, run) && whole(a.q_out, a.ldqo, 8)));
  const dim3 grid((unsigned)(a.r.n / kGroup + 2 * (int64_t)a.r.B), a.Hkv);
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
  const AttnPlan plan = plan_of(r.n, r.B, a.Hq, a.Hkv, a.hd, a.max_new, r.max_pages * r.page, a.shared, a.ws, nullptr);
  const Mask mask{a.window, a.sinks};
  const float sl2 = (float)(1.4426950408889634 * (double)a.scale);
  auto go = [&](auto h) {
    constexpr int HD = decltype(h)::value;
    if (plan.cut) {
      const dim3 grid(plan.pre, (unsigned)(((int64_t)r.n * G + 15) / 16 * a.Hkv));
      hipLaunchKernelGGL((attn_paged_split_kernel<HD, 1, true>), grid, kWaves * 64, 0, s, a.q, a.ldq, a.kc, a.vc, r, a.max_new, a.Hkv, G, plan, mask, sl2, a.out);
    }
    const dim3 grid(plan.split.most, (unsigned)(((int64_t)a.max_new * G + 15) / 16 * a.Hkv), r.B);
    hipLaunchKernelGGL((attn_paged_split_kernel<HD, 1, false>), grid, kWaves * 64, 0, s, a.q, a.ldq, a.kc, a.vc, r, a.max_new, a.Hkv, G, plan, mask, sl2, a.out);
    if (plan.cut || plan.split.most > 1)
      hipLaunchKernelGGL((attn_paged_join_kernel<HD>), (unsigned)(((int64_t)r.n * a.Hq + 3) / 4), 256, 0, s, r, a.max_new, a.Hkv, G, plan, mask, a.out);
  };
  if (a.hd == 64) go(std::integral_constant<int, 64>{});
  else go(std::integral_constant<int, 128>{});
  return hipGetLastError();
}

}  // namespace lmgc
