// The key/value cache in 8 bits and attention over it.
//
// Cache of one layer: for every sequence and key/value head, blocks of 64
// tokens in e4m3 with one float32 scale (a power of two) per block, keys and
// values apart.  Inside a block the codes lie in the order in which the lanes
// of the 16x16x32 matrix instruction take them:
//   key   (t, d): ((t/16) (hd/64) + d/64) 1024 + ((t%16) + 16 ((d%64)/16)) 16 + d%16
//   value (t, d): (d/16) 1024 + ((d%16) + 16 ((t%16)/4)) 16 + 4 (t/16) + t%4
// so a lane's 16 bytes are its operand of two instructions, a wave's load is
// 1 KB of consecutive memory, and the value order is the one in which the
// scores come out of the first product: the probabilities are the second
// product's operand where they are, with no exchange between lanes.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "mx.h"

namespace lmgc {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kBlk = 64;        // tokens per block
constexpr int kMinScale = 63;   // exponent byte of the smallest block scale, 2^-64

__device__ inline int key_at(int t, int d, int hd) {
  return ((t >> 4) * (hd >> 6) + (d >> 6)) * 1024 + ((t & 15) + 16 * ((d & 63) >> 4)) * 16 + (d & 15);
}
__device__ inline int value_at(int t, int d) {
  return (d >> 4) * 1024 + ((d & 15) + 16 * ((t & 15) >> 2)) * 16 + 4 * (t >> 4) + (t & 3);
}

// New tokens of a sequence that fit the cache: rows past this are left alone.
__device__ inline int new_tokens(const int32_t* lens, const int32_t* counts, int b, int T, int cap, int& len) {
  len = lens[b];
  const int n = counts ? min(T, counts[b]) : T;
  return len < 0 || len >= cap ? 0 : min(n, cap - len);
}

// ------------------------------------------------------------------ append
// A workgroup per (block of the cache that new tokens may fall into, key/value
// head, sequence x {key, value}).
//
// A block that gets its first token is read once, 16 bytes a load, and written
// once, 16 bytes of codes a lane, 1 KB in a row.  A key's 16 codes are 32
// bytes of its row.  A value's are 16 tokens of one dim: a thread takes 4
// tokens x 8 dims, packs the 4 tokens of each dim into the word they are in
// the block, and the words meet in LDS.  A block that has tokens already is
// the rare one (one per sequence and call): its new tokens are written byte by
// byte, and the earlier codes are gone over only when the scale grows.  4 x 32
// heads of 128, 4096 tokens: 73 us, 5.5 TB/s (bytes of k, v and the codes); a
// token each for 32 sequences 3 us, the launch and a round trip to memory.
__device__ inline uint32_t abs_max2(uint32_t a, uint32_t w) { return max(a, max(w & 0x7fffu, (w >> 16) & 0x7fffu)); }

__device__ inline uint32_t block_max(uint32_t a, uint32_t* part) {
  for (int o = 32; o; o >>= 1) a = max(a, (uint32_t)__shfl_xor((int)a, o, 64));
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = a;
  __syncthreads();
  return max(max(part[0], part[1]), max(part[2], part[3]));
}

template <int HD>
__global__ __launch_bounds__(256) void kv8_append_kernel(const uint16_t* __restrict__ kin, const uint16_t* __restrict__ vin,
                                                         int Hkv, int T, int cap, const int32_t* __restrict__ lens,
                                                         const int32_t* __restrict__ counts, uint8_t* __restrict__ kc,
                                                         float* __restrict__ ks, uint8_t* __restrict__ vc,
                                                         float* __restrict__ vs) {
  __shared__ uint32_t part[4];
  __shared__ uint32_t words[kBlk * HD / 4];
  const int b = blockIdx.z >> 1, is_v = blockIdx.z & 1, h = blockIdx.y, tid = threadIdx.x, lane = tid & 63;
  int len;
  const int n = new_tokens(lens, counts, b, T, cap, len);
  if (n <= 0) return;
  const int blk = len / kBlk + blockIdx.x, t0 = blk * kBlk;
  if (t0 >= len + n) return;
  const int lo = max(0, len - t0), hi = min(kBlk, len + n - t0);  // new tokens of the block
  const int64_t hb = (int64_t)b * Hkv + h;
  const uint16_t* src = (is_v ? vin : kin) + (hb * T + (t0 - len)) * HD;  // row of token t0 (rows lo .. hi - 1 exist)
  uint8_t* codes = (is_v ? vc : kc) + (hb * (cap / kBlk) + blk) * (kBlk * HD);
  float* scale = (is_v ? vs : ks) + hb * (cap / kBlk) + blk;
  // bf16 bits of a magnitude -> block scale (NaN for a NaN or an infinity)
  auto scale_of = [](uint32_t a) __attribute__((always_inline)) {
    return a >= 0x7f80u ? __builtin_bit_cast(float, 0x7fc00000u) : mx_scale(max(mx_scale_byte<LMGC_MX_FP8>(a << 16), kMinScale));
  };
  auto lo16 = [](uint32_t w) __attribute__((always_inline)) { return __builtin_bit_cast(float, w << 16); };
  auto hi16 = [](uint32_t w) __attribute__((always_inline)) { return __builtin_bit_cast(float, w & 0xffff0000u); };
  auto pack4 = [](float a, float b2, float c, float d) __attribute__((always_inline)) {
    const int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b2, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
  };
  const u32x4 zero = {0, 0, 0, 0};
  if (lo == 0 && !is_v) {
    constexpr int NP = HD / 64, NC = HD / 64;  // pieces of a thread; chunks of 64 dims
    u32x4 w[NP][2];
    uint32_t a = 0;
#pragma unroll
    for (int i = 0; i < NP; i++) {
      const int p = (tid >> 6) + 4 * i, t = 16 * (p / NC) + (lane & 15), d = 64 * (p % NC) + 16 * (lane >> 4);
      const u32x4* q = reinterpret_cast<const u32x4*>(src + (int64_t)t * HD + d);
      w[i][0] = t < hi ? q[0] : zero;
      w[i][1] = t < hi ? q[1] : zero;
    }
#pragma unroll
    for (int i = 0; i < NP; i++)
#pragma unroll
      for (int e = 0; e < 8; e++) a = abs_max2(a, w[i][e >> 2][e & 3]);
    const float s = scale_of(block_max(a, part));
    const bool nan = s != s;
    const float inv = nan ? 0.f : 1.0f / s;
    if (tid == 0) *scale = s;
#pragma unroll
    for (int i = 0; i < NP; i++) {
      u32x4 o = zero;
#pragma unroll
      for (int e = 0; e < 4; e++) {
        const uint32_t x = w[i][e >> 1][2 * (e & 1)], y = w[i][e >> 1][2 * (e & 1) + 1];
        if (!nan) o[e] = pack4(lo16(x) * inv, hi16(x) * inv, lo16(y) * inv, hi16(y) * inv);
      }
      reinterpret_cast<u32x4*>(codes)[((tid >> 6) + 4 * i) * 64 + lane] = o;
    }
  } else if (lo == 0) {
    const int quad = tid & 15, d0 = (tid >> 4) * 8;  // tokens 4 quad .. + 3, dims d0 .. + 7
    u32x4 w[4];
    uint32_t a = 0;
#pragma unroll
    for (int r = 0; r < 4; r++) {
      const int t = 4 * quad + r;
      w[r] = t < hi && d0 < HD ? *reinterpret_cast<const u32x4*>(src + (int64_t)t * HD + d0) : zero;
#pragma unroll
      for (int e = 0; e < 4; e++) a = abs_max2(a, w[r][e]);
    }
    const float s = scale_of(block_max(a, part));
    const bool nan = s != s;
    const float inv = nan ? 0.f : 1.0f / s;
    if (tid == 0) *scale = s;
    if (d0 < HD) {
#pragma unroll
      for (int e = 0; e < 8; e++) {
        const int d = d0 + e;
        float v[4];
#pragma unroll
        for (int r = 0; r < 4; r++) v[r] = (e & 1 ? hi16(w[r][e >> 1]) : lo16(w[r][e >> 1])) * inv;
        words[(d >> 4) * 256 + ((d & 15) + 16 * (quad & 3)) * 4 + (quad >> 2)] = nan ? 0u : pack4(v[0], v[1], v[2], v[3]);
      }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < HD / 64; i++)
      reinterpret_cast<u32x4*>(codes)[i * 256 + tid] = *reinterpret_cast<const u32x4*>(words + (i * 256 + tid) * 4);
  } else {
    uint32_t a = 0;
    for (int i = tid; i < (hi - lo) * HD; i += 256) a = max(a, (uint32_t)src[(int64_t)lo * HD + i] & 0x7fffu);
    const float s_old = *scale;
    const float s_new = scale_of(block_max(a, part));  // (the barrier in it: every thread has read the old scale)
    const bool nan = s_new != s_new || s_old != s_old;
    const float s = nan ? __builtin_bit_cast(float, 0x7fc00000u) : fmaxf(s_old, s_new);
    const float inv = 1.0f / s, grow = s_old * inv;
    if (tid == 0) *scale = s;
    if (!nan && s != s_old)
      for (int i = tid; i < lo * HD; i += 256) {
        const int t = i / HD, d = i - t * HD;
        uint8_t* p = codes + (is_v ? value_at(t, d) : key_at(t, d, HD));
        const float v = __builtin_amdgcn_cvt_f32_fp8((int)*p, 0) * grow;
        *p = (uint8_t)__builtin_amdgcn_cvt_pk_fp8_f32(v, v, 0, false);
      }
    for (int i = tid; i < (hi - lo) * HD; i += 256) {
      const int t = lo + i / HD, d = i % HD;
      const float v = nan ? 0.f : bf16_to_f32(src[(int64_t)t * HD + d]) * inv;
      codes[is_v ? value_at(t, d) : key_at(t, d, HD)] = (uint8_t)__builtin_amdgcn_cvt_pk_fp8_f32(v, v, 0, false);
    }
  }
}

// --------------------------------------------------------------- attention
// Keys that a query at position pos sees: j <= pos and, with a window, j >
// pos - window or j < sinks.
struct Mask {
  int window, sinks;
  // low(pos): the last key before the window (no short circuits: a select costs less than a branch)
  __device__ inline int low(int pos) const { return window ? pos - window : -1; }
  __device__ inline bool sees(int pos, int low, int j) const { return (j <= pos) & ((j > low) | (j < sinks)); }
  // whether any query at positions p0 .. p1 may see a key of [j0, j1)
  __device__ inline bool any(int p0, int p1, int j0, int j1) const {
    return j0 <= p1 && (window == 0 || j1 - 1 > p0 - window || j0 < sinks);
  }
  // whether every query at positions p0 .. p1 sees every key of [j0, j1)
  __device__ inline bool all(int p0, int p1, int j0, int j1) const {
    return j1 - 1 <= p0 && (window == 0 || j0 > p1 - window || j1 <= sinks);
  }
  // the tokens of the block at j0 that some query at positions p0 .. p1 sees, a bit each
  __device__ inline uint64_t seen(int p0, int p1, int j0) const {
    auto first = [](int n) __attribute__((always_inline)) { return n >= kBlk ? ~0ull : (1ull << max(n, 0)) - 1; };
    return first(p1 + 1 - j0) & (~first(max(low(p0), -1) + 1 - j0) | first(sinks - j0));
  }
  // whether split [j0, j1) of the cache is the only one that any of them sees
  __device__ inline bool only(int p0, int p1, int j0, int j1) const { return j1 > p1 && (j0 == 0 || !any(p0, p1, 0, j0)); }
};

// Codes of values that no query sees may be anything, a NaN among it, and a
// probability of zero times that is NaN: they are cleared.  The bytes that stay
// in word e of a lane's 16 codes of a block, tokens 16 e + 4 g .. + 3 of `seen`.
__device__ inline uint32_t seen_bytes(uint64_t seen, int e, int g) {
  const uint32_t four = (uint32_t)(seen >> (e & 2 ? 32 : 0)) >> (4 * g) >> (16 * (e & 1)) & 15;
  const uint32_t ones = four * 0x204081 & 0x01010101;  // a bit to a byte
  return (ones << 8) - ones;
}

__device__ inline bf16x8 fp8_bf16(uint32_t w0, uint32_t w1) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, 1.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, 1.0f, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, 1.0f, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, 1.0f, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// Columns: column c = t G + i of a (sequence, key/value head) is query head
// kvh G + i of new token t.  A column's result is a function of the column's
// query and of the cache, whatever columns, sequences and splits run with it:
// blocks that a column does not see add exact zeros.

// (in integers: a block's scales are the same in all lanes, and so stay scalar)
__device__ inline bool is_nan(float v) { return (__builtin_bit_cast(uint32_t, v) & 0x7fffffffu) > 0x7f800000u; }
// log2 of a block's scale, a power of two; NaN stays NaN.
__device__ inline float log2_scale(float v) {
  return is_nan(v) ? v : (float)((int)(__builtin_bit_cast(uint32_t, v) >> 23) - 127);
}

// Buffer over the codes of one block (stride 0, word 3 of gfx9).
template <int HD>
__device__ inline __amdgpu_buffer_rsrc_t block_buffer(const uint8_t* codes, int64_t blk) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(codes + blk * (kBlk * HD)), (short)0, kBlk * HD, 0x00020000);
}

// ---- few columns
// Up to kFewCols columns whose tiles of 16, times Hkv, the cache's blocks and
// the head's halves, are at most kFewBlocks, and up to 32 anyway: every tile
// walks the cache by itself, eight waves at a time, which takes less time than
// the form for many columns as long as the sequences do not fill the chip.  12
// heads of 64, 1000 queries from the start: 9.9 us (the other form 29.5), 4
// such sequences 27 (31), 8 of them 47 (42); 32 heads on 8 of 128, 50 queries
// over 3900 tokens: 19 us (31), 4 of them 46 (37).  So the limits are those of a
// sequence by itself, and several in one call lose some of it: the choice may
// not go by their number, or a sequence's bits would.
//
// Grid: (splits, tiles of 16 columns x Hkv, B), 512 threads.  A cache of up to
// kOneBytes is one split (and the call one launch), a longer one is cut into
// kSplitBytes (more where that were over kMaxSplits).  Wave w takes its blocks
// w, w + 8, ..: S^T = K Q^T, so lane (col, g) holds the scores of its column
// and tokens 16 i + 4 g + r of a block, an online softmax, O^T += V^T P^T.
// The waves' parts meet in LDS.
//
// Bound by the bytes of the cache, with many tiles by the vector unit (codes to
// bf16, exponentials), and with few tokens by a chain of dependent loads (5.9 us
// for 512 + 4 of them).  ONCE, a single tile of columns: nothing reads the codes
// again before the next step, so they are loaded past the caches' order of use.
// From memory, 8 sequences x 32 heads of 128 over 4094 tokens, 268 MB: 48 to 49 us,
// 5.5 TB/s (55 without ONCE); 32 sequences 170 us, 6.2 TB/s (187); one sequence
// 11.6 us (12.5).  With two tiles the second one misses them (23.7 us for 21.7
// at 8 x 8 heads, 32 columns over 2000).
constexpr int kFewCols = 2048, kFewBlocks = 16384;
constexpr int kNonTemporal = 2;  // the instruction's nt bit
constexpr int kOneBytes = 256 << 10, kSplitBytes = 128 << 10;
constexpr int kSplitWaves = 8;
constexpr int kMaxSplits = 64;  // a lane each in the join

template <int HD, bool ONCE>
__global__ __launch_bounds__(kSplitWaves * 64, HD == 64 ? 6 : 4) void attn_kv8_split_kernel(
    const uint16_t* __restrict__ q, const uint8_t* __restrict__ kc, const float* __restrict__ ks,
    const uint8_t* __restrict__ vc, const float* __restrict__ vs, const int32_t* __restrict__ lens,
    const int32_t* __restrict__ counts, int Hkv, uint32_t hinv, int G, uint32_t ginv, int T, int cap, int nsplit, int chunk, Mask mask,
    float sl2, float* __restrict__ part_o, float2* __restrict__ part_ml, uint16_t* __restrict__ out) {
  constexpr int NC = HD / 64, ND = HD / 16, NW = kSplitWaves;
  __shared__ float so[NW][16][HD + 4];
  __shared__ float sm[NW][16], sl[NW][16];
  const int tile = Hkv > 1 ? (int)__umulhi(blockIdx.y, hinv) : (int)blockIdx.y;  // blockIdx.y / Hkv
  const int split = blockIdx.x, c0 = 16 * tile, kvh = blockIdx.y - tile * Hkv, b = blockIdx.z;
  const int tid = threadIdx.x, lane = tid & 63, col = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  auto over_g = [&](int c) __attribute__((always_inline)) { return G > 1 ? (int)__umulhi(c, ginv) : c; };  // c / G
  int len;
  const int n = new_tokens(lens, counts, b, T, cap, len);
  const int ncol = min(16, n * G - c0);
  if (ncol <= 0) return;
  const int p0 = len + over_g(c0), p1 = len + over_g(c0 + ncol - 1);  // positions of the tile's queries
  const int jlo = split * chunk, jhi = min(cap, jlo + chunk);
  if (!mask.any(p0, p1, jlo, jhi)) return;
  const int c = c0 + min(col, ncol - 1), t = over_g(c), pos = len + t, low = mask.low(pos);
  const int64_t hb = (int64_t)b * Hkv + kvh, nblk = cap / kBlk;
  const uint16_t* qp = q + ((hb * G + (c - t * G)) * T + t) * HD + 16 * g;
  bf16x8 qf[NC][2];
#pragma unroll
  for (int x = 0; x < NC; x++)
#pragma unroll
    for (int y = 0; y < 2; y++) qf[x][y] = *reinterpret_cast<const bf16x8*>(qp + 64 * x + 8 * y);

  float m = -INFINITY;
  f32x4 l = {};  // the row sum, four times: a product of the probabilities with ones
  f32x4 o[ND] = {};
  const int jend = min(jhi, p1 + 1);
  for (int j0 = jlo + wave * kBlk; j0 < jend; j0 += NW * kBlk) {
    if (!mask.any(p0, p1, j0, j0 + kBlk)) continue;
    const int64_t blk = hb * nblk + j0 / kBlk;
    // (through buffers of a block each: their addresses take no vector registers)
    const __amdgpu_buffer_rsrc_t kb = block_buffer<HD>(kc, blk), vb = block_buffer<HD>(vc, blk);
    auto codes = [&](__amdgpu_buffer_rsrc_t block, int i) __attribute__((always_inline)) {
      return __builtin_amdgcn_raw_buffer_load_b128(block, lane * 16, i * 1024, ONCE ? kNonTemporal : 0);
    };
    u32x4 kr[4][NC], vr[ND];
#pragma unroll
    for (int i = 0; i < 4; i++)
#pragma unroll
      for (int x = 0; x < NC; x++) kr[i][x] = codes(kb, i * NC + x);
#pragma unroll
    for (int i = 0; i < ND / 2; i++) vr[i] = codes(vb, i);
    const float kscale = ks[blk];
    float fk = kscale * sl2, fv = vs[blk];
    f32x4 s[4] = {};
    // tile by tile, half of the values asked for behind the first tile: mixed
    // with each other and with what follows, 128 dims do not fit the registers
#pragma unroll
    for (int i = 0; i < 4; i++) {
      __builtin_amdgcn_sched_barrier(0);
      if (i == 1)
#pragma unroll
        for (int e = ND / 2; e < ND; e++) vr[e] = codes(vb, e);
#pragma unroll
      for (int x = 0; x < NC; x++)
#pragma unroll
        for (int y = 0; y < 2; y++)
          s[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fp8_bf16(kr[i][x][2 * y], kr[i][x][2 * y + 1]), qf[x][y], s[i], 0, 0, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
    if (!mask.all(p0, p1, j0, j0 + kBlk)) {
      // NaN in a scale: the visible tokens' scores take it, and the others are
      // left out as ever
      if (is_nan(kscale) || is_nan(fv)) {
#pragma unroll
        for (int i = 0; i < 4; i++) s[i] *= __builtin_bit_cast(float, 0x7fc00000u);
        fk = fv = 1.0f;
      }
#pragma unroll
      for (int i = 0; i < 4; i++)
#pragma unroll
        for (int r = 0; r < 4; r++)
          if (!mask.sees(pos, low, j0 + 16 * i + 4 * g + r)) s[i][r] = -INFINITY;
      const uint64_t seen = mask.seen(p0, p1, j0);
#pragma unroll
      for (int e = 0; e < 4; e++) {
        const uint32_t keep = seen_bytes(seen, e, g);
#pragma unroll
        for (int i = 0; i < ND; i++) vr[i][e] &= keep;
      }
    }
    float mx = -INFINITY;
#pragma unroll
    for (int i = 0; i < 4; i++)
#pragma unroll
      for (int r = 0; r < 4; r++) mx = fmaxf(mx, s[i][r]);  // (drops a NaN; it comes back through the exponential)
    mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
    mx = fmaxf(mx, __shfl_xor(mx, 32, 64)) * fk;
    if (mx > m) {
      const float a = __builtin_amdgcn_exp2f(m - mx);
      l *= a;
#pragma unroll
      for (int i = 0; i < ND; i++) o[i] *= a;
      m = mx;
    }
    // the keys' scale is the exponent's factor, the values' (a power of two) a
    // summand of it: log2_scale; the row sum has ones over that scale
    const float sub = log2_scale(fv) - (m == -INFINITY ? 0.f : m);
    const __bf16 unscale = (__bf16)(is_nan(fv) ? 1.0f : __builtin_amdgcn_rcpf(fv));  // exact
    const bf16x8 ones = {unscale, unscale, unscale, unscale, unscale, unscale, unscale, unscale};
    bf16x8 pf[2];  // rounded to bf16 for the second product; the sum is of the rounded values
#pragma unroll
    for (int i = 0; i < 4; i++)
#pragma unroll
      for (int r = 0; r < 4; r++) pf[i >> 1][(i & 1) * 4 + r] = (__bf16)__builtin_amdgcn_exp2f(fmaf(s[i][r], fk, sub));
#pragma unroll
    for (int y = 0; y < 2; y++) l = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, pf[y], l, 0, 0, 0);
#pragma unroll
    for (int i = 0; i < ND; i++)
#pragma unroll
      for (int y = 0; y < 2; y++)
        o[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fp8_bf16(vr[i][2 * y], vr[i][2 * y + 1]), pf[y], o[i], 0, 0, 0);
  }
  if (g == 0) {
    sm[wave][col] = m;
    sl[wave][col] = l[0];
  }
#pragma unroll
  for (int i = 0; i < ND; i++) *reinterpret_cast<f32x4*>(&so[wave][col][16 * i + 4 * g]) = o[i];
  __syncthreads();
  // HD / 32 dims of a column to a thread
  typedef float f32xd __attribute__((ext_vector_type(HD / 32)));
  const int oc = tid >> 5, d0 = (tid & 31) * (HD / 32);
  if (oc >= ncol) return;
  float M = sm[0][oc];
#pragma unroll
  for (int w = 1; w < NW; w++) M = fmaxf(M, sm[w][oc]);
  float L = 0.f;
  f32xd r = {};
#pragma unroll
  for (int w = 0; w < NW; w++) {
    // waves without a token they see (m = -inf, l = 0) count for nothing
    const float mw = sm[w][oc], lw = sl[w][oc], a = mw == -INFINITY && lw == 0.f ? 0.f : __builtin_amdgcn_exp2f(mw - M);
    L += a * lw;
    r += a * *reinterpret_cast<const f32xd*>(&so[w][oc][d0]);
  }
  const int ot = over_g(c0 + oc);
  if (mask.only(p0, p1, jlo, jhi)) {
    const float inv = 1.0f / L;
    uint32_t* op = reinterpret_cast<uint32_t*>(out + (((int64_t)b * T + ot) * Hkv + kvh) * ((int64_t)G * HD) + (c0 + oc - ot * G) * HD + d0);
#pragma unroll
    for (int e = 0; e < HD / 64; e++)
      op[e] = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)(r[2 * e] * inv), (__bf16)(r[2 * e + 1] * inv)});
  } else {
    const int64_t row = (hb * T * G + c0 + oc) * nsplit + split;
    *reinterpret_cast<f32xd*>(part_o + row * HD + d0) = r;
    if (d0 == 0) part_ml[row] = make_float2(M, L);
  }
}

// Joins the splits of a column: a wave per column, first a lane per split (its
// weight), then HD / 64 dims to a lane.  TILE: columns whose positions decide
// together which splits have run.
template <int HD, int TILE>
__global__ __launch_bounds__(64) void attn_kv8_join_kernel(const float* __restrict__ part_o, const float2* __restrict__ part_ml,
                                                           const int32_t* __restrict__ lens, const int32_t* __restrict__ counts,
                                                           int Hkv, int G, int T, int cap, int nsplit, int chunk, Mask mask,
                                                           uint16_t* __restrict__ out) {
  const int c = blockIdx.x, kvh = blockIdx.y, b = blockIdx.z, lane = threadIdx.x;
  int len;
  const int n = new_tokens(lens, counts, b, T, cap, len);
  if (c >= n * G) return;
  const int c0 = c / TILE * TILE, ncol = min(TILE, n * G - c0), p0 = len + c0 / G, p1 = len + (c0 + ncol - 1) / G;
  const int64_t hb = (int64_t)b * Hkv + kvh, row = hb * T * G + c;
  const bool ran = lane < nsplit && mask.any(p0, p1, lane * chunk, min(cap, lane * chunk + chunk));
  const uint64_t used = __ballot(ran);
  if ((used & (used - 1)) == 0) return;  // written by the only split
  const float2 ml = ran ? part_ml[row * nsplit + lane] : make_float2(-INFINITY, 0.f);
  float M = ml.x;
  for (int o = 32; o; o >>= 1) M = fmaxf(M, __shfl_xor(M, o, 64));
  // splits without a token that the column sees (m = -inf, l = 0) count for nothing
  const float a = ml.x == -INFINITY && ml.y == 0.f ? 0.f : __builtin_amdgcn_exp2f(ml.x - M);
  float L = a * ml.y;
  for (int o = 32; o; o >>= 1) L += __shfl_xor(L, o, 64);
  typedef float f32xd __attribute__((ext_vector_type(HD / 64)));
  f32xd acc = {};
  const f32xd* p = reinterpret_cast<const f32xd*>(part_o + row * nsplit * HD) + lane;
  // 16 at a time, so that their loads are under way together (those of splits
  // that have not run, between the sinks and the window, are dropped)
  for (int x0 = 0; x0 < nsplit; x0 += 16) {
    f32xd v[16];
#pragma unroll
    for (int x = 0; x < 16; x++) v[x] = p[min(x0 + x, nsplit - 1) * 64];
#pragma unroll
    for (int x = 0; x < 16; x++) {
      const float ax = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, a), x0 + x));
      if (used >> (x0 + x) & 1) acc += ax * v[x];
    }
  }
  const int t = c / G, hq = kvh * G + c % G;
  const float inv = 1.0f / L;  // as where a single split writes the result: a column's tile decides which does
  uint16_t* op = out + ((int64_t)b * T + t) * ((int64_t)Hkv * G * HD) + hq * HD + lane * (HD / 64);
#pragma unroll
  for (int i = 0; i < HD / 64; i++) op[i] = f32_to_bf16(acc[i] * inv);
}

// ---- many columns
// A workgroup of eight waves takes 256 columns of one (sequence, key/value
// head), each wave 32, and walks the cache block by block.  A block's codes
// come straight to LDS kAhead steps ahead, are converted once and stored as
// bf16 in the order of the matrix operands, so a conversion serves 256 columns
// and the products read a lane's 16 bytes in a row.
//
// A step has two phases, a barrier after each: one for the vector unit
// (maxima, exponentials), one for the matrix unit (the block's values, the
// next block's scores; behind them the conversion, which evens them out).  The
// waves of a SIMD, w and w + 4, are a phase apart, so that the units work side
// by side: in a wave's own stream, vector instructions between products only
// delay them (64 products took 2000 cycles by themselves and 2900 with 110
// vector instructions among them), and with both waves in the same phase a
// step took 5500 cycles.  Bound by the two units' turns: 2 x 32 heads of 128 on
// 8 key/value heads, 3001 queries behind 1000 tokens, 232 to 242 us, 1.01 to
// 1.05 PFLOP/s (a bf16 library product of 8192^3 reaches 1.40 to 1.45).
//
// The block scales cost nothing per score: the keys' goes into the exponent's
// factor, the values' (a power of two) into its summand, and the row sums
// are a product too, with ones over that scale.
//
// Where a sequence has fewer than 128 tiles the length is split too: for 128
// workgroups as long as a split has kShortSplit tokens, for 256 where it has
// kLongSplit.  A split's sums go twice through memory: 1 x 12 heads of 64, 50
// queries over 1000 tokens take 16 us in splits of 512 and 24 of 1024, 8 x 12
// heads, 256 over 768, take 40 and 31; 2 x 32 heads of 128, 1000 over 4000
// tokens, take 118 us whole and 164 in halves; 1 x 32 heads, 4 queries to a
// key/value head, 512 over 30000 take 233 us in quarters and 392 in halves.
constexpr int kTileCols = 256;
constexpr int kShortSplit = 576, kLongSplit = 2048;
constexpr int kMaxPromptSplits = 16;
constexpr int kAhead = 3;  // steps that a block's codes are asked for ahead
constexpr int kReads = 8;  // operands read ahead of their products

// 16 bytes a lane from memory to LDS, lane l's at lds + 16 l.  In assembly:
// with the builtin the compiler waits for every load before any read of the
// ring; the waits are written out where they belong.
__device__ inline void load_lds(const uint8_t* p, u32x4* lds) {
  const uint32_t at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) u32x4*)lds;
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off"
               :: "s"(__builtin_amdgcn_readfirstlane((int)at)), "v"(p) : "m0", "memory");
}

// s_waitcnt vmcnt(n) alone
constexpr int vmcnt_imm(int n) { return (n & 15) | ((n >> 4) << 14) | 0xF70; }

template <int HD>
__global__ __launch_bounds__(512, 2) void attn_kv8_prompt_kernel(
    const uint16_t* __restrict__ q, const uint8_t* __restrict__ kc, const float* __restrict__ ks,
    const uint8_t* __restrict__ vc, const float* __restrict__ vs, const int32_t* __restrict__ lens,
    const int32_t* __restrict__ counts, int B, int Hkv, int G, int T, int cap, int ntile, int nsplit, int chunk, Mask mask, float sl2,
    float* __restrict__ part_o, float2* __restrict__ part_ml, uint16_t* __restrict__ out) {
  constexpr int ND = HD / 16, KQ = HD / 32;  // dim tiles; 32-dim steps of a score
  constexpr int NP = HD / 64;                // 4 KB of codes of keys (and of values) of a block
  __shared__ u32x4 sk[2][NP * 512], sv[2][NP * 512];
  __shared__ u32x4 raw[kAhead][8][NP][64];  // codes on their way, by wave
  const int npair = B * Hkv;
  // pairs fastest: with a multiple of eight pairs all tiles of a pair run on
  // one XCD and share its L2; the longest tiles first
  const int pair = blockIdx.x % npair, rest = blockIdx.x / npair, split = rest % nsplit;
  const int c0 = (ntile - 1 - rest / nsplit) * kTileCols;
  const int b = pair / Hkv, kvh = pair % Hkv;
  int len;
  const int n = new_tokens(lens, counts, b, T, cap, len);
  const int ncol = min(kTileCols, n * G - c0);
  if (ncol <= 0) return;
  const int p0 = len + c0 / G, p1 = len + (c0 + ncol - 1) / G;
  const int jlo = split * chunk, jhi = min(cap, jlo + chunk);
  if (!mask.any(p0, p1, jlo, jhi)) return;
  const int tid = threadIdx.x, lane = tid & 63, col = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // the wave's columns (past the last: the last one's again)
  const int w0 = min(c0 + wave * 32, c0 + ncol - 1), w1 = min(c0 + wave * 32 + 31, c0 + ncol - 1);
  const bool works = wave * 32 < ncol;
  const int q0 = len + w0 / G, q1 = len + w1 / G;
  int pos[2];
  bf16x8 qf[2][KQ];
#pragma unroll
  for (int i = 0; i < 2; i++) {
    const int c = min(w0 + 16 * i + col, w1), t = c / G;
    pos[i] = len + t;
    const uint16_t* qp = q + (((int64_t)b * Hkv * G + kvh * G + c % G) * T + t) * HD + 16 * g;
#pragma unroll
    for (int x = 0; x < KQ; x++) qf[i][x] = *reinterpret_cast<const bf16x8*>(qp + 64 * (x >> 1) + 8 * (x & 1));
  }
  const int64_t blk0 = (int64_t)pair * (cap / kBlk);
  const uint8_t *kp = kc + blk0 * (kBlk * HD), *vp = vc + blk0 * (kBlk * HD);
  // blocks bfirst .. bend - 1 of this split, those between the sinks and the
  // window left out
  const int bend = min(jhi - 1, p1) / kBlk + 1;
  const int bwin = mask.window ? max(0, p0 - mask.window + 1) / kBlk : 0;  // first block that the window reaches
  auto skip = [&](int x) __attribute__((always_inline)) { return x * kBlk >= mask.sinks && x < bwin ? bwin : x; };
  auto after = [&](int x) __attribute__((always_inline)) { return skip(x + 1); };
  const u32x4 zero = {0, 0, 0, 0};
  // a thread's 16 bytes of a block's codes: of keys and of values (128 dims),
  // or of one of them (64 dims: waves 0 to 3 keys, 4 to 7 values)
  constexpr bool kBoth = HD == 128;
  const bool keys = kBoth || wave < 4, values = kBoth || wave >= 4;
  const int at = kBoth ? tid : tid & 255;
  // a block's codes straight to the wave's place in LDS (past the end: the
  // last block's again, so that the loads in flight stay countable)
  auto fetch = [&](int slot, int xk, int xv) __attribute__((always_inline)) {
    if (keys) load_lds(kp + (int64_t)min(xk, bend - 1) * (kBlk * HD) + at * 16, raw[slot][wave][0]);
    if (values) load_lds(vp + (int64_t)min(xv, bend - 1) * (kBlk * HD) + at * 16, raw[slot][wave][NP - 1]);
  };
  auto stash = [&](u32x4* to, u32x4 w) __attribute__((always_inline)) {
    u32x4* d = to + (at >> 6) * 128 + lane;
    d[0] = __builtin_bit_cast(u32x4, fp8_bf16(w[0], w[1]));
    d[64] = __builtin_bit_cast(u32x4, fp8_bf16(w[2], w[3]));
  };
  auto stash_values = [&](u32x4* to, u32x4 w, uint64_t seen) __attribute__((always_inline)) {
    if (seen != ~0ull) {
#pragma unroll
      for (int e = 0; e < 4; e++) w[e] &= seen_bytes(seen, e, g);
    }
    stash(to, w);
  };
  f32x4 acc[ND][2] = {};
  f32x4 sc[4][2];   // scores of a block
  bf16x8 pf[2][2];  // its probabilities
  float m[2] = {-INFINITY, -INFINITY};
  f32x4 l[2] = {};  // row sums: the product of the probabilities with ones, four times
  // (two tiles by turns: a product waits for none of the three before it)
  auto scores = [&](const u32x4* k) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 4; i += 2)
#pragma unroll
      for (int x = 0; x < KQ; x++)
#pragma unroll
        for (int e = 0; e < 2; e++) {
          const bf16x8 kf = __builtin_bit_cast(bf16x8, k[((i + e) * KQ + x) * 64 + lane]);
#pragma unroll
          for (int y = 0; y < 2; y++)
            sc[i + e][y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[y][x], x == 0 ? f32x4{} : sc[i + e][y], 0, 0, 0);
        }
  };
  bf16x8 ones;  // over the values' scale, which the probabilities hold
  auto add_values = [&](const u32x4* v) __attribute__((always_inline)) {
#pragma unroll
    for (int x = 0; x < 2; x++)
#pragma unroll
      for (int y = 0; y < 2; y++) l[y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, pf[y][x], l[y], 0, 0, 0);
#pragma unroll
    for (int i = 0; i < ND; i += 2)
#pragma unroll
      for (int x = 0; x < 2; x++)
#pragma unroll
        for (int e = 0; e < 2; e++) {
          const bf16x8 vf = __builtin_bit_cast(bf16x8, v[((i + e) * 2 + x) * 64 + lane]);
#pragma unroll
          for (int y = 0; y < 2; y++) acc[i + e][y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[y][x], acc[i + e][y], 0, 0, 0);
        }
  };
  // Waits for the wave's LDS accesses and meets the others; the loads go on
  // (__syncthreads would wait for them).
  auto phase = [&]() __attribute__((always_inline)) {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };

  // a step works on block x[0], the ones after it are x[1], x[2], ..
  int x[kAhead + 3];
  x[0] = skip(jlo / kBlk);
#pragma unroll
  for (int i = 1; i < kAhead + 3; i++) x[i] = after(x[i - 1]);
  if (keys) {
    const u32x4* p = reinterpret_cast<const u32x4*>(kp + at * 16);
    stash(sk[0], p[(int64_t)x[0] * (kBlk * HD / 16)]);
    stash(sk[1], x[1] < bend ? p[(int64_t)x[1] * (kBlk * HD / 16)] : zero);
  }
  if (values) stash_values(sv[0], reinterpret_cast<const u32x4*>(vp + at * 16)[(int64_t)x[0] * (kBlk * HD / 16)], mask.seen(p0, p1, x[0] * kBlk));
#pragma unroll
  for (int i = 0; i < kAhead; i++) fetch(i, x[i + 2], x[i + 1]);
  float fk = ks[blk0 + x[0]] * sl2, fv = vs[blk0 + x[0]];
  __syncthreads();
  scores(sk[0]);
  __syncthreads();
  // Step t, phase one (the vector unit): the probabilities of x[0] from its
  // scores.  Phase two (the matrix unit): x[0]'s values, x[1]'s scores; then
  // the keys of x[2] and the values of x[1] are stored, at places that the
  // last wave has read a phase ago.
  int par = 0, slot = 0;
  if (wave >= 4) phase();
  while (x[0] < bend) {
    // the next block's scales, asked for before the phase's work, and its tokens that count
    const int64_t bn = blk0 + min(x[1], bend - 1);
    const float nk = ks[bn], nv = vs[bn];
    const uint64_t next_seen = mask.seen(p0, p1, x[1] * kBlk);
    __builtin_amdgcn_sched_barrier(0);
    if (works) {
      const int j0 = x[0] * kBlk;
      if (!mask.all(q0, q1, j0, j0 + kBlk)) {
        // NaN in a scale: the visible tokens' scores take it, and the others
        // are left out as ever
        const bool nan = fk != fk || fv != fv;
#pragma unroll
        for (int i = 0; i < 4; i++)
#pragma unroll
          for (int y = 0; y < 2; y++)
#pragma unroll
            for (int r = 0; r < 4; r++) {
              const bool sees = mask.sees(pos[y], mask.low(pos[y]), j0 + 16 * i + 4 * g + r);
              if (nan) sc[i][y][r] = __builtin_bit_cast(float, 0x7fc00000u);
              if (!sees) sc[i][y][r] = -INFINITY;
            }
        if (nan) fk = fv = 1.0f;
      }
      float mx[2];
#pragma unroll
      for (int y = 0; y < 2; y++) {
        float v = -INFINITY;
#pragma unroll
        for (int i = 0; i < 4; i++)
#pragma unroll
          for (int r = 0; r < 4; r++) v = fmaxf(v, sc[i][y][r]);
        mx[y] = v * fk;
      }
      // a column's reference moves only when a score passes it by 2^8
      if (__ballot(mx[0] > m[0] + 8.0f || mx[1] > m[1] + 8.0f)) {
#pragma unroll
        for (int y = 0; y < 2; y++) {
          float v = fmaxf(mx[y], __shfl_xor(mx[y], 16, 64));
          v = fmaxf(v, __shfl_xor(v, 32, 64));
          if (v > m[y] + 8.0f) {
            const float a = __builtin_amdgcn_exp2f(m[y] - v);
            l[y] *= a;
#pragma unroll
            for (int i = 0; i < ND; i++) acc[i][y] *= a;
            m[y] = v;
          }
        }
      }
      const float ev = log2_scale(fv);
      const __bf16 unscale = (__bf16)(fv == fv ? __builtin_amdgcn_rcpf(fv) : 1.0f);  // exact
      ones = bf16x8{unscale, unscale, unscale, unscale, unscale, unscale, unscale, unscale};
#pragma unroll
      for (int y = 0; y < 2; y++) {
        const float sub = ev - (m[y] == -INFINITY ? 0.f : m[y]);
#pragma unroll
        for (int i = 0; i < 4; i++) {
          float p[4];
#pragma unroll
          for (int r = 0; r < 4; r++) p[r] = __builtin_amdgcn_exp2f(fmaf(sc[i][y][r], fk, sub));
          const bf16x2 u = {(__bf16)p[0], (__bf16)p[1]}, w = {(__bf16)p[2], (__bf16)p[3]};
#pragma unroll
          for (int r = 0; r < 2; r++) {
            pf[y][i >> 1][(i & 1) * 4 + r] = u[r];
            pf[y][i >> 1][(i & 1) * 4 + 2 + r] = w[r];
          }
        }
      }
      // (kept here: the compiler would move the exponentials to their use)
#pragma unroll
      for (int y = 0; y < 2; y++)
#pragma unroll
        for (int e = 0; e < 2; e++) asm volatile("" : "+v"(pf[y][e]));
    }
    __builtin_amdgcn_sched_barrier(0);
    fk = nk * sl2;
    fv = nv;
    phase();
    __builtin_amdgcn_s_waitcnt(vmcnt_imm((kAhead - 1) * NP));
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    u32x4 kr = zero, vr = zero;
    if (keys) kr = raw[slot][wave][0][lane];
    if (values) vr = raw[slot][wave][NP - 1][lane];
    __builtin_amdgcn_sched_barrier(0);
    if (works) {
      add_values(sv[par]);
      scores(sk[par ^ 1]);
      // operands read kReads ahead, two products to a read
      __builtin_amdgcn_sched_group_barrier(0x100, kReads, 0);
#pragma unroll
      for (int i = 0; i < 2 + 2 * ND + 4 * KQ; i++) {
        __builtin_amdgcn_sched_group_barrier(0x008, 2, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    if (keys) stash(sk[par], kr);
    if (values) stash_values(sv[par ^ 1], vr, next_seen);
    __builtin_amdgcn_sched_barrier(0);
    phase();
    __builtin_amdgcn_sched_barrier(0);
    fetch(slot, x[kAhead + 2], x[kAhead + 1]);  // into what this step has read
    slot = slot == kAhead - 1 ? 0 : slot + 1;
    par ^= 1;
#pragma unroll
    for (int i = 0; i < kAhead + 2; i++) x[i] = x[i + 1];
    x[kAhead + 2] = after(x[kAhead + 1]);
  }
  if (wave < 4) phase();
  __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));  // no load to LDS outlives the workgroup
  if (!works) return;
  const bool only = mask.only(p0, p1, jlo, jhi);
#pragma unroll
  for (int y = 0; y < 2; y++) {
    const int c = w0 + 16 * y + col;
    const float L = l[y][0];
    if (c > w1) continue;
    if (only) {
      const float inv = 1.0f / L;
      uint16_t* op = out + ((int64_t)b * T + c / G) * ((int64_t)Hkv * G * HD) + (kvh * G + c % G) * HD + 4 * g;
#pragma unroll
      for (int i = 0; i < ND; i++) {
        mx_u32x2 w;
#pragma unroll
        for (int e = 0; e < 2; e++)
          w[e] = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)(acc[i][y][2 * e] * inv), (__bf16)(acc[i][y][2 * e + 1] * inv)});
        *reinterpret_cast<mx_u32x2*>(op + 16 * i) = w;
      }
    } else {
      const int64_t row = (int64_t)pair * T * G + c;
#pragma unroll
      for (int i = 0; i < ND; i++) *reinterpret_cast<f32x4*>(part_o + (row * nsplit + split) * HD + 16 * i + 4 * g) = acc[i][y];
      if (g == 0) part_ml[row * nsplit + split] = make_float2(m[y], L);
    }
  }
}

int64_t tiles_of(int64_t cols) { return (cols + kTileCols - 1) / kTileCols; }

// The form and the tokens in a split of the length: by the columns, heads and
// cache of one sequence, so that a query's result does not depend on the others.
bool few(int64_t cols, int Hkv, int hd, int cap) {
  return cols <= 32 || (cols <= kFewCols && (cols + 15) / 16 * Hkv * (cap / kBlk) * (hd / 64) <= kFewBlocks);
}
// Whole blocks, so that n of them hold cap tokens.
int64_t round_up(int64_t cap, int64_t n) { return ((cap + n - 1) / n + kBlk - 1) / kBlk * kBlk; }
int chunk_of(int64_t cols, int Hkv, int hd, int cap) {
  if (few(cols, Hkv, hd, cap) && cap <= kOneBytes / (2 * hd)) return cap;
  const int64_t tokens = kSplitBytes / (2 * hd);
  // a few queries: splits of `tokens`, longer ones where that were too many;
  // more queries: as many splits as have an eighth more than that
  if (cols <= 32) return (int)std::max(tokens, round_up(cap, kMaxSplits));
  int64_t n;
  if (few(cols, Hkv, hd, cap)) {
    n = std::min<int64_t>(cap / (tokens + tokens / 8), kMaxSplits);
  } else {
    const int64_t groups = tiles_of(cols) * Hkv;
    n = groups >= 128 ? 1 : std::max(std::min<int64_t>(128 / groups, cap / kShortSplit), std::min<int64_t>(256 / groups, cap / kLongSplit));
    n = std::min<int64_t>(n, kMaxPromptSplits);
  }
  return (int)round_up(cap, std::max<int64_t>(n, 1));
}
int splits_of(int chunk, int cap) { return (cap + chunk - 1) / chunk; }

}  // namespace

int64_t kv8_workspace_bytes(int B, int Hq, int Hkv, int T, int hd, int cap) {
  const int64_t nsplit = splits_of(chunk_of((int64_t)T * (Hq / Hkv), Hkv, hd, cap), cap);
  return nsplit > 1 ? (int64_t)B * Hq * T * nsplit * (hd + 2) * 4 : 0;
}

int64_t kv8_workgroups(int B, int Hq, int Hkv, int T, int hd, int cap) {
  const int64_t cols = (int64_t)T * (Hq / Hkv);
  return few(cols, Hkv, hd, cap) ? 1 : tiles_of(cols) * splits_of(chunk_of(cols, Hkv, hd, cap), cap) * B * Hkv;
}

hipError_t launch_kv8_append(const uint16_t* k, const uint16_t* v, int B, int Hkv, int T, int hd, int cap,
                             const int32_t* lens, const int32_t* counts, uint8_t* kc, float* ks, uint8_t* vc, float* vs,
                             hipStream_t s) {
  const dim3 grid((std::min(T, cap) + kBlk - 2) / kBlk + 1, Hkv, 2 * B);
  if (hd == 64) kv8_append_kernel<64><<<grid, 256, 0, s>>>(k, v, Hkv, T, cap, lens, counts, kc, ks, vc, vs);
  else kv8_append_kernel<128><<<grid, 256, 0, s>>>(k, v, Hkv, T, cap, lens, counts, kc, ks, vc, vs);
  return hipGetLastError();
}

hipError_t launch_attention_kv8(const uint16_t* q, int B, int Hq, int Hkv, int T, int hd, int cap, const int32_t* lens,
                                const int32_t* counts, const uint8_t* kc, const float* ks, const uint8_t* vc,
                                const float* vs, int window, int sinks, void* ws, uint16_t* out, hipStream_t s) {
  const int G = Hq / Hkv;
  const int64_t cols = (int64_t)T * G;
  const int chunk = chunk_of(cols, Hkv, hd, cap), nsplit = splits_of(chunk, cap);
  const Mask mask{window, sinks};
  const float sl2 = (float)(1.4426950408889634 / sqrt((double)hd));
  float* po = (float*)ws;
  float2* pml = nsplit > 1 ? (float2*)(po + (int64_t)B * Hq * T * nsplit * hd) : nullptr;
  auto go = [&](auto h) {
    constexpr int HD = decltype(h)::value;
    const dim3 join((unsigned)cols, Hkv, B);
    if (few(cols, Hkv, hd, cap)) {
      // exact quotients of numbers below 2^16: x / n = x (2^32 / n + 1) / 2^32
      const uint32_t hinv = (uint32_t)((1ull << 32) / Hkv + 1), ginv = (uint32_t)((1ull << 32) / G + 1);
      const dim3 grid(nsplit, (unsigned)((cols + 15) / 16) * Hkv, B);
      auto split = [&](auto once) {
        attn_kv8_split_kernel<HD, decltype(once)::value><<<grid, kSplitWaves * 64, 0, s>>>(
            q, kc, ks, vc, vs, lens, counts, Hkv, hinv, G, ginv, T, cap, nsplit, chunk, mask, sl2, po, pml, out);
      };
      if (cols > 16) split(std::false_type{});
      else split(std::true_type{});
      if (nsplit > 1)
        attn_kv8_join_kernel<HD, 16><<<join, 64, 0, s>>>(po, pml, lens, counts, Hkv, G, T, cap, nsplit, chunk, mask, out);
    } else {
      const int ntile = (int)tiles_of(cols);
      attn_kv8_prompt_kernel<HD><<<(unsigned)((int64_t)ntile * nsplit * B * Hkv), 512, 0, s>>>(
          q, kc, ks, vc, vs, lens, counts, B, Hkv, G, T, cap, ntile, nsplit, chunk, mask, sl2, po, pml, out);
      if (nsplit > 1)
        attn_kv8_join_kernel<HD, kTileCols><<<join, 64, 0, s>>>(po, pml, lens, counts, Hkv, G, T, cap, nsplit, chunk, mask, out);
    }
  };
  if (hd == 64) go(std::integral_constant<int, 64>{});
  else go(std::integral_constant<int, 128>{});
  return hipGetLastError();
}

}  // namespace lmgc
