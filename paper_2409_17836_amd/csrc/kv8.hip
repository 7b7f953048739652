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
  if (len < 0 || len >= cap) return 0;
  int n = min(T, cap - len);
  if (counts) n = min(n, counts[b]);
  return n;
}

// ------------------------------------------------------------------ append
// A workgroup per (block of the cache that new tokens may fall into, key/value
// head, sequence x {key, value}).
template <int HD>
__global__ __launch_bounds__(256) void kv8_append_kernel(const uint16_t* __restrict__ kin, const uint16_t* __restrict__ vin,
                                                         int Hkv, int T, int cap, const int32_t* __restrict__ lens,
                                                         const int32_t* __restrict__ counts, uint8_t* __restrict__ kc,
                                                         float* __restrict__ ks, uint8_t* __restrict__ vc,
                                                         float* __restrict__ vs) {
  __shared__ uint32_t part[4];
  const int b = blockIdx.z >> 1, is_v = blockIdx.z & 1, h = blockIdx.y;
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
  uint32_t a = 0;
  for (int i = threadIdx.x; i < (hi - lo) * HD; i += 256) a = max(a, abs_bits(load1(src + (int64_t)lo * HD + i)));
  for (int o = 32; o; o >>= 1) a = max(a, (uint32_t)__shfl_xor((int)a, o, 64));
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = a;
  __syncthreads();
  a = max(max(part[0], part[1]), max(part[2], part[3]));
  const float s_old = lo ? *scale : 0.f;
  float s_new = a >= 0x7f800000u ? __builtin_bit_cast(float, 0x7fc00000u)
                                 : mx_scale(max(mx_scale_byte<LMGC_MX_FP8>(a), kMinScale));
  const bool nan = s_new != s_new || s_old != s_old;
  const float s = nan ? __builtin_bit_cast(float, 0x7fc00000u) : fmaxf(s_old, s_new);
  const float inv = nan ? 1.0f : 1.0f / s, grow = nan ? 1.0f : s_old * inv;
  __syncthreads();  // every thread has read the old scale
  if (threadIdx.x == 0) *scale = s;
  for (int i = threadIdx.x; i < kBlk * HD; i += 256) {
    const int t = i / HD, d = i - t * HD;
    uint8_t* p = codes + (is_v ? value_at(t, d) : key_at(t, d, HD));
    float v;
    if (t >= lo && t < hi) {
      v = load1(src + (int64_t)t * HD + d) * inv;
      if (nan) v = 0.f;
    } else if (lo == 0) {
      v = 0.f;  // a new block is cleared behind its tokens
    } else {
      if (t >= hi || grow == 1.0f) continue;
      v = __builtin_amdgcn_cvt_f32_fp8((int)*p, 0) * grow;
    }
    *p = (uint8_t)__builtin_amdgcn_cvt_pk_fp8_f32(v, v, 0, false);
  }
}

// --------------------------------------------------------------- attention
// Keys that a query at position pos sees: j <= pos and, with a window, j >
// pos - window or j < sinks.
struct Mask {
  int window, sinks;
  __device__ inline bool sees(int pos, int j) const {
    return j <= pos && (window == 0 || j > pos - window || j < sinks);
  }
  // whether any query at positions p0 .. p1 may see a key of [j0, j1)
  __device__ inline bool any(int p0, int p1, int j0, int j1) const {
    return j0 <= p1 && (window == 0 || j1 - 1 > p0 - window || j0 < sinks);
  }
  // whether every query at positions p0 .. p1 sees every key of [j0, j1)
  __device__ inline bool all(int p0, int p1, int j0, int j1) const {
    return j1 - 1 <= p0 && (window == 0 || j0 > p1 - window || j1 <= sinks);
  }
};

__device__ inline bf16x8 fp8_bf16(uint32_t w0, uint32_t w1) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, 1.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, 1.0f, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, 1.0f, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, 1.0f, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

constexpr int kChunk = 256;  // tokens of a split: one block for each of four waves

// Column c = t G + g of a (sequence, key/value head): query head kvh G + g of
// new token t.
//
// Grid: (splits x column tiles, Hkv, B); a workgroup computes 16 columns over
// kChunk tokens, wave w over its block w.  S^T = K Q^T: lane (col, g) holds
// the scores of its column and tokens 16 i + 4 g + r.
template <int HD>
__global__ __launch_bounds__(256) void attn_kv8_split_kernel(
    const uint16_t* __restrict__ q, const uint8_t* __restrict__ kc, const float* __restrict__ ks,
    const uint8_t* __restrict__ vc, const float* __restrict__ vs, const int32_t* __restrict__ lens,
    const int32_t* __restrict__ counts, int Hkv, int G, int T, int cap, int nsplit, Mask mask, float sl2,
    float* __restrict__ part_o, float2* __restrict__ part_ml, uint16_t* __restrict__ out) {
  constexpr int NC = HD / 64, ND = HD / 16;
  __shared__ float so[4][16][HD + 4];
  __shared__ float sm[4][16], sl[4][16];
  const int split = blockIdx.x % nsplit, c0 = blockIdx.x / nsplit * 16, kvh = blockIdx.y, b = blockIdx.z;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, col = lane & 15, g = lane >> 4;
  int len;
  const int n = new_tokens(lens, counts, b, T, cap, len);
  const int ncol = min(16, n * G - c0);
  if (ncol <= 0) return;
  const int p0 = len + c0 / G, p1 = len + (c0 + ncol - 1) / G;  // positions of the tile's queries
  const int j0 = split * kChunk + wave * kBlk;
  if (!mask.any(p0, p1, split * kChunk, split * kChunk + kChunk)) return;
  const int c = c0 + min(col, ncol - 1), t = c / G, pos = len + t;
  const int64_t hb = (int64_t)b * Hkv + kvh, nblk = cap / kBlk;

  float m = -INFINITY, l = 0.f;
  f32x4 o[ND] = {};
  if (j0 < cap && mask.any(p0, p1, j0, j0 + kBlk)) {
    const uint16_t* qp = q + (((int64_t)b * Hkv * G + kvh * G + c % G) * T + t) * HD;
    const int64_t blk = hb * nblk + j0 / kBlk;
    const u32x4* kp = reinterpret_cast<const u32x4*>(kc + blk * (kBlk * HD)) + lane;
    const u32x4* vp = reinterpret_cast<const u32x4*>(vc + blk * (kBlk * HD)) + lane;
    u32x4 kr[4][NC], vr[ND];
#pragma unroll
    for (int i = 0; i < 4; i++)
#pragma unroll
      for (int x = 0; x < NC; x++) kr[i][x] = kp[(i * NC + x) * 64];
#pragma unroll
    for (int i = 0; i < ND; i++) vr[i] = vp[i * 64];
    const float sk = ks[blk] * sl2, sv = vs[blk];
    f32x4 s[4] = {};
#pragma unroll
    for (int x = 0; x < NC; x++)
#pragma unroll
      for (int y = 0; y < 2; y++) {
        const bf16x8 qf = *reinterpret_cast<const bf16x8*>(qp + 64 * x + 16 * g + 8 * y);
#pragma unroll
        for (int i = 0; i < 4; i++)
          s[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fp8_bf16(kr[i][x][2 * y], kr[i][x][2 * y + 1]), qf, s[i], 0, 0, 0);
      }
    const bool whole = mask.all(p0, p1, j0, j0 + kBlk);
    bool see[4][4];
#pragma unroll
    for (int i = 0; i < 4; i++)
#pragma unroll
      for (int r = 0; r < 4; r++) {
        see[i][r] = whole || mask.sees(pos, j0 + 16 * i + 4 * g + r);
        s[i][r] = see[i][r] ? s[i][r] * sk : -INFINITY;
        m = fmaxf(m, s[i][r]);
        // (fmaxf drops a NaN; it comes back through the exponential)
      }
    m = fmaxf(m, __shfl_xor(m, 16, 64));
    m = fmaxf(m, __shfl_xor(m, 32, 64));
    const float ref = m == -INFINITY ? 0.f : m;
    bf16x8 pf[2];
#pragma unroll
    for (int i = 0; i < 4; i++)
#pragma unroll
      for (int r = 0; r < 4; r++) {
        // rounded to bf16 for the second product; the sum is of the rounded values
        const __bf16 p = (__bf16)__builtin_amdgcn_exp2f(s[i][r] - ref);
        l += (float)p;
        pf[i >> 1][(i & 1) * 4 + r] = see[i][r] ? (__bf16)((float)p * sv) : (__bf16)0.f;
      }
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
#pragma unroll
    for (int i = 0; i < ND; i++)
#pragma unroll
      for (int y = 0; y < 2; y++)
        o[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fp8_bf16(vr[i][2 * y], vr[i][2 * y + 1]), pf[y], o[i], 0, 0, 0);
  }
  if (g == 0) {
    sm[wave][col] = m;
    sl[wave][col] = l;
  }
#pragma unroll
  for (int i = 0; i < ND; i++) *reinterpret_cast<f32x4*>(&so[wave][col][16 * i + 4 * g]) = o[i];
  __syncthreads();
  // whether this chunk is all that the tile's queries see
  bool only = true;
  for (int x = 0; x < nsplit; x++)
    if (x != split && mask.any(p0, p1, x * kChunk, x * kChunk + kChunk)) only = false;
  for (int i = tid; i < ncol * HD; i += 256) {
    const int cc = i / HD, d = i - cc * HD;
    const float M = fmaxf(fmaxf(sm[0][cc], sm[1][cc]), fmaxf(sm[2][cc], sm[3][cc]));
    float acc = 0.f, L = 0.f;
#pragma unroll
    for (int w = 0; w < 4; w++) {
      const float a = sm[w][cc] == -INFINITY && sl[w][cc] == 0.f ? 0.f : __builtin_amdgcn_exp2f(sm[w][cc] - M);
      acc += a * so[w][cc][d];
      L += a * sl[w][cc];
    }
    const int64_t row = (hb * T) * G + c0 + cc;
    if (only) {
      const int ct = (c0 + cc) / G, hq = kvh * G + (c0 + cc) % G;
      out[((int64_t)b * T + ct) * (Hkv * G * HD) + hq * HD + d] = f32_to_bf16(acc / L);
    } else {
      part_o[(row * nsplit + split) * HD + d] = acc;
      if (d == 0) part_ml[row * nsplit + split] = make_float2(M, L);
    }
  }
}

// Joins the splits of a column: a wave per column, HD / 64 dims to a lane.
template <int HD>
__global__ __launch_bounds__(64) void attn_kv8_join_kernel(const float* __restrict__ part_o, const float2* __restrict__ part_ml,
                                                           const int32_t* __restrict__ lens, const int32_t* __restrict__ counts,
                                                           int Hkv, int G, int T, int cap, int nsplit, Mask mask,
                                                           uint16_t* __restrict__ out) {
  const int c = blockIdx.x, kvh = blockIdx.y, b = blockIdx.z, lane = threadIdx.x;
  int len;
  const int n = new_tokens(lens, counts, b, T, cap, len);
  if (c >= n * G) return;
  const int c0 = c & ~15, ncol = min(16, n * G - c0), p0 = len + c0 / G, p1 = len + (c0 + ncol - 1) / G;
  const int64_t hb = (int64_t)b * Hkv + kvh, row = hb * T * G + c;
  float M = -INFINITY;
  int used = 0;
  for (int x = 0; x < nsplit; x++)
    if (mask.any(p0, p1, x * kChunk, x * kChunk + kChunk)) {
      M = fmaxf(M, part_ml[row * nsplit + x].x);
      used++;
    }
  if (used <= 1) return;  // written by the only split
  float acc[HD / 64] = {}, L = 0.f;
  for (int x = 0; x < nsplit; x++) {
    if (!mask.any(p0, p1, x * kChunk, x * kChunk + kChunk)) continue;
    const float2 ml = part_ml[row * nsplit + x];
    const float a = ml.x == -INFINITY && ml.y == 0.f ? 0.f : __builtin_amdgcn_exp2f(ml.x - M);
    L += a * ml.y;
#pragma unroll
    for (int i = 0; i < HD / 64; i++) acc[i] += a * part_o[(row * nsplit + x) * HD + lane + 64 * i];
  }
  const int t = c / G, hq = kvh * G + c % G;
#pragma unroll
  for (int i = 0; i < HD / 64; i++)
    out[((int64_t)b * T + t) * (Hkv * G * HD) + hq * HD + lane + 64 * i] = f32_to_bf16(acc[i] / L);
}

// Prompts: a workgroup of eight waves takes 256 columns of one (sequence,
// key/value head), each wave 32, and walks the cache in steps of 8 KB of keys
// and of values (64 tokens of 128 dims, 128 of 64).  Each thread fetches 16
// bytes of codes of both a step ahead, converts them and stores them as bf16
// in the order of the matrix operands, so a conversion serves 256 columns and
// the products read LDS a lane's 16 bytes in a row.  Keys run one step ahead
// of values: the scores of step s + 1 are multiplied while the exponentials
// of step s are taken.  The block scales cost nothing per score: the keys'
// goes into the exponent's factor, the values' (a power of two) into its
// summand, from which the row sums are freed once per block.
template <int HD>
__global__ __launch_bounds__(512, 2) void attn_kv8_prompt_kernel(
    const uint16_t* __restrict__ q, const uint8_t* __restrict__ kc, const float* __restrict__ ks,
    const uint8_t* __restrict__ vc, const float* __restrict__ vs, const int32_t* __restrict__ lens,
    const int32_t* __restrict__ counts, int B, int Hkv, int G, int T, int cap, int ntile, Mask mask, float sl2,
    uint16_t* __restrict__ out) {
  constexpr int NC = HD / 64, ND = HD / 16, NB = 128 / HD, TB = NB * kBlk;  // blocks and tokens of a step
  constexpr int KQ = HD / 32;                                               // 32-dim steps of a score
  __shared__ u32x4 sk[2][1024], sv[2][1024];  // 16 KB each
  const int npair = B * Hkv;
  // pairs fastest: with a multiple of eight pairs all tiles of a pair run on
  // one XCD and share its L2; the longest tiles first
  const int pair = blockIdx.x % npair, c0 = (ntile - 1 - (int)blockIdx.x / npair) * 256;
  const int b = pair / Hkv, kvh = pair % Hkv;
  int len;
  const int n = new_tokens(lens, counts, b, T, cap, len);
  const int ncol = min(256, n * G - c0);
  if (ncol <= 0) return;
  const int tid = threadIdx.x, lane = tid & 63, col = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int p0 = len + c0 / G, p1 = len + (c0 + ncol - 1) / G;
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
  const int nsteps = p1 / TB + 1;
  const int64_t bytes = (int64_t)cap * HD;
  const int w_step = mask.window ? max(0, p0 - mask.window + 1) / TB : 0;  // first step that the window reaches
  auto after = [&](int s) __attribute__((always_inline)) {
    const int x = s + 1;
    return x * TB >= mask.sinks && x < w_step ? w_step : x;
  };
  const u32x4 zero = {0, 0, 0, 0};
  auto fetch = [&](const uint8_t* p, int s) __attribute__((always_inline)) {
    const int64_t off = (int64_t)s * 8192 + tid * 16;
    return s < nsteps && off < bytes ? *reinterpret_cast<const u32x4*>(p + off) : zero;
  };
  auto stash = [&](u32x4* to, u32x4 w) __attribute__((always_inline)) {
    u32x4* at = to + (tid >> 6) * 128 + lane;
    at[0] = __builtin_bit_cast(u32x4, fp8_bf16(w[0], w[1]));
    at[64] = __builtin_bit_cast(u32x4, fp8_bf16(w[2], w[3]));
  };
  // scores of step s: token tile i of the step, column tile x
  f32x4 sc[NB * 4][2], sn[NB * 4][2];
  auto scores = [&](f32x4(&o)[NB * 4][2], const u32x4* k) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < NB * 4; i++)
#pragma unroll
      for (int x = 0; x < KQ; x++) {
        const bf16x8 kf = __builtin_bit_cast(bf16x8, k[(i * KQ + x) * 64 + lane]);
#pragma unroll
        for (int y = 0; y < 2; y++)
          o[i][y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[y][x], x == 0 ? f32x4{} : o[i][y], 0, 0, 0);
      }
  };
  f32x4 acc[ND][2] = {};
  float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};

  int s = mask.window && mask.sinks == 0 ? w_step : 0;
  int s1 = after(s);
  u32x4 kr = fetch(kp, s), vr = fetch(vp, s);
  stash(sk[0], kr);
  stash(sv[0], vr);
  kr = fetch(kp, s1);
  vr = fetch(vp, s1);
  __syncthreads();
  scores(sc, sk[0]);
  stash(sk[1], kr);
  kr = fetch(kp, after(s1));
  __syncthreads();
  for (int it = 0; s < nsteps; it++) {
    // here: sc the scores of s; sk[(it + 1) & 1] the keys of s1, kr the next
    // ones; sv[it & 1] the values of s, vr those of s1
    const int s2 = after(s1);
    stash(sv[(it + 1) & 1], vr);
    vr = fetch(vp, s2);
    if (works) {
      scores(sn, sk[(it + 1) & 1]);
#pragma unroll
      for (int h = 0; h < NB; h++) {
        const int j0 = s * TB + h * kBlk;
        if (j0 >= cap || !mask.any(q0, q1, j0, j0 + kBlk)) continue;
        const float fk = ks[blk0 + j0 / kBlk] * sl2, fv = vs[blk0 + j0 / kBlk];
        // log2 of the values' scale (a power of two; NaN stays NaN)
        const float ev = fv == fv ? (float)((int)(__builtin_bit_cast(uint32_t, fv) >> 23) - 127) : fv;
        const float unscale = fv == fv ? 1.0f / fv : 1.0f;
        const bool whole = mask.all(q0, q1, j0, j0 + kBlk);
        bf16x8 pf[2][2];
#pragma unroll
        for (int y = 0; y < 2; y++) {
          float mx = -INFINITY;
          if (!whole) {
#pragma unroll
            for (int i = 0; i < 4; i++)
#pragma unroll
              for (int r = 0; r < 4; r++)
                if (!mask.sees(pos[y], j0 + 16 * i + 4 * g + r)) sc[4 * h + i][y][r] = -INFINITY;
          }
#pragma unroll
          for (int i = 0; i < 4; i++)
#pragma unroll
            for (int r = 0; r < 4; r++) mx = fmaxf(mx, sc[4 * h + i][y][r]);
          mx *= fk;
          // a column's reference moves only when a score passes it by 2^8
          if (__ballot(mx > m[y] + 8.0f)) {
            mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
            mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
            if (mx > m[y] + 8.0f) {
              const float a = __builtin_amdgcn_exp2f(m[y] - mx);
              l[y] *= a;
#pragma unroll
              for (int i = 0; i < ND; i++) acc[i][y] *= a;
              m[y] = mx;
            }
          }
          const float sub = ev - (m[y] == -INFINITY ? 0.f : m[y]);
          float sum = 0.f;
#pragma unroll
          for (int i = 0; i < 4; i++) {
            float p[4];
#pragma unroll
            for (int r = 0; r < 4; r++) {
              p[r] = __builtin_amdgcn_exp2f(fmaf(sc[4 * h + i][y][r], fk, sub));
              if (!whole && sc[4 * h + i][y][r] == -INFINITY) p[r] = 0.f;
            }
            const bf16x2 a = {(__bf16)p[0], (__bf16)p[1]}, c = {(__bf16)p[2], (__bf16)p[3]}, one = {(__bf16)1.0f, (__bf16)1.0f};
            sum = __builtin_amdgcn_fdot2_f32_bf16(a, one, sum, false);
            sum = __builtin_amdgcn_fdot2_f32_bf16(c, one, sum, false);
#pragma unroll
            for (int r = 0; r < 2; r++) {
              pf[y][i >> 1][(i & 1) * 4 + r] = a[r];
              pf[y][i >> 1][(i & 1) * 4 + 2 + r] = c[r];
            }
          }
          l[y] = fmaf(sum, unscale, l[y]);
        }
#pragma unroll
        for (int i = 0; i < ND; i++)
#pragma unroll
          for (int x = 0; x < 2; x++) {
            const bf16x8 vf = __builtin_bit_cast(bf16x8, sv[it & 1][((h * ND + i) * 2 + x) * 64 + lane]);
#pragma unroll
            for (int y = 0; y < 2; y++) acc[i][y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[y][x], acc[i][y], 0, 0, 0);
          }
      }
#pragma unroll
      for (int i = 0; i < NB * 4; i++)
#pragma unroll
        for (int y = 0; y < 2; y++) sc[i][y] = sn[i][y];
    }
    stash(sk[it & 1], kr);
    kr = fetch(kp, after(s2));
    __syncthreads();
    s = s1;
    s1 = s2;
  }
  if (!works) return;
#pragma unroll
  for (int y = 0; y < 2; y++) {
    const int c = w0 + 16 * y + col;
    float L = l[y];
    L += __shfl_xor(L, 16, 64);
    L += __shfl_xor(L, 32, 64);
    if (c > w1) continue;
    const float inv = 1.0f / L;
    uint16_t* op = out + ((int64_t)b * T + c / G) * ((int64_t)Hkv * G * HD) + (kvh * G + c % G) * HD + 4 * g;
#pragma unroll
    for (int i = 0; i < ND; i++) {
      mx_u32x2 w;
#pragma unroll
      for (int e = 0; e < 2; e++)
        w[e] = (uint32_t)f32_to_bf16(acc[i][y][2 * e] * inv) | ((uint32_t)f32_to_bf16(acc[i][y][2 * e + 1] * inv) << 16);
      *reinterpret_cast<mx_u32x2*>(op + 16 * i) = w;
    }
  }
}

// Columns up to which a (sequence, key/value head) takes the split form.
constexpr int kSplitCols = 64;

}  // namespace

int64_t kv8_workspace_bytes(int B, int Hq, int Hkv, int T, int hd, int cap) {
  const int64_t nsplit = (cap + kChunk - 1) / kChunk;
  if (nsplit <= 1 || (int64_t)T * (Hq / Hkv) > kSplitCols) return 0;
  return (int64_t)B * Hq * T * nsplit * (hd + 2) * 4;
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
  const int G = Hq / Hkv, nsplit = (cap + kChunk - 1) / kChunk, ntile = (T * G + 15) / 16;
  const Mask mask{window, sinks};
  const float sl2 = (float)(1.4426950408889634 / sqrt((double)hd));
  float* po = (float*)ws;
  float2* pml = (float2*)(po + (int64_t)B * Hq * T * nsplit * hd);
  auto go = [&](auto h) {
    constexpr int HD = decltype(h)::value;
    if ((int64_t)T * G > kSplitCols) {
      const int tiles = (int)(((int64_t)T * G + 255) / 256);
      attn_kv8_prompt_kernel<HD><<<dim3((unsigned)tiles * B * Hkv), 512, 0, s>>>(q, kc, ks, vc, vs, lens, counts, B, Hkv, G, T,
                                                                               cap, tiles, mask, sl2, out);
      return;
    }
    attn_kv8_split_kernel<HD><<<dim3(nsplit * ntile, Hkv, B), 256, 0, s>>>(q, kc, ks, vc, vs, lens, counts, Hkv, G, T, cap,
                                                                           nsplit, mask, sl2, po, pml, out);
    if (nsplit > 1)
      attn_kv8_join_kernel<HD><<<dim3(T * G, Hkv, B), 64, 0, s>>>(po, pml, lens, counts, Hkv, G, T, cap, nsplit, mask, out);
  };
  if (hd == 64) go(std::integral_constant<int, 64>{});
  else go(std::integral_constant<int, 128>{});
  return hipGetLastError();
}

}  // namespace lmgc
