// Product of microscaled operands: C[M, N] = A[M, K] * B[N, K]^T (+ add) with
// A in e4m3 or e2m1 (rows), B in e2m1 (blocks), on the scaled matrix
// instruction of 16 x 16 x 128, which multiplies each lane's 32 products by
// both blocks' scales and accumulates in float32.
//
// Every output element is one chain of these instructions over rising k,
// whatever M, N and the tile, so a row's result depends on that row of A and
// on B alone.
#include <algorithm>

#include "mx.h"

namespace lmgc {
namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// Lane l = r + 16 g of the instruction: e2m1 operands: columns 32 g .. + 31
// of row r; e4m3 operands: columns 16 g .. + 15 and 64 + 16 g .. + 15.  In
// both the lane gives the scale of columns 32 g .. + 31.
template <int FMT>
__device__ inline i32x8 load_a(const uint8_t* row, int k, int g) {
  i32x8 a = {};
  if constexpr (FMT == LMGC_MX_FP8) {
    const i32x4 lo = *reinterpret_cast<const i32x4*>(row + (int64_t)k * 128 + 16 * g);
    const i32x4 hi = *reinterpret_cast<const i32x4*>(row + (int64_t)k * 128 + 64 + 16 * g);
#pragma unroll
    for (int i = 0; i < 4; i++) {
      a[i] = lo[i];
      a[4 + i] = hi[i];
    }
  } else {
    const i32x4 lo = *reinterpret_cast<const i32x4*>(row + (int64_t)k * 64 + 16 * g);
#pragma unroll
    for (int i = 0; i < 4; i++) a[i] = lo[i];
  }
  return a;
}

template <int FMT>
__device__ inline f32x4 mma(const i32x8& a, const i32x4& b4, f32x4 c, uint32_t sa, uint32_t sb) {
  constexpr int cbsz = FMT == LMGC_MX_FP8 ? 0 : 4;
  const i32x8 b = {b4[0], b4[1], b4[2], b4[3], 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, cbsz, 4, 0, (int)sa, 0, (int)sb);
}

// A wave per 32 x 32 outputs, operands straight from memory.
template <int FMT>
__global__ __launch_bounds__(64) void gemm_mx_kernel(const uint8_t* __restrict__ A, const uint8_t* __restrict__ As,
                                                     const uint8_t* __restrict__ B, const uint8_t* __restrict__ Bs,
                                                     int M, int N, int K, const float* add, void* out, int bf16) {
  const int lane = threadIdx.x, r = lane & 15, g = lane >> 4;
  const int nk = (int)(mx_cols(K) / 128), ns = (int)mx_row_scales(K);
  const int64_t lda = FMT == LMGC_MX_FP8 ? (int64_t)nk * 128 : (int64_t)nk * 64;
  const int64_t m0 = (int64_t)blockIdx.y * 32;
  const int n0 = blockIdx.x * 32, groups = (N + 15) / 16;
  const uint8_t *pa[2], *psa[2], *pb[2], *psb[2];
#pragma unroll
  for (int i = 0; i < 2; i++) {
    const int64_t m = min<int64_t>(m0 + 16 * i + r, M - 1);
    pa[i] = A + m * lda;
    psa[i] = As + m * ns + 4 * g;
    const int64_t grp = min(n0 / 16 + i, groups - 1);
    pb[i] = B + grp * nk * 1024 + lane * 16;
    psb[i] = Bs + grp * (ns / 16) * 256 + lane * 4;
  }
  f32x4 acc[2][2] = {};
  for (int k = 0; k < nk; k++) {
    i32x8 a[2];
    i32x4 b[2];
    uint32_t sa[2], sb[2];
#pragma unroll
    for (int i = 0; i < 2; i++) {
      a[i] = load_a<FMT>(pa[i], k, g);
      b[i] = *reinterpret_cast<const i32x4*>(pb[i] + (int64_t)k * 1024);
      sa[i] = *reinterpret_cast<const uint32_t*>(psa[i] + (k >> 2) * 16) >> (8 * (k & 3));
      sb[i] = *reinterpret_cast<const uint32_t*>(psb[i] + (int64_t)(k >> 2) * 256) >> (8 * (k & 3));
    }
#pragma unroll
    for (int i = 0; i < 2; i++)
#pragma unroll
      for (int j = 0; j < 2; j++) acc[i][j] = mma<FMT>(a[i], b[j], acc[i][j], sa[i], sb[j]);
  }
#pragma unroll
  for (int i = 0; i < 2; i++)
#pragma unroll
    for (int j = 0; j < 2; j++)
#pragma unroll
      for (int e = 0; e < 4; e++) {
        const int64_t m = m0 + 16 * i + 4 * g + e;
        const int n = n0 + 16 * j + r;
        if (m >= M || n >= N) continue;
        float v = acc[i][j][e];
        if (add) v += add[m * N + n];
        if (bf16) ((uint16_t*)out)[m * N + n] = f32_to_bf16(v);
        else ((float*)out)[m * N + n] = v;
      }
}

}  // namespace

hipError_t launch_gemm_mx(const uint8_t* a, const uint8_t* as, int a_fmt, const uint8_t* b, const uint8_t* bs, int M,
                          int N, int K, const float* add, void* out, int bf16, hipStream_t s) {
  const dim3 grid((N + 31) / 32, (M + 31) / 32);
  if (a_fmt == LMGC_MX_FP8) gemm_mx_kernel<LMGC_MX_FP8><<<grid, 64, 0, s>>>(a, as, b, bs, M, N, K, add, out, bf16);
  else gemm_mx_kernel<LMGC_MX_FP4><<<grid, 64, 0, s>>>(a, as, b, bs, M, N, K, add, out, bf16);
  return hipGetLastError();
}

}  // namespace lmgc
