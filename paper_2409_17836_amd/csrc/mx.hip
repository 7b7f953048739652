// Microscaled operands of the 4- and 8-bit products: quantisation of rows,
// the way back, the block layout of weights, and the residual add with
// RMSNorm whose output is microscaled.  All are bound by the bytes they move
// (times below: from and to memory, a copy kernel reaches 5.3 TB/s) and, when
// small, by the launch and one round trip to memory (2.2 to 4 us).
#include <algorithm>
#include <type_traits>

#include "mx.h"

namespace lmgc {
namespace {

// ---------------------------------------------------------------- quantise
// Unit: one row x 512 columns, a wave; lane l takes columns 8 l .. 8 l + 7, so
// four lanes hold a block and its largest magnitude takes two exchanges between
// neighbours.  VEC: rows are whole 16-byte pieces (base, ld and cols), so a
// lane reads its columns in one or two loads.  32768 x 4096 bf16 to e4m3 75 us
// (5.4 TB/s), 22016 x 4096 to e2m1 46 us (4.9).
template <int FMT, typename T, bool VEC>
__global__ __launch_bounds__(256) void mx_quantize_kernel(const T* __restrict__ src, int64_t rows, int cols, int64_t ld,
                                                          uint8_t* __restrict__ codes, uint8_t* __restrict__ scales) {
  const int kcols = (int)mx_cols(cols), ns = (int)mx_row_scales(cols), n512 = ns / 16;
  const int lane = threadIdx.x & 63;
  const int64_t units = rows * n512, stride = (int64_t)gridDim.x * 4;
  for (int64_t u = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); u < units; u += stride) {
    const int64_t row = u / n512;
    const int c = (int)(u - row * n512) * 64 + lane;
    float v[8] = {};
    const T* p = src + row * ld + 8 * (int64_t)c;
    if (VEC) {
      if (8 * c < cols) load8(p, v);
    } else {
#pragma unroll
      for (int i = 0; i < 8; i++)
        if (8 * c + i < cols) v[i] = load1(p + i);
    }
    mx_store8<FMT>(v, c, kcols, ns, codes + row * (FMT == LMGC_MX_FP8 ? kcols : kcols / 2), scales + row * ns);
  }
}

// -------------------------------------------------------------- dequantise
__device__ inline void store8(float* p, const float (&v)[8]) {
  *reinterpret_cast<mx_f32x4*>(p) = mx_f32x4{v[0], v[1], v[2], v[3]};
  *reinterpret_cast<mx_f32x4*>(p + 4) = mx_f32x4{v[4], v[5], v[6], v[7]};
}
__device__ inline void store8(uint16_t* p, const float (&v)[8]) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  mx_u32x4 w;
#pragma unroll
  for (int i = 0; i < 4; i++) w[i] = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)v[2 * i], (__bf16)v[2 * i + 1]});
  *reinterpret_cast<mx_u32x4*>(p) = w;
}

// A thread: 8 columns.  VEC: as above, for the output.  32768 x 4096 e4m3 to
// bf16 73 us (5.6 TB/s), 22016 x 4096 e2m1 50 us (4.6).
template <int FMT, typename T, bool VEC>
__global__ __launch_bounds__(256) void mx_dequantize_kernel(const uint8_t* __restrict__ codes,
                                                            const uint8_t* __restrict__ scales, int64_t rows, int cols,
                                                            T* __restrict__ out, int64_t ld) {
  const int kcols = (int)mx_cols(cols), ns = (int)mx_row_scales(cols), nc = (cols + 7) / 8;
  const int64_t stride = (int64_t)gridDim.x * 256;
  for (int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x; t < rows * nc; t += stride) {
    const int64_t row = t / nc;
    const int c = (int)(t - row * nc);
    const float s = mx_scale(scales[row * ns + mx_scale_pos(c >> 2)]);
    float v[8];
    if constexpr (FMT == LMGC_MX_FP8) {
      const mx_u32x2 w = *reinterpret_cast<const mx_u32x2*>(codes + row * kcols + 8 * c);
#pragma unroll
      for (int i = 0; i < 2; i++) {
        v[4 * i] = __builtin_amdgcn_cvt_f32_fp8((int)w[i], 0);
        v[4 * i + 1] = __builtin_amdgcn_cvt_f32_fp8((int)w[i], 1);
        v[4 * i + 2] = __builtin_amdgcn_cvt_f32_fp8((int)w[i], 2);
        v[4 * i + 3] = __builtin_amdgcn_cvt_f32_fp8((int)w[i], 3);
      }
    } else {
      typedef float f32x2 __attribute__((ext_vector_type(2)));
      const uint32_t w = *reinterpret_cast<const uint32_t*>(codes + row * (kcols / 2) + 4 * c);
      const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 1);
      const f32x2 d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 2), e = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 3);
      v[0] = a[0], v[1] = a[1], v[2] = b[0], v[3] = b[1], v[4] = d[0], v[5] = d[1], v[6] = e[0], v[7] = e[1];
    }
    T* p = out + row * ld + 8 * (int64_t)c;
#pragma unroll
    for (int i = 0; i < 8; i++) v[i] *= s;
    if constexpr (VEC) {
      store8(p, v);
    } else {
#pragma unroll
      for (int i = 0; i < 8; i++) {
        if (8 * c + i >= cols) continue;
        if constexpr (sizeof(T) == 2) p[i] = f32_to_bf16(v[i]);
        else p[i] = v[i];
      }
    }
  }
}

// ------------------------------------------------------------------ blocks
// Row-major 4-bit codes and scales -> blocks (lmgc.h): thread t moves the
// 16-byte piece (32 columns of a row) that is piece t of the blocks, and the
// threads whose piece opens a 512-column group its word of scales.  Writes are
// in order, a wave 1 KB; reads are 16 rows' 64 bytes.  22016 x 4096 19 us.
__global__ __launch_bounds__(256) void mx_block_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales,
                                                       int64_t N, int K, uint8_t* __restrict__ bcodes,
                                                       uint8_t* __restrict__ bscales) {
  const int nk = (int)(mx_cols(K) / 128), n512 = (int)(mx_row_scales(K) / 16);
  const int64_t pieces = (N + 15) / 16 * nk * 64, stride = (int64_t)gridDim.x * 256;
  for (int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x; t < pieces; t += stride) {
    const int lane = (int)(t & 63), r = lane & 15, g = lane >> 4;
    const int64_t blk = t >> 6, grp = blk / nk, n = grp * 16 + r;
    const int k = (int)(blk - grp * nk);
    mx_u32x4 v = {};
    if (n < N) v = *reinterpret_cast<const mx_u32x4*>(codes + n * (nk * 64) + k * 64 + 16 * g);
    *reinterpret_cast<mx_u32x4*>(bcodes + t * 16) = v;
    if ((k & 3) == 0) {
      const int s = k >> 2;
      uint32_t w = 0;
      if (n < N) w = *reinterpret_cast<const uint32_t*>(scales + n * (n512 * 16) + s * 16 + 4 * g);
      *reinterpret_cast<uint32_t*>(bscales + (grp * n512 + s) * 256 + lane * 4) = w;
    }
  }
}

// -------------------------------------------------------- add and RMSNorm
// NT threads per row: a wave up to 1024 columns, then 256 to 1024, so that a
// thread has one piece of 8 columns (two past 8192) and the code stays short:
// with 256 threads throughout, 8 x 4096 took 0.9 us more and 32768 x 4096 8 us
// more.  From a graph 8 x 4096 takes 4.2 us, 32768 x 4096 from float32 259 (5.7
// TB/s), from bf16 to e2m1 182 (4.8).  Thread t keeps columns 8 (t + NT i) .. + 7 in
// registers between the sum of squares and the codes, so a row is read once.
// The sum that is normalised is the one that is stored.
//
// A code is the rounding of y, and an error in y of e turns some e / 2^-4 of
// the codes into their neighbours, so y is kept closer than a float32: the sum
// of the squares, the root and the products are float64 (which has room for
// rows, gains and values of any size too), and y becomes a float32 with its last
// bit set wherever bits are left behind it, so that it lies on a border between
// two codes only if the value does.  The float32s of twice the precision that
// did this before took as long, and failed near the ends of float32.  The
// kernel is bound by its memory traffic either way.
template <int FMT, typename TH, typename TX, typename TG, int NC, int NT>
__global__ __launch_bounds__(NT < 256 ? 256 : NT) void add_norm_mx_kernel(
    const TH* h, const TX* __restrict__ x, const TG* __restrict__ gain, float eps, int64_t M, int d, TH* out,
    uint8_t* __restrict__ codes, uint8_t* __restrict__ scales) {
#pragma clang fp contract(off)
  constexpr int NW = NT / 64, kRows = NT < 256 ? 256 / NT : 1;  // waves of a row, rows of a block
  __shared__ double part[NW];
  const int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / NT;
  if (kRows > 1 && row >= M) return;
  const int t = threadIdx.x % NT, nchunks = d / 8;
  const int kcols = (int)mx_cols(d), ns = (int)mx_row_scales(d);
  float v[NC][8], w[NC][8], gn[NC][8];
#pragma unroll
  for (int i = 0; i < NC; i++) {
    const int c = t + NT * i;
#pragma unroll
    for (int e = 0; e < 8; e++) v[i][e] = w[i][e] = gn[i][e] = 0.f;
    if (c >= nchunks) continue;
    load8(h + row * d + 8 * c, v[i]);
    if (x) load8(x + row * d + 8 * c, w[i]);
    load8(gain + 8 * c, gn[i]);
  }
  double sd = 0.0;
#pragma unroll
  for (int i = 0; i < NC; i++) {
    const int c = t + NT * i;
    if (x) {
#pragma unroll
      for (int e = 0; e < 8; e++) {
        v[i][e] += w[i][e];
        if constexpr (sizeof(TH) == 2) v[i][e] = bf16_to_f32(f32_to_bf16(v[i][e]));
      }
    }
    if (out && c < nchunks) store8(out + row * d + 8 * c, v[i]);
#pragma unroll
    for (int e = 0; e < 8; e++) sd = fma((double)v[i][e], (double)v[i][e], sd);
  }
#pragma unroll
  for (int o = 32; o; o >>= 1) sd += __shfl_xor(sd, o, 64);
  if constexpr (NW > 1) {
    if ((t & 63) == 0) part[t >> 6] = sd;
    __syncthreads();
    sd = 0.0;
#pragma unroll
    for (int w = 0; w < NW; w++) sd += part[w];
  }
  const double r = 1.0 / sqrt(sd / (double)d + (double)eps);
#pragma unroll
  for (int i = 0; i < NC; i++) {
    const int c = t + NT * i;
#pragma unroll
    for (int e = 0; e < 8; e++) {
      // (converted here: with two pieces the float64s, made earlier, took the
      // registers of a second block on the CU, 4096 x 16384 bf16 119 us)
      if constexpr (NC > 1) asm volatile("" : "+v"(v[i][e]), "+v"(gn[i][e]));
      const uint64_t u = __builtin_bit_cast(uint64_t, (double)v[i][e] * r * (double)gn[i][e]);
      constexpr uint32_t kBelow = 0x1fffffffu;  // the bits behind a float32's last
      const uint32_t lo = ((uint32_t)u | (((uint32_t)u & kBelow) + kBelow)) & ~kBelow;
      const float y = (float)__builtin_bit_cast(double, (u & 0xffffffff00000000ull) | lo);
      v[i][e] = c < nchunks ? y : 0.f;  // (zero times a NaN or infinite root is NaN)
    }
    mx_store8<FMT>(v[i], c, kcols, ns, codes + row * (FMT == LMGC_MX_FP8 ? kcols : kcols / 2), scales + row * ns);
  }
}

int grid_of(int64_t blocks) { return (int)std::max<int64_t>(1, std::min<int64_t>(blocks, 1 << 16)); }

template <int FMT, typename T>
void quantize(const T* src, int64_t rows, int cols, int64_t ld, uint8_t* codes, uint8_t* scales, hipStream_t s) {
  const bool vec = cols % 8 == 0 && ld * sizeof(T) % 16 == 0 && ((uintptr_t)src & 15) == 0;
  const int grid = grid_of((rows * (mx_row_scales(cols) / 16) + 3) / 4);
  if (vec) mx_quantize_kernel<FMT, T, true><<<grid, 256, 0, s>>>(src, rows, cols, ld, codes, scales);
  else mx_quantize_kernel<FMT, T, false><<<grid, 256, 0, s>>>(src, rows, cols, ld, codes, scales);
}

template <int FMT, typename TH, typename TX, typename TG>
void add_norm(const void* h, const void* x, const void* gain, float eps, int64_t M, int d, void* out, uint8_t* codes,
              uint8_t* scales, hipStream_t s) {
  const int nc = (int)mx_row_scales(d) / 16;  // groups of 512 columns, 64 threads each
  constexpr int64_t kLaunch = 1 << 21;  // rows of a launch: under 2^32 threads
  const int64_t nc_row = FMT == LMGC_MX_FP8 ? mx_cols(d) : mx_cols(d) / 2, ns_row = mx_row_scales(d);
  auto go = [&](auto n, auto nt) {
    constexpr int NT = decltype(nt)::value, kRows = NT < 256 ? 256 / NT : 1;
    for (int64_t m = 0; m < M; m += kLaunch) {
      const int64_t rows = std::min(kLaunch, M - m);
      add_norm_mx_kernel<FMT, TH, TX, TG, decltype(n)::value, NT><<<(unsigned)((rows + kRows - 1) / kRows), kRows * NT, 0, s>>>(
          (const TH*)h + m * d, x ? (const TX*)x + m * d : nullptr, (const TG*)gain, eps, rows, d,
          out ? (TH*)out + m * d : nullptr, codes + m * nc_row, scales + m * ns_row);
    }
  };
  using one = std::integral_constant<int, 1>;
  using two = std::integral_constant<int, 2>;
  if (nc <= 1) go(one{}, std::integral_constant<int, 64>{});
  else if (nc <= 2) go(two{}, std::integral_constant<int, 64>{});
  else if (nc <= 4) go(one{}, std::integral_constant<int, 256>{});
  else if (nc <= 8) go(one{}, std::integral_constant<int, 512>{});
  else if (nc <= 16) go(one{}, std::integral_constant<int, 1024>{});
  else go(two{}, std::integral_constant<int, 1024>{});
}

}  // namespace

hipError_t launch_mx_quantize(const void* src, int dtype, int64_t rows, int cols, int64_t ld, int fmt, uint8_t* codes,
                              uint8_t* scales, hipStream_t s) {
  const bool bf = dtype == LMGC_DTYPE_BF16;
  if (fmt == LMGC_MX_FP8) {
    if (bf) quantize<LMGC_MX_FP8>((const uint16_t*)src, rows, cols, ld, codes, scales, s);
    else quantize<LMGC_MX_FP8>((const float*)src, rows, cols, ld, codes, scales, s);
  } else {
    if (bf) quantize<LMGC_MX_FP4>((const uint16_t*)src, rows, cols, ld, codes, scales, s);
    else quantize<LMGC_MX_FP4>((const float*)src, rows, cols, ld, codes, scales, s);
  }
  return hipGetLastError();
}

hipError_t launch_mx_dequantize(const uint8_t* codes, const uint8_t* scales, int fmt, int64_t rows, int cols, void* out,
                                int dtype, int64_t ld, hipStream_t s) {
  const int grid = grid_of((rows * ((cols + 7) / 8) + 255) / 256);
  const bool vec = cols % 8 == 0 && ld * (dtype == LMGC_DTYPE_BF16 ? 2 : 4) % 16 == 0 && ((uintptr_t)out & 15) == 0;
  auto go = [&](auto f, auto t, auto v) {
    using T = decltype(t);
    mx_dequantize_kernel<decltype(f)::value, T, decltype(v)::value><<<grid, 256, 0, s>>>(codes, scales, rows, cols, (T*)out, ld);
  };
  auto go_t = [&](auto f, auto t) {
    if (vec) go(f, t, std::true_type{});
    else go(f, t, std::false_type{});
  };
  auto go_f = [&](auto f) {
    if (dtype == LMGC_DTYPE_BF16) go_t(f, uint16_t{});
    else go_t(f, float{});
  };
  if (fmt == LMGC_MX_FP8) go_f(std::integral_constant<int, LMGC_MX_FP8>{});
  else go_f(std::integral_constant<int, LMGC_MX_FP4>{});
  return hipGetLastError();
}

hipError_t launch_mx_block(const uint8_t* codes, const uint8_t* scales, int64_t N, int K, uint8_t* bcodes,
                           uint8_t* bscales, hipStream_t s) {
  const int grid = grid_of(((N + 15) / 16 * (mx_cols(K) / 128) * 64 + 255) / 256);
  mx_block_kernel<<<grid, 256, 0, s>>>(codes, scales, N, K, bcodes, bscales);
  return hipGetLastError();
}

hipError_t launch_add_norm_mx(const void* h, int h_dtype, const void* x, int x_dtype, const void* gain, int g_dtype,
                              float eps, int64_t M, int d, int fmt, void* out, uint8_t* codes, uint8_t* scales,
                              hipStream_t s) {
  auto go3 = [&](auto f, auto th, auto tx) {
    using TH = decltype(th);
    using TX = decltype(tx);
    constexpr int F = decltype(f)::value;
    if (g_dtype == LMGC_DTYPE_BF16) add_norm<F, TH, TX, uint16_t>(h, x, gain, eps, M, d, out, codes, scales, s);
    else add_norm<F, TH, TX, float>(h, x, gain, eps, M, d, out, codes, scales, s);
  };
  auto go2 = [&](auto f, auto th) {
    if (x_dtype == LMGC_DTYPE_BF16) go3(f, th, uint16_t{});
    else go3(f, th, float{});
  };
  auto go1 = [&](auto f) {
    if (h_dtype == LMGC_DTYPE_BF16) go2(f, uint16_t{});
    else go2(f, float{});
  };
  if (fmt == LMGC_MX_FP8) go1(std::integral_constant<int, LMGC_MX_FP8>{});
  else go1(std::integral_constant<int, LMGC_MX_FP4>{});
  return hipGetLastError();
}

}  // namespace lmgc
