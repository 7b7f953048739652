// Launches of the operators in fewer bits.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace lmgc {

// Columns of codes in a row (a whole number of 128-wide matrix steps) and
// bytes of scales in a row (whole groups of 512 columns).
__host__ __device__ inline int64_t mx_cols(int64_t cols) { return (cols + 127) / 128 * 128; }
__host__ __device__ inline int64_t mx_row_scales(int64_t cols) { return (cols + 511) / 512 * 16; }

// Microscaled operands (mx.hip, gemm_mx.hip) and the 8-bit key/value cache
// (kv8.hip); arguments as in lmgc.h, checked by the callers.
hipError_t launch_mx_quantize(const void* src, int dtype, int64_t rows, int cols, int64_t ld, int fmt, uint8_t* codes,
                              uint8_t* scales, hipStream_t s);
hipError_t launch_mx_dequantize(const uint8_t* codes, const uint8_t* scales, int fmt, int64_t rows, int cols, void* out,
                                int dtype, int64_t ld, hipStream_t s);
hipError_t launch_mx_block(const uint8_t* codes, const uint8_t* scales, int64_t N, int K, uint8_t* bcodes,
                           uint8_t* bscales, hipStream_t s);
hipError_t launch_add_norm_mx(const void* h, int h_dtype, const void* x, int x_dtype, const void* gain, int g_dtype,
                              float eps, int64_t M, int d, int fmt, void* out, uint8_t* codes, uint8_t* scales,
                              hipStream_t s);
hipError_t launch_gemm_mx(const uint8_t* a, const uint8_t* as, int a_fmt, const uint8_t* b, const uint8_t* bs, int M,
                          int N, int K, const float* add, void* out, int bf16, int tile, hipStream_t s);
int64_t kv8_workspace_bytes(int B, int Hq, int Hkv, int T, int hd, int cap);
// Workgroups of the attention over its columns, where they are one dimension of the grid.
int64_t kv8_workgroups(int B, int Hq, int Hkv, int T, int hd, int cap);
hipError_t launch_kv8_append(const uint16_t* k, const uint16_t* v, int B, int Hkv, int T, int hd, int cap,
                             const int32_t* lens, const int32_t* counts, uint8_t* kc, float* ks, uint8_t* vc, float* vs,
                             hipStream_t s);
hipError_t launch_attention_kv8(const uint16_t* q, int B, int Hq, int Hkv, int T, int hd, int cap, const int32_t* lens,
                                const int32_t* counts, const uint8_t* kc, const float* ks, const uint8_t* vc,
                                const float* vs, int window, int sinks, void* ws, uint16_t* out, hipStream_t s);

}  // namespace lmgc
