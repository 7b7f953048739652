// Microscaled numbers (OCP MX formats): blocks of 32 values along a row share
// a scale 2^(byte - 127); a value is an e4m3 or an e2m1 number times it.
// Device helpers shared by the kernels that write and read them.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "common.h"
#include "lowbit.h"

namespace lmgc {

typedef uint32_t mx_u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t mx_u32x2 __attribute__((ext_vector_type(2)));
typedef float mx_f32x4 __attribute__((ext_vector_type(4)));

// Where the scale of block j of a row sits: a lane of the 16x16x128 matrix
// instruction takes the scale of block 4 s + g at step s, so the four steps
// of a 512-column group are the bytes of one 32-bit word.
__host__ __device__ inline int mx_scale_pos(int j) { return (j & ~15) + 4 * (j & 3) + ((j & 15) >> 2); }

// The scale byte of a block whose largest magnitude has the bits `amax`
// (sign cleared): the smallest power of two s, 2^-127 at least, with
// amax <= largest code * s, so that no code saturates; 255 (NaN) when the
// block holds a NaN or an infinity.  e4m3 ends at 1.75 * 2^8, e2m1 at
// 1.5 * 2^2.
template <int FMT>
__device__ inline int mx_scale_byte(uint32_t amax) {
  constexpr int emax = FMT == LMGC_MX_FP8 ? 8 : 2;
  constexpr uint32_t top = FMT == LMGC_MX_FP8 ? 0x600000u : 0x400000u;
  if (amax >= 0x7f800000u) return 255;
  const int e = (int)(amax >> 23) - emax + ((amax & 0x7fffffu) > top ? 1 : 0);
  return e > 0 ? e : 0;
}

// 2^(127 - byte): multiplying by it is exact for every value of the block.
__device__ inline float mx_inverse(int byte) { return __builtin_bit_cast(float, (uint32_t)(254 - min(byte, 254)) << 23); }

// 2^(byte - 127), NaN for byte 255.
__device__ inline float mx_scale(int byte) {
  const uint32_t u = byte == 255 ? 0x7fc00000u : byte ? (uint32_t)byte << 23 : 0x00400000u;
  return __builtin_bit_cast(float, u);
}

__device__ inline uint32_t abs_bits(float v) { return __builtin_bit_cast(uint32_t, v) & 0x7fffffffu; }

// Eight values, already divided by the scale -> 8 bytes (e4m3) or 4 bytes
// (e2m1, the first value in the low half of the byte), round to nearest even.
__device__ inline mx_u32x2 pack_fp8(const float (&v)[8]) {
  mx_u32x2 r;
#pragma unroll
  for (int i = 0; i < 2; i++) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i], v[4 * i + 1], 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i + 2], v[4 * i + 3], w, true);
    r[i] = (uint32_t)w;
  }
  return r;
}
__device__ inline uint32_t pack_fp4(const float (&v)[8]) {
  uint32_t w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, v[0], v[1], 1.0f, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2], v[3], 1.0f, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[4], v[5], 1.0f, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[6], v[7], 1.0f, 3);
}

// max over the four neighbouring lanes 4 q .. 4 q + 3.
__device__ inline uint32_t quad_max(uint32_t v) {
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, false));
  return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xF, 0xF, false));
}

// Columns 8 c .. 8 c + 7 of a row, four neighbouring lanes to a block: the
// block's scale, the codes to code_row and (one lane in four) the scale to
// scale_row.  Every lane of a wave calls it; c past the row's last group of
// 128 columns writes no codes, c past its last group of 512 nothing.
template <int FMT>
__device__ inline void mx_store8(float (&v)[8], int c, int kcols, int nscales, uint8_t* code_row, uint8_t* scale_row) {
  uint32_t a = 0;
#pragma unroll
  for (int i = 0; i < 8; i++) a = max(a, abs_bits(v[i]));
  const int byte = mx_scale_byte<FMT>(quad_max(a));
  const float inv = mx_inverse(byte);
#pragma unroll
  for (int i = 0; i < 8; i++) v[i] = byte == 255 ? 0.f : v[i] * inv;
  if (8 * c < kcols) {
    if constexpr (FMT == LMGC_MX_FP8) *reinterpret_cast<mx_u32x2*>(code_row + 8 * c) = pack_fp8(v);
    else *reinterpret_cast<uint32_t*>(code_row + 4 * c) = pack_fp4(v);
  }
  const int j = c >> 2;
  if ((c & 3) == 0 && j < nscales) scale_row[mx_scale_pos(j)] = (uint8_t)byte;
}

// Eight values at p (float32 or bf16), 16-byte aligned.
__device__ inline void load8(const float* p, float (&v)[8]) {
  const mx_f32x4 a = *reinterpret_cast<const mx_f32x4*>(p), b = *reinterpret_cast<const mx_f32x4*>(p + 4);
#pragma unroll
  for (int i = 0; i < 4; i++) {
    v[i] = a[i];
    v[4 + i] = b[i];
  }
}
__device__ inline void load8(const uint16_t* p, float (&v)[8]) {
  const mx_u32x4 a = *reinterpret_cast<const mx_u32x4*>(p);
#pragma unroll
  for (int i = 0; i < 4; i++) {
    v[2 * i] = __builtin_bit_cast(float, a[i] << 16);
    v[2 * i + 1] = __builtin_bit_cast(float, a[i] & 0xffff0000u);
  }
}
__device__ inline float load1(const float* p) { return *p; }
__device__ inline float load1(const uint16_t* p) { return bf16_to_f32(*p); }

}  // namespace lmgc
