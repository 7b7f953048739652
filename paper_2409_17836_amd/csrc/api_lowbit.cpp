// C ABI of the operators in fewer bits: argument checks and launches.
#include <hip/hip_runtime.h>

#include "common.h"
#include "host.h"
#include "lowbit.h"

using namespace lmgc;

namespace {

constexpr int64_t kMaxCols = 1 << 20;

bool aligned(const void* p) { return ((uintptr_t)p & 15) == 0; }
bool overlap(const void* a, int64_t na, const void* b, int64_t nb) {
  return a && b && (const char*)a < (const char*)b + nb && (const char*)b < (const char*)a + na;
}
bool is_dtype(int32_t t) { return t == LMGC_DTYPE_F32 || t == LMGC_DTYPE_BF16; }
int64_t dtype_bytes(int32_t t) { return t == LMGC_DTYPE_BF16 ? 2 : 4; }
bool is_fmt(int32_t f) { return f == LMGC_MX_FP8 || f == LMGC_MX_FP4; }

int check_shape(int64_t rows, int64_t cols) {
  if (rows < 0 || rows > INT32_MAX) return set_error(LMGC_EINVAL, "rows must be in [0, 2^31 - 1]");
  if (cols < 1 || cols > kMaxCols) return set_error(LMGC_EINVAL, "cols must be in [1, 2^20]");
  return LMGC_OK;
}

// rows `ld` elements apart, their extent within the address space (2^46 elements: its bytes do not pass 64 bits)
int check_ld(int64_t rows, int64_t cols, int64_t ld) {
  if (ld < cols || ld > ((int64_t)1 << 40)) return set_error(LMGC_EINVAL, "ld must be in [cols, 2^40]");
  if (rows > 1 && rows - 1 > ((int64_t)1 << 46) / ld) return set_error(LMGC_EINVAL, "rows ld passes 2^46 elements");
  return LMGC_OK;
}

int64_t code_bytes(int32_t fmt, int64_t rows, int64_t cols) { return rows * (fmt == LMGC_MX_FP8 ? mx_cols(cols) : mx_cols(cols) / 2); }

int done(hipError_t e, const char* what) {
  if (e != hipSuccess) return set_error(LMGC_EDEVICE, "%s launch: %s", what, hipGetErrorString(e));
  return LMGC_OK;
}

int check_cache(int32_t B, int32_t Hkv, int32_t T, int32_t hd, int32_t cap, const int32_t* lens, const uint8_t* kc,
                const float* ks, const uint8_t* vc, const float* vs) {
  if (B <= 0 || Hkv <= 0 || T <= 0 || cap <= 0) return set_error(LMGC_EINVAL, "B, Hkv, T and cap must be positive");
  if (B > 16383 || Hkv > 32767 || T > (1 << 24) || cap > (1 << 24))
    return set_error(LMGC_EINVAL, "B above 16383, Hkv above 32767, or T or cap above 2^24");
  if (cap % 64) return set_error(LMGC_EINVAL, "cap must be a multiple of 64");
  if (hd != 64 && hd != 128) return set_error(LMGC_EUNSUPPORTED, "need hd in {64, 128}");
  if (!lens || !kc || !ks || !vc || !vs) return set_error(LMGC_EINVAL, "NULL device buffer");
  if (!aligned(kc) || !aligned(ks) || !aligned(vc) || !aligned(vs) || ((uintptr_t)lens & 3))
    return set_error(LMGC_EINVAL, "cache pointers must be 16-byte aligned");
  const int64_t blocks = (int64_t)B * Hkv * (cap / 64), codes = blocks * 64 * hd;
  const void* p[4] = {kc, vc, ks, vs};
  const int64_t bytes[4] = {codes, codes, 4 * blocks, 4 * blocks};
  for (int i = 0; i < 4; i++)
    for (int j = 0; j < i; j++)
      if (overlap(p[i], bytes[i], p[j], bytes[j])) return set_error(LMGC_EINVAL, "the cache's buffers overlap");
  return LMGC_OK;
}
// whether n bytes at p share memory with the cache
bool in_cache(const void* p, int64_t n, int32_t B, int32_t Hkv, int32_t hd, int32_t cap, const void* kc, const void* ks,
              const void* vc, const void* vs) {
  const int64_t blocks = (int64_t)B * Hkv * (cap / 64), codes = blocks * 64 * hd;
  return overlap(p, n, kc, codes) || overlap(p, n, vc, codes) || overlap(p, n, ks, 4 * blocks) || overlap(p, n, vs, 4 * blocks);
}

}  // namespace

extern "C" {

int64_t lmgc_mx_code_bytes(int32_t fmt, int64_t rows, int64_t cols) {
  clear_error();
  if (!is_fmt(fmt)) return set_error(LMGC_EINVAL, "unknown format %d", fmt);
  int rc = check_shape(rows, cols);
  return rc ? rc : code_bytes(fmt, rows, cols);
}

int64_t lmgc_mx_scale_bytes(int64_t rows, int64_t cols) {
  clear_error();
  int rc = check_shape(rows, cols);
  return rc ? rc : rows * mx_row_scales(cols);
}

int64_t lmgc_mx_block_code_bytes(int64_t rows, int64_t cols) {
  clear_error();
  int rc = check_shape(rows, cols);
  return rc ? rc : code_bytes(LMGC_MX_FP4, (rows + 15) / 16 * 16, cols);
}

int64_t lmgc_mx_block_scale_bytes(int64_t rows, int64_t cols) {
  clear_error();
  int rc = check_shape(rows, cols);
  return rc ? rc : (rows + 15) / 16 * 16 * mx_row_scales(cols);
}

int lmgc_op_mx_quantize(const void* d_src, int32_t dtype, int64_t rows, int64_t cols, int64_t ld, int32_t fmt,
                        uint8_t* d_codes, uint8_t* d_scales, void* stream) {
  clear_error();
  int rc = check_shape(rows, cols);
  if (rc) return rc;
  if (!is_dtype(dtype)) return set_error(LMGC_EINVAL, "unknown dtype %d", dtype);
  if (!is_fmt(fmt)) return set_error(LMGC_EINVAL, "unknown format %d", fmt);
  if ((rc = check_ld(rows, cols, ld))) return rc;
  if (rows == 0) return LMGC_OK;
  if (!d_src || !d_codes || !d_scales) return set_error(LMGC_EINVAL, "NULL device buffer");
  if ((uintptr_t)d_src % dtype_bytes(dtype) || !aligned(d_codes) || !aligned(d_scales))
    return set_error(LMGC_EINVAL, "codes and scales must be 16-byte aligned, the source aligned to its elements");
  const int64_t nsrc = ((rows - 1) * ld + cols) * dtype_bytes(dtype), nc = code_bytes(fmt, rows, cols), ns = rows * mx_row_scales(cols);
  if (overlap(d_src, nsrc, d_codes, nc) || overlap(d_src, nsrc, d_scales, ns) || overlap(d_codes, nc, d_scales, ns))
    return set_error(LMGC_EINVAL, "buffers overlap");
  return done(launch_mx_quantize(d_src, dtype, rows, (int)cols, ld, fmt, d_codes, d_scales, (hipStream_t)stream), "mx quantize");
}

int lmgc_op_mx_dequantize(const uint8_t* d_codes, const uint8_t* d_scales, int32_t fmt, int64_t rows, int64_t cols,
                          void* d_out, int32_t dtype, int64_t ld, void* stream) {
  clear_error();
  int rc = check_shape(rows, cols);
  if (rc) return rc;
  if (!is_dtype(dtype)) return set_error(LMGC_EINVAL, "unknown dtype %d", dtype);
  if (!is_fmt(fmt)) return set_error(LMGC_EINVAL, "unknown format %d", fmt);
  if ((rc = check_ld(rows, cols, ld))) return rc;
  if (rows == 0) return LMGC_OK;
  if (!d_out || !d_codes || !d_scales) return set_error(LMGC_EINVAL, "NULL device buffer");
  if ((uintptr_t)d_out % dtype_bytes(dtype) || !aligned(d_codes) || !aligned(d_scales))
    return set_error(LMGC_EINVAL, "codes and scales must be 16-byte aligned, the output aligned to its elements");
  const int64_t nout = ((rows - 1) * ld + cols) * dtype_bytes(dtype);
  if (overlap(d_out, nout, d_codes, code_bytes(fmt, rows, cols)) || overlap(d_out, nout, d_scales, rows * mx_row_scales(cols)))
    return set_error(LMGC_EINVAL, "buffers overlap");
  return done(launch_mx_dequantize(d_codes, d_scales, fmt, rows, (int)cols, d_out, dtype, ld, (hipStream_t)stream), "mx dequantize");
}

int lmgc_op_mx_block(const uint8_t* d_codes, const uint8_t* d_scales, int64_t N, int64_t K, uint8_t* d_block_codes,
                     uint8_t* d_block_scales, void* stream) {
  clear_error();
  int rc = check_shape(N, K);
  if (rc) return rc;
  if (N == 0) return LMGC_OK;
  if (!d_codes || !d_scales || !d_block_codes || !d_block_scales) return set_error(LMGC_EINVAL, "NULL device buffer");
  if (!aligned(d_codes) || !aligned(d_scales) || !aligned(d_block_codes) || !aligned(d_block_scales))
    return set_error(LMGC_EINVAL, "pointers must be 16-byte aligned");
  const int64_t nc = code_bytes(LMGC_MX_FP4, N, K), ns = N * mx_row_scales(K), n16 = (N + 15) / 16 * 16;
  const int64_t bc = code_bytes(LMGC_MX_FP4, n16, K), bs = n16 * mx_row_scales(K);
  if (overlap(d_codes, nc, d_block_codes, bc) || overlap(d_codes, nc, d_block_scales, bs) ||
      overlap(d_scales, ns, d_block_codes, bc) || overlap(d_scales, ns, d_block_scales, bs) ||
      overlap(d_block_codes, bc, d_block_scales, bs))
    return set_error(LMGC_EINVAL, "buffers overlap");
  return done(launch_mx_block(d_codes, d_scales, N, (int)K, d_block_codes, d_block_scales, (hipStream_t)stream), "mx block");
}

int lmgc_op_add_norm_mx(const void* d_h, int32_t h_dtype, const void* d_x, int32_t x_dtype, const void* d_gain,
                        int32_t g_dtype, float eps, int64_t M, int64_t d, int32_t fmt, void* d_out, uint8_t* d_codes,
                        uint8_t* d_scales, void* stream) {
  clear_error();
  int rc = check_shape(M, d);
  if (rc) return rc;
  if (!is_dtype(h_dtype) || !is_dtype(g_dtype) || (d_x && !is_dtype(x_dtype))) return set_error(LMGC_EINVAL, "unknown dtype");
  if (!is_fmt(fmt)) return set_error(LMGC_EINVAL, "unknown format %d", fmt);
  if (!(eps >= 0.f)) return set_error(LMGC_EINVAL, "eps must be >= 0");
  if (d % 32 || d > 16384) return set_error(LMGC_EUNSUPPORTED, "need d %% 32 == 0 and d <= 16384");
  if (M == 0) return LMGC_OK;
  if (!d_h || !d_gain || !d_codes || !d_scales) return set_error(LMGC_EINVAL, "NULL device buffer");
  if (!aligned(d_h) || !aligned(d_x) || !aligned(d_gain) || !aligned(d_out) || !aligned(d_codes) || !aligned(d_scales))
    return set_error(LMGC_EINVAL, "pointers must be 16-byte aligned");
  const int64_t nh = M * d * dtype_bytes(h_dtype), nx = d_x ? M * d * dtype_bytes(x_dtype) : 0, ng = d * dtype_bytes(g_dtype);
  const void* w[3] = {d_out == d_h ? nullptr : d_out, d_codes, d_scales};
  const int64_t nw[3] = {nh, code_bytes(fmt, M, d), M * mx_row_scales(d)};
  for (int i = 0; i < 3; i++)
    if (overlap(w[i], nw[i], d_h, nh) || overlap(w[i], nw[i], d_x, nx) || overlap(w[i], nw[i], d_gain, ng) ||
        overlap(w[i], nw[i], w[(i + 1) % 3], nw[(i + 1) % 3]))
      return set_error(LMGC_EINVAL, "buffers overlap");
  if (d_out == d_h && (overlap(d_out, nh, d_x, nx) || overlap(d_out, nh, d_gain, ng)))
    return set_error(LMGC_EINVAL, "buffers overlap");
  return done(launch_add_norm_mx(d_h, h_dtype, d_x, x_dtype, d_gain, g_dtype, eps, M, (int)d, fmt, d_out, d_codes, d_scales,
                                 (hipStream_t)stream), "add norm");
}

int lmgc_op_gemm_mx(const uint8_t* d_a, const uint8_t* d_a_scales, int32_t a_fmt, const uint8_t* d_b,
                    const uint8_t* d_b_scales, const float* d_add, void* d_out, int32_t M, int32_t N, int32_t K,
                    int32_t kind, void* stream) {
  return lmgc_op_gemm_mx_tile(d_a, d_a_scales, a_fmt, d_b, d_b_scales, d_add, d_out, M, N, K, kind, -1, stream);
}

int lmgc_op_gemm_mx_tile(const uint8_t* d_a, const uint8_t* d_a_scales, int32_t a_fmt, const uint8_t* d_b,
                         const uint8_t* d_b_scales, const float* d_add, void* d_out, int32_t M, int32_t N, int32_t K,
                         int32_t kind, int32_t tile, void* stream) {
  clear_error();
  if (M < 0 || M > (1 << 26) || N <= 0 || N > kMaxCols || K <= 0 || K > kMaxCols)
    return set_error(LMGC_EINVAL, "need 0 <= M <= 2^26 and N, K in [1, 2^20]");
  if (!is_fmt(a_fmt)) return set_error(LMGC_EINVAL, "unknown format %d", a_fmt);
  if (tile > LMGC_MX_TILE_256X256 || (tile == LMGC_MX_TILE_256X256 && a_fmt == LMGC_MX_FP4))
    return set_error(LMGC_EINVAL, "unknown tile %d", tile);
  if (kind != LMGC_OP_STORE && kind != LMGC_OP_STORE_BF16) return set_error(LMGC_EINVAL, "unknown kind %d", kind);
  if (M == 0) return LMGC_OK;
  if (!d_a || !d_a_scales || !d_b || !d_b_scales || !d_out) return set_error(LMGC_EINVAL, "NULL device buffer");
  if (!aligned(d_a) || !aligned(d_a_scales) || !aligned(d_b) || !aligned(d_b_scales) || !aligned(d_add) || !aligned(d_out))
    return set_error(LMGC_EINVAL, "pointers must be 16-byte aligned");
  const int64_t n16 = ((int64_t)N + 15) / 16 * 16;
  const int64_t nout = (int64_t)M * N * (kind == LMGC_OP_STORE ? 4 : 2);
  if (d_add && (const void*)d_add != d_out && overlap(d_add, (int64_t)M * N * 4, d_out, nout))
    return set_error(LMGC_EINVAL, "d_add overlaps d_out without being equal to it");
  if (d_add && (const void*)d_add == d_out && kind != LMGC_OP_STORE)
    return set_error(LMGC_EINVAL, "d_add may be d_out only for a float32 result");
  if (overlap(d_out, nout, d_a, code_bytes(a_fmt, M, K)) || overlap(d_out, nout, d_a_scales, M * mx_row_scales(K)) ||
      overlap(d_out, nout, d_b, code_bytes(LMGC_MX_FP4, n16, K)) || overlap(d_out, nout, d_b_scales, n16 * mx_row_scales(K)))
    return set_error(LMGC_EINVAL, "d_out overlaps an operand");
  return done(launch_gemm_mx(d_a, d_a_scales, a_fmt, d_b, d_b_scales, M, N, K, d_add, d_out, kind == LMGC_OP_STORE_BF16,
                             tile, (hipStream_t)stream), "gemm");
}

int lmgc_op_kv8_append(const uint16_t* d_k, const uint16_t* d_v, int32_t B, int32_t Hkv, int32_t T, int32_t hd,
                       int32_t cap, const int32_t* d_lens, const int32_t* d_counts, uint8_t* d_kc, float* d_ks,
                       uint8_t* d_vc, float* d_vs, void* stream) {
  clear_error();
  int rc = check_cache(B, Hkv, T, hd, cap, d_lens, d_kc, d_ks, d_vc, d_vs);
  if (rc) return rc;
  if (!d_k || !d_v) return set_error(LMGC_EINVAL, "NULL device buffer");
  if (!aligned(d_k) || !aligned(d_v) || ((uintptr_t)d_counts & 3)) return set_error(LMGC_EINVAL, "pointers must be 16-byte aligned");
  const int64_t nk = (int64_t)B * Hkv * T * hd * 2;
  if (in_cache(d_k, nk, B, Hkv, hd, cap, d_kc, d_ks, d_vc, d_vs) || in_cache(d_v, nk, B, Hkv, hd, cap, d_kc, d_ks, d_vc, d_vs))
    return set_error(LMGC_EINVAL, "d_k or d_v overlaps the cache");
  for (const int32_t* p : {d_lens, d_counts})
    if (in_cache(p, (int64_t)B * 4, B, Hkv, hd, cap, d_kc, d_ks, d_vc, d_vs))
      return set_error(LMGC_EINVAL, "d_lens or d_counts overlaps the cache");
  return done(launch_kv8_append(d_k, d_v, B, Hkv, T, hd, cap, d_lens, d_counts, d_kc, d_ks, d_vc, d_vs, (hipStream_t)stream),
              "append");
}

int64_t lmgc_kv8_workspace(int32_t B, int32_t Hq, int32_t Hkv, int32_t T, int32_t hd, int32_t cap) {
  clear_error();
  if (B <= 0 || B > 16383 || Hkv <= 0 || Hq <= 0 || Hq > 65535 || Hq % Hkv || T <= 0 || T > (1 << 24) || cap <= 0 || cap > (1 << 24) || cap % 64 ||
      (int64_t)T * (Hq / Hkv) > (1 << 30))
    return set_error(LMGC_EINVAL, "bad sizes");
  if (hd != 64 && hd != 128) return set_error(LMGC_EUNSUPPORTED, "need hd in {64, 128}");
  return kv8_workspace_bytes(B, Hq, Hkv, T, hd, cap);
}

int lmgc_op_attention_kv8(const uint16_t* d_q, int32_t B, int32_t Hq, int32_t Hkv, int32_t T, int32_t hd, int32_t cap,
                          const int32_t* d_lens, const int32_t* d_counts, const uint8_t* d_kc, const float* d_ks,
                          const uint8_t* d_vc, const float* d_vs, int32_t window, int32_t sinks, uint16_t* d_out,
                          void* d_ws, size_t ws_bytes, void* stream) {
  clear_error();
  int rc = check_cache(B, Hkv, T, hd, cap, d_lens, d_kc, d_ks, d_vc, d_vs);
  if (rc) return rc;
  if (Hq <= 0 || Hq > 65535 || Hq % Hkv) return set_error(LMGC_EINVAL, "Hq must be a positive multiple of Hkv");
  if ((int64_t)T * (Hq / Hkv) > (1 << 30)) return set_error(LMGC_EINVAL, "T Hq / Hkv above 2^30");
  if (kv8_workgroups(B, Hq, Hkv, T, hd, cap) >= 1 << 23)  // 2^32 threads
    return set_error(LMGC_EUNSUPPORTED, "too many columns for one launch");
  if (window < 0 || sinks < 0) return set_error(LMGC_EINVAL, "window and sinks must be >= 0");
  if (!d_q || !d_out) return set_error(LMGC_EINVAL, "NULL device buffer");
  if (!aligned(d_q) || !aligned(d_out) || !aligned(d_ws) || ((uintptr_t)d_counts & 3))
    return set_error(LMGC_EINVAL, "pointers must be 16-byte aligned");
  const int64_t nq = (int64_t)B * Hq * T * hd * 2, need = kv8_workspace_bytes(B, Hq, Hkv, T, hd, cap);
  if (need > 0 && (!d_ws || ws_bytes < (size_t)need))
    return set_error(LMGC_ESIZE, "workspace too small: %zu < %lld", d_ws ? ws_bytes : (size_t)0, (long long)need);
  if (overlap(d_q, nq, d_out, nq) || overlap(d_ws, need, d_q, nq) || overlap(d_ws, need, d_out, nq) ||
      in_cache(d_out, nq, B, Hkv, hd, cap, d_kc, d_ks, d_vc, d_vs) || in_cache(d_ws, need, B, Hkv, hd, cap, d_kc, d_ks, d_vc, d_vs))
    return set_error(LMGC_EINVAL, "buffers overlap");
  for (const int32_t* p : {d_lens, d_counts})
    if (overlap(p, (int64_t)B * 4, d_out, nq) || overlap(p, (int64_t)B * 4, d_ws, need))
      return set_error(LMGC_EINVAL, "d_lens or d_counts overlaps what the call writes");
  return done(launch_attention_kv8(d_q, B, Hq, Hkv, T, hd, cap, d_lens, d_counts, d_kc, d_ks, d_vc, d_vs, window, sinks,
                                   d_ws, d_out, (hipStream_t)stream), "attention");
}

}  // extern "C"
