// C ABI of the rotary positions and the paged key/value cache: argument checks
// and launches.
#include <hip/hip_runtime.h>
#include <math.h>

#include <algorithm>

#include "common.h"
#include "host.h"
#include "paged.h"

using namespace lmgc;

namespace {

constexpr int kMaxTokens = 1 << 24;
constexpr int64_t kMaxLd = (int64_t)1 << 40, kMaxExtent = (int64_t)1 << 46;

bool aligned(const void* p, int64_t n) { return (uintptr_t)p % n == 0; }
bool overlap(const void* a, int64_t na, const void* b, int64_t nb) {
  return a && b && na > 0 && nb > 0 && (const char*)a < (const char*)b + nb && (const char*)b < (const char*)a + na;
}
bool is_dtype(int32_t t) { return t == LMGC_DTYPE_F32 || t == LMGC_DTYPE_BF16; }
int64_t dtype_bytes(int32_t t) { return t == LMGC_DTYPE_BF16 ? 2 : 4; }

int done(hipError_t e, const char* what) {
  if (e != hipSuccess) return set_error(LMGC_EDEVICE, "%s launch: %s", what, hipGetErrorString(e));
  return LMGC_OK;
}

// Rows of `cols` numbers, ld apart: their extent in numbers, or < 0 (an error is set).
int64_t extent(int64_t rows, int64_t cols, int64_t ld, const char* what) {
  if (ld < cols || ld > kMaxLd) return set_error(LMGC_EINVAL, "%s must be in [columns of a row, 2^40]", what);
  if (rows > 1 && rows - 1 > kMaxExtent / ld) return set_error(LMGC_EINVAL, "rows of %s pass 2^46 numbers", what);
  return rows > 0 ? (rows - 1) * ld + cols : 0;
}

int check_table(const float* table, int64_t n_pos, int32_t rot, int32_t hd, int32_t layout) {
  if (rot < 2 || rot % 2 || rot > hd || rot > kMaxRot) return set_error(LMGC_EINVAL, "rot must be even, in [2, hd] and at most %d", kMaxRot);
  if (layout != LMGC_ROPE_HALF && layout != LMGC_ROPE_INTERLEAVED) return set_error(LMGC_EINVAL, "unknown layout %d", layout);
  if (n_pos < 1 || n_pos > kMaxTokens) return set_error(LMGC_EINVAL, "n_pos must be in [1, 2^24]");
  if (!table) return set_error(LMGC_EINVAL, "NULL device buffer");
  if (!aligned(table, 16)) return set_error(LMGC_EINVAL, "the table must be 16-byte aligned");
  return LMGC_OK;
}

int check_sizes(int64_t n, int64_t B, int64_t Hq, int64_t Hkv, int64_t hd) {
  if (n < 0 || n > kMaxTokens || B < 1 || B > 65535) return set_error(LMGC_EINVAL, "need 0 <= n <= 2^24 and 1 <= B <= 65535");
  if (Hkv < 1 || Hkv > 4096 || Hq < 1 || Hq > 65535 || Hq % Hkv)
    return set_error(LMGC_EINVAL, "need 1 <= Hkv <= 4096, and Hq a multiple of it, at most 65535");
  if (hd != 64 && hd != 128) return set_error(LMGC_EUNSUPPORTED, "need hd in {64, 128}");
  return LMGC_OK;
}

struct Cache {
  const void *kc, *vc;
  int64_t bytes;
  bool with(const void* p, int64_t n) const { return overlap(p, n, kc, bytes) || overlap(p, n, vc, bytes); }
};

int check_cache(const Cache& c, const Ragged& r) {
  if (r.page != 32 && r.page != 64 && r.page != 128 && r.page != 256) return set_error(LMGC_EUNSUPPORTED, "need page in {32, 64, 128, 256}");
  if (r.n_pages < 1) return set_error(LMGC_EINVAL, "n_pages must be positive");
  if (r.max_pages < 1 || (int64_t)r.max_pages * r.page > kMaxTokens) return set_error(LMGC_EINVAL, "max_pages page must be in [1, 2^24]");
  if (!c.kc || !c.vc || !r.pages || !r.starts || !r.lens) return set_error(LMGC_EINVAL, "NULL device buffer");
  if (!aligned(c.kc, 16) || !aligned(c.vc, 16)) return set_error(LMGC_EINVAL, "the pools must be 16-byte aligned");
  if (!aligned(r.pages, 4) || !aligned(r.starts, 4) || !aligned(r.lens, 4)) return set_error(LMGC_EINVAL, "pages, starts and lens must be 4-byte aligned");
  if (overlap(c.kc, c.bytes, c.vc, c.bytes)) return set_error(LMGC_EINVAL, "the pools overlap");
  return LMGC_OK;
}

// Whether n bytes at p share memory with what describes the batch.
bool in_batch(const void* p, int64_t n, const Ragged& r) {
  return overlap(p, n, r.pages, (int64_t)r.B * r.max_pages * 4) || overlap(p, n, r.starts, ((int64_t)r.B + 1) * 4) ||
         overlap(p, n, r.lens, (int64_t)r.B * 4);
}

}  // namespace

extern "C" {

int lmgc_rope_frequencies(double theta, int32_t rot, int32_t scaling, double factor, double orig, double slow, double fast, double* freqs) {
  clear_error();
  if (rot < 2 || rot % 2 || rot > kMaxRot) return set_error(LMGC_EINVAL, "rot must be even and in [2, %d]", kMaxRot);
  if (!(theta > 0) || !isfinite(theta)) return set_error(LMGC_EINVAL, "theta must be positive");
  if (!freqs) return set_error(LMGC_EINVAL, "NULL buffer");
  if (scaling < LMGC_ROPE_PLAIN || scaling > LMGC_ROPE_YARN) return set_error(LMGC_EINVAL, "unknown scaling %d", scaling);
  if (scaling != LMGC_ROPE_PLAIN && (!(factor >= 1) || !isfinite(factor))) return set_error(LMGC_EINVAL, "factor must be at least 1");
  if (scaling == LMGC_ROPE_NTK && rot < 4) return set_error(LMGC_EINVAL, "NTK scaling needs rot of 4 at least");
  if (scaling == LMGC_ROPE_YARN && (!(orig > 0) || !isfinite(orig) || !(slow >= 0) || !(fast > slow) || !isfinite(fast)))
    return set_error(LMGC_EINVAL, "need orig > 0 and 0 <= slow < fast");
  if (scaling == LMGC_ROPE_NTK) theta *= pow(factor, rot / (rot - 2.0));
  for (int i = 0; i < rot / 2; i++) {
    double f = pow(theta, -2.0 * i / rot);
    if (scaling == LMGC_ROPE_LINEAR) f /= factor;
    if (scaling == LMGC_ROPE_YARN) {
      const double turns = orig * f / (2.0 * M_PI), keep = std::min(1.0, std::max(0.0, (turns - slow) / (fast - slow)));
      f = f * keep + f / factor * (1.0 - keep);
    }
    freqs[i] = f;
  }
  return LMGC_OK;
}

int lmgc_op_rope_table(const double* freqs, int32_t rot, double mscale, int64_t n_pos, float* d_table, void* stream) {
  clear_error();
  int rc = check_table(d_table, n_pos, rot, kMaxRot, LMGC_ROPE_HALF);
  if (rc) return rc;
  if (!freqs) return set_error(LMGC_EINVAL, "NULL buffer");
  if (!isfinite(mscale)) return set_error(LMGC_EINVAL, "mscale must be finite");
  for (int i = 0; i < rot / 2; i++)
    if (!isfinite(freqs[i])) return set_error(LMGC_EINVAL, "frequency %d is not finite", i);
  return done(launch_rope_table(freqs, rot, mscale, n_pos, d_table, (hipStream_t)stream), "rope table");
}

int lmgc_op_rope(const void* d_x, int32_t dtype, int64_t n, int32_t heads, int32_t hd, int64_t ldx, int64_t ldhx,
                 const int32_t* d_pos, const float* d_table, int64_t n_pos, int32_t rot, int32_t layout, int32_t backward,
                 void* d_out, int64_t ldo, int64_t ldho, void* stream) {
  clear_error();
  if (!is_dtype(dtype)) return set_error(LMGC_EINVAL, "unknown dtype %d", dtype);
  if (n < 0 || n > kMaxTokens) return set_error(LMGC_EINVAL, "n must be in [0, 2^24]");
  if (heads < 1 || heads > (1 << 20) || hd < 2 || hd > kMaxRot) return set_error(LMGC_EINVAL, "need heads in [1, 2^20] and hd in [2, %d]", kMaxRot);
  int rc = check_table(d_table, n_pos, rot, hd, layout);
  if (rc) return rc;
  // rows and heads, either of them the outer: the inner ones lie apart from each other
  int64_t ext[2];
  for (int i = 0; i < 2; i++) {
    const int64_t ld = i ? ldo : ldx, ldh = i ? ldho : ldhx;
    const int64_t in = extent(heads, hd, ldh, "ldh");
    if (in < 0) return (int)in;
    if (ld >= in) {
      ext[i] = extent(n, in, ld, "ld");
    } else {
      const int64_t rows = extent(n, hd, ld, "ld");
      if (rows < 0) return (int)rows;
      if (ldh < rows) return set_error(LMGC_EINVAL, "rows and heads overlap");
      ext[i] = extent(heads, rows, ldh, "ldh");
    }
    if (ext[i] < 0) return (int)ext[i];
  }
  if (n == 0) return LMGC_OK;
  if (!d_x || !d_out || !d_pos) return set_error(LMGC_EINVAL, "NULL device buffer");
  const int64_t size = dtype_bytes(dtype);
  if (!aligned(d_x, size) || !aligned(d_out, size) || !aligned(d_pos, 4)) return set_error(LMGC_EINVAL, "pointers must be aligned to their elements");
  const int64_t nx = ext[0] * size, no = ext[1] * size;
  if (d_out == d_x ? ldx != ldo || ldhx != ldho : overlap(d_x, nx, d_out, no))
    return set_error(LMGC_EINVAL, "d_out overlaps d_x without being equal to it");
  if (overlap(d_out, no, d_pos, n * 4) || overlap(d_out, no, d_table, n_pos * rot * 4)) return set_error(LMGC_EINVAL, "buffers overlap");
  const RopeArgs a{d_x, d_out, ldx, ldhx, ldo, ldho, dtype, (int)n, heads, hd, rot, layout, backward != 0, d_pos, d_table, n_pos};
  return done(launch_rope(a, (hipStream_t)stream), "rope");
}

int lmgc_op_paged_append(const void* d_k, const void* d_v, int32_t dtype, int64_t ldk, int64_t ldv, int32_t n, int32_t B, int32_t Hkv,
                         int32_t hd, uint16_t* d_kc, uint16_t* d_vc, int32_t n_pages, int32_t page, const int32_t* d_pages,
                         int32_t max_pages, const int32_t* d_starts, const int32_t* d_lens, const float* d_table, int64_t n_pos,
                         int32_t rot, int32_t layout, const void* d_q, int64_t ldq, int32_t Hq, uint16_t* d_q_out, int64_t ldqo,
                         void* stream) {
  clear_error();
  if (!is_dtype(dtype)) return set_error(LMGC_EINVAL, "unknown dtype %d", dtype);
  int rc = check_sizes(n, B, d_q ? Hq : Hkv, Hkv, hd);
  if (rc) return rc;
  const Ragged r{d_pages, d_starts, d_lens, B, n, max_pages, page, n_pages};
  const Cache cache{d_kc, d_vc, (int64_t)n_pages * Hkv * page * hd * 2};
  if ((rc = check_cache(cache, r))) return rc;
  if (d_table && (rc = check_table(d_table, n_pos, rot, hd, layout))) return rc;
  if (d_q && !d_table) return set_error(LMGC_EINVAL, "queries without a table: nothing to do for them");
  if (!d_q != !d_q_out) return set_error(LMGC_EINVAL, "d_q and d_q_out go together");
  const int64_t size = dtype_bytes(dtype), ek = extent(n, (int64_t)Hkv * hd, ldk, "ldk");
  if (ek < 0) return (int)ek;
  const int64_t ev = extent(n, (int64_t)Hkv * hd, ldv, "ldv");
  if (ev < 0) return (int)ev;
  const int64_t eq = d_q ? extent(n, (int64_t)Hq * hd, ldq, "ldq") : 0;
  if (eq < 0) return (int)eq;
  const int64_t eo = d_q ? extent(n, (int64_t)Hq * hd, ldqo, "ldqo") : 0;
  if (eo < 0) return (int)eo;
  if (n == 0) return LMGC_OK;
  if (!d_k || !d_v) return set_error(LMGC_EINVAL, "NULL device buffer");
  if (!aligned(d_k, size) || !aligned(d_v, size) || !aligned(d_q, size) || !aligned(d_q_out, 2))
    return set_error(LMGC_EINVAL, "k, v and q must be aligned to their elements");
  const int64_t nt = d_table ? n_pos * rot * 4 : 0;
  if (cache.with(d_k, ek * size) || cache.with(d_v, ev * size) || cache.with(d_q, eq * size) || cache.with(d_q_out, eo * 2) ||
      cache.with(d_table, nt))
    return set_error(LMGC_EINVAL, "a buffer overlaps the cache");
  if (in_batch(d_kc, cache.bytes, r) || in_batch(d_vc, cache.bytes, r) || in_batch(d_q_out, eo * 2, r))
    return set_error(LMGC_EINVAL, "pages, starts or lens overlap what the call writes");
  if (overlap(d_q_out, eo * 2, d_k, ek * size) || overlap(d_q_out, eo * 2, d_v, ev * size) || overlap(d_q_out, eo * 2, d_q, eq * size) ||
      overlap(d_q_out, eo * 2, d_table, nt))
    return set_error(LMGC_EINVAL, "d_q_out overlaps an input");
  const AppendArgs a{d_k, d_v, d_q, ldk, ldv, ldq, ldqo, dtype, d_q ? Hq : Hkv, Hkv, hd, d_table ? rot : 0, layout, d_kc, d_vc, d_q_out,
                     d_table, n_pos, r};
  return done(launch_paged_append(a, (hipStream_t)stream), "append");
}

int64_t lmgc_paged_workspace(int32_t n, int32_t B, int32_t Hq, int32_t Hkv, int32_t hd, int32_t max_new, int32_t tokens, int32_t shared) {
  clear_error();
  int rc = check_sizes(n, B, Hq, Hkv, hd);
  if (rc) return rc;
  if (max_new < 1 || max_new > kMaxTokens || tokens < 1 || tokens > kMaxTokens || shared < 0)
    return set_error(LMGC_EINVAL, "need max_new and tokens in [1, 2^24] and shared >= 0");
  return n ? paged_workspace_bytes(n, B, Hq, Hkv, hd, max_new, tokens, shared) : 0;
}

int lmgc_op_attention_paged(const uint16_t* d_q, int64_t ldq, int32_t n, int32_t B, int32_t Hq, int32_t Hkv, int32_t hd,
                            const uint16_t* d_kc, const uint16_t* d_vc, int32_t n_pages, int32_t page, const int32_t* d_pages,
                            int32_t max_pages, const int32_t* d_starts, const int32_t* d_lens, int32_t max_new, int32_t window,
                            int32_t sinks, int32_t shared, float scale, uint16_t* d_out, void* d_ws, size_t ws_bytes, void* stream) {
  clear_error();
  int rc = check_sizes(n, B, Hq, Hkv, hd);
  if (rc) return rc;
  const Ragged r{d_pages, d_starts, d_lens, B, n, max_pages, page, n_pages};
  const Cache cache{d_kc, d_vc, (int64_t)n_pages * Hkv * page * hd * 2};
  if ((rc = check_cache(cache, r))) return rc;
  if (max_new < 1 || max_new > kMaxTokens) return set_error(LMGC_EINVAL, "max_new must be in [1, 2^24]");
  if (window < 0 || sinks < 0 || shared < 0) return set_error(LMGC_EINVAL, "window, sinks and shared must be >= 0");
  if (!(scale > 0) || !isfinite(scores_scale(scale))) return set_error(LMGC_EINVAL, "scale must be positive and log2(e) of it finite");
  const int64_t eq = extent(n, (int64_t)Hq * hd, ldq, "ldq");
  if (eq < 0) return (int)eq;
  if (n == 0) return LMGC_OK;
  if (!d_q || !d_out) return set_error(LMGC_EINVAL, "NULL device buffer");
  if (!aligned(d_q, 16) || ldq % 8 || !aligned(d_out, 16) || !aligned(d_ws, 16))
    return set_error(LMGC_EINVAL, "pointers must be 16-byte aligned and ldq a multiple of 8");
  const int tokens = max_pages * page;
  if (paged_workgroups(n, B, Hq, Hkv, hd, max_new, tokens, shared, window, sinks) >= 1 << 23)  // 2^32 threads
    return set_error(LMGC_EUNSUPPORTED, "too many columns for one launch");
  const int64_t need = paged_workspace_bytes(n, B, Hq, Hkv, hd, max_new, tokens, shared), no = (int64_t)n * Hq * hd * 2;
  if (need > 0 && (!d_ws || ws_bytes < (size_t)need))
    return set_error(LMGC_ESIZE, "workspace too small: %zu < %lld", d_ws ? ws_bytes : (size_t)0, (long long)need);
  if (overlap(d_q, eq * 2, d_out, no) || overlap(d_ws, need, d_q, eq * 2) || overlap(d_ws, need, d_out, no) || cache.with(d_out, no) ||
      cache.with(d_ws, need))
    return set_error(LMGC_EINVAL, "buffers overlap");
  if (in_batch(d_out, no, r) || in_batch(d_ws, need, r)) return set_error(LMGC_EINVAL, "pages, starts or lens overlap what the call writes");
  const PagedAttnArgs a{d_q, d_kc, d_vc, ldq, Hq, Hkv, hd, max_new, window, sinks, shared, scale, d_out, d_ws, r};
  return done(launch_attention_paged(a, (hipStream_t)stream), "attention");
}

}  // extern "C"
