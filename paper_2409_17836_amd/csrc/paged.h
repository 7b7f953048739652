// Launches of the rotary positions (rope.hip) and of the paged key/value cache
// (paged.hip); arguments as in lmgc.h, checked by the callers.
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

namespace lmgc {

constexpr int kMaxRot = 512;  // dims of a head that rotate, at most

// A batch of ragged rows over a paged cache: sequence b has rows starts[b] ..
// starts[b + 1] - 1, lens[b] tokens before them, and its tokens on pages[b, :].
struct Ragged {
  const int32_t* pages;
  const int32_t* starts;
  const int32_t* lens;
  int B, n, max_pages, page, n_pages;
};

// (a, b) turned by the angle of (c, s): the same bits wherever it is done.
__device__ inline float turn_first(float a, float b, float c, float s) { return fmaf(a, c, -(b * s)); }
__device__ inline float turn_second(float a, float b, float c, float s) { return fmaf(a, s, b * c); }

hipError_t launch_rope_table(const double* freqs, int rot, double mscale, int64_t n_pos, float* table, hipStream_t s);

// Rows ld, heads ldh elements apart (x and out).
struct RopeArgs {
  const void* x;
  void* out;
  int64_t ldx, ldhx, ldo, ldho;
  int dtype, n, heads, hd, rot, layout, backward;
  const int32_t* pos;
  const float* table;
  int64_t n_pos;
};
hipError_t launch_rope(const RopeArgs& a, hipStream_t s);

struct AppendArgs {
  const void *k, *v, *q;  // q: nullable
  int64_t ldk, ldv, ldq, ldqo;
  int dtype, Hq, Hkv, hd, rot, layout;
  uint16_t *kc, *vc, *q_out;
  const float* table;  // nullable: no rotation
  int64_t n_pos;
  Ragged r;
};
hipError_t launch_paged_append(const AppendArgs& a, hipStream_t s);

struct PagedAttnArgs {
  const uint16_t *q, *kc, *vc;
  int64_t ldq;
  int Hq, Hkv, hd, max_new, window, sinks, shared;
  float scale;
  uint16_t* out;
  void* ws;
  Ragged r;
};
// Of scores in powers of two.
inline float scores_scale(float scale) { return (float)(1.4426950408889634 * (double)scale); }
int64_t paged_workspace_bytes(int n, int B, int Hq, int Hkv, int hd, int max_new, int tokens, int shared);
// Workgroups of the largest launch in one dimension (other launches have heads and
// sequences in two of their own).
int64_t paged_workgroups(int n, int B, int Hq, int Hkv, int hd, int max_new, int tokens, int shared, int window, int sinks);
hipError_t launch_attention_paged(const PagedAttnArgs& a, hipStream_t s);

}  // namespace lmgc
