// The kernels of the paged cache on the CPU (tests/cpu_hip): appending to it and
// attention over it for batches whose pages, rows and lengths are partly out of
// range, against plain loops in float64.  Pools, batch and results lie against
// pages that may not be touched.  Prints "ok".
#include <sys/mman.h>

#include <hip/hip_runtime.h>

typedef __bf16 cpu_bf16x8 __attribute__((ext_vector_type(8)));
typedef float cpu_f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t cpu_u32x4 __attribute__((ext_vector_type(4)));

// The 16x16x32 matrix instruction: lane (i, g) gives row (column) i and 8 of the
// products' terms from 8 g on, and takes rows 4 g .. of column i.
static cpu_bf16x8 g_a[64 * 16], g_b[64 * 16];
static cpu_f32x4 cpu_mfma(cpu_bf16x8 a, cpu_bf16x8 b, cpu_f32x4 c) {
  const unsigned t = threadIdx.x, w = t & ~63u, l = t & 63;
  g_a[t] = a;
  g_b[t] = b;
  cpu_hip::wait(cpu_hip::kWave);
  for (int r = 0; r < 4; r++)
    for (int k = 0; k < 32; k++)
      c[r] = fmaf((float)g_a[w + 4 * (l >> 4) + r + 16 * (k / 8)][k % 8], (float)g_b[w + (l & 15) + 16 * (k / 8)][k % 8], c[r]);
  cpu_hip::wait(cpu_hip::kWave);
  return c;
}
// The 32x32x16 one: lane (i, h) gives row (column) i and 8 terms from 8 h on, and
// takes rows 8 (r / 4) + 4 h + r % 4 of column i.
typedef float cpu_f32x16 __attribute__((ext_vector_type(16)));
static cpu_f32x16 cpu_mfma32(cpu_bf16x8 a, cpu_bf16x8 b, cpu_f32x16 c) {
  const unsigned t = threadIdx.x, w = t & ~63u, l = t & 63;
  g_a[t] = a;
  g_b[t] = b;
  cpu_hip::wait(cpu_hip::kWave);
  for (int r = 0; r < 16; r++)
    for (int k = 0; k < 16; k++)
      c[r] = fmaf((float)g_a[w + 8 * (r / 4) + 4 * (l >> 5) + r % 4 + 32 * (k / 8)][k % 8], (float)g_b[w + (l & 31) + 32 * (k / 8)][k % 8], c[r]);
  cpu_hip::wait(cpu_hip::kWave);
  return c;
}
typedef __bf16 cpu_bf16x2 __attribute__((ext_vector_type(2)));
static float cpu_dot2(cpu_bf16x2 a, cpu_bf16x2 b, float c) { return fmaf((float)a[1], (float)b[1], fmaf((float)a[0], (float)b[0], c)); }
struct CpuBuffer {
  const char* p;
  int n;
};
static cpu_u32x4 cpu_load(CpuBuffer b, int v, int s) {
  if (v + s < 0 || v + s + 16 > b.n) abort();
  return *(const cpu_u32x4*)(b.p + v + s);
}
#define __amdgpu_buffer_rsrc_t CpuBuffer
#define __builtin_amdgcn_make_buffer_rsrc(p, stride, n, flags) (CpuBuffer{(const char*)(p), n})
#define __builtin_amdgcn_raw_buffer_load_b128(b, v, s, aux) cpu_load(b, v, s)
#define __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, x, y, z) cpu_mfma(a, b, c)
#define __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, x, y, z) cpu_mfma32(a, b, c)
#define __builtin_amdgcn_fdot2_f32_bf16(a, b, c, x) cpu_dot2(a, b, c)
#define __builtin_amdgcn_readfirstlane(x) __shfl(x, 0)
#define __builtin_amdgcn_exp2f(x) exp2f(x)
#define __builtin_amdgcn_sched_barrier(x)
#define __builtin_amdgcn_sched_group_barrier(a, b, c)
#undef hipLaunchKernelGGL
#define hipLaunchKernelGGL(kernel, grid, block, lds, stream, ...) launch_3d(grid, block, [&] { kernel(__VA_ARGS__); })
// csrc/async_lds.h for the CPU: loads take place as early (when they are asked
// for) or as late (when they are waited for) as they may.
#define LMGC_ASYNC_LDS_H
#include <deque>
static bool g_late;
struct CpuLoad {
  const void* p;
  void* to;
};
static std::deque<CpuLoad> g_loads[1024];
namespace lmgc {
typedef char* LdsAt;
inline LdsAt lds_at(void* p) { return (LdsAt)p; }
inline void load_lds(const void* p, uint32_t at, LdsAt lds) {
  p = (const char*)p + at;
  volatile char probe = *(const volatile char*)p;
  (void)probe;
  const CpuLoad l{p, lds + 16 * (threadIdx.x & 63)};
  if (g_late) g_loads[threadIdx.x].push_back(l);
  else memcpy(l.to, l.p, 16);
}
template <int n>
void wait_loads() {
  auto& q = g_loads[threadIdx.x];
  for (; (int)q.size() > n; q.pop_front()) memcpy(q.front().to, q.front().p, 16);
}
inline void meet() { __syncthreads(); }
template <class T, int n>
void keep(T (&)[n]) {}
}  // namespace lmgc
inline float2 make_float2(float a, float b) { return {a, b}; }
static int min(int a, int b) { return a < b ? a : b; }
static int max(int a, int b) { return a > b ? a : b; }
static int64_t min(int64_t a, int64_t b) { return a < b ? a : b; }
static int64_t max(int64_t a, int64_t b) { return a > b ? a : b; }
template <class F>
static void launch_3d(dim3 grid, dim3 block, F body) {
  const std::function<void()> f = body;
  cpu_hip::g_grid_dim = grid;
  cpu_hip::g_block_dim = block;
  for (unsigned z = 0; z < grid.z; z++)
    for (unsigned y = 0; y < grid.y; y++)
      for (unsigned x = 0; x < grid.x; x++) {
        cpu_hip::g_block = dim3(x, y, z);
        cpu_hip::run_block(block.x, f);
      }
}

#include "../paper_2409_17836_amd/csrc/paged.hip"

#include <random>

using namespace lmgc;

static char* guarded(size_t bytes) {
  const size_t gap = 64 << 20, page = 4096, body = (bytes + page - 1) / page * page + page;
  char* p = (char*)mmap(nullptr, 2 * gap + body, PROT_NONE, MAP_PRIVATE | MAP_ANONYMOUS | MAP_NORESERVE, -1, 0);
  if (p == MAP_FAILED || mprotect(p + gap, body, PROT_READ | PROT_WRITE)) abort();
  return p + gap + (body - bytes) / 16 * 16;
}
template <class T>
static T* copy(const std::vector<T>& v) {
  T* p = (T*)guarded(v.size() * sizeof(T));
  std::copy(v.begin(), v.end(), p);
  return p;
}
static void check(bool ok, const char* what, int at) {
  if (ok) return;
  printf("%s (%d)\n", what, at);
  exit(1);
}

struct Case {
  int hd, page, Hkv, G, window, sinks, shared, max_new, rot, layout;
  std::vector<int> starts, lens, pages;  // pages: max_pages of each sequence
  int n, n_pages;
};

static int at_key(int t, int d, int hd) { return ((t / 16) * (hd / 32) + d / 32) * 512 + ((t % 16) + 16 * ((d % 32) / 8)) * 8 + d % 8; }
static int at_value(int t, int d) { return (d / 16) * 512 + ((d % 16) + 16 * ((t % 16) / 4)) * 8 + 4 * (t / 16) + t % 4; }

static void run(const Case& c, int id) {
  const int B = (int)c.lens.size(), most = (int)c.pages.size() / B, tokens = most * c.page, Hq = c.Hkv * c.G, hd = c.hd;
  std::mt19937 rng(id + 1);
  std::normal_distribution<float> normal;
  const size_t pool = (size_t)c.n_pages * c.Hkv * c.page * hd;
  std::vector<uint16_t> kc(pool), vc(pool), q((size_t)c.n * Hq * hd), k((size_t)c.n * c.Hkv * hd), v(k.size());
  for (auto* x : {&q, &k, &v})
    for (auto& e : *x) e = f32_to_bf16(normal(rng));
  for (auto* x : {&kc, &vc})
    for (auto& e : *x) e = rng() % 4 == 0 ? 0x7fc1 : f32_to_bf16(normal(rng));  // stale places: NaN among them
  std::vector<float> table((size_t)tokens * c.rot);
  for (int p = 0; p < tokens; p++)
    for (int i = 0; i < c.rot / 2; i++) {
      table[(size_t)p * c.rot + 2 * i] = (float)cos(p * pow(100.0, -2.0 * i / c.rot));
      table[(size_t)p * c.rot + 2 * i + 1] = (float)sin(p * pow(100.0, -2.0 * i / c.rot));
    }
  // what of the batch counts
  std::vector<int> T(B);
  for (int b = 0; b < B; b++) {
    const bool ok = c.starts[b] >= 0 && c.starts[b + 1] >= c.starts[b] && c.starts[b + 1] <= c.n && c.lens[b] >= 0 && c.lens[b] < tokens;
    T[b] = ok ? std::min(c.starts[b + 1] - c.starts[b], tokens - c.lens[b]) : 0;
  }
  auto place = [&](int b, int p, int h) -> int64_t {
    const int page = c.pages[b * most + p / c.page];
    return page < 0 || page >= c.n_pages ? -1 : (((int64_t)page * c.Hkv + h) * c.page + p % c.page / 32 * 32) * hd;
  };
  auto rotate = [&](const uint16_t* x, int p, std::vector<float>& y) {
    for (int d = 0; d < hd; d++) y[d] = bf16_to_f32(x[d]);
    for (int i = 0; i < c.rot / 2; i++) {
      const int d0 = c.layout == LMGC_ROPE_HALF ? i : 2 * i, d1 = c.layout == LMGC_ROPE_HALF ? i + c.rot / 2 : 2 * i + 1;
      const float a = y[d0], b = y[d1], co = table[(size_t)p * c.rot + 2 * i], si = table[(size_t)p * c.rot + 2 * i + 1];
      y[d0] = a * co - b * si;
      y[d1] = a * si + b * co;
    }
  };
  // earlier tokens: finite numbers in their places
  for (int b = 0; b < B; b++)
    for (int p = 0; p < (T[b] ? c.lens[b] : 0); p++)
      for (int h = 0; h < c.Hkv; h++) {
        const int64_t at = place(b, p, h);
        for (int d = 0; d < hd && at >= 0; d++) {
          kc[at + at_key(p % 32, d, hd)] = f32_to_bf16(normal(rng));
          vc[at + at_value(p % 32, d)] = f32_to_bf16(normal(rng));
        }
      }
  uint16_t *gk = copy(kc), *gv = copy(vc), *gq = (uint16_t*)guarded(q.size() * 2);
  std::fill(gq, gq + q.size(), (uint16_t)0x1234);
  const Ragged r{copy(c.pages), copy(c.starts), copy(c.lens), B, c.n, most, c.page, c.n_pages};
  AppendArgs a{copy(k), copy(v), copy(q), c.Hkv * hd, c.Hkv * hd, Hq * hd, Hq * hd, LMGC_DTYPE_BF16, Hq, c.Hkv, hd, c.rot, c.layout,
               gk, gv, gq, copy(table), tokens, r};
  launch_paged_append(a, nullptr);
  std::vector<uint16_t> wq(q.size(), 0x1234);
  std::vector<float> y(hd);
  for (int b = 0; b < B; b++)
    for (int t = 0; t < T[b]; t++) {
      const int row = c.starts[b] + t, p = c.lens[b] + t;
      for (int h = 0; h < c.Hkv; h++) {
        const int64_t at = place(b, p, h);
        rotate(&k[((size_t)row * c.Hkv + h) * hd], p, y);
        for (int d = 0; d < hd && at >= 0; d++) {
          kc[at + at_key(p % 32, d, hd)] = f32_to_bf16(y[d]);
          vc[at + at_value(p % 32, d)] = v[((size_t)row * c.Hkv + h) * hd + d];
        }
      }
      for (int h = 0; h < Hq; h++) {
        rotate(&q[((size_t)row * Hq + h) * hd], p, y);
        for (int d = 0; d < hd; d++) wq[((size_t)row * Hq + h) * hd + d] = f32_to_bf16(y[d]);
      }
    }
  auto near = [](uint16_t a, uint16_t b) { return abs((int)(a & 0x7fff) - (int)(b & 0x7fff)) <= 1; };  // (a contraction may move a rounding)
  for (size_t i = 0; i < pool; i++) check(near(gk[i], kc[i]), "key", (int)i);
  for (size_t i = 0; i < pool; i++) check(gv[i] == vc[i], "value", (int)i);
  for (size_t i = 0; i < q.size(); i++) check(near(gq[i], wq[i]), "query", (int)i);
  std::copy(gk, gk + pool, kc.begin());

  // attention, with rows of no token marked
  std::copy(gq, gq + q.size(), wq.begin());
  uint16_t* out = (uint16_t*)guarded(q.size() * 2);
  std::fill(out, out + q.size(), (uint16_t)0x1234);
  const int max_new = c.max_new;
  const int64_t bytes = paged_workspace_bytes(c.n, B, Hq, c.Hkv, hd, max_new, tokens, c.shared);
  char* ws = guarded(bytes);
  memset(ws, 0xff, bytes);
  const PagedAttnArgs p{gq, gk, gv, Hq * hd, Hq, c.Hkv, hd, max_new, c.window, c.sinks, c.shared, 0.125f, out, ws, r};
  launch_attention_paged(p, nullptr);
  for (auto& l : g_loads) check(l.empty(), "a load outlives its kernel", id);
  std::vector<bool> token(c.n, false);
  for (int b = 0; b < B; b++)
    for (int t = 0; t < std::min(T[b], c.max_new); t++) {
      const int row = c.starts[b] + t, pos = c.lens[b] + t;
      token[row] = true;
      for (int h = 0; h < Hq; h++) {
        std::vector<double> s(pos + 1), o(hd, 0.0);
        double sum = 0, mx = -1e300;
        for (int j = 0; j <= pos; j++) {
          const int64_t at = place(b, j, h / c.G);
          s[j] = -1e300;
          if (at < 0 || (c.window && j <= pos - c.window && j >= c.sinks)) continue;
          double z = 0;
          for (int d = 0; d < hd; d++) z += (double)bf16_to_f32(wq[((size_t)row * Hq + h) * hd + d]) * bf16_to_f32(kc[at + at_key(j % 32, d, hd)]);
          s[j] = 0.125 * z;
          mx = std::max(mx, s[j]);
        }
        for (int j = 0; j <= pos; j++) {
          if (s[j] == -1e300) continue;
          const double e = exp(s[j] - mx);
          const int64_t at = place(b, j, h / c.G);
          sum += e;
          for (int d = 0; d < hd; d++) o[d] += e * bf16_to_f32(vc[at + at_value(j % 32, d)]);
        }
        for (int d = 0; d < hd; d++) {
          const double want = sum > 0 ? o[d] / sum : 0.0, got = bf16_to_f32(out[((size_t)row * Hq + h) * hd + d]);
          // each probability, and the result, is off by half a step of bf16 at most (and by float32 sums)
          double dev = 0;
          for (int j = 0; j <= pos; j++)
            if (s[j] != -1e300) dev += exp(s[j] - mx) / sum * fabs(bf16_to_f32(vc[place(b, j, h / c.G) + at_value(j % 32, d)]) - want);
          if (!(fabs(got - want) <= dev * (0x1p-8 + 0x1p-12) + fabs(want) * 0x1p-8)) {
            printf("row %d head %d dim %d: %g, not %g\n", row, h, d, got, want);
            check(false, "attention", id);
          }
        }
      }
    }
  for (int row = 0; row < c.n; row++)
    for (int i = 0; i < Hq * hd && !token[row]; i++) check(out[(size_t)row * Hq * hd + i] == 0x1234, "a row of no token", row);
}

int main() {
  const int big = 1 << 30;
  std::vector<Case> cases = {
      // a whole batch, lengths on every side of groups and pages, rows behind the last
      {64, 32, 2, 2, 0, 0, 0, 99, 64, LMGC_ROPE_HALF, {0, 1, 36, 36, 37}, {40, 0, 5, 31}, {3, 4, 7, 0, 1, 2, 5, 6, 7, 8, 9, 10}, 40, 12},
      // pages outside the pool, lengths and rows outside theirs
      {64, 32, 1, 4, 0, 0, 0, 99, 32, LMGC_ROPE_INTERLEAVED, {0, 20, 21, 22, 23, 24}, {35, 70, -1, 96, 20}, {0, -1, 2, 3, 99, 5, 6, 7, 8, 9, 10, 11, -5, big, 12}, 30, 13},
      {64, 32, 1, 1, 0, 0, 0, 99, 64, LMGC_ROPE_HALF, {-3, 2, 4, 3, 900, big}, {1, 2, 3, 4, 5}, {0, 1, 2, 3, 4, 5, 6, 7, 8, 9}, 6, 10},
      {64, 32, 1, 1, 0, 0, 0, 99, 64, LMGC_ROPE_HALF, {0, 2, 5}, {10, 60}, {-1, -1, 3, -1}, 5, 4},
      // rows past the pages' end, more rows than max_new
      {128, 64, 1, 2, 0, 0, 0, 3, 128, LMGC_ROPE_HALF, {0, 30, 36}, {110, 64}, {0, 1, 2, 3}, 36, 4},
      // windows and sinks, part of the head, a rotation that is no multiple of 16
      {128, 32, 1, 1, 20, 3, 0, 99, 36, LMGC_ROPE_HALF, {0, 3, 4}, {90, 7}, {0, 1, 2, 3, 4, 5, 6, 7}, 4, 8},
      {64, 32, 2, 1, 33, 0, 0, 99, 6, LMGC_ROPE_INTERLEAVED, {0, 50}, {70}, {5, 3, 1, 0}, 50, 6},
      // a prefix of two pages in common, one sequence without rows, one inside the prefix
      {64, 32, 1, 4, 0, 0, 66, 99, 64, LMGC_ROPE_HALF, {1, 2, 2, 9}, {70, 80, 66}, {0, 1, 2, 0, 1, 3, 0, 1, 4}, 11, 5},
      {64, 32, 2, 1, 40, 5, 64, 99, 64, LMGC_ROPE_HALF, {0, 1, 3}, {64, 90}, {0, 1, 2, 3, 0, 1, 4, 5}, 3, 6},
      {64, 32, 1, 1, 0, 0, 64, 99, 64, LMGC_ROPE_HALF, {0, 1, 3}, {64, 70}, {-1, 1, 2, -1, 1, 3}, 3, 4},
      // many columns: several tiles, ragged ends, a page that is not there, few columns beside them
      {64, 32, 1, 8, 0, 0, 0, 999, 64, LMGC_ROPE_HALF, {0, 70, 71, 83}, {0, 40, 50}, {3, 4, 5, 6, 0, -1, 7, 8, 1, 2, 99, 9}, 84, 10},
      {128, 64, 1, 3, 70, 5, 0, 999, 128, LMGC_ROPE_HALF, {0, 90}, {260}, {0, 1, 2, 3, 4, 5}, 90, 6},
      {64, 32, 2, 2, 0, 0, 0, 40, 64, LMGC_ROPE_HALF, {0, 60}, {550}, {19, 18, 17, 16, 15, 14, 13, 12, 11, 10, 9, 8, 7, 6, 5, 4, 3, 2, 1, 0}, 60, 20},
      // many columns behind a prefix, rows of no token among them
      {64, 32, 1, 4, 0, 0, 64, 999, 64, LMGC_ROPE_HALF, {2, 40, 41, 61}, {64, 80, 70}, {0, 1, 2, 3, 0, 1, 4, 5, 0, 1, 6, 7}, 63, 8},
      {64, 32, 1, 4, 50, 3, 64, 999, 64, LMGC_ROPE_HALF, {0, 40, 60}, {64, 90}, {0, 1, 2, 3, 0, 1, 4, 5}, 60, 8},
      // more rows than max_new, which has many columns; and few of one part, beside others
      {64, 32, 1, 16, 0, 0, 0, 40, 64, LMGC_ROPE_HALF, {0, 50, 52}, {20, 70}, {0, 1, 2, 3, 4, 5}, 53, 6},
      {64, 32, 1, 8, 0, 0, 0, 60, 64, LMGC_ROPE_HALF, {0, 30, 33, 93}, {20, 70, 10}, {0, 1, 2, 3, 4, 5, 6, 7, 8}, 94, 9},
      {128, 32, 1, 8, 40, 2, 64, 60, 64, LMGC_ROPE_HALF, {0, 30, 33}, {64, 70}, {0, 1, 2, 3, 0, 1, 4, 5}, 34, 6},
      {128, 64, 1, 4, 0, 0, 0, 20, 128, LMGC_ROPE_HALF, {0, 17, 20}, {500, 40}, {8, 7, 6, 5, 4, 3, 2, 1, 0, 9, 10, 11, 12, 13, 14, 15, 16, 17}, 20, 18},
  };
  // more sequences than a wave has lanes, some without rows, behind a prefix: 140 columns, 280, more than 512
  for (int G : {2, 4, 8}) {
    Case c{64, 32, 1, G, 0, 0, 64, 999, 64, LMGC_ROPE_HALF, {1}, {}, {}, 73, 72};
    for (int b = 0; b < 70; b++) {
      c.starts.push_back(c.starts[b] + (b % 9 == 4 ? 0 : b % 9 == 5 ? 2 : 1));
      c.lens.push_back(64 + b % 30);
      c.pages.insert(c.pages.end(), {0, 1, 2 + b});
    }
    cases.push_back(c);
  }
  for (int late = 0; late < 2; late++) {
    g_late = late;
    for (size_t i = 0; i < cases.size(); i++) run(cases[i], (int)i);
  }
  printf("ok\n");
}
