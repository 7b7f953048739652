// Rotary positions: the table of angles, and the rotation of rows of heads.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "common.h"
#include "paged.h"

namespace lmgc {
namespace {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// ------------------------------------------------------------------- table
// table[p, i] = mscale (cos, sin)(p freqs[i]), angles and functions in float64:
// at position 2^17 a float32 angle is off by 2^-7.  A thread has kPositions
// positions of a frequency, from a multiple of kPositions on: it turns the first
// one's (cos, sin) by the frequency, in float64, for the next ones.  A step adds
// two roundings, 2^-49 to the last of a run; the angle p f itself is rounded, 2^-53 of it
// (2^-36 at 2^17 and 2^-29 at 2^24 radians, of float32's 2^-24).
// 131072 positions of 64 frequencies, 67 MB, take 12.7 us (5.3 TB/s), bound by the
// stores; 31 with a sine and a cosine for each.
struct Freqs {
  double f[kMaxRot / 2];
};
constexpr int kPositions = 8;

__global__ __launch_bounds__(256) void rope_table_kernel(Freqs freqs, int half, double mscale, int n_pos, float2* __restrict__ table) {
  // thread number / half, of which the block's first is the same for all lanes
  const int64_t first = (int64_t)blockIdx.x * 256;
  const int64_t p0 = first / half;
  const int rest = (int)(first - p0 * half) + threadIdx.x, more = rest / half, i = rest - more * half;
  const int64_t p = (p0 + more) * kPositions;
  if (p >= n_pos) return;
  const double f = freqs.f[i];
  double s, c, ds, dc;
  sincos((double)p * f, &s, &c);
  sincos(f, &ds, &dc);
  float2* o = table + p * half + i;
  const int n = (int)min((int64_t)kPositions, n_pos - p);
  for (int k = 0; k < n; k++) {
    o[(int64_t)k * half] = make_float2((float)(c * mscale), (float)(s * mscale));
    const double t = c * dc - s * ds;
    s = s * dc + c * ds;
    c = t;
  }
}

// ---------------------------------------------------------------- rotation
// 16 bytes of a row to a run; a thread has the two runs of as many pairs, of
// the same place in kHeads heads, so a pair's cos and sin are read once for them.
// Bound by memory: 8191 rows of 36 heads of 64, float32, 151 MB, take 35.6 us (4.27
// TB/s; a copy 5.15); 37.4 with one head's loads at a time.  16384 rows of 64 heads of
// 128, bf16, take 96 us; number by number (not FAST) 211, and 298 where rot is 100.
template <class T>
struct Run;
template <>
struct Run<float> {
  static constexpr int n = 4;
  f32x4 v;
  __device__ inline float get(int i) const { return v[i]; }
  __device__ inline void set(const float* y) { v = f32x4{y[0], y[1], y[2], y[3]}; }
};
template <>
struct Run<uint16_t> {
  static constexpr int n = 8;
  u32x4 v;
  __device__ inline float get(int i) const { return __builtin_bit_cast(float, i & 1 ? v[i >> 1] & 0xffff0000u : v[i >> 1] << 16); }
  __device__ inline void set(const float* y) {
#pragma unroll
    for (int i = 0; i < 4; i++) v[i] = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)y[2 * i], (__bf16)y[2 * i + 1]});
  }
};

__device__ inline float load1(const float* p) { return *p; }
__device__ inline float load1(const uint16_t* p) { return bf16_to_f32(*p); }
__device__ inline void store1(float* p, float x) { *p = x; }
__device__ inline void store1(uint16_t* p, float x) { *p = f32_to_bf16(x); }

// Grid: (heads / kHeads, blocks of rows), 256 threads: np places of a row side
// by side.  FAST: rot a multiple of two runs, hd of a run, everything 16-byte
// aligned.
constexpr int kHeads = 2;
constexpr int kRowBlocks = 32768;  // in one plane of the grid

template <class T, bool FAST>
__global__ __launch_bounds__(256) void rope_kernel(RopeArgs a, int np, int rows, int per) {
  constexpr int R = Run<T>::n;
  const int place = threadIdx.x % np;
  const int64_t row = ((int64_t)blockIdx.z * kRowBlocks + blockIdx.y) * rows + threadIdx.x / np;
  if ((int)threadIdx.x >= rows * np || row >= a.n) return;
  const int64_t pos = a.pos[row];
  if (pos < 0 || pos >= a.n_pos) return;
  const int half = a.rot / 2, h0 = blockIdx.x * per, h1 = min(a.heads, h0 + per);
  const float2* tab = reinterpret_cast<const float2*>(a.table) + pos * half;
  const T* x = static_cast<const T*>(a.x) + row * a.ldx;
  T* o = static_cast<T*>(a.out) + row * a.ldo;
  const bool copy = a.x != a.out;  // (in place, what does not rotate stays)
  if (FAST) {
    const int nrot = half / R;
    if (place < nrot) {
      const int d0 = a.layout == LMGC_ROPE_HALF ? place * R : place * 2 * R, d1 = a.layout == LMGC_ROPE_HALF ? d0 + half : d0 + R;
      float c[R], s[R];
#pragma unroll
      for (int i = 0; i < R; i += 2) {
        const f32x4 w = *reinterpret_cast<const f32x4*>(tab + place * R + i);
        c[i] = w[0], s[i] = a.backward ? -w[1] : w[1], c[i + 1] = w[2], s[i + 1] = a.backward ? -w[3] : w[3];
      }
      // the numbers of kHeads heads are asked for at once
      for (int g0 = h0; g0 < h1; g0 += kHeads) {
        Run<T> us[kHeads], vs[kHeads];
#pragma unroll
        for (int k = 0; k < kHeads; k++) {
          const int h = min(g0 + k, h1 - 1);
          us[k].v = *reinterpret_cast<const decltype(us[k].v)*>(x + h * a.ldhx + d0);
          vs[k].v = *reinterpret_cast<const decltype(us[k].v)*>(x + h * a.ldhx + d1);
        }
#pragma unroll
        for (int k = 0; k < kHeads; k++) {
          const int h = g0 + k;
          if (h >= h1) break;
          const Run<T> u = us[k], v = vs[k];
          float y[R], z[R];
          if (a.layout == LMGC_ROPE_HALF) {
#pragma unroll
            for (int i = 0; i < R; i++) {
              const float p = u.get(i), q = v.get(i);
              y[i] = turn_first(p, q, c[i], s[i]);
              z[i] = turn_second(p, q, c[i], s[i]);
            }
          } else {
#pragma unroll
            for (int i = 0; i < R; i++) {
              const float p = i < R / 2 ? u.get(2 * i) : v.get(2 * i - R), q = i < R / 2 ? u.get(2 * i + 1) : v.get(2 * i + 1 - R);
              (i < R / 2 ? y[2 * i] : z[2 * i - R]) = turn_first(p, q, c[i], s[i]);
              (i < R / 2 ? y[2 * i + 1] : z[2 * i + 1 - R]) = turn_second(p, q, c[i], s[i]);
            }
          }
          Run<T> out;
          out.set(y);
          *reinterpret_cast<decltype(out.v)*>(o + h * a.ldho + d0) = out.v;
          out.set(z);
          *reinterpret_cast<decltype(out.v)*>(o + h * a.ldho + d1) = out.v;
        }
      }
    } else if (copy) {
      const int d0 = a.rot + (place - nrot) * 2 * R;
      for (int h = h0; h < h1; h++)
        for (int d = d0; d < min(a.hd, d0 + 2 * R); d += R)
          *reinterpret_cast<decltype(Run<T>::v)*>(o + h * a.ldho + d) = *reinterpret_cast<const decltype(Run<T>::v)*>(x + h * a.ldhx + d);
    }
  } else {
    // a pair, or two numbers that do not rotate
    for (int i = place; i < (a.hd + 1) / 2; i += np)
      for (int h = h0; h < h1; h++) {
        const T* xh = x + h * a.ldhx;
        T* oh = o + h * a.ldho;
        if (i < half) {
          const int d0 = a.layout == LMGC_ROPE_HALF ? i : 2 * i, d1 = a.layout == LMGC_ROPE_HALF ? i + half : 2 * i + 1;
          const float c = tab[i].x, s = a.backward ? -tab[i].y : tab[i].y, p = load1(xh + d0), q = load1(xh + d1);
          store1(oh + d0, turn_first(p, q, c, s));
          store1(oh + d1, turn_second(p, q, c, s));
        } else if (copy) {
          for (int d = 2 * i; d < min(a.hd, 2 * i + 2); d++) oh[d] = xh[d];
        }
      }
  }
}

}  // namespace

hipError_t launch_rope_table(const double* freqs, int rot, double mscale, int64_t n_pos, float* table, hipStream_t s) {
  Freqs f{};
  for (int i = 0; i < rot / 2; i++) f.f[i] = freqs[i];
  const int64_t n = (n_pos + kPositions - 1) / kPositions * (rot / 2);
  rope_table_kernel<<<(unsigned)((n + 255) / 256), 256, 0, s>>>(f, rot / 2, mscale, (int)n_pos, (float2*)table);
  return hipGetLastError();
}

hipError_t launch_rope(const RopeArgs& a, hipStream_t s) {
  auto go = [&](auto t) {
    using T = decltype(t);
    constexpr int R = Run<T>::n;
    auto whole = [](int64_t x) { return x % R == 0; };
    const bool fast = a.rot % (2 * R) == 0 && whole(a.hd) && whole(a.ldx) && whole(a.ldhx) && whole(a.ldo) && whole(a.ldho) &&
                      ((uintptr_t)a.x & 15) == 0 && ((uintptr_t)a.out & 15) == 0;
    const int np = fast ? a.rot / 2 / R + (a.hd - a.rot + 2 * R - 1) / (2 * R) : std::min((a.hd + 1) / 2, 64);
    const int rows = 256 / np;
    const int64_t blocks = ((int64_t)a.n + rows - 1) / rows;
    // two heads to a thread where one fills the chip: 8 rows of 64 heads of 128 take 2.17
    // us with one and 2.30 with two, 512 rows 4.47 and 3.98 (four: 3.97), 8192 47.0 and 45.6
    // (47.2)
    const int per = blocks * a.heads >= 512 ? kHeads : 1;
    const dim3 grid((a.heads + per - 1) / per, std::min<int64_t>(blocks, kRowBlocks), (blocks + kRowBlocks - 1) / kRowBlocks);
    if (fast) rope_kernel<T, true><<<grid, 256, 0, s>>>(a, np, rows, per);
    else rope_kernel<T, false><<<grid, 256, 0, s>>>(a, np, rows, per);
  };
  if (a.dtype == LMGC_DTYPE_BF16) go(uint16_t{});
  else go(float{});
  return hipGetLastError();
}

}  // namespace lmgc
