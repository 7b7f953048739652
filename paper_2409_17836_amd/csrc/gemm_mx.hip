// Product of microscaled operands: C[M, N] = A[M, K] * B[N, K]^T (+ add) with
// A in e4m3 or e2m1 (rows), B in e2m1 (blocks), on the scaled matrix
// instruction of 16 x 16 x 128, which multiplies each lane's 32 products by
// both blocks' scales and accumulates in float32.
//
// Every output element is one chain of these instructions over rising k,
// whatever M, N and the tile, so a row's result depends on that row of A and
// on B alone.
#include <algorithm>
#include <type_traits>

#include "mx.h"

namespace lmgc {
namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// Lane l = r + 16 g of the instruction: e2m1 operands: columns 32 g .. + 31
// of row r; e4m3 operands: columns 16 g .. + 15 and 64 + 16 g .. + 15.  In
// both the lane gives the scale of columns 32 g .. + 31.
//
// weights x activations: element e of the result is column 4 g + e of the
// block, row r; KS: the stage's byte of the scale words
template <int FMT, int KS>
__device__ inline f32x4 mma(const i32x4& w4, const i32x8& a, f32x4 c, uint32_t sw, uint32_t sa) {
  constexpr int blgp = FMT == LMGC_MX_FP8 ? 0 : 4;
  const i32x8 w = {w4[0], w4[1], w4[2], w4[3], 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, a, c, 4, blgp, KS, (int)sw, KS, (int)sa);
}

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) char* lds_bytes_t;

constexpr int kXcds = 8;
constexpr int kNonTemporal = 2;  // the load's nt bit

// Two floats -> a packed bf16 pair, round to nearest even.
__device__ inline uint32_t pack_bf16(float a, float b) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  const bf16x2 v = {(__bf16)a, (__bf16)b};
  return __builtin_bit_cast(uint32_t, v);
}

// s_waitcnt vmcnt(n) alone (vmcnt bits 3:0 and 15:14)
constexpr int vmcnt_imm(int n) { return (n & 15) | ((n >> 4) << 14) | 0xF70; }
// mask that adds lgkmcnt(0) to it
constexpr int kLgkm0 = 0xF0FF;

// Buffer resource over `bytes` bytes at p (gfx9: stride 0, word 3
// 0x00020000); a lane offset at or past them loads zero.  The scalar offset is
// not counted on in that check: with one, lanes past the end are also past the
// bytes without it.
__device__ inline __amdgpu_buffer_rsrc_t buffer_of(const uint8_t* p, int bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(p), (short)0, bytes, 0x00020000);
}

// 16 bytes a lane from the buffer straight to LDS: lane l's piece lands at
// lds + 16 l.
template <int AUX = 0>
__device__ inline void load_lds(__amdgpu_buffer_rsrc_t rsrc, lds_bytes_t lds, int voff, int soff) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (__attribute__((address_space(3))) void*)lds, 16, voff, soff, 0, AUX);
}

// Rows of COLS float32 values in LDS (COLS + 4 apart) to the output: `rows`
// rows of `nc` columns from element `at` on, N apart.
template <int COLS>
__device__ inline void store_rows(const float* src, int64_t at, int rows, int nc, int N, int lane, const float* add, void* out,
                                  int bf16) {
  constexpr int RS = COLS + 4;
  static_assert(COLS >= 32, "at most 16 rows at once");
  if (bf16) {
    constexpr int PER = 8, LPR = COLS / PER, RPI = 64 / LPR;  // values a lane, lanes a row, rows at once
    const bool vec = (N & 7) == 0;
#pragma unroll
    for (int q = 0; q < 16 / RPI; q++) {
      const int row = q * RPI + lane / LPR, c = lane % LPR * PER;
      if (row >= rows || c >= nc) continue;
      f32x4 v[2] = {*reinterpret_cast<const f32x4*>(src + row * RS + c), *reinterpret_cast<const f32x4*>(src + row * RS + c + 4)};
      const int64_t p = at + (int64_t)row * N + c;
      if (vec) {
        if (add) {
          v[0] += *reinterpret_cast<const f32x4*>(add + p);
          v[1] += *reinterpret_cast<const f32x4*>(add + p + 4);
        }
        const u32x4 w = {pack_bf16(v[0][0], v[0][1]), pack_bf16(v[0][2], v[0][3]), pack_bf16(v[1][0], v[1][1]),
                         pack_bf16(v[1][2], v[1][3])};
        *reinterpret_cast<u32x4*>((uint16_t*)out + p) = w;
      } else {
#pragma unroll
        for (int e = 0; e < 8; e++)
          if (c + e < nc) ((uint16_t*)out)[p + e] = f32_to_bf16(add ? v[e >> 2][e & 3] + add[p + e] : v[e >> 2][e & 3]);
      }
    }
  } else {
    constexpr int PER = 4, LPR = COLS / PER, RPI = 64 / LPR;
    const bool vec = (N & 3) == 0;
#pragma unroll
    for (int q = 0; q < 16 / RPI; q++) {
      const int row = q * RPI + lane / LPR, c = lane % LPR * PER;
      if (row >= rows || c >= nc) continue;
      f32x4 v = *reinterpret_cast<const f32x4*>(src + row * RS + c);
      const int64_t p = at + (int64_t)row * N + c;
      if (vec) {
        if (add) v += *reinterpret_cast<const f32x4*>(add + p);
        *reinterpret_cast<f32x4*>((float*)out + p) = v;
      } else {
#pragma unroll
        for (int e = 0; e < 4; e++)
          if (c + e < nc) ((float*)out)[p + e] = add ? v[e] + add[p + e] : v[e];
      }
    }
  }
}

// Tiles.  A workgroup of WM x WN waves computes BM x BN outputs, a wave BM /
// WM x BN / WN of them as 16 x 16 blocks with the weights as the
// instruction's first operand, so a lane ends up with four neighbouring
// columns of one row.
//
// K advances in stages of 128 bytes of a row of A (one step of 128 columns in
// e4m3, two in e2m1) through a ring of ST stages in LDS.  A load of A takes 8
// rows x 128 bytes: whole cache lines (16 rows x 64 bytes, the lanes' own
// order, moved 37 KB a microsecond and CU where this moves 90 to 117).  Chunk
// c of row r lies at slot c ^ ((r >> 1) & 7) of its row, so that the 16 rows
// that one cycle of an LDS read serves fall on 16 different quads of banks.
// B's 1 KB blocks lie as they are, in the lanes' order.  Scales come in groups
// of four steps, PS groups ahead, through a ring of their own.
//
// Step k: its operands are in registers.  Before the operands of the next
// stage are read: wait for that stage's loads and for the wave's reads of
// this one; barrier; load the stage ST further on into this one's place.
// Then the operands of step k + 1 are read into a second set of registers
// while step k is multiplied.  Past the last stage the loads go on with an
// empty buffer: they move nothing, and the counts of loads in flight stay
// constants.
//
// Large products are bound by the matrix units at the clock that the power
// limit leaves (1.8 to 1.9 GHz): 16384 x 12288 x 4096 in e4m3 567 to 622 us,
// 2.7 to 2.9 PFLOP/s from one machine to the next, in e2m1 470 to 495, 3.4
// (instructions alone, from registers: 4.9 and 5.2; an 8-bit library product of
// 8192^3 2.7); middle ones by a stage's round, waits and barrier included:
// 1000 x 2048 x 5632 in e2m1 12 us from a graph, 14 to 16 with everything from
// memory, 0.27 a step.
//
// ONCE, a single row of tiles: nothing reads the weights again before the next
// step, so they are loaded past the caches' order of use (64 x 22016 x 4096
// from memory 18.4 us for 19.3; with more rows of tiles the others miss them).
template <int FMT, int BM, int BN, int WM, int WN, int ST>
struct Tile {
  static constexpr int NW = WM * WN, PA = FMT == LMGC_MX_FP8 ? 2 : 1, KPS = 2 / PA;  // steps per stage
  static constexpr int G = 4 / KPS;                                                   // stages per group of scales
  static constexpr int LA = BM / 8, LB = BN / 16 * KPS, L = LA + LB;                  // pieces of a stage
  static constexpr int LPA = LA / NW, LPB = LB / NW, LPW = LPA + LPB;                 // loads of a stage, each wave
  static constexpr int SA = (BM + 63) / 64, SB = (BN + 63) / 64, S = SA + SB;  // pieces of a group's scales
  // with fewer pieces than waves, some waves load one again, so that all have
  // the same loads in flight
  static constexpr int SPA = (SA + NW - 1) / NW, SPB = (SB + NW - 1) / NW, SPW = SPA + SPB;
  static constexpr int PS = (ST + G - 1) / G;  // the scales of a group are asked for before the operands of its stages
  static constexpr int FM = BM / WM / 16, FN = BN / WN / 16;
  static constexpr int kStage = L * 1024, kScale = S * 1024;
  static constexpr int kLds = ST * kStage + (PS + 1) * kScale;
  static_assert(LA % NW == 0 && LB % NW == 0 && kLds <= 160 * 1024, "stage does not fit");
  static_assert((ST - 2) * LPW + PS * SPW < 64, "more loads in flight than the wait counts");
  // loads that may be in flight when stage G u + s + 1 is needed: those of
  // the ST - 2 stages after it, and the scales asked for among them
  static constexpr int in_flight(int s) {
    int n = (ST - 2) * LPW;
    for (int i = s - ST + 2; i <= s - 1; i++)
      if (((i % G) + G) % G == 0) n += SPW;
    return n;
  }
};

template <int FMT, int BM, int BN, int WM, int WN, int ST, bool ONCE>
__global__ __launch_bounds__(WM * WN * 64, 1) void gemm_mx_tile_kernel(
    const uint8_t* __restrict__ A, const uint8_t* __restrict__ As, const uint8_t* __restrict__ B,
    const uint8_t* __restrict__ Bs, int M, int N, int nk, int ns, int ntm, int ntn, int gm, const float* add, void* out,
    int bf16) {
  using C = Tile<FMT, BM, BN, WM, WN, ST>;
  __shared__ u32x4 smem[C::kLds / 16];
  int tm, tn;
  {
    // XCD x (workgroups x, x + 8, ..) walks a contiguous range of the tiles,
    // in groups of gm row tiles
    const int per = gridDim.x / kXcds, t = ((int)blockIdx.x % kXcds) * per + (int)blockIdx.x / kXcds;
    if (t >= ntm * ntn) return;
    const int grp = t / (gm * ntn), first = grp * gm, gs = min(ntm - first, gm), r = t - grp * gm * ntn;
    tm = __builtin_amdgcn_readfirstlane(first + r % gs);
    tn = __builtin_amdgcn_readfirstlane(r / gs);
  }
  const int tid = threadIdx.x, lane = tid & 63, r = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave / WN, wn = wave % WN;
  const int64_t m0 = (int64_t)tm * BM;
  const int n0 = tn * BN, mrows = (int)min<int64_t>(BM, M - m0), groups = min(BN / 16, (N + 15) / 16 - n0 / 16);
  const int lda = FMT == LMGC_MX_FP8 ? nk * 128 : nk * 64, nst = (nk + C::KPS - 1) / C::KPS;
  const uint8_t *pa = A + m0 * lda, *psa = As + m0 * ns, *pb = B + (int64_t)(n0 / 16) * nk * 1024,
                *psb = Bs + (int64_t)(n0 / 16) * ns * 16;
  const __amdgpu_buffer_rsrc_t rsa = buffer_of(psa, mrows * ns), rsb = buffer_of(psb, groups * ns * 16);
  const lds_bytes_t lds0 = (lds_bytes_t)(char*)smem;

  // wave w loads pieces w LPA .. of A's part of a stage and w LPB .. of B's,
  // and so with the scales of a group
  int va[C::LPA], vb[C::LPB], vsa[C::SPA], vsb[C::SPB];
#pragma unroll
  for (int i = 0; i < C::LPA; i++) {
    const int row = (wave * C::LPA + i) * 8 + (lane >> 3);
    va[i] = row * lda + (((lane & 7) ^ ((row >> 1) & 7)) << 4);
  }
#pragma unroll
  for (int i = 0; i < C::LPB; i++) {
    const int q = wave * C::LPB + i;
    vb[i] = (q / C::KPS * nk + q % C::KPS) * 1024 + lane * 16;
  }
#pragma unroll
  for (int i = 0; i < C::SPA; i++) vsa[i] = (min(wave * C::SPA + i, C::SA - 1) * 64 + lane) * ns;
#pragma unroll
  for (int i = 0; i < C::SPB; i++)
    vsb[i] = (min(wave * C::SPB + i, C::SB - 1) * 4 + (lane >> 4)) * ns * 16 + (lane & 15) * 16;
  auto load_stage = [&](int s, int slot) __attribute__((always_inline)) {
    const lds_bytes_t at = lds0 + slot * C::kStage;
    // e4m3: stages are whole steps, and their place a scalar offset.  e2m1: of
    // a last stage with one step of two (an odd number of steps) the last row's
    // second half is past the end, so the buffers begin at the stage (590 us
    // for 570 at 16384 x 12288 x 4096 in e4m3, which does not need it).
    const int ka = s * 128, kb = s * (C::KPS * 1024), shift = C::KPS > 1 ? 1 : 0;
    const __amdgpu_buffer_rsrc_t ra = buffer_of(pa + shift * ka, s < nst ? mrows * lda - shift * ka : 0),
                                 rb = buffer_of(pb + shift * kb, s < nst ? groups * nk * 1024 - shift * kb : 0);
#pragma unroll
    for (int i = 0; i < C::LPA; i++) load_lds(ra, at + (wave * C::LPA + i) * 1024, va[i], shift ? 0 : ka);
#pragma unroll
    for (int i = 0; i < C::LPB; i++) load_lds<ONCE ? kNonTemporal : 0>(rb, at + (C::LA + wave * C::LPB + i) * 1024, vb[i], shift ? 0 : kb);
  };
  const int nu = ns / 16;
  auto load_scales = [&](int u) __attribute__((always_inline)) {
    const int uu = min(u, nu - 1);
    const lds_bytes_t at = lds0 + ST * C::kStage + (u % (C::PS + 1)) * C::kScale;
#pragma unroll
    for (int i = 0; i < C::SPA; i++) load_lds(rsa, at + min(wave * C::SPA + i, C::SA - 1) * 1024, vsa[i], uu * 16);
#pragma unroll
    for (int i = 0; i < C::SPB; i++) load_lds(rsb, at + (C::SA + min(wave * C::SPB + i, C::SB - 1)) * 1024, vsb[i], uu * 256);
  };

  f32x4 acc[C::FM][C::FN] = {};
  uint32_t sa[C::FM], sb[C::FN];
  u32x4 a[C::FM][C::PA], b[2][C::FN];
  auto sync = [&](auto s_tag) __attribute__((always_inline)) {
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(vmcnt_imm(C::in_flight(decltype(s_tag)::value)) & kLgkm0);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  };
  // chunk g of the lane's row; chunk 4 + g is 64 bytes away under the xor
  const int arow = (r >> 3) * 64 + (r & 7) * 8 + (g ^ ((r >> 1) & 7));
  // operands of step h of the stage at `slot`: the weights into set p, a row
  // block of A
  auto read_b = [&](int p, int slot, int h) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < C::FN; j++) b[p][j] = smem[slot * (C::kStage / 16) + (C::LA + (wn * C::FN + j) * C::KPS + h) * 64 + lane];
  };
  auto read_a = [&](int i, int slot, int h) __attribute__((always_inline)) {
#pragma unroll
    for (int q = 0; q < C::PA; q++) a[i][q] = smem[slot * (C::kStage / 16) + (wm * C::FM + i) * 128 + (arow ^ (4 * (q + h)))];
  };
  auto scales_at = [&](int u) __attribute__((always_inline)) {
    return (const char*)smem + ST * C::kStage + (u % (C::PS + 1)) * C::kScale;
  };
  auto read_sa = [&](int i, int u) __attribute__((always_inline)) {
    sa[i] = *reinterpret_cast<const uint32_t*>(scales_at(u) + (wm * C::FM + i) * 256 + r * 16 + 4 * g);
  };
  auto read_sb = [&](uint32_t* to, int u) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < C::FN; j++) to[j] = *reinterpret_cast<const uint32_t*>(scales_at(u) + C::SA * 1024 + (wn * C::FN + j) * 256 + lane * 4);
  };
  // what the stages before the first do: the loads alone
#pragma unroll
  for (int u = 0; u < C::PS; u++)
    if (C::G * (u - C::PS) < -ST) load_scales(u);
#pragma unroll
  for (int i = -ST; i < -1; i++) {
    if (i % C::G == 0) load_scales(i / C::G + C::PS);
    load_stage(i + ST, i + ST);
  }
  sync(std::integral_constant<int, C::G - 1>{});
  load_stage(ST - 1, ST - 1);
  read_b(0, 0, 0);
  read_sb(sb, 0);
#pragma unroll
  for (int i = 0; i < C::FM; i++) {
    read_a(i, 0, 0);
    read_sa(i, 0);
  }
  int slot = 0;  // of the stage of step k
  // A step: rows of blocks 0 .. HALF - 1; then (if the next step opens a
  // stage) the meeting of the waves; then the other rows, while the next
  // step's weights are read into the other set and its rows of A into the
  // registers of rows already multiplied.
  constexpr int HALF = C::FM / 2;
  auto step = [&](auto ks_tag, int k) __attribute__((always_inline)) {
    constexpr int KS = decltype(ks_tag)::value, P = KS & 1, H = KS % C::KPS, SG = KS / C::KPS;
    constexpr bool kNext = H == C::KPS - 1;
    auto row = [&](int i) __attribute__((always_inline)) {
      i32x8 av = {};
#pragma unroll
      for (int e = 0; e < 4; e++) {
        av[e] = (int)a[i][0][e];
        av[4 + e] = FMT == LMGC_MX_FP8 ? (int)a[i][C::PA - 1][e] : 0;
      }
#pragma unroll
      for (int j = 0; j < C::FN; j++) acc[i][j] = mma<FMT, KS>(__builtin_bit_cast(i32x4, b[P][j]), av, acc[i][j], sb[j], sa[i]);
    };
#pragma unroll
    for (int i = 0; i < HALF; i++) row(i);
    if constexpr (kNext) {
      const int s = k / C::KPS;
      sync(std::integral_constant<int, SG>{});
      if (SG == 0) load_scales(s / C::G + C::PS);
      load_stage(s + ST, slot);
      slot = slot == ST - 1 ? 0 : slot + 1;
    }
    constexpr int HN = kNext ? 0 : H + 1;
    read_b(P ^ 1, slot, HN);
#pragma unroll
    for (int i = 0; i < HALF; i++) {
      read_a(i, slot, HN);
      if (KS == 3) read_sa(i, (k >> 2) + 1);
    }
#pragma unroll
    for (int i = HALF; i < C::FM; i++) {
      row(i);
      if (i == HALF) {
        // the reads above between this row's products
#pragma unroll
        for (int j = 0; j < C::FN; j++) {
          __builtin_amdgcn_sched_group_barrier(0x100, (C::FN + HALF * C::PA + C::FN - 1) / C::FN, 0);
          __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      read_a(i, slot, HN);
      if (KS == 3) read_sa(i, (k >> 2) + 1);
    }
    if (KS == 3) read_sb(sb, (k >> 2) + 1);
  };
  int k = 0;
  for (; k + 4 <= nk; k += 4) {
    step(std::integral_constant<int, 0>{}, k);
    step(std::integral_constant<int, 1>{}, k + 1);
    step(std::integral_constant<int, 2>{}, k + 2);
    step(std::integral_constant<int, 3>{}, k + 3);
  }
  if (k < nk) {
    step(std::integral_constant<int, 0>{}, k);
    if (k + 1 < nk) {
      step(std::integral_constant<int, 1>{}, k + 1);
      if (k + 2 < nk) step(std::integral_constant<int, 2>{}, k + 2);
    }
  }

  // Results through LDS, a row block of the wave (16 rows x 16 FN columns) at
  // a time, so that memory sees whole lines (8 bytes of 16 rows at once, as
  // the registers have them, made the stores a fifth of the large product's
  // time).  Rows are 16 bytes longer than their values, against bank
  // conflicts.
  __builtin_amdgcn_s_waitcnt(vmcnt_imm(0) & kLgkm0);  // no load to LDS is in flight past this
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  constexpr int COLS = C::FN * 16, RS = COLS + 4;  // floats of a row
  static_assert(C::NW * 16 * RS * 4 <= C::kLds, "epilogue does not fit");
  float* mine = reinterpret_cast<float*>(smem) + wave * 16 * RS;
  const int nw = n0 + wn * COLS, nc = min(COLS, N - nw);  // the wave's columns
#pragma unroll
  for (int i = 0; i < C::FM; i++) {
#pragma unroll
    for (int j = 0; j < C::FN; j++) *reinterpret_cast<f32x4*>(mine + r * RS + 16 * j + 4 * g) = acc[i][j];
    __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
    asm volatile("" ::: "memory");
    const int ml0 = wm * (BM / WM) + 16 * i;
    if (nc > 0 && ml0 < mrows) store_rows<COLS>(mine, (m0 + ml0) * N + nw, min(16, mrows - ml0), nc, N, lane, add, out, bf16);
    asm volatile("" ::: "memory");
  }
}

// Few rows.  A wave by itself takes 16 rows x 16 FN columns and needs no LDS:
// B's blocks and A's rows lie in the operands' order, so a load fills the
// instruction's registers.  D steps are under way: step k's operands are used
// and the loads of step k + D go into their registers.  Bound by the latency
// of memory and then by the bytes of the weights, and with 16 rows by the rows
// of A that every tile fetches, hence wider tiles for more columns.  One matrix
// of weights again and again (out of the Infinity Cache) 1 x 4096 x 4096 3.2 us,
// 16 x 4096 x 11008 8.7 us, 1 x 22016 x 4096 8.6 us; with the operands through
// LDS, whose latency was a step's time, 5.7, 11.5 and 10.4.  Weights from memory
// 3.6, 9.9 and 10.3 us (4.6 TB/s).
template <int FMT, int FN, int D, bool ONCE>
__global__ __launch_bounds__(64) void gemm_mx_rows_kernel(const uint8_t* __restrict__ A, const uint8_t* __restrict__ As,
                                                          const uint8_t* __restrict__ B, const uint8_t* __restrict__ Bs,
                                                          int M, int N, int nk, int ns, const float* add, void* out,
                                                          int bf16) {
  constexpr int PA = FMT == LMGC_MX_FP8 ? 2 : 1, AUX = ONCE ? kNonTemporal : 0;
  static_assert(D % 4 == 0, "whole groups of scales");
  const int lane = threadIdx.x, r = lane & 15, g = lane >> 4;
  const int64_t m0 = (int64_t)blockIdx.y * 16;
  const int n0 = blockIdx.x * 16 * FN, mrows = (int)min<int64_t>(16, M - m0), groups = min(FN, (N + 15) / 16 - n0 / 16);
  const int lda = nk * 64 * PA;
  const uint8_t *pa = A + m0 * lda, *psa = As + m0 * ns, *pb = B + (int64_t)(n0 / 16) * nk * 1024,
                *psb = Bs + (int64_t)(n0 / 16) * ns * 16;
  const int va = r * lda + 16 * g, vsa = r * ns + 4 * g;
  u32x4 a[D][PA], b[D][FN];
  uint32_t sa[D / 4], sb[D / 4][FN];
  // past the last step the buffers are empty: such loads give zeros and move nothing
  auto load = [&](int s, int k) __attribute__((always_inline)) {
    const __amdgpu_buffer_rsrc_t ra = buffer_of(pa, k < nk ? mrows * lda : 0), rb = buffer_of(pb, k < nk ? groups * nk * 1024 : 0);
#pragma unroll
    for (int j = 0; j < FN; j++) b[s][j] = __builtin_amdgcn_raw_buffer_load_b128(rb, j * nk * 1024 + lane * 16, k * 1024, AUX);
#pragma unroll
    for (int q = 0; q < PA; q++) a[s][q] = __builtin_amdgcn_raw_buffer_load_b128(ra, va + 64 * q, k * 64 * PA, 0);
    if (s % 4 == 0) {
      const __amdgpu_buffer_rsrc_t rsa = buffer_of(psa, k < nk ? mrows * ns : 0), rsb = buffer_of(psb, k < nk ? groups * ns * 16 : 0);
      sa[s / 4] = __builtin_amdgcn_raw_buffer_load_b32(rsa, vsa, k * 4, 0);
#pragma unroll
      for (int j = 0; j < FN; j++) sb[s / 4][j] = __builtin_amdgcn_raw_buffer_load_b32(rsb, j * ns * 16 + lane * 4, k * 64, AUX);
    }
  };
  f32x4 acc[FN] = {};
  auto step = [&](auto s_tag) __attribute__((always_inline)) {
    constexpr int S = decltype(s_tag)::value;
    i32x8 av = {};
#pragma unroll
    for (int e = 0; e < 4; e++) {
      av[e] = (int)a[S][0][e];
      av[4 + e] = PA == 2 ? (int)a[S][PA - 1][e] : 0;
    }
#pragma unroll
    for (int j = 0; j < FN; j++) acc[j] = mma<FMT, S % 4>(__builtin_bit_cast(i32x4, b[S][j]), av, acc[j], sb[S / 4][j], sa[S / 4]);
  };
  auto steps = [&](auto self, auto s_tag, int k0, auto loads) __attribute__((always_inline)) -> void {
    constexpr int S = decltype(s_tag)::value;
    if constexpr (S < D) {
      if (!decltype(loads)::value && k0 + S >= nk) return;
      step(s_tag);
      // (the scales of a group are in use to its last step)
      if constexpr (decltype(loads)::value && S % 4 == 3) {
#pragma unroll
        for (int i = S - 3; i <= S; i++) load(i, k0 + D + i);
      }
      self(self, std::integral_constant<int, S + 1>{}, k0, loads);
    }
  };
#pragma unroll
  for (int s = 0; s < D; s++) load(s, s);
  int k = 0;
  for (; k + D < nk; k += D) steps(steps, std::integral_constant<int, 0>{}, k, std::true_type{});
  steps(steps, std::integral_constant<int, 0>{}, k, std::false_type{});

  if (r >= mrows) return;
#pragma unroll
  for (int j = 0; j < FN; j++) {
    const int n = n0 + 16 * j + 4 * g;
    if (n >= N) continue;
    const int64_t at = (m0 + r) * N + n;
    f32x4 v = acc[j];
    if ((N & 3) == 0) {
      if (add) v += *reinterpret_cast<const f32x4*>(add + at);
      if (bf16) *reinterpret_cast<mx_u32x2*>((uint16_t*)out + at) = mx_u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
      else *reinterpret_cast<f32x4*>((float*)out + at) = v;
    } else {
#pragma unroll
      for (int e = 0; e < 4; e++) {
        if (n + e >= N) continue;
        const float x = add ? v[e] + add[at + e] : v[e];
        if (bf16) ((uint16_t*)out)[at + e] = f32_to_bf16(x);
        else ((float*)out)[at + e] = x;
      }
    }
  }
}

template <int FMT, int FN, int D>
void launch_rows(const uint8_t* a, const uint8_t* as, const uint8_t* b, const uint8_t* bs, int M, int N, int K,
                 const float* add, void* out, int bf16, hipStream_t s) {
  const int nk = (int)(mx_cols(K) / 128), ns = (int)mx_row_scales(K);
  const dim3 grid((N + 16 * FN - 1) / (16 * FN), (M + 15) / 16);
  if (M <= 16) gemm_mx_rows_kernel<FMT, FN, D, true><<<grid, 64, 0, s>>>(a, as, b, bs, M, N, nk, ns, add, out, bf16);
  else gemm_mx_rows_kernel<FMT, FN, D, false><<<grid, 64, 0, s>>>(a, as, b, bs, M, N, nk, ns, add, out, bf16);
}

// Row tiles per group of the tile order: an XCD's 32 workgroups then cover
// about as many bytes of A as of B (16384 x 12288 x 4096, e4m3: 573 us with 4,
// 594 with 8, 604 with 16).
constexpr int kGroupM = 4;

template <int FMT, int BM, int BN, int WM, int WN, int ST>
void launch_tile(const uint8_t* a, const uint8_t* as, const uint8_t* b, const uint8_t* bs, int M, int N, int K,
                 const float* add, void* out, int bf16, hipStream_t s) {
  const int nk = (int)(mx_cols(K) / 128), ns = (int)mx_row_scales(K);
  const int ntm = (M + BM - 1) / BM, ntn = (N + BN - 1) / BN;
  const int64_t grid = ((int64_t)ntm * ntn + kXcds - 1) / kXcds * kXcds;
  auto go = [&](auto once) {
    gemm_mx_tile_kernel<FMT, BM, BN, WM, WN, ST, decltype(once)::value><<<(unsigned)grid, WM * WN * 64, 0, s>>>(
        a, as, b, bs, M, N, nk, ns, ntm, ntn, kGroupM, add, out, bf16);
  };
  if (ntm == 1) go(std::true_type{});
  else go(std::false_type{});
}

// The tile with the least modelled time: a fixed part, and for every round of
// tiles over the 256 CUs a part per tile and one per step of 128 columns
// (microseconds, fitted to launches from a graph with N x K of 768 x 768 to
// 22016 x 4096 and 1 to 16384 rows).  At K = 4096, e4m3, the choice and what
// the next tile would take:
//   16 x 4096    16x16   4.3 us   16x32  4.9      16 x 22016    16x64  10.2   16x32 10.5
//   32 x 4096    16x32   4.7      16x64  5.4      64 x 4096     16x64  5.6    16x32 7.0
//   500 x 2048   64x64   8.2      128x64 11.6     512 x 4096    128x64 12.3   64x64 13.0
//   1000 x 4096  128x128 17.6     128x64 22.4     2048 x 4096   128x256 28.9  128x128 30.5
//   4096 x 4096  256x256 51.2     128x128 56.6    16384 x 12288 256x256 567   128x256 630
// The first three are gemm_mx_rows_kernel's: many waves to a CU, so their
// rounds are counted in fractions.  256x256 is left to e4m3: with e2m1 128x256
// is as fast (16384 x 4096 x 11008: 364 and 365 us).
int pick_tile(int fmt, int64_t M, int64_t N, int K) {
  struct Cost {
    int bm, bn;
    double fixed, tile, step;
  };
  constexpr int kTiles = LMGC_MX_TILE_256X256 + 1;
  static const Cost cost[2][kTiles] = {
      {{16, 16, 2.0, 0, 0.080}, {16, 32, 2.0, 0, 0.085}, {16, 64, 2.0, 0, 0.118}, {64, 64, 2.0, 0.7, 0.146}, {128, 64, 2.5, 0.9, 0.285},
       {128, 128, 2.5, 0.9, 0.400}, {128, 256, 2.5, 2.5, 0.720}, {256, 256, 4.0, 3.5, 1.330}},
      {{16, 16, 2.0, 0, 0.052}, {16, 32, 2.0, 0, 0.062}, {16, 64, 2.0, 0, 0.092}, {64, 64, 2.3, 0.9, 0.125}, {128, 64, 2.5, 0.9, 0.210},
       {128, 128, 2.5, 1.2, 0.290}, {128, 256, 2.5, 3.0, 0.530}, {256, 256, 0, 1e30, 0}}};
  const int nk = (int)(mx_cols(K) / 128);
  int best = LMGC_MX_TILE_64X64;
  double least = 1e300;
  for (int t = 0; t < kTiles; t++) {
    const Cost& c = cost[fmt == LMGC_MX_FP8 ? 0 : 1][t];
    const int64_t tiles = (M + c.bm - 1) / c.bm * ((N + c.bn - 1) / c.bn);
    const bool rows = t <= LMGC_MX_TILE_16X64;
    if (rows && M > 1 << 19) continue;  // their grid is two-dimensional
    const double rounds = rows ? std::max(1.0, tiles / 256.0) : (double)((tiles + 255) / 256);
    const double us = c.fixed + rounds * (c.tile + c.step * nk);
    if (us < least) {
      least = us;
      best = t;
    }
  }
  return best;
}

template <int FMT>
void launch_fmt(const uint8_t* a, const uint8_t* as, const uint8_t* b, const uint8_t* bs, int M, int N, int K,
                const float* add, void* out, int bf16, int tile, hipStream_t s) {
  constexpr bool F8 = FMT == LMGC_MX_FP8;
  switch (tile < 0 ? pick_tile(FMT, M, N, K) : tile) {
    case LMGC_MX_TILE_16X16: return launch_rows<FMT, 1, 16>(a, as, b, bs, M, N, K, add, out, bf16, s);
    case LMGC_MX_TILE_16X32: return launch_rows<FMT, 2, 16>(a, as, b, bs, M, N, K, add, out, bf16, s);
    case LMGC_MX_TILE_16X64: return launch_rows<FMT, 4, 8>(a, as, b, bs, M, N, K, add, out, bf16, s);
    case LMGC_MX_TILE_64X64: return launch_tile<FMT, 64, 64, 2, 2, 4>(a, as, b, bs, M, N, K, add, out, bf16, s);
    case LMGC_MX_TILE_128X64: return launch_tile<FMT, 128, 64, 4, F8 ? 1 : 2, F8 ? 4 : 3>(a, as, b, bs, M, N, K, add, out, bf16, s);
    case LMGC_MX_TILE_128X128: return launch_tile<FMT, 128, 128, 4, 2, F8 ? 3 : 2>(a, as, b, bs, M, N, K, add, out, bf16, s);
    case LMGC_MX_TILE_128X256: return launch_tile<FMT, 128, 256, 2, 4, F8 ? 4 : 2>(a, as, b, bs, M, N, K, add, out, bf16, s);
    default:
      if constexpr (F8) launch_tile<FMT, 256, 256, 4, 2, 3>(a, as, b, bs, M, N, K, add, out, bf16, s);
  }
}

}  // namespace

hipError_t launch_gemm_mx(const uint8_t* a, const uint8_t* as, int a_fmt, const uint8_t* b, const uint8_t* bs, int M,
                          int N, int K, const float* add, void* out, int bf16, int tile, hipStream_t s) {
  if (a_fmt == LMGC_MX_FP8) launch_fmt<LMGC_MX_FP8>(a, as, b, bs, M, N, K, add, out, bf16, tile, s);
  else launch_fmt<LMGC_MX_FP4>(a, as, b, bs, M, N, K, add, out, bf16, tile, s);
  return hipGetLastError();
}

}  // namespace lmgc
