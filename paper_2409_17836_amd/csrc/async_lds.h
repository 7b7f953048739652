// Loads from memory straight to LDS that stay under way across barriers.
#ifndef LMGC_ASYNC_LDS_H
#define LMGC_ASYNC_LDS_H

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace lmgc {

// A place in LDS.
typedef uint32_t LdsAt;
__device__ inline LdsAt lds_at(void* p) { return (LdsAt)(uintptr_t)(__attribute__((address_space(3))) char*)p; }

// 16 bytes a lane from p (the same for all lanes) + at bytes to LDS, lane l's at
// to + 16 l.  In assembly: with the builtin the compiler waits for every load
// before any read of the ring; the waits are written out where they belong
// (wait_loads).
__device__ inline void load_lds(const void* p, uint32_t at, LdsAt to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" :: "s"(to), "v"(at), "s"(p) : "m0", "memory");
}

// Waits until at most n of the wave's loads are under way.
template <int n>
__device__ inline void wait_loads() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((n & 15) | ((n >> 4) << 14) | 0xF70);  // vmcnt(n) alone
  asm volatile("" ::: "memory");
}

// Waits for the wave's LDS accesses and meets the others; its loads go on
// (__syncthreads would wait for them).
__device__ inline void meet() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// Holds values where they are: the compiler would move what makes them to their
// use.
template <class T, int n>
__device__ inline void keep(T (&x)[n]) {
#pragma unroll
  for (int i = 0; i < n; i++) asm volatile("" : "+v"(x[i]));
}

}  // namespace lmgc

#endif
