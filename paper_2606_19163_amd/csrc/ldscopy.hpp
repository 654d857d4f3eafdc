// Tiles that go straight from memory to LDS, and waves that meet over them
// (kgrad.hip, lin8.hip).  LDS is read by ordinary loads, whose registers the
// compiler keeps until they have arrived; the copies are inline, since behind its
// own builtin the compiler makes every LDS read wait for all copies in flight.  A
// copy writes no register, and as it and the meetings count as touching all
// memory, no read moves across them.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace pulse {

__device__ __forceinline__ uint32_t lds_at(const void* p) {
  return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) char*)p;
}

// 16 bytes of each lane from `from` to LDS, lane l's to lds + 16 l (the same lds on
// all lanes).  It counts in vmcnt; m0 takes a wait state to be read.
__device__ __forceinline__ void lds_copy16(const void* from, uint32_t lds) {
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(from), "{m0}"(lds) : "memory");
#endif
}

// All waves of the block meet: this wave's reads of LDS have arrived, and of its
// copies all but the last N.  What the others copied before their own meeting, as
// far as they waited for it, may be read, and what was read may be overwritten.
template <int N>
__device__ __forceinline__ void lds_meet() {
#if defined(__HIP_DEVICE_COMPILE__)
  static_assert(N >= 0 && N < 64, "vmcnt");
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"i"(N) : "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
#endif
}

// a contiguous range of n blocks per XCD, of which the hardware takes turns
__device__ __forceinline__ int xcd_order(int b, int n) {
  const int q = n >> 3, r = n & 7, x = b & 7;
  return x * q + (x < r ? x : r) + (b >> 3);
}

}  // namespace pulse
