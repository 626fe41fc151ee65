// Global -> LDS loads and the waits of an LDS ring: what the contractions' tile
// loops share.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace fxpq {

// s_waitcnt immediate that waits until at most n vector memory operations are
// outstanding (gfx9 encoding: vmcnt split over bits 3:0 and 15:14; expcnt and
// lgkmcnt left at their maxima, i.e. not waited for).
template <int N>
__device__ inline void wait_vmcnt() {
  static_assert(N >= 0 && N < 64, "vmcnt range");
  __builtin_amdgcn_s_waitcnt((N & 0xF) | ((N >> 4) << 14) | (0x7 << 4) | (0xF << 8));
}

// One 16-byte global -> LDS load per lane (global_load_lds_dwordx4): lane l's
// bytes land at lds + 16 l.  Issued as inline asm so that the compiler does
// not add its own conservative wait for these LDS writes before later LDS
// reads (it cannot tell the ring stages apart); the ring waits explicitly
// (wait_vmcnt) and orders with ring_barrier().  M0 holds the wave-uniform LDS
// address; the s_nop separates its write from the load.
__device__ inline void dma16(const int8_t* g, int8_t* lds) {
  const uint32_t l = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)lds);
  asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(g), "{m0}"(l) : "memory");
}

// The same from a wave-uniform address and a byte offset of each lane.
__device__ inline void dma16(const void* base, uint32_t offset, int8_t* lds) {
  const uint32_t l = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)lds);
  asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(offset), "s"(base), "{m0}"(l) : "memory");
}

// One 4-byte load per lane: lane l's bytes land at lds + 4 l.
__device__ inline void dma4(const void* g, int8_t* lds) {
  const uint32_t l = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)lds);
  asm volatile("s_nop 0\n\tglobal_load_lds_dword %0, off" ::"v"(g), "{m0}"(l) : "memory");
}

// Workgroup barrier without the memory fence __syncthreads() adds: that fence
// would wait for every outstanding LDS-ring load.  The empty asm statements
// keep the compiler from moving memory accesses across it.
__device__ inline void ring_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

}  // namespace fxpq
