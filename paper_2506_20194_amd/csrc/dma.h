// Loads from global memory into LDS that the compiler does not see as such.  It would
// wait for all of them before every transposing LDS read (it cannot tell that they go
// elsewhere), which takes away what loading ahead is for; here the caller waits, with
// wait_vm, before it reads what they bring.  There is no output register: the wave's
// data go to the 64 consecutive places from `lds` on, in lane order.
#pragma once

#include "common.h"

namespace duo {

// LDS address of a pointer into shared memory.
__device__ __forceinline__ uint32_t lds_addr(const void* p) {
  return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void*)p;
}

// m0 says where in LDS the loads go, and is named as changed.  The compiler warns (400 times, silenced
// here) that it may not keep what it has in m0 itself across such a block: nothing else in the kernels
// that use this file may need m0, and tests/test_dma_listing_cpu.py looks at what was compiled.
//
// A scalar address is moved here, by a scalar instruction: a load needs five wait states behind a
// vector instruction that wrote its address (a lane read, such as brings back a spilled register),
// and the compiler inserts none for loads that it does not see.  The move is also the one
// wait state that a load needs behind a write of m0.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
#define DUO_DMA_TO "s_mov_b32 m0, %1\n\ts_mov_b64 %0, %2\n\t"

// 16 or 4 bytes per lane from base + off; base and lds are the same for all lanes.
__device__ __forceinline__ void dma16(const void* base, uint32_t off, uint32_t lds) {
  const void* at;
  asm volatile(DUO_DMA_TO "global_load_lds_dwordx4 %3, %0" : "=&s"(at) : "s"(lds), "s"(base), "v"(off) : "memory", "m0");
}
__device__ __forceinline__ void dma4(const void* base, uint32_t off, uint32_t lds) {
  const void* at;
  asm volatile(DUO_DMA_TO "global_load_lds_dword %3, %0" : "=&s"(at) : "s"(lds), "s"(base), "v"(off) : "memory", "m0");
}
// N (2, 4 or 8) loads of 16 bytes per lane from consecutive KiB: load i from base + 1024 i +
// off[i] to lds + 1024 i (the instruction's offset counts for both sides).
template <int N>
__device__ __forceinline__ void dma16_run(const uint8_t* base, const uint32_t (&off)[N], uint32_t lds) {
  static_assert(N == 2 || N % 4 == 0, "");
  const void* at;
  if constexpr (N == 2)
    asm volatile(DUO_DMA_TO
                 "global_load_lds_dwordx4 %3, %0\n\t"
                 "global_load_lds_dwordx4 %4, %0 offset:1024"
                 : "=&s"(at) : "s"(lds), "s"(base), "v"(off[0]), "v"(off[1]) : "memory", "m0");
  else
#pragma unroll
    for (int i = 0; i < N; i += 4)
      asm volatile(DUO_DMA_TO
                   "global_load_lds_dwordx4 %3, %0\n\t"
                   "global_load_lds_dwordx4 %4, %0 offset:1024\n\tglobal_load_lds_dwordx4 %5, %0 offset:2048\n\t"
                   "global_load_lds_dwordx4 %6, %0 offset:3072"
                   : "=&s"(at)
                   : "s"(lds + 1024 * i), "s"(base + 1024 * i), "v"(off[i]), "v"(off[i + 1]), "v"(off[i + 2]), "v"(off[i + 3])
                   : "memory", "m0");
}
#undef DUO_DMA_TO
// The same from an address per lane.
__device__ __forceinline__ void dma16(const void* at, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds), "v"(at) : "memory", "m0");
}
__device__ __forceinline__ void dma4(const void* at, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(lds), "v"(at) : "memory", "m0");
}
#pragma clang diagnostic pop

}  // namespace duo
