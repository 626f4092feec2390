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

// 16 or 4 bytes per lane from base + off; base and lds are the same for all lanes.
__device__ __forceinline__ void dma16(const void* base, uint32_t off, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(off), "s"(base) : "memory");
}
__device__ __forceinline__ void dma4(const void* base, uint32_t off, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(lds), "v"(off), "s"(base) : "memory");
}
// The same from an address per lane.
__device__ __forceinline__ void dma16(const void* at, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds), "v"(at) : "memory");
}
__device__ __forceinline__ void dma4(const void* at, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(lds), "v"(at) : "memory");
}

}  // namespace duo
