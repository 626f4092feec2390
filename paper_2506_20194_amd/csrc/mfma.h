// Packed bf16 pairs and the 32-wide MFMA, shared by the attention kernels.
#pragma once

#include "common.h"

namespace duo {

typedef __bf16 bf16v2 __attribute__((ext_vector_type(2)));
typedef float f32v2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const bf16v2 v = __builtin_convertvector(f32v2{lo, hi}, bf16v2);  // round to nearest even
  uint32_t u;
  __builtin_memcpy(&u, &v, 4);
  return u;
}

typedef short s16v4 __attribute__((ext_vector_type(4)));
typedef float f16x __attribute__((ext_vector_type(16)));

__device__ __forceinline__ f16x mma32_bf16(const u32x4& a, const u32x4& b, f16x c) {
  bf16x8 av, bv;
  __builtin_memcpy(&av, &a, 16);
  __builtin_memcpy(&bv, &b, 16);
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(av, bv, c, 0, 0, 0);
}

}  // namespace duo
