// Device helpers shared by grad_rows.hip and grad_products.hip.
#pragma once

#include <hip/hip_runtime.h>

#include "grad.h"

namespace lm {
namespace {

typedef __bf16 bf16;
typedef _Float16 f16;
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

// 16 bytes at the address of a 16-bit or a 32-bit element, with the non-temporal hint.
typedef unsigned u32x4_at2 __attribute__((ext_vector_type(4), aligned(2)));
typedef unsigned u32x4_at4 __attribute__((ext_vector_type(4), aligned(4)));
template <typename T>
__device__ __forceinline__ void store16_nt(T* p, u32x4 v) {
  if constexpr (sizeof(T) == 2) __builtin_nontemporal_store(u32x4_at2(v), reinterpret_cast<u32x4_at2*>(p));
  else __builtin_nontemporal_store(u32x4_at4(v), reinterpret_cast<u32x4_at4*>(p));
}

// The factor 2^e of a scale byte e + 127.
__device__ __forceinline__ float scale_of(uint32_t byte) { return __builtin_bit_cast(float, byte << 23); }

// Values of eight codes of one block.
__device__ __forceinline__ void decode8(u32x2 c, float scale, float v[8]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(c[h], false);
    const f32x2 hi = __builtin_amdgcn_cvt_pk_f32_fp8(c[h], true);
    v[4 * h] = lo[0] * scale;
    v[4 * h + 1] = lo[1] * scale;
    v[4 * h + 2] = hi[0] * scale;
    v[4 * h + 3] = hi[1] * scale;
  }
}

}  // namespace
}  // namespace lm
