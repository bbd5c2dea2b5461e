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

// Eight consecutive elements of a row as floats. The 16-byte accesses are
// unaligned ones as far as the compiler knows (the hardware takes any address,
// and aligned ones at full speed), so one path serves every stride; only the last
// elements of a row, n < 8 of them, go one at a time.
template <typename T>
__device__ __forceinline__ void load8(const T* p, int64_t n, float v[8]) {
  if (n >= 8) {
    T t[8];
    __builtin_memcpy(t, p, sizeof(t));
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = float(t[j]);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = j < n ? float(p[j]) : 0.0f;
  }
}

// 16 bytes at the address of a 16-bit or a 32-bit element, with the non-temporal hint.
typedef unsigned u32x4_at2 __attribute__((ext_vector_type(4), aligned(2)));
typedef unsigned u32x4_at4 __attribute__((ext_vector_type(4), aligned(4)));
template <typename T>
__device__ __forceinline__ void store16_nt(T* p, u32x4 v) {
  if constexpr (sizeof(T) == 2) __builtin_nontemporal_store(u32x4_at2(v), reinterpret_cast<u32x4_at2*>(p));
  else __builtin_nontemporal_store(u32x4_at4(v), reinterpret_cast<u32x4_at4*>(p));
}

// 16-bit results leave with the non-temporal hint: a wave writes whole lines of
// tensors that no cache on the way will be asked for (32768 x 4096 bf16 from a
// checkpoint: 112 us without, 58 with it, 6.9 TB/s; gated activation's gradient 314 -> 230).
// In fp32 a lane's 32 bytes are two stores that each fill half a line, and the hint
// costs more than it gives (restore 41 -> 67 us at 32768 x 1280).
template <typename T>
__device__ __forceinline__ void store8(T* p, int64_t n, const float v[8]) {
  if (n >= 8) {
    T t[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) t[j] = T(v[j]);
    if constexpr (sizeof(T) == 2) {
      u32x4 x;
      __builtin_memcpy(&x, t, 16);
      store16_nt(p, x);
    } else {
      __builtin_memcpy(p, t, sizeof(t));
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < n) p[j] = T(v[j]);
  }
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
