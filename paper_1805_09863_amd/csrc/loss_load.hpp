// What the losses' kernels share for values in memory and in lanes: 16 bytes at any element's address, and DPP moves.
#pragma once

#include "kb_common.hpp"

namespace kb {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 AnyU32x4 __attribute__((aligned(2)));  // 16 bytes at any element
typedef f32x4 AnyF32x4 __attribute__((aligned(4)));

// An element as float32.
__device__ __forceinline__ float widen(const uint16_t* p, size_t i) { return __uint_as_float((uint32_t)p[i] << 16); }
__device__ __forceinline__ float widen(const float* p, size_t i) { return p[i]; }

// 16 bytes from p on as float32.
__device__ __forceinline__ void load16(const uint16_t* p, float* x) {
  const u32x4 w = *reinterpret_cast<const AnyU32x4*>(p);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void load16(const float* p, float* x) {
  const f32x4 v = *reinterpret_cast<const AnyF32x4*>(p);
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = v[i];
}

template <int CTRL>
__device__ __forceinline__ float dpp_of(float x) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, true));
}

}  // namespace kb
