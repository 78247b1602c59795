// Element types and activations shared by the float operators (norm, products, gated block, optimizer).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "axconv.h"

namespace ax {

__device__ __forceinline__ float bf16_to_f32(uint32_t b) { return __uint_as_float(b << 16); }
// To nearest, ties to even; NaN stays NaN.
__device__ __forceinline__ uint32_t f32_to_bf16(float f) {
  __bf16 h = (__bf16)f;
  return (uint32_t)__builtin_bit_cast(unsigned short, h);
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) { return f32_to_bf16(lo) | (f32_to_bf16(hi) << 16); }

// Activations in float32: one exponential and one reciprocal (both good to a few units in the last place), against
// results that are rounded to bf16 or compared at 2e-5.
__device__ __forceinline__ float act_of(float z, int act) {
  switch (act) {
    case AX_ACT_RELU: return z < 0.f ? 0.f : z;  // NaN stays
    case AX_ACT_SILU: return z / (1.f + __expf(-z));
    case AX_ACT_GELU: return 0.5f * z * (1.f + erff(z * 0.70710678118654752f));
    default: return z;
  }
}
__device__ __forceinline__ float act_slope(float z, int act) {
  switch (act) {
    case AX_ACT_RELU: return z > 0.f ? 1.f : 0.f;
    case AX_ACT_SILU: {
      const float s = 1.f / (1.f + __expf(-z));
      return s * (1.f + z * (1.f - s));
    }
    case AX_ACT_GELU:
      return 0.5f * (1.f + erff(z * 0.70710678118654752f)) + z * __expf(-0.5f * z * z) * 0.39894228040143268f;
    default: return 1.f;
  }
}

}  // namespace ax
