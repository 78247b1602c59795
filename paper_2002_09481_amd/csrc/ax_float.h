// Element types and activations shared by the float operators (norm, products, gated block, optimizer).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>
#include <type_traits>

#include "ax_internal.h"

namespace ax {

// Stores, like load_any, at an address of any alignment: rows of odd length start anywhere, and global memory takes
// accesses of 16 bytes there too, at the cost of the extra lines that they touch.
template <typename T>
__device__ __forceinline__ void store_any(void* p, const T& v) {
  __builtin_memcpy(p, &v, sizeof(T));
}

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float bf16_to_f32(uint32_t b) { return __uint_as_float(b << 16); }
// To nearest, ties to even; NaN stays NaN.
__device__ __forceinline__ uint32_t f32_to_bf16(float f) {
  __bf16 h = (__bf16)f;
  return (uint32_t)__builtin_bit_cast(unsigned short, h);
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) { return f32_to_bf16(lo) | (f32_to_bf16(hi) << 16); }

// E (4 or 8) elements from element i of p on, `left` of them in the row (zeros behind).
template <bool F32, int E>
__device__ __forceinline__ void load_elems(const void* p, long long i, int left, float (&v)[E]) {
  if (left >= E) {
    if (F32) {
#pragma unroll
      for (int h = 0; h < E / 4; ++h) {
        const f32x4 t = load_any<f32x4>((const float*)p + i + 4 * h);
        for (int e = 0; e < 4; ++e) v[4 * h + e] = t[e];
      }
    } else if (E == 8) {
      const u32x4 t = load_any<u32x4>((const uint16_t*)p + i);
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] = bf16_to_f32((t[e >> 1] >> (16 * (e & 1))) & 0xffffu);
    } else {
      const u32x2 t = load_any<u32x2>((const uint16_t*)p + i);
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] = bf16_to_f32((t[(e >> 1) & 1] >> (16 * (e & 1))) & 0xffffu);
    }
    return;
  }
#pragma unroll
  for (int e = 0; e < E; ++e)
    v[e] = e >= left ? 0.f : F32 ? ((const float*)p)[i + e] : bf16_to_f32(((const uint16_t*)p)[i + e]);
}
template <bool F32, int E>
__device__ __forceinline__ void store_elems(void* p, long long i, int left, const float (&v)[E]) {
  if (left >= E) {
    if (F32) {
#pragma unroll
      for (int h = 0; h < E / 4; ++h) store_any((float*)p + i + 4 * h, f32x4{v[4 * h], v[4 * h + 1], v[4 * h + 2], v[4 * h + 3]});
    } else if (E == 8) {
      store_any((uint16_t*)p + i, u32x4{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4 % E], v[5 % E]),
                                        pack_bf16(v[6 % E], v[7 % E])});
    } else {
      store_any((uint16_t*)p + i, u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])});
    }
    return;
  }
#pragma unroll
  for (int e = 0; e < E; ++e)
    if (e < left) {
      if (F32) ((float*)p)[i + e] = v[e];
      else ((uint16_t*)p)[i + e] = (uint16_t)f32_to_bf16(v[e]);
    }
}

// Eight float32 values in three pieces, smallest pieces last: v = p0 + p1 + p2 exactly (down to 2^-133, the least that a bf16
// holds), each piece what is left, rounded to nearest.  So the pieces of a product that are left out (p1 q2, p2 q1, p2 q2) are
// within 2^-24 (1 + 2^-8) of it, of either sign: 2^-27 in the root mean square over normal factors.  (Pieces that are cut
// instead have the value's sign: up to 7.8 2^-24 left out, 0.7 on average, always towards zero.)  A value that would round to
// infinity has its first piece cut.  An infinity or a NaN goes into the first piece alone; what it meets comes out as NaN
// or infinity (not always the one that float32 gives: a piece of the other factor may be zero).
__device__ __forceinline__ void pieces_of(const float (&v)[8], u32x4 (&p)[3]) {
  uint32_t top = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(v[e]) & 0x7fffffffu);
  const bool plain = top < 0x7f7f8000u;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    float r[2] = {v[2 * e], v[2 * e + 1]};
    uint32_t q = pack_bf16(r[0], r[1]);
    if (!plain) {
      q = 0;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t b = __float_as_uint(r[h]), a = b & 0x7fffffffu;
        q |= (a < 0x7f7f8000u ? f32_to_bf16(r[h]) : (b >> 16) | (a > 0x7f800000u ? 0x40u : 0u)) << (16 * h);
      }
    }
    p[0][e] = q;
    r[0] -= __uint_as_float(q << 16);
    r[1] -= __uint_as_float(q & 0xffff0000u);
    if (!plain) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
        if ((__float_as_uint(v[2 * e + h]) & 0x7f800000u) == 0x7f800000u) r[h] = 0.f;
    }
    p[1][e] = q = pack_bf16(r[0], r[1]);
    r[0] -= __uint_as_float(q << 16);
    r[1] -= __uint_as_float(q & 0xffff0000u);
    p[2][e] = (__float_as_uint(r[0]) >> 16) | (__float_as_uint(r[1]) & 0xffff0000u);
  }
}

// Activations in float32, with the fast exponential and reciprocal (a few units in the last place each), against results
// that are rounded to bf16 or compared in the norm.  The normal distribution function of gelu is 7.1.26 of Abramowitz and
// Stegun's Handbook of Mathematical Functions: erfc(x) = (a1 t + ... + a5 t^5) exp(-x^2) with t = 1 / (1 + 0.3275911 x),
// off by at most 1.5e-7 for x >= 0, here with the halves of the coefficients and x = |z| / sqrt 2.  (The library's erf
// takes three times as many instructions: 17 us for a 256 x 256 tile of a compute unit, of 86 for the whole tile.)
__device__ __forceinline__ float normal_cdf(float z, float gauss) {  // gauss = exp(-z^2 / 2)
  const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(fabsf(z), 0.231641888f, 1.0f));
  float p = __builtin_fmaf(t, 0.5307027145f, -0.7265760135f);
  p = __builtin_fmaf(t, p, 0.7107068705f);
  p = __builtin_fmaf(t, p, -0.142248368f);
  p = __builtin_fmaf(t, p, 0.127414796f);
  const float tail = p * t * gauss;
  return z > 0.f ? 1.f - tail : tail;
}
__device__ __forceinline__ float sigmoid(float z) { return __builtin_amdgcn_rcpf(1.f + __expf(-z)); }
__device__ __forceinline__ float gelu(float z) {
  const float y = z * normal_cdf(z, __expf(-0.5f * z * z));
  return z < -14.f ? -0.f : y;  // (-infinity times zero; the product is below float32 there)
}

template <int E>
__device__ __forceinline__ void apply_act(float (&v)[E], int act) {
  switch (act) {
    case AX_ACT_RELU:
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] = v[e] < 0.f ? 0.f : v[e];  // NaN stays
      break;
    case AX_ACT_SILU:
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] *= sigmoid(v[e]);
      break;
    case AX_ACT_GELU:
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] = gelu(v[e]);
      break;
    default: break;
  }
}
// v = act(z), s = act'(z)
template <int E>
__device__ __forceinline__ void act_and_slope(const float (&z)[E], int act, float (&v)[E], float (&s)[E]) {
  switch (act) {
    case AX_ACT_RELU:
#pragma unroll
      for (int e = 0; e < E; ++e) {
        v[e] = z[e] < 0.f ? 0.f : z[e];
        s[e] = z[e] > 0.f ? 1.f : 0.f;
      }
      break;
    case AX_ACT_SILU:
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float g = sigmoid(z[e]);
        v[e] = z[e] * g;
        s[e] = g * (1.f + z[e] * (1.f - g));
      }
      break;
    case AX_ACT_GELU:
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float x = __expf(-0.5f * z[e] * z[e]), c = normal_cdf(z[e], x);
        v[e] = z[e] < -14.f ? -0.f : z[e] * c;
        s[e] = c + (x > 0.f ? z[e] * x * 0.39894228040143268f : 0.f);
      }
      break;
    default:
#pragma unroll
      for (int e = 0; e < E; ++e) {
        v[e] = z[e];
        s[e] = 1.f;
      }
  }
}

}  // namespace ax
