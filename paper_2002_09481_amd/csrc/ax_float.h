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

// Activations.  EXACT: for results in float32, otherwise for results that are rounded to bf16, with the fast exponential and
// reciprocal: relative errors of 1.2e-4 at most, far out, where 2^-9 is half a unit.
//
// The normal distribution function of gelu is exp(-z^2 / 2) t P(t) for z < 0 and one minus that for z > 0, t = 1 / (1 + c |z|).
// P is fitted to the scaled function over 0 <= |z| <= 14.2, so that the tail keeps its leading digits where it is far below one:
// nine coefficients for the smallest largest relative error, 1.3e-8, and six within 5.4e-8 and, where that says less, relatively
// within 1.1e-4.  Evaluated in float32, over -12.5 < z < 12.5: z times the long form within 7.7 2^-24 of it, the short form
// within 2.2e-7 and relatively within 1.2e-4.  (The library's erf takes three times the instructions of the short form, and
// 1 + erf has no digits left in the tail.)
__device__ __forceinline__ float rcp_near(float d) {  // 1 / d of normal d, to within a unit in the last place
  const float t = __builtin_amdgcn_rcpf(d);
  return __builtin_fmaf(__builtin_fmaf(-d, t, 1.0f), t, t);
}
// exp(x + low) of a finite x <= 0 and a low below x's last place: 2^(x log2 e) with what the product loses put back.
__device__ __forceinline__ float exp_near(float x, float low) {
  const float q = x * 1.44269504f, r = __builtin_fmaf(x, 1.44269504f, -q);
  const float e = __builtin_amdgcn_exp2f(q);
  return __builtin_fmaf(e, __builtin_fmaf(x, 1.92596303e-8f * 0.693147181f, __builtin_fmaf(r, 0.693147181f, low)), e);
}
template <bool EXACT>
__device__ __forceinline__ float gauss_of(float x) {  // exp(-x^2 / 2) of x >= 0 (EXACT: up to 64)
  if (!EXACT) return __expf(-0.5f * x * x);
  const float q = x * x;
  return exp_near(-0.5f * q, -0.5f * __builtin_fmaf(x, x, -q));
}
template <bool EXACT>
__device__ __forceinline__ float normal_cdf(float z, float& gauss) {  // gauss = exp(-z^2 / 2)
  const float x = EXACT && fabsf(z) > 64.f ? 64.f : fabsf(z);  // (NaN stays; both are 0 or 1 from there on)
  gauss = gauss_of<EXACT>(x);
  float p;
  const float d = __builtin_fmaf(x, EXACT ? 0.265f : 0.29f, 1.0f);
  const float t = EXACT ? rcp_near(d) : __builtin_amdgcn_rcpf(d);
  if (EXACT) {
    p = __builtin_fmaf(t, 0.0307411347f, -0.143851921f);
    p = __builtin_fmaf(t, p, 0.217057899f);
    p = __builtin_fmaf(t, p, -0.115519196f);
    p = __builtin_fmaf(t, p, 0.137384608f);
    p = __builtin_fmaf(t, p, 0.0605500154f);
    p = __builtin_fmaf(t, p, 0.102641486f);
    p = __builtin_fmaf(t, p, 0.105254889f);
    p = __builtin_fmaf(t, p, 0.105741084f);
  } else {
    p = __builtin_fmaf(t, -0.0892740786f, 0.286521465f);
    p = __builtin_fmaf(t, p, -0.0954555646f);
    p = __builtin_fmaf(t, p, 0.181015849f);
    p = __builtin_fmaf(t, p, 0.100275196f);
    p = __builtin_fmaf(t, p, 0.116917126f);
  }
  const float tail = p * t * gauss;
  return z > 0.f ? 1.f - tail : tail;
}
// 1 / (1 + exp(-z)), and one minus it
template <bool EXACT>
__device__ __forceinline__ float sigmoid(float z, float& rest) {
  if (!EXACT) {
    const float g = __builtin_amdgcn_rcpf(1.f + __expf(-z));
    rest = 1.f - g;
    return g;
  }
  const float x = fabsf(z) > 128.f ? 128.f : fabsf(z);  // (NaN stays; the exponential is 0 from there on)
  const float e = exp_near(-x, 0.f), r = rcp_near(1.f + e), s = e * r;
  rest = z > 0.f ? s : r;
  return z > 0.f ? r : s;
}

template <bool EXACT, int E>
__device__ __forceinline__ void apply_act(float (&v)[E], int act) {
  switch (act) {
    case AX_ACT_RELU:
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] = v[e] < 0.f ? 0.f : v[e];  // NaN stays
      break;
    case AX_ACT_SILU:
#pragma unroll
      for (int e = 0; e < E; ++e) {
        float rest;
        v[e] *= sigmoid<EXACT>(v[e], rest);
      }
      break;
    case AX_ACT_GELU:
#pragma unroll
      for (int e = 0; e < E; ++e) {
        float gauss;
        const float y = v[e] * normal_cdf<EXACT>(v[e], gauss);
        v[e] = v[e] < -14.2f ? -0.f : y;  // (-infinity times zero; the product is below float32 there)
      }
      break;
    default: break;
  }
}
// v = act(z), s = act'(z)
template <bool EXACT, int E>
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
        float rest;
        const float g = sigmoid<EXACT>(z[e], rest);
        v[e] = z[e] * g;
        s[e] = g * (1.f + z[e] * rest);
      }
      break;
    case AX_ACT_GELU:
#pragma unroll
      for (int e = 0; e < E; ++e) {
        float gauss;
        const float c = normal_cdf<EXACT>(z[e], gauss);
        v[e] = z[e] < -14.2f ? -0.f : z[e] * c;
        s[e] = c + (gauss > 0.f ? z[e] * gauss * 0.39894228040143268f : 0.f);
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
