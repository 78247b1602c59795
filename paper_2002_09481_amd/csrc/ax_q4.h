// Weights of 4 bits in the library's layout (ax_q4.hip), as the kernels read them.
#pragma once

#include "ax_gemm.h"

namespace ax {

typedef uint32_t q4_words __attribute__((ext_vector_type(4)));

struct Q4Weights {
  const uint8_t* codes[2];    // one matrix, or a gated pair
  const uint16_t* scales[2];
  int tiles, blocks;          // of 16 rows and of 128 columns, of an expert's matrix
  int group;
};

// A word holds eight codes, plus eight each: the even ones in the lower half, the odd ones in the upper, so that pairs are a
// shift away from where bf16 pairs have their leading digits.
__host__ __device__ __forceinline__ int q4_shift(int i) { return (i >> 1) * 4 + (i & 1) * 16; }  // of code i

// The eight codes as bf16, exact.  (The conversion takes a code for sixteenths: what comes out is c / 16.)
__device__ __forceinline__ q4_words widen(uint32_t d) {
  q4_words v;
  d ^= 0x88888888u;
  uint32_t odd = d >> 4;
  asm("" : "+v"(odd));  // (kept as it is: the conversions then take bytes of the two words as they lie)
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t b = (i & 1 ? odd : d) >> (8 * (i >> 1));
    const uint32_t lo = __float_as_uint(__builtin_amdgcn_cvt_off_f32_i4((int)(b & 0xffu)));
    const uint32_t hi = __float_as_uint(__builtin_amdgcn_cvt_off_f32_i4((int)(b >> 16 & 0xffu)));
    v[i] = __builtin_amdgcn_perm(hi, lo, 0x07060302u);  // (the upper halves: four significant bits)
  }
  return v;
}
// The eight codes plus 24, 16 to 31, as bf16: the four bits behind the leading one of 16.  A third of the instructions; products with
// them are 24 times the sum of x too large, which a product with -24 (kQ4Less) in front takes off again.
__device__ __forceinline__ q4_words widen_more(uint32_t d) {
  const uint32_t at[4] = {d << 3, d >> 1, d >> 5, d >> 9};
  uint32_t digits = 0x00780078u;
  asm("" : "+v"(digits));  // (in a vector register: an instruction takes one other constant, and does both steps then)
  q4_words v;
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = (at[i] & digits) | 0x41804180u;
  return v;
}
constexpr uint32_t kQ4Less = 0xc1c0c1c0u;  // -24, twice

// Many rows of x (ax_q4_tile.hip).  g as for launch_gemm_experts, without right operands; N columns of each weight.
int q4_tile_rows(const GemmArgs& g, const Groups& e);  // of a workgroup
bool q4_tiles_fit(const GemmArgs& g, const Groups& e);  // whether they are as many as one launch can have
hipError_t launch_q4_tiles(const GemmArgs& g, const Groups& e, const Q4Weights& w, hipStream_t s);

}  // namespace ax
