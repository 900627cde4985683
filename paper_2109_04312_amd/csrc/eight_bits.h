// Activations in 8 bits: e4m3 codes (one sign, four exponent and three mantissa bits, largest value 448) and one scale
// for each block of 32 features of a token, a power of two 2^(s - 127) stored as the byte s, 1 <= s <= 254.
//
// s is the smallest with (block's largest finite magnitude) <= 448 x 2^(s - 127): no value saturates, and the largest
// keeps all four of its significant bits.  (The usual choice, the exponent of the largest value less 8, is one smaller for
// largest mantissas above 1.75, which then saturate, off by up to an eighth.)  Values are rounded to nearest even.
// A power of two makes the rest exact: dividing by it, and code x scale in bf16, which has four spare mantissa
// bits and the scale's exponents.  (But for scales 1 and 2: below 2^-130 their values have more bits than bf16's denormal numbers, and are rounded to
// nearest even; fp32 holds all.)  Infinities and NaN are stored as NaN and do not enter the scale; a block of zeros
// has s = 1.
#pragma once
#include <hip/hip_runtime.h>

#include "mfma_common.h"

namespace mate {

constexpr int kScaleBlock = 32;
__host__ __device__ inline int scale_blocks(int features) { return (features + kScaleBlock - 1) / kScaleBlock; }

typedef short s16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

constexpr unsigned kInfBits = 0x7f800000u;

// The largest value below 2^128 with four significant bits: what rounds up from there would be no number of either type.
constexpr unsigned kLargestBits = 0x7f700000u;

// A block's largest finite magnitude, as bits, which compare like it: of a lane's values, then across() the block's lanes.
// Only if that is not finite, or close to the end of the range, are values looked at one by one (rare, so the common path has no test
// per value); those above the largest are replaced by it.  (A comparison of numbers takes the sign off for nothing, and two values at a time.  One
// with a NaN gives the other value, or the NaN, which is not finite.)
__device__ __forceinline__ unsigned magnitude(float x) { return __float_as_uint(x) & 0x7fffffffu; }
template <int kValues, class Across>
__device__ __forceinline__ unsigned block_magnitude(float (&v)[kValues], Across&& across) {
  float most = __builtin_fabsf(v[0]);
#pragma unroll
  for (int e = 1; e < kValues; ++e) most = __builtin_fmaxf(most, __builtin_fabsf(v[e]));
  unsigned m = across(magnitude(most));
  if (__builtin_expect(__any(m > kLargestBits), 0)) {
    m = 0;
#pragma unroll
    for (int e = 0; e < kValues; ++e) {
      const unsigned x = magnitude(v[e]);
      if (x < kInfBits) {
        if (x > kLargestBits) v[e] = __uint_as_float((__float_as_uint(v[e]) & 0x80000000u) | kLargestBits);
        m = max(m, min(x, kLargestBits));
      }
    }
    m = across(m);
  }
  return m;
}
// Across the four lanes of a quad.
__device__ __forceinline__ unsigned quad_maximum(unsigned m) {
  m = max(m, (unsigned)__builtin_amdgcn_update_dpp(0, (int)m, 0xb1, 0xf, 0xf, false));
  return max(m, (unsigned)__builtin_amdgcn_update_dpp(0, (int)m, 0x4e, 0xf, 0xf, false));
}
// The scale's byte for the bits of a block's largest magnitude: its exponent less 8, one more above 1.75.
__device__ __forceinline__ unsigned scale_byte(unsigned magnitude_bits) {
  const int s = (int)((magnitude_bits + 0x1fffffu) >> 23) - 8;
  return (unsigned)max(s, 1);
}
__device__ __forceinline__ float scale_value(unsigned byte) { return __uint_as_float(byte << 23); }

// Four values as codes in a word (divided by the scale, rounded to nearest even; not finite: NaN).
__device__ __forceinline__ unsigned to_codes(float a, float b, float c, float d, float scale) {
  s16x2 r = {0, 0};
  r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, a, b, scale, false);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, c, d, scale, true);
  return __builtin_bit_cast(unsigned, r);
}
// And back: exact in fp32.
__device__ __forceinline__ f32x4 from_codes(unsigned w, float scale) {
  const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, scale, true);
  return f32x4{a[0], a[1], b[0], b[1]};
}
// As four bf16 in two words.
__device__ __forceinline__ uint2 bf16_from_codes(unsigned w, float scale) {
  return make_uint2(__builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, false)),
                    __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, true)));
}

// Two bf16 in a word.
__device__ __forceinline__ float low_bf16(unsigned w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float high_bf16(unsigned w) { return __uint_as_float(w & 0xffff0000u); }

}  // namespace mate
