// Activations and their derivatives, in fp32 (codes: mate_activation).
//
// Exponentials are 2^x of the hardware, quotients its reciprocal (1 ulp each).  With p = 1 / (1 + e^-u):
//   silu       z p(z);                          derivative p + z p (1 - p)
//   gelu_tanh  z p(z (a + b z^2)), a = sqrt(8 / pi), b = 0.044715 a   (0.5 (1 + tanh u) = p(2 u))
//              derivative p + z p (1 - p) (a + 3 b z^2)
//   tanh       2 p(2 z) - 1, and below 1/16, where that cancels, z - z^3 / 3 + 2 z^5 / 15; derivative 4 p(2 |z|) (1 - p(2 |z|))
//   gelu       z F(z), F the normal distribution function;  derivative F(z) + z f(z), f its density
// F(-|z|) = 0.5 erfc(|z| / sqrt(2)) by formula 7.1.26 of Abramowitz and Stegun, t (a1 + .. + a5 t^4) e^(-z^2 / 2) with
// t = 1 / (1 + 0.3275911 |z| / sqrt(2)), off by 1.5e-7 at most: no branch, one exponential, which the derivative's
// density is as well, and an error that shrinks with e^(-z^2 / 2) in the tail instead of staying at an ulp of 1.
// (A product's epilogue evaluates it for 67 million values of a large layer, 19 instruction slots each.)
#pragma once
#include <hip/hip_runtime.h>

#include <type_traits>

#include "mfma_common.h"

namespace mate {

enum Activation { kActNone = 0, kActRelu = 1, kActGelu = 2, kActGeluTanh = 3, kActSilu = 4, kActTanh = 5 };

__device__ __forceinline__ float logistic(float u) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-kLog2e * u)); }

// F(-|z|) and e^(-z^2 / 2)
struct Normal { float tail, bell; };
__device__ __forceinline__ Normal normal(float z) {
  const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.3275911f * 0.70710678f, __builtin_fabsf(z), 1.f));
  float s = __builtin_fmaf(t, 0.5f * 1.061405429f, 0.5f * -1.453152027f);
  s = __builtin_fmaf(t, s, 0.5f * 1.421413741f);
  s = __builtin_fmaf(t, s, 0.5f * -0.284496736f);
  s = __builtin_fmaf(t, s, 0.5f * 0.254829592f);
  const float bell = __builtin_amdgcn_exp2f(z * z * (-0.5f * kLog2e));
  return {t * s * bell, bell};
}

// Is z above 0, or not a number?  (A comparison alone would lose a NaN in relu.)
__device__ __forceinline__ bool passes(float z) {
  const unsigned u = __float_as_uint(z);
  return (int)u > 0 || u > 0xff800000u;
}

constexpr float kTanhSlope = 1.5957691216057308f, kTanhCubic = 0.044715f * kTanhSlope;  // a, b above

template <int kAct>
__device__ __forceinline__ float activate(float z) {
  if constexpr (kAct == kActRelu) return passes(z) ? z : 0.f;
  // z F(z) = max(z, 0) - |z| F(-|z|).  (A NaN comes through F; where |z| is cut, F is zero, and infinity times zero would not be.)
  if constexpr (kAct == kActGelu) return __builtin_fmaf(-__builtin_fminf(__builtin_fabsf(z), 64.f), normal(z).tail, __builtin_fmaxf(z, 0.f));
  if constexpr (kAct == kActGeluTanh) return z * logistic(z * __builtin_fmaf(kTanhCubic, z * z, kTanhSlope));
  if constexpr (kAct == kActSilu) return z * logistic(z);
  if constexpr (kAct == kActTanh) {
    const float z2 = z * z, small = __builtin_fmaf(z * z2, __builtin_fmaf(z2, 2.f / 15, -1.f / 3), z);
    return __builtin_fabsf(z) < 0.0625f ? small : __builtin_fmaf(2.f, logistic(2.f * z), -1.f);
  }
  return z;
}

// (|z| is cut at 64 where a factor is zero by then: infinity times zero would not be.)
template <int kAct>
__device__ __forceinline__ float slope(float z) {
  const float zc = __builtin_fminf(__builtin_fmaxf(z, -64.f), 64.f);
  if constexpr (kAct == kActRelu) return passes(z) ? 1.f : 0.f;
  if constexpr (kAct == kActGelu) {
    const Normal n = normal(z);
    return __builtin_fmaf(zc * 0.3989422804f, n.bell, z < 0.f ? n.tail : 1.f - n.tail);
  }
  if constexpr (kAct == kActGeluTanh || kAct == kActSilu) {
    const float p = logistic(kAct == kActSilu ? z : z * __builtin_fmaf(kTanhCubic, z * z, kTanhSlope));
    const float inner = kAct == kActSilu ? zc : zc * __builtin_fmaf(3.f * kTanhCubic, zc * zc, kTanhSlope);
    return __builtin_fmaf(p * (1.f - p), inner, p);
  }
  if constexpr (kAct == kActTanh) {
    const float e = __builtin_amdgcn_exp2f(-2.f * kLog2e * __builtin_fabsf(z)), p = __builtin_amdgcn_rcpf(1.f + e);
    return 4.f * e * p * p;
  }
  return 1.f;
}

// f(std::integral_constant<int, act>()) for an activation that is the same in all lanes: one scalar branch.
template <class F>
__device__ __forceinline__ void with_activation(int act, F&& f) {
  switch (act) {
    case kActRelu: return f(std::integral_constant<int, kActRelu>());
    case kActGelu: return f(std::integral_constant<int, kActGelu>());
    case kActGeluTanh: return f(std::integral_constant<int, kActGeluTanh>());
    case kActSilu: return f(std::integral_constant<int, kActSilu>());
    case kActTanh: return f(std::integral_constant<int, kActTanh>());
    default: return f(std::integral_constant<int, kActNone>());
  }
}

}  // namespace mate
