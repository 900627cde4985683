// Activations and their derivatives, in fp32 (codes: mate_activation).
//
// Exponentials are 2^x of the hardware, quotients its reciprocal (1 ulp each).  With p = 1 / (1 + e^-u):
//   silu       z p(z);                          derivative p + z p (1 - p)
//   gelu_tanh  z p(z (a + b z^2)), a = sqrt(8 / pi), b = 0.044715 a   (0.5 (1 + tanh u) = p(2 u))
//              derivative p + z p (1 - p) (a + 3 b z^2)
//   tanh       2 p(2 z) - 1, and below 1/16, where that cancels, z - z^3 / 3 + 2 z^5 / 15; derivative 4 p(2 |z|) (1 - p(2 |z|))
//   gelu       z F(z), F the normal distribution function;  derivative F(z) + z f(z), f its density
// gelu is max(z, 0) - |z| F(-|z|), and F(-t) = 2^p(t): its logarithm is smooth, so that a polynomial of degree 7 does (fitted here, for the
// least largest error; relative to F it is below 2^-10 up to t = 9, and |z| F(-|z|) is off by 2.8e-7 at most, rounding included; above 0 the
// result's own rounding to fp32 comes on top).  Beyond, p goes on
// falling.  The derivative is S(-z) below 0 and 1 - S(z) above, S(t) = F(-t) - t f(t) = e^(-t^2 / 2) m(t), m a polynomial of degree 10 up
// to t = 6.5, off by 4.4e-7 below 0 and, where 1 - S is rounded once more, 5e-7 above (at z = -4 that is a 1700th of the slope, at -5 a 250th, which
// is bf16's own half step; a polynomial of higher degree would take another slot a value); beyond, where S is below 1e-8, m stays what it is there.
// gelu and its derivative take one exponential each and no quotient (a
// hardware one takes as long as four additions): 14 and 21 instruction slots a value, where formula 7.1.26 of Abramowitz and Stegun
// takes 20 and 24.  The others have one exponential and one reciprocal each.
#pragma once
#include <hip/hip_runtime.h>

#include <type_traits>

#include "mfma_common.h"

namespace mate {

enum Activation { kActNone = 0, kActRelu = 1, kActGelu = 2, kActGeluTanh = 3, kActSilu = 4, kActTanh = 5 };

__device__ __forceinline__ float logistic_base2(float u) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(u)); }   // 1 / (1 + 2^u)
__device__ __forceinline__ float logistic(float u) { return logistic_base2(-kLog2e * u); }

// F(-t), t >= 0
__device__ __forceinline__ float normal_tail(float t) {
  float p = __builtin_fmaf(t, -1.330662257714721e-06f, 5.147118281456642e-05f);
  p = __builtin_fmaf(t, p, -0.000856266007758677f);
  p = __builtin_fmaf(t, p, 0.008262364193797112f);
  p = __builtin_fmaf(t, p, -0.05358245596289635f);
  p = __builtin_fmaf(t, p, -0.45871248841285706f);
  p = __builtin_fmaf(t, p, -1.1511999368667603f);
  return __builtin_amdgcn_exp2f(__builtin_fmaf(t, p, -0.9999955296516418f));
}
// S(|z|); a NaN comes through the exponential.
__device__ __forceinline__ float gelu_tail_slope(float z) {
  const float t = __builtin_fminf(__builtin_fabsf(z), 6.5f);
  float m = __builtin_fmaf(t, 7.85023814842134e-07f, -2.0947529264958575e-05f);
  m = __builtin_fmaf(t, m, 0.00024150629178620875f);
  m = __builtin_fmaf(t, m, -0.001614499487914145f);
  m = __builtin_fmaf(t, m, 0.007173601072281599f);
  m = __builtin_fmaf(t, m, -0.023348676040768623f);
  m = __builtin_fmaf(t, m, 0.06044773757457733f);
  m = __builtin_fmaf(t, m, -0.13223105669021606f);
  m = __builtin_fmaf(t, m, 0.2498626410961151f);
  m = __builtin_fmaf(t, m, -0.7978750467300415f);
  m = __builtin_fmaf(t, m, 0.49999988079071045f);
  return m * __builtin_amdgcn_exp2f(z * z * (-0.5f * kLog2e));
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
  // (A NaN comes through F; where |z| is cut, F is zero, and infinity times zero would not be.)
  if constexpr (kAct == kActGelu) return __builtin_fmaf(-__builtin_fminf(__builtin_fabsf(z), 64.f), normal_tail(__builtin_fabsf(z)), __builtin_fmaxf(z, 0.f));
  if constexpr (kAct == kActGeluTanh) return z * logistic_base2(z * __builtin_fmaf(-kLog2e * kTanhCubic, z * z, -kLog2e * kTanhSlope));
  if constexpr (kAct == kActSilu) return z * logistic(z);
  if constexpr (kAct == kActTanh) {
    const float z2 = z * z, small = __builtin_fmaf(z * z2, __builtin_fmaf(z2, 2.f / 15, -1.f / 3), z);
    float large = __builtin_fmaf(2.f, logistic(2.f * z), -1.f);
    asm volatile("" : "+v"(large));   // (computed for all: a branch around it, which the compiler would make, costs more)
    return __builtin_fabsf(z) < 0.0625f ? small : large;
  }
  return z;
}

// (|z| is cut at 64 where another factor is below 2^-92 by then: infinity times zero would not be zero.)
template <int kAct>
__device__ __forceinline__ float slope(float z) {
  const float zc = __builtin_fminf(__builtin_fmaxf(z, -64.f), 64.f);
  if constexpr (kAct == kActRelu) return passes(z) ? 1.f : 0.f;
  if constexpr (kAct == kActGelu) {
    const float s = gelu_tail_slope(z);
    return z < 0.f ? s : 1.f - s;
  }
  if constexpr (kAct == kActGeluTanh || kAct == kActSilu) {
    const float p = logistic_base2(z * (kAct == kActSilu ? -kLog2e : __builtin_fmaf(-kLog2e * kTanhCubic, z * z, -kLog2e * kTanhSlope)));
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
