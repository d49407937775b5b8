// Activations of the linear layers' epilogues and their derivatives, in fp32.
#pragma once

#include "common.h"

namespace numbat {

enum { kActNone = 0, kActRelu = 1, kActGelu = 2, kActGeluTanh = 3, kActSilu = 4 };

constexpr float kInvSqrt2Pi = 0.39894228040143268f;
constexpr float kGeluTanhA = 1.5957691216057308f;  // 2 sqrt(2 / pi): 1 + tanh(u) = 2 sigmoid(2 u)
constexpr float kGeluTanhB = 0.044715f;

// GELU's normal distribution function Phi, and e = exp(-z^2 / 2), from which its density follows.
// With x = |z| / sqrt(2) the tail beyond |z| is erfc(x) / 2 = t (a1 + t (a2 + ... + t a5)) exp(-x^2) / 2,
// t = 1 / (1 + p x): formula 7.1.26 of Abramowitz and Stegun's Handbook of Mathematical Functions,
// within 1.5e-7 / 2 everywhere, the size of fp32's own rounding of 1 + erf.  That is an absolute bound:
// GELU's measured error is at most 3.4e-7 (|z| up to 12; of fp32 operations with erf 4.5e-7), but for
// |z| < 1 its root mean square is 3.2e-8 against 1.4e-8, between -4 and -1 it is 0.8 to 1.6e-7 against 2 to
// 3e-8, and relative to the tail itself it grows from 5e-4 at -4 to 4e-3 at -6 and 3e-2 at -12, where
// the value is below 1e-8 (1 + erf has lost it altogether from -6 on).  About 16 instruction
// slots and no branch, where a library erf takes some 45 on both of its ranges: an epilogue of
// 256 x 256 elements is VALU work that nothing hides.
// half the tail: erfc(|z| / sqrt(2)) / 2, and e
__device__ __forceinline__ float normal_tail(float z, float& e) {
  const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.3275911f * 0.70710678f, fabsf(z), 1.0f));
  float q = __builtin_fmaf(t, 0.5f * 1.061405429f, 0.5f * -1.453152027f);
  q = __builtin_fmaf(t, q, 0.5f * 1.421413741f);
  q = __builtin_fmaf(t, q, 0.5f * -0.284496736f);
  q = __builtin_fmaf(t, q, 0.5f * 0.254829592f);
  e = __builtin_amdgcn_exp2f((z * z) * -0.72134752f);  // log2(e) / 2
  return q * (t * e);
}
// z Phi(z) = max(z, 0) - |z| tail: on either side of 0 the smaller term is what is computed (the tail
// is zero in fp32 from |z| = 20 on, so the product's bound changes nothing but an infinite z)
__device__ __forceinline__ float gelu(float z) {
  float e;
  const float q = normal_tail(z, e);
  return __builtin_fmaf(-fminf(fabsf(z), 64.f), q, z > 0.f ? z : (z == z ? 0.f : z));
}

__device__ __forceinline__ float act_apply(float z, int act) {
  switch (act) {
    case kActRelu: return z > 0.f ? z : (z == z ? 0.f : z);
    case kActGelu: return gelu(z);
    case kActGeluTanh: return z * sigmoidf_fast(kGeluTanhA * z * __builtin_fmaf(kGeluTanhB * z, z, 1.0f));
    case kActSilu: return z * sigmoidf_fast(z);
    default: return z;
  }
}

__device__ __forceinline__ float act_slope(float z, int act) {
  switch (act) {
    case kActRelu: return z > 0.f ? 1.f : 0.f;
    case kActGelu: {
      float e;
      const float q = normal_tail(z, e);
      return __builtin_fmaf(z * kInvSqrt2Pi, e, z > 0.f ? 1.0f - q : q);
    }
    case kActGeluTanh: {
      const float q = sigmoidf_fast(kGeluTanhA * z * __builtin_fmaf(kGeluTanhB * z, z, 1.0f)), p = z * q * (1.0f - q);
      // (p is 0 long before z^2 passes fp32's range; its factor stays finite, so that the product is 0 too)
      return __builtin_fmaf(p, kGeluTanhA * fminf(__builtin_fmaf(3.0f * kGeluTanhB * z, z, 1.0f), 1e38f), q);
    }
    case kActSilu: {
      const float q = sigmoidf_fast(z);
      return q * __builtin_fmaf(z, 1.0f - q, 1.0f);
    }
    default: return 1.f;
  }
}

}  // namespace numbat
