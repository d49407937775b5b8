// Activations of the linear layers' epilogues and their derivatives, in fp32.
#pragma once

#include "common.h"

namespace numbat {

enum { kActNone = 0, kActRelu = 1, kActGelu = 2, kActGeluTanh = 3, kActSilu = 4 };

constexpr float kSqrtHalf = 0.70710678118654752f;
constexpr float kInvSqrt2Pi = 0.39894228040143268f;
constexpr float kGeluTanhA = 1.5957691216057308f;  // 2 sqrt(2 / pi): 1 + tanh(u) = 2 sigmoid(2 u)
constexpr float kGeluTanhB = 0.044715f;

__device__ __forceinline__ float act_apply(float z, int act) {
  switch (act) {
    case kActRelu: return z > 0.f ? z : (z == z ? 0.f : z);
    case kActGelu: return z * (0.5f * (1.0f + erff(z * kSqrtHalf)));
    case kActGeluTanh: return z * sigmoidf_fast(kGeluTanhA * z * __builtin_fmaf(kGeluTanhB * z, z, 1.0f));
    case kActSilu: return z * sigmoidf_fast(z);
    default: return z;
  }
}

__device__ __forceinline__ float act_slope(float z, int act) {
  switch (act) {
    case kActRelu: return z > 0.f ? 1.f : 0.f;
    case kActGelu:
      return __builtin_fmaf(z * kInvSqrt2Pi, __expf(-0.5f * z * z), 0.5f * (1.0f + erff(z * kSqrtHalf)));
    case kActGeluTanh: {
      const float q = sigmoidf_fast(kGeluTanhA * z * __builtin_fmaf(kGeluTanhB * z, z, 1.0f));
      return __builtin_fmaf(z * q * (1.0f - q), kGeluTanhA * __builtin_fmaf(3.0f * kGeluTanhB * z, z, 1.0f), q);
    }
    case kActSilu: {
      const float q = sigmoidf_fast(z);
      return q * __builtin_fmaf(z, 1.0f - q, 1.0f);
    }
    default: return 1.f;
  }
}

}  // namespace numbat
