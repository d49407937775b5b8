// Vectors of consecutive bf16 or fp32 values as fp32 registers, at 16-byte aligned or at any addresses.
#pragma once

#include "common.h"

namespace numbat {

namespace {

struct __attribute__((packed, aligned(2))) Any16 {
  uint32_t u[4];
};
template <bool ALIGNED>
__device__ __forceinline__ uint4 get16(const void* p) {
  if constexpr (ALIGNED) return *static_cast<const uint4*>(p);
  const Any16 v = *static_cast<const Any16*>(p);
  return make_uint4(v.u[0], v.u[1], v.u[2], v.u[3]);
}
template <bool ALIGNED>
__device__ __forceinline__ void put16(void* p, uint4 v) {
  if constexpr (ALIGNED) *static_cast<uint4*>(p) = v;
  else *static_cast<Any16*>(p) = Any16{{v.x, v.y, v.z, v.w}};
}

__device__ __forceinline__ float get1(const bf16_t* p) { return bf2f(*p); }
__device__ __forceinline__ float get1(const float* p) { return *p; }
__device__ __forceinline__ void put1(bf16_t* p, float f) { *p = (bf16_t)f2bf(f); }
__device__ __forceinline__ void put1(float* p, float f) { *p = f; }

// values that 16 bytes hold
template <typename T>
constexpr int kVec = 16 / (int)sizeof(T);

// N values, N a multiple of what 16 bytes hold
template <bool ALIGNED, int N>
__device__ __forceinline__ void get_vec(const bf16_t* p, float (&f)[N]) {
  static_assert(N == 8, "eight values of bf16");
  unpack8(get16<ALIGNED>(p), f);
}
template <bool ALIGNED, int N>
__device__ __forceinline__ void get_vec(const float* p, float (&f)[N]) {
#pragma unroll
  for (int i = 0; i < N; i += 4) {
    const uint4 v = get16<ALIGNED>(p + i);
    f[i] = __uint_as_float(v.x);
    f[i + 1] = __uint_as_float(v.y);
    f[i + 2] = __uint_as_float(v.z);
    f[i + 3] = __uint_as_float(v.w);
  }
}
template <bool ALIGNED, int N>
__device__ __forceinline__ void put_vec(bf16_t* p, const float (&f)[N]) {
  static_assert(N == 8, "eight values of bf16");
  put16<ALIGNED>(p, pack8(f));
}
template <bool ALIGNED, int N>
__device__ __forceinline__ void put_vec(float* p, const float (&f)[N]) {
#pragma unroll
  for (int i = 0; i < N; i += 4)
    put16<ALIGNED>(p + i, make_uint4(__float_as_uint(f[i]), __float_as_uint(f[i + 1]), __float_as_uint(f[i + 2]),
                                     __float_as_uint(f[i + 3])));
}

// the first `count` of N values, zeros behind them; a whole vector in 16-byte accesses
template <bool ALIGNED, int N, typename T>
__device__ __forceinline__ void get_some(const T* p, int count, float (&f)[N]) {
  if (count >= N) {
    get_vec<ALIGNED>(p, f);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) f[i] = i < count ? get1(p + i) : 0.f;
  }
}
template <bool ALIGNED, int N, typename T>
__device__ __forceinline__ void put_some(T* p, int count, const float (&f)[N]) {
  if (count >= N) {
    put_vec<ALIGNED>(p, f);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (i < count) put1(p + i, f[i]);
  }
}

}  // namespace

}  // namespace numbat
