// The element-wise work on a matrix product's fp32 sums, shared by the kernels that form them.
#pragma once

#include "act.h"
#include "mlp_kernels.h"

namespace numbat {

namespace {

// The epilogue on NV consecutive columns of one row (NV = 8: 16-byte accesses, or 1).
template <int NV>
__device__ __forceinline__ void load_cols(const bf16_t* p, float (&f)[NV]) {
  if constexpr (NV == 8) unpack8(*reinterpret_cast<const uint4*>(p), f);
  else f[0] = bf2f(*p);
}
template <int NV>
__device__ __forceinline__ void load_cols(const float* p, float (&f)[NV]) {
  if constexpr (NV == 8) {
    const float4 lo = reinterpret_cast<const float4*>(p)[0], hi = reinterpret_cast<const float4*>(p)[1];
    f[0] = lo.x; f[1] = lo.y; f[2] = lo.z; f[3] = lo.w;
    f[4] = hi.x; f[5] = hi.y; f[6] = hi.z; f[7] = hi.w;
  } else {
    f[0] = *p;
  }
}
template <int NV>
__device__ __forceinline__ void store_cols(bf16_t* p, const float (&f)[NV]) {
  if constexpr (NV == 8) {
    const uint4 v = pack8(f);
    __builtin_nontemporal_store(u32x4{v.x, v.y, v.z, v.w}, reinterpret_cast<u32x4*>(p));
  } else {
    *p = (bf16_t)f2bf(f[0]);
  }
}
template <int NV>
__device__ __forceinline__ void store_cols(float* p, const float (&f)[NV]) {
  if constexpr (NV == 8) {
    __builtin_nontemporal_store(f32x4{f[0], f[1], f[2], f[3]}, reinterpret_cast<f32x4*>(p));
    __builtin_nontemporal_store(f32x4{f[4], f[5], f[6], f[7]}, reinterpret_cast<f32x4*>(p) + 1);
  } else {
    *p = f[0];
  }
}

// The matrix that the epilogue reads beside the sums: the residual (forward), z (data gradient
// through an activation) or the old values (weight gradient that accumulates).  Raw, so that its
// loads can be issued early and cost few registers.
template <int NV>
struct Aux {
  uint4 lo, hi;  // 8 bf16, or 8 fp32; element 0 alone for NV = 1
};
template <int KIND>
__device__ __forceinline__ const void* aux_base(const GemmEpilogue& e, int64_t* ld, bool* f32) {
  *f32 = KIND == kGemmWgrad || (KIND == kGemmFwd && e.out_f32);
  *ld = KIND == kGemmFwd ? e.ldr : KIND == kGemmDgrad ? e.ldz : e.ldo;
  return KIND == kGemmFwd     ? e.res
         : KIND == kGemmDgrad ? (e.act != kActNone ? e.z : nullptr)
                              : (e.accumulate ? e.out : nullptr);
}
template <int KIND, int NV>
__device__ __forceinline__ void load_aux(const GemmEpilogue& e, int64_t row, int col, Aux<NV>& x) {
  int64_t ld;
  bool f32;
  const void* base = aux_base<KIND>(e, &ld, &f32);
  if (base == nullptr) return;
  const char* p = static_cast<const char*>(base) + (row * ld + col) * (f32 ? 4 : 2);
  if constexpr (NV == 8) {
    x.lo = *reinterpret_cast<const uint4*>(p);
    if (f32) x.hi = *reinterpret_cast<const uint4*>(p + 16);
  } else {
    x.lo.x = f32 ? *reinterpret_cast<const uint32_t*>(p) : *reinterpret_cast<const uint16_t*>(p);
  }
}
template <int NV>
__device__ __forceinline__ void aux_values(const Aux<NV>& x, bool f32, float (&f)[NV]) {
  if constexpr (NV == 8) {
    if (f32) {
      const uint32_t u[8] = {x.lo.x, x.lo.y, x.lo.z, x.lo.w, x.hi.x, x.hi.y, x.hi.z, x.hi.w};
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = __uint_as_float(u[i]);
    } else {
      unpack8(x.lo, f);
    }
  } else {
    f[0] = f32 ? __uint_as_float(x.lo.x) : bf2f(x.lo.x);
  }
}

template <int NV, typename F>
__device__ __forceinline__ void each(float (&f)[NV], F&& fn) {
#pragma unroll
  for (int i = 0; i < NV; ++i) f[i] = fn(i);
}

// f: the sums; bias: those of the columns; x: loaded by load_aux
template <int KIND, int NV>
__device__ __forceinline__ void finish_cols(const GemmEpilogue& e, int64_t row, int col, float (&f)[NV],
                                            const float (&bias)[NV], const Aux<NV>& x) {
  float o[NV];
  if constexpr (KIND == kGemmFwd) {
    each(f, [&](int i) { return f[i] + bias[i]; });
    if (e.z != nullptr) store_cols<NV>(e.z + row * e.ldz + col, f);
    // (one branch for the vector, not one per element)
    switch (e.act) {
      case kActRelu: each(f, [&](int i) { return act_apply(f[i], kActRelu); }); break;
      case kActGelu: each(f, [&](int i) { return act_apply(f[i], kActGelu); }); break;
      case kActGeluTanh: each(f, [&](int i) { return act_apply(f[i], kActGeluTanh); }); break;
      case kActSilu: each(f, [&](int i) { return act_apply(f[i], kActSilu); }); break;
      default: break;
    }
    if (e.res != nullptr) {
      aux_values<NV>(x, e.out_f32, o);
      each(f, [&](int i) { return f[i] + o[i]; });
    }
    if (e.out_f32) store_cols<NV>(static_cast<float*>(e.out) + row * e.ldo + col, f);
    else store_cols<NV>(static_cast<bf16_t*>(e.out) + row * e.ldo + col, f);
  } else if constexpr (KIND == kGemmDgrad) {
    if (e.act != kActNone) aux_values<NV>(x, false, o);
    switch (e.act) {
      case kActRelu: each(f, [&](int i) { return f[i] * act_slope(o[i], kActRelu); }); break;
      case kActGelu: each(f, [&](int i) { return f[i] * act_slope(o[i], kActGelu); }); break;
      case kActGeluTanh: each(f, [&](int i) { return f[i] * act_slope(o[i], kActGeluTanh); }); break;
      case kActSilu: each(f, [&](int i) { return f[i] * act_slope(o[i], kActSilu); }); break;
      default: break;
    }
    bf16_t* p = static_cast<bf16_t*>(e.out) + row * e.ldo + col;
    if (e.accumulate) {
      load_cols<NV>(p, o);
      each(f, [&](int i) { return f[i] + o[i]; });
    }
    store_cols<NV>(p, f);
  } else {
    if (e.accumulate) {
      aux_values<NV>(x, true, o);
      each(f, [&](int i) { return f[i] + o[i]; });
    }
    store_cols<NV>(static_cast<float*>(e.out) + row * e.ldo + col, f);
  }
}

template <int KIND, int NV>
__device__ __forceinline__ void load_bias(const GemmEpilogue& e, int col, int n, float (&b)[NV]) {
#pragma unroll
  for (int i = 0; i < NV; ++i) b[i] = 0.f;
  if constexpr (KIND == kGemmFwd) {
    if (e.bias != nullptr && col < n) load_cols<NV>(e.bias + col, b);
  }
}

}  // namespace

}  // namespace numbat
