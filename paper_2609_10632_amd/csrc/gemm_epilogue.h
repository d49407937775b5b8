// The element-wise work on a matrix product's fp32 sums, shared by the kernels that form them.
#pragma once

#include "act.h"
#include "mlp_kernels.h"

namespace numbat {

namespace {

// A vector of columns whose row starts at any element: unaligned 16-byte accesses, which the hardware
// splits where they cross a line.
struct __attribute__((packed, aligned(2))) AnyVec {
  uint32_t u[4];
};
template <bool ALIGNED>
__device__ __forceinline__ uint4 load16(const void* p) {
  if constexpr (ALIGNED) return *static_cast<const uint4*>(p);
  const AnyVec v = *static_cast<const AnyVec*>(p);
  return make_uint4(v.u[0], v.u[1], v.u[2], v.u[3]);
}
// how results are stored: at any address, in 16-byte vectors, or in those past the caches (see
// EpiloguePtr)
enum { kStoreAny, kStoreVec, kStoreStream };
template <int HOW>
__device__ __forceinline__ void store16(void* p, u32x4 v) {
  if constexpr (HOW == kStoreAny) *static_cast<AnyVec*>(p) = AnyVec{{v.x, v.y, v.z, v.w}};
  else if constexpr (HOW == kStoreStream) __builtin_nontemporal_store(v, static_cast<u32x4*>(p));
  else *static_cast<u32x4*>(p) = v;
}

struct __attribute__((packed, aligned(2))) AnyHalf {
  uint32_t u[2];
};
// NV consecutive columns: 8 or 4 of bf16, 4 of fp32 (16 bytes a lane, so that neighbouring lanes'
// accesses join to whole lines), or 1
template <int NV, bool ALIGNED = true>
__device__ __forceinline__ void load_cols(const bf16_t* p, float (&f)[NV]) {
  if constexpr (NV == 8) {
    unpack8(load16<ALIGNED>(p), f);
  } else if constexpr (NV == 4) {
    const AnyHalf v = *reinterpret_cast<const AnyHalf*>(p);
    f[0] = bf2f(v.u[0] & 0xffffu);
    f[1] = bf2f(v.u[0] >> 16);
    f[2] = bf2f(v.u[1] & 0xffffu);
    f[3] = bf2f(v.u[1] >> 16);
  } else {
    f[0] = bf2f(*p);
  }
}
template <int NV, bool ALIGNED = true>
__device__ __forceinline__ void load_cols(const float* p, float (&f)[NV]) {
  static_assert(NV == 4 || NV == 1, "four columns of fp32 at a time");
  if constexpr (NV == 4) {
    const uint4 v = load16<ALIGNED>(p);
    f[0] = __uint_as_float(v.x);
    f[1] = __uint_as_float(v.y);
    f[2] = __uint_as_float(v.z);
    f[3] = __uint_as_float(v.w);
  } else {
    f[0] = *p;
  }
}
template <int NV, int HOW = kStoreVec>
__device__ __forceinline__ void store_cols(bf16_t* p, const float (&f)[NV]) {
  if constexpr (NV == 8) {
    const uint4 v = pack8(f);
    store16<HOW>(p, u32x4{v.x, v.y, v.z, v.w});
  } else if constexpr (NV == 4) {
    *reinterpret_cast<AnyHalf*>(p) = AnyHalf{{pack2(f[0], f[1]), pack2(f[2], f[3])}};
  } else {
    *p = (bf16_t)f2bf(f[0]);
  }
}
template <int NV, int HOW = kStoreVec>
__device__ __forceinline__ void store_cols(float* p, const float (&f)[NV]) {
  if constexpr (NV == 4) store16<HOW>(p, __builtin_bit_cast(u32x4, f32x4{f[0], f[1], f[2], f[3]}));
  else if constexpr (NV == 1) *p = f[0];
}

// The matrix that the epilogue reads beside the sums: the residual (forward), z (data gradient
// through an activation) or the old values (weight gradient that accumulates).  Raw, so that its
// loads can be issued early and cost few registers.
typedef uint4 Aux;  // 8 or 4 bf16, 4 fp32, or one element

// The epilogue's matrices from one element of theirs, a tile's first as a rule: bases that are the
// same for a whole block and 32-bit byte offsets from there (a tile is at most 256 rows of 2^21
// elements), which cost a lane one multiply-add where 64-bit addresses cost it ten instructions.
struct EpiloguePtr {
  char *out, *z;
  const char* aux;            // nullptr: none
  uint32_t ldo, ldz, ldx;     // bytes between rows
  bool out_f32, aux_f32;
  // Whether results go past the caches: they are written once and read by a later kernel, and 102400 x
  // 192 -> 768 with z takes 84 us so against 111.  Only where rows are whole 128-byte lines: elsewhere
  // neighbouring tiles write parts of the same lines, which the L2 then joins (24 x 11576 x 6712's fp32
  // gradient 56 us against 133).
  bool stream;
};
template <int KIND>
__device__ __forceinline__ EpiloguePtr epilogue_at(const GemmEpilogue& e, int64_t row, int64_t col) {
  EpiloguePtr p;
  p.out_f32 = KIND == kGemmWgrad || (KIND == kGemmFwd && e.out_f32);
  p.aux_f32 = KIND != kGemmDgrad && p.out_f32;
  const int so = p.out_f32 ? 4 : 2, sx = p.aux_f32 ? 4 : 2;
  const void* aux = KIND == kGemmFwd     ? e.res
                    : KIND == kGemmDgrad ? (e.act != kActNone ? e.z : nullptr)
                                         : (e.accumulate ? e.out : nullptr);
  const int64_t ldx = KIND == kGemmFwd ? e.ldr : KIND == kGemmDgrad ? e.ldz : e.ldo;
  p.ldo = (uint32_t)e.ldo * so;
  p.ldz = (uint32_t)e.ldz * 2;
  p.ldx = (uint32_t)ldx * sx;
  p.out = static_cast<char*>(e.out) + (row * e.ldo + col) * so;
  p.z = KIND == kGemmFwd && e.z != nullptr ? reinterpret_cast<char*>(e.z + row * e.ldz + col) : nullptr;
  p.stream = (((uint32_t)(uintptr_t)e.out | p.ldo | (p.z != nullptr ? (uint32_t)(uintptr_t)e.z | p.ldz : 0)) & 127u) == 0;
  p.aux = aux != nullptr ? static_cast<const char*>(aux) + (row * ldx + col) * sx : nullptr;
  return p;
}

// row r and column c count from the element that p points to
template <int NV, bool ALIGNED = true>
__device__ __forceinline__ void load_aux(const EpiloguePtr& p, uint32_t r, uint32_t c, Aux& x) {
  if (p.aux == nullptr) return;
  const char* at = p.aux + (uint32_t)(r * p.ldx + c * (p.aux_f32 ? 4 : 2));
  if constexpr (NV == 8) {
    x = load16<ALIGNED>(at);
  } else if constexpr (NV == 4) {
    if (p.aux_f32) {
      x = load16<ALIGNED>(at);
    } else {
      const AnyHalf v = *reinterpret_cast<const AnyHalf*>(at);
      x.x = v.u[0];
      x.y = v.u[1];
    }
  } else {
    x.x = p.aux_f32 ? *reinterpret_cast<const uint32_t*>(at) : *reinterpret_cast<const uint16_t*>(at);
  }
}
template <int NV>
__device__ __forceinline__ void aux_values(const Aux& x, bool f32, float (&f)[NV]) {
  if constexpr (NV == 8) {
    unpack8(x, f);
  } else if constexpr (NV == 4) {
    f[0] = f32 ? __uint_as_float(x.x) : bf2f(x.x & 0xffffu);
    f[1] = f32 ? __uint_as_float(x.y) : bf2f(x.x >> 16);
    f[2] = f32 ? __uint_as_float(x.z) : bf2f(x.y & 0xffffu);
    f[3] = f32 ? __uint_as_float(x.w) : bf2f(x.y >> 16);
  } else {
    f[0] = f32 ? __uint_as_float(x.x) : bf2f(x.x);
  }
}

template <int NV, typename F>
__device__ __forceinline__ void each(float (&f)[NV], F&& fn) {
#pragma unroll
  for (int i = 0; i < NV; ++i) f[i] = fn(i);
}

// f: the sums; bias: those of the columns; x: loaded by load_aux
template <int KIND, int NV, int HOW = kStoreVec>
__device__ __forceinline__ void finish_cols(const GemmEpilogue& e, const EpiloguePtr& p, uint32_t r, uint32_t c,
                                            float (&f)[NV], const float* bias, const Aux& x) {
  float o[NV];
  char* out = p.out + (uint32_t)(r * p.ldo + c * (p.out_f32 ? 4 : 2));
  if constexpr (KIND == kGemmFwd) {
    each(f, [&](int i) { return f[i] + bias[i]; });
    if (p.z != nullptr) store_cols<NV, HOW>(reinterpret_cast<bf16_t*>(p.z + (uint32_t)(r * p.ldz + c * 2)), f);
    // (one branch for the vector, not one per element)
    switch (e.act) {
      case kActRelu: each(f, [&](int i) { return act_apply(f[i], kActRelu); }); break;
      case kActGelu: each(f, [&](int i) { return act_apply(f[i], kActGelu); }); break;
      case kActGeluTanh: each(f, [&](int i) { return act_apply(f[i], kActGeluTanh); }); break;
      case kActSilu: each(f, [&](int i) { return act_apply(f[i], kActSilu); }); break;
      default: break;
    }
    if (p.aux != nullptr) {
      aux_values<NV>(x, p.aux_f32, o);
      each(f, [&](int i) { return f[i] + o[i]; });
    }
  } else if constexpr (KIND == kGemmDgrad) {
    if (e.act != kActNone) aux_values<NV>(x, false, o);
    switch (e.act) {
      case kActRelu: each(f, [&](int i) { return f[i] * act_slope(o[i], kActRelu); }); break;
      case kActGelu: each(f, [&](int i) { return f[i] * act_slope(o[i], kActGelu); }); break;
      case kActGeluTanh: each(f, [&](int i) { return f[i] * act_slope(o[i], kActGeluTanh); }); break;
      case kActSilu: each(f, [&](int i) { return f[i] * act_slope(o[i], kActSilu); }); break;
      default: break;
    }
    if (e.accumulate) {
      load_cols<NV, HOW != kStoreAny>(reinterpret_cast<const bf16_t*>(out), o);
      each(f, [&](int i) { return f[i] + o[i]; });
    }
  } else {
    if (e.accumulate) {
      aux_values<NV>(x, true, o);
      each(f, [&](int i) { return f[i] + o[i]; });
    }
  }
  if constexpr (NV != 8) {  // (fp32 results never come in eights)
    if (p.out_f32) return store_cols<NV, HOW>(reinterpret_cast<float*>(out), f);
  }
  if constexpr (KIND != kGemmWgrad) store_cols<NV, HOW>(reinterpret_cast<bf16_t*>(out), f);
}

// the bias of NV columns from col (it may start at any float; zeros past the last column)
template <int KIND, int NV>
__device__ __forceinline__ void load_bias(const GemmEpilogue& e, int col, int n, float* b) {
#pragma unroll
  for (int i = 0; i < NV; ++i) b[i] = 0.f;
  if constexpr (KIND == kGemmFwd) {
    if (e.bias == nullptr) return;
    if (NV >= 4 && col + NV <= n) {
#pragma unroll
      for (int i = 0; i < NV / 4; ++i) {
        const uint4 v = load16<false>(e.bias + col + 4 * i);
        b[4 * i] = __uint_as_float(v.x);
        b[4 * i + 1] = __uint_as_float(v.y);
        b[4 * i + 2] = __uint_as_float(v.z);
        b[4 * i + 3] = __uint_as_float(v.w);
      }
    } else {
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (col + i < n) b[i] = e.bias[col + i];
    }
  }
}

// NV columns, of which `cols` are left in the row (rows that are not whole vectors): a whole vector as
// one, the last of a row by elements.
template <int KIND, int NV>
__device__ __forceinline__ void finish_any(const GemmEpilogue& e, const EpiloguePtr& p, uint32_t r, uint32_t c, int cols,
                                           float (&f)[NV], const float* bias) {
  Aux x;
  if (cols >= NV) {
    load_aux<NV, false>(p, r, c, x);
    finish_cols<KIND, NV, kStoreAny>(e, p, r, c, f, bias, x);
    return;
  }
  float rest[NV];
#pragma unroll
  for (int j = 0; j < NV; ++j) rest[j] = bias[j];
#pragma unroll 1
  for (int i = 0; i < cols; ++i) {  // (registers shift down: none is indexed by a variable)
    float g[1] = {f[0]}, b[1] = {rest[0]};
    load_aux<1>(p, r, c + i, x);
    finish_cols<KIND, 1>(e, p, r, c + i, g, b, x);
#pragma unroll
    for (int j = 0; j < NV - 1; ++j) {
      f[j] = f[j + 1];
      rest[j] = rest[j + 1];
    }
  }
}

}  // namespace

}  // namespace numbat
