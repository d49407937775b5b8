// The AdamW step over a table of parameter tensors, with moments in fp32 or in 8 bits, on gfx950.
//   g = c grad;  m = b1 m + (1 - b1) g;  v = b2 v + (1 - b2) g^2
//   w = w (1 - lr wd) - lr / (1 - b1^t) * m / (sqrt(v / (1 - b2^t)) + eps)
// c is 1, or the global-norm clip's min(1, max_norm / (norm + 1e-6)) from a first pass over the
// gradients (fp64 partials per block, added in a fixed order by every block of the update).
//
// 8-bit moments are held in blocks of 256 elements of a tensor with one fp32 unit each:
//   m = u q |q|, q in -127 .. 127, u = max|m| / 127^2
//   v = r^2,  r = u q^2,  q in 0 .. 255, u = max r / 255^2
// The square spaces the codes evenly in sqrt|m| and sqrt(r): a moment that is a thousandth of its
// block's largest still has 4 codes below it.  v is held by its root, whose size is what the
// update divides by, and a v above zero never takes the code 0: a denominator that rounded away
// to zero would make a step of lr m / eps.  The step itself uses the new moments before they are
// rounded.  The arithmetic up to the codes is plain IEEE fp32 without contraction, so that codes
// do not depend on how a compiler joins multiplies and adds.
//
// A wave takes a block of 256 elements, four per lane, so a block's largest moment is one wave
// reduction; 4096-element chunks of all tensors are numbered in table order and dealt to thread
// blocks in contiguous ranges.  A thread loads everything of its four rounds of a whole, aligned
// chunk before it computes any of it.  Bound by the bytes, read and written: 30 per element with fp32
// moments, gradients and a bf16 copy (25.9 million elements of 243 tensors 143 us, 5.5 TB/s; the norm's
// pass over 104 MB of gradients 32 to 38 us, what reading alone reaches here), 16 with 8-bit moments and bf16
// gradients (134 million 470 us, 4.6 TB/s).
#include <type_traits>

#include "mlp_kernels.h"

namespace numbat {

namespace {

constexpr int kThreads = 256;
constexpr int kChunk = 4096;

// s_first[t] = chunks of the tensors before t, s_first[count] = all
__device__ __forceinline__ void count_chunks(const AdamTensor* tab, int count, int64_t* s_first) {
  __shared__ int64_t s_wave[kThreads / 64];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  // thread t counts the chunks of tensors 4 t .. 4 t + 3; an inclusive scan over the wave, then the
  // waves before it
  int64_t n[4], c[4], local = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) n[j] = 4 * t + j < count ? tab[4 * t + j].n : 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    c[j] = n[j] > 0 ? (n[j] + kChunk - 1) / kChunk : 0;
    local += c[j];
  }
  int64_t run = local;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int64_t v = __shfl_up(run, d);
    run += lane >= d ? v : 0;
  }
  if (lane == 63) s_wave[wave] = run;
  __syncthreads();
  run -= local;
  for (int w = 0; w < wave; ++w) run += s_wave[w];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int i = 4 * t + j;
    if (i < count) s_first[i] = run;
    run += c[j];
  }
  if (t == kThreads - 1) s_first[count] = run;
  __syncthreads();
}

// f(T, first element, elements) for every chunk of this block; the entries are read by scalar loads
template <typename F>
__device__ __forceinline__ void for_my_chunks(const AdamTensor* tab, const int64_t* s_first, int count, F&& f) {
  const int64_t total = s_first[count];
  int64_t k = total * blockIdx.x / gridDim.x;
  const int64_t kend = total * (blockIdx.x + 1) / gridDim.x;
  if (k >= kend) return;
  int lo = 0, hi = count - 1;  // the last tensor whose first chunk is at or before k
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (s_first[mid] <= k) lo = mid;
    else hi = mid - 1;
  }
  typedef const __attribute__((address_space(4))) AdamTensor* Entry;
  for (int t = lo; k < kend; ++k) {
    while (s_first[t + 1] <= k) ++t;  // (tensors without elements have no chunks)
    t = __builtin_amdgcn_readfirstlane(t);
    const Entry e = (Entry)(tab + t);
    AdamTensor T;
    T.w = e->w;
    T.g = e->g;
    T.m = e->m;
    T.v = e->v;
    T.m_unit = e->m_unit;
    T.v_unit = e->v_unit;
    T.w_copy = e->w_copy;
    T.n = e->n;
    T.group = e->group;
    T.g_type = e->g_type;
    const int64_t off = (k - s_first[t]) * kChunk;
    f(T, off, (int)(T.n - off < kChunk ? T.n - off : kChunk));
  }
}

__device__ __forceinline__ bool aligned(const void* p, int bytes) {
  return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0;
}

// Pointers out of the table, as the global memory's that they are.
template <typename T>
using Global = __attribute__((address_space(1))) T*;
template <typename T>
__device__ __forceinline__ Global<T> global(const void* p, int64_t i) {
  return (Global<T>)(const_cast<T*>(static_cast<const T*>(p)) + i);
}
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// Four elements from element i of a tensor of which `left` remain from there (none or fewer: zeros).
// WHOLE: there are four, and the place allows one access.
template <bool WHOLE>
__device__ __forceinline__ void load4(const float* base, int64_t i, int left, float (&f)[4]) {
  const Global<float> p = global<float>(base, i);
  if (WHOLE || (left >= 4 && aligned(base + i, 16))) {
    const f32x4 v = *(Global<f32x4>)p;
#pragma unroll
    for (int e = 0; e < 4; ++e) f[e] = v[e];
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) f[e] = e < left ? p[e] : 0.f;
  }
}
template <bool WHOLE>
__device__ __forceinline__ void load_grad(const AdamTensor& T, int64_t i, int left, float (&g)[4]) {
  if (T.g_type != 0) return load4<WHOLE>(static_cast<const float*>(T.g), i, left, g);
  const bf16_t* at = static_cast<const bf16_t*>(T.g) + i;
  const Global<bf16_t> p = global<bf16_t>(at, 0);
  if (WHOLE || (left >= 4 && aligned(at, 8))) {
    const u32x2 v = *(Global<u32x2>)p;
    g[0] = bf2f(v.x & 0xffffu);
    g[1] = __uint_as_float(v.x & 0xffff0000u);
    g[2] = bf2f(v.y & 0xffffu);
    g[3] = __uint_as_float(v.y & 0xffff0000u);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) g[e] = e < left ? bf2f(p[e]) : 0.f;
  }
}
template <bool WHOLE>
__device__ __forceinline__ void store4(float* base, int64_t i, int left, const float (&f)[4]) {
  const Global<float> p = global<float>(base, i);
  if (WHOLE || (left >= 4 && aligned(base + i, 16))) {
    *(Global<f32x4>)p = f32x4{f[0], f[1], f[2], f[3]};
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < left) p[e] = f[e];
  }
}
template <bool WHOLE>
__device__ __forceinline__ void store4(bf16_t* base, int64_t i, int left, const float (&f)[4]) {
  const Global<bf16_t> p = global<bf16_t>(base, i);
  if (WHOLE || (left >= 4 && aligned(base + i, 8))) {
    *(Global<u32x2>)p = u32x2{pack2(f[0], f[1]), pack2(f[2], f[3])};
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < left) p[e] = (bf16_t)f2bf(f[e]);
  }
}
template <bool WHOLE>
__device__ __forceinline__ uint32_t load_codes(const void* q, int64_t i, int left) {
  const Global<uint8_t> p = global<uint8_t>(q, i);
  if (WHOLE || (left >= 4 && aligned(static_cast<const uint8_t*>(q) + i, 4))) return *(Global<uint32_t>)p;
  uint32_t v = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (e < left) v |= (uint32_t)p[e] << (8 * e);
  return v;
}
template <bool WHOLE>
__device__ __forceinline__ void store_codes(void* q, int64_t i, int left, uint32_t v) {
  const Global<uint8_t> p = global<uint8_t>(q, i);
  if (WHOLE || (left >= 4 && aligned(static_cast<uint8_t*>(q) + i, 4))) {
    *(Global<uint32_t>)p = v;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < left) p[e] = (uint8_t)(v >> (8 * e));
  }
}

// The largest of the wave's values, by their bits: floats at or above zero are ordered as their bits
// are, and an integer maximum needs no care for NaNs.
__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
  // shifts by 1, 2, 4 and 8 lanes within rows of 16, then each row's last lane to the next rows: lane
  // 63 ends with the largest of all (lanes that nothing is shifted into take 0)
#define NUMBAT_DPP_MAX(ctrl, rows)                                                              \
  {                                                                                             \
    const uint32_t y = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, ctrl, rows, 0xf, false); \
    x = x > y ? x : y;                                                                          \
  }
  NUMBAT_DPP_MAX(0x111, 0xf);
  NUMBAT_DPP_MAX(0x112, 0xf);
  NUMBAT_DPP_MAX(0x114, 0xf);
  NUMBAT_DPP_MAX(0x118, 0xf);
  NUMBAT_DPP_MAX(0x142, 0xa);
  NUMBAT_DPP_MAX(0x143, 0xc);
#undef NUMBAT_DPP_MAX
  return (uint32_t)__builtin_amdgcn_readlane((int)x, 63);
}
constexpr uint32_t kInfBits = 0x7f800000u;
// of four values per lane, none below zero; those that are not finite do not count
__device__ __forceinline__ uint32_t largest_of(const float (&f)[4]) {
  uint32_t b[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) b[e] = __float_as_uint(f[e]) & 0x7fffffffu;
  auto m4 = [&]() { return max(max(b[0], b[1]), max(b[2], b[3])); };
  uint32_t x = wave_max(m4());
  if (x >= kInfBits) {
#pragma unroll
    for (int e = 0; e < 4; ++e) b[e] = b[e] < kInfBits ? b[e] : 0u;
    x = wave_max(m4());
  }
  return x;
}

// Codes: rint(sqrt(x inv)) of the IEEE root, at most `most`, for four x >= 0.  The hardware's root
// gives the same integer unless it lies next to a half; then, for about one wave in twenty, all four
// are formed again from the library's.
__device__ __forceinline__ void encode4(const float (&x)[4], float inv, float most, float (&q)[4]) {
#pragma clang fp contract(off)
  float s[4], far = 0.f;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    s[e] = __builtin_amdgcn_sqrtf(x[e] * inv);
    q[e] = rintf(s[e]);
    far = fmaxf(far, fabsf(s[e] - q[e]));  // exact; 0.5 is a tie, and an ulp of 255 is 2^-16
  }
  if (far > 0.5f - 0x1p-13f) {
#pragma unroll
    for (int e = 0; e < 4; ++e) q[e] = rintf(sqrtf(x[e] * inv));
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) q[e] = fminf(q[e], most);
}

// A block's units (zero where one would not be a normal number: those moments are stored as zeros)
// and their reciprocals, both from one division: the first half of the wave forms those of m, the
// second those of v.
__device__ __forceinline__ void units_of(uint32_t largest_m, uint32_t largest_v, float& um, float& im, float& uv,
                                         float& iv) {
  const bool second = (threadIdx.x & 32) != 0;
  float u = __uint_as_float(second ? largest_v : largest_m) * (second ? 1.0f / (255.0f * 255.0f) : 1.0f / (127.0f * 127.0f));
  if (u < 1.17549435e-38f) u = 0.f;
  const float inv = u > 0.f ? 1.0f / u : 0.f;
  um = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(u), 0));
  uv = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(u), 32));
  im = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(inv), 0));
  iv = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(inv), 32));
}

// the value of code q of a first moment / of the root of a second one
__device__ __forceinline__ float m_value(float u, float q) { return u * (q * fabsf(q)); }
__device__ __forceinline__ float r_value(float u, float q) { return u * (q * q); }

constexpr int kRounds = kChunk / (4 * kThreads);

__global__ __launch_bounds__(kThreads) void adamw_norm_kernel(AdamArgs a) {
  __shared__ int64_t s_first[kAdamMaxTensors + 1];
  __shared__ double s_w[kThreads / 64];
  count_chunks(a.tab, a.count, s_first);
  double acc = 0.0;
  for_my_chunks(a.tab, s_first, a.count, [&](const AdamTensor& T, int64_t off, int len) {
    auto chunk = [&](auto wc) __attribute__((always_inline)) {
      float g[kRounds][4];
#pragma unroll
      for (int r = 0; r < kRounds; ++r) {
        const int i = 4 * ((int)threadIdx.x + r * kThreads);
        load_grad<decltype(wc)::value>(T, off + i, len - i, g[r]);
      }
#pragma unroll
      for (int r = 0; r < kRounds; ++r)
        acc += ((double)g[r][0] * g[r][0] + (double)g[r][1] * g[r][1]) +
               ((double)g[r][2] * g[r][2] + (double)g[r][3] * g[r][3]);
    };
    if (len == kChunk && aligned(T.g, T.g_type == 0 ? 8 : 16)) chunk(std::true_type{});
    else chunk(std::false_type{});
  });
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) acc += __shfl_xor(acc, d);
  if ((threadIdx.x & 63) == 0) s_w[threadIdx.x >> 6] = acc;
  __syncthreads();
  if (threadIdx.x == 0) a.part[blockIdx.x] = (s_w[0] + s_w[1]) + (s_w[2] + s_w[3]);
}

// what a thread holds of four consecutive elements
template <int BITS>
struct Quad {
  float w[4], g[4];
  float m[4], v[4];  // 32-bit state
  uint32_t qm, qv;   // 8-bit state
  float um, uv;
};

template <bool WHOLE, int BITS>
__device__ __forceinline__ void load_quad(const AdamTensor& T, int64_t at, int left, Quad<BITS>& q) {
  load4<WHOLE>(T.w, at, left, q.w);
  load_grad<WHOLE>(T, at, left, q.g);
  if constexpr (BITS == 32) {
    load4<WHOLE>(static_cast<float*>(T.m), at, left, q.m);
    load4<WHOLE>(static_cast<float*>(T.v), at, left, q.v);
  } else {
    q.qm = load_codes<WHOLE>(T.m, at, left);
    q.qv = load_codes<WHOLE>(T.v, at, left);
    const int64_t blk = WHOLE || left > 0 ? at / kAdamBlock : 0;
    q.um = *global<float>(T.m_unit, blk);
    q.uv = *global<float>(T.v_unit, blk);
  }
}

// the update of four elements, of which `left` are in the tensor (every lane of a wave calls it)
template <bool WHOLE, int BITS>
__device__ __forceinline__ void update_quad(const AdamArgs& a, const AdamTensor& T, int64_t at, int left, float lr,
                                            float keep, float coef, Quad<BITS>& q) {
#pragma clang fp contract(off)
  float m[4], v[4], root[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if constexpr (BITS == 32) {
      m[e] = q.m[e];
      v[e] = q.v[e];
    } else {
      m[e] = m_value(q.um, (float)(int8_t)(q.qm >> (8 * e)));
      const float r = r_value(q.uv, (float)((q.qv >> (8 * e)) & 255u));
      v[e] = r * r;
    }
    const float d = q.g[e] * coef;  // (1 without clipping)
    m[e] = m[e] * a.b1 + d * a.omb1;
    v[e] = v[e] * a.b2 + (d * d) * a.omb2;
  }
  // (the codes of 8-bit state need the root as IEEE rounds it; the step takes the hardware's root and
  // reciprocal, 1 ulp each)
  if constexpr (BITS == 32) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      // (the hardware's root takes a v below the normal numbers for zero: scaled by powers of two, exact)
      const bool small = v[e] < 0x1p-126f;
      root[e] = __builtin_amdgcn_sqrtf(small ? v[e] * 0x1p48f : v[e]) * (small ? 0x1p-24f : 1.0f);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) root[e] = sqrtf(v[e]);
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float step = m[e] * __builtin_amdgcn_rcpf(__builtin_fmaf(root[e], a.rsqrt_bc2, a.eps));
    q.w[e] = __builtin_fmaf(-lr, step, q.w[e] * keep);
  }
  store4<WHOLE>(T.w, at, left, q.w);
  if (T.w_copy != nullptr) store4<WHOLE>(T.w_copy, at, left, q.w);
  if constexpr (BITS == 32) {
    store4<WHOLE>(static_cast<float*>(T.m), at, left, m);
    store4<WHOLE>(static_cast<float*>(T.v), at, left, v);
  } else {
    // (elements past the end hold zeros: they change neither maximum; a moment that is not finite
    // takes the largest code and leaves the block's unit to the others)
    float um, im, uv, iv, cm[4], cv[4], am[4];
    units_of(largest_of(m), largest_of(root), um, im, uv, iv);
#pragma unroll
    for (int e = 0; e < 4; ++e) am[e] = fabsf(m[e]);
    encode4(am, im, 127.f, cm);
    encode4(root, iv, 255.f, cv);
    uint32_t qm = 0, qv = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      qm |= ((uint32_t)(int)__builtin_copysignf(cm[e], m[e]) & 255u) << (8 * e);
      qv |= (uint32_t)(int)(root[e] > 0.f ? fmaxf(cv[e], 1.f) : cv[e]) << (8 * e);
    }
    store_codes<WHOLE>(T.m, at, left, qm);
    store_codes<WHOLE>(T.v, at, left, qv);
    if ((threadIdx.x & 63) == 0 && (WHOLE || left > 0)) {
      *global<float>(T.m_unit, at / kAdamBlock) = um;
      *global<float>(T.v_unit, at / kAdamBlock) = uv;
    }
  }
}

template <int BITS>
__global__ __launch_bounds__(kThreads) void adamw_kernel(AdamArgs a) {
  __shared__ int64_t s_first[kAdamMaxTensors + 1];
  __shared__ float s_coef;
  if (threadIdx.x < 64) {
    float coef = 1.f;
    if (a.max_norm > 0.f) {
      // lane l sums partials l, l + 64, ..., then a fixed butterfly over the wave
      double p[kAdamNormBlocks / 64], s = 0.0;
#pragma unroll
      for (int i = 0; i < kAdamNormBlocks / 64; ++i) p[i] = a.part[threadIdx.x + 64 * i];
#pragma unroll
      for (int i = 0; i < kAdamNormBlocks / 64; ++i) s += p[i];
#pragma unroll
      for (int d = 32; d >= 1; d >>= 1) s += __shfl_xor(s, d);
      const double total = sqrt(s), c = (double)a.max_norm / (total + 1e-6);
      coef = (float)(c < 1.0 ? c : 1.0);
      if (blockIdx.x == 0 && threadIdx.x == 0 && a.total_norm != nullptr) *a.total_norm = (float)total;
    }
    if (threadIdx.x == 0) s_coef = coef;
  }
  count_chunks(a.tab, a.count, s_first);  // (its barriers also publish s_coef)
  const float coef = s_coef;
  for_my_chunks(a.tab, s_first, a.count, [&](const AdamTensor& T, int64_t off, int len) {
    if (T.group < 0 || T.group >= a.ngroups) return;  // outside the given groups: left unchanged
    const float lr = a.lr[T.group], keep = a.keep[T.group];
    const bool whole = len == kChunk && aligned(T.w, 16) && aligned(T.g, T.g_type == 0 ? 8 : 16) &&
                       aligned(T.m, BITS == 32 ? 16 : 4) && aligned(T.v, BITS == 32 ? 16 : 4) && aligned(T.w_copy, 8);
    auto chunk = [&](auto wc) __attribute__((always_inline)) {
      constexpr bool WHOLE = decltype(wc)::value;
      Quad<BITS> q[kRounds];
#pragma unroll
      for (int r = 0; r < kRounds; ++r) {
        const int i = 4 * ((int)threadIdx.x + r * kThreads);
        load_quad<WHOLE>(T, off + i, len - i, q[r]);
      }
#pragma unroll
      for (int r = 0; r < kRounds; ++r) {
        const int i = 4 * ((int)threadIdx.x + r * kThreads);
        update_quad<WHOLE>(a, T, off + i, len - i, lr, keep, coef, q[r]);
      }
    };
    if (whole) chunk(std::true_type{});
    else chunk(std::false_type{});
  });
}

// a thread takes four elements of each of four groups of 1024
__global__ __launch_bounds__(256) void adamw_values_kernel(int64_t n, const int8_t* m, const float* m_unit,
                                                           const uint8_t* v, const float* v_unit, float* mo, float* vo) {
  const bool apart = !(aligned(m, 4) && aligned(v, 4) && aligned(mo, 16) && aligned(vo, 16));
  auto chunk = [&](auto wc, int64_t base) __attribute__((always_inline)) {
    constexpr bool WHOLE = decltype(wc)::value;
    uint32_t qm[kRounds], qv[kRounds];
    float um[kRounds], uv[kRounds];
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
      const int64_t i = base + 4 * ((int)threadIdx.x + r * kThreads);
      const int left = n - i < 4 ? (int)(n - i > 0 ? n - i : 0) : 4;
      qm[r] = load_codes<WHOLE>(m, i, left);
      qv[r] = load_codes<WHOLE>(v, i, left);
      um[r] = left > 0 ? m_unit[i / kAdamBlock] : 0.f;
      uv[r] = left > 0 ? v_unit[i / kAdamBlock] : 0.f;
    }
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
      const int64_t i = base + 4 * ((int)threadIdx.x + r * kThreads);
      const int left = n - i < 4 ? (int)(n - i > 0 ? n - i : 0) : 4;
      float x[4], y[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[e] = m_value(um[r], (float)(int8_t)(qm[r] >> (8 * e)));
        const float root = r_value(uv[r], (float)((qv[r] >> (8 * e)) & 255u));
        y[e] = root * root;
      }
      store4<WHOLE>(mo, i, left, x);
      store4<WHOLE>(vo, i, left, y);
    }
  };
  for (int64_t base = (int64_t)blockIdx.x * kChunk; base < n; base += (int64_t)gridDim.x * kChunk) {
    if (!apart && n - base >= kChunk) chunk(std::true_type{}, base);
    else chunk(std::false_type{}, base);
  }
}

}  // namespace

hipError_t adamw_launch(const AdamArgs& a, int bits, hipStream_t s) {
  if (a.max_norm > 0.f) {
    trace_begin(KC_ADAMW_NORM);
    NUMBAT_LAUNCH(adamw_norm_kernel, dim3(kAdamNormBlocks), dim3(kThreads), 0, s, a);
    trace_end(KC_ADAMW_NORM);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  trace_begin(KC_ADAMW);
  if (bits == 8) NUMBAT_LAUNCH(adamw_kernel<8>, dim3(kAdamBlocks), dim3(kThreads), 0, s, a);
  else NUMBAT_LAUNCH(adamw_kernel<32>, dim3(kAdamBlocks), dim3(kThreads), 0, s, a);
  trace_end(KC_ADAMW);
  return hipGetLastError();
}

hipError_t adamw_values_launch(int64_t n, const int8_t* m, const float* m_unit, const uint8_t* v, const float* v_unit,
                               float* mo, float* vo, hipStream_t s) {
  const int64_t blocks = (n + kChunk - 1) / kChunk;
  trace_begin(KC_ADAMW);
  NUMBAT_LAUNCH(adamw_values_kernel, dim3((unsigned)(blocks < 16384 ? blocks : 16384)), dim3(256), 0, s, n, m, m_unit, v,
                v_unit, mo, vo);
  trace_end(KC_ADAMW);
  return hipGetLastError();
}

}  // namespace numbat
