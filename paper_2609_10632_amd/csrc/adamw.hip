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
// reduction; 4096-element chunks of all tensors are numbered in table order and dealt to blocks in
// contiguous ranges.  Bound by the bytes: 28 per element with fp32 moments, 16 with 8-bit ones.
#include "mlp_kernels.h"

namespace numbat {

namespace {

constexpr int kThreads = 256;
constexpr int kChunk = 4096;

// the table in LDS, and s_first[t] = chunks of the tensors before t (s_first[count] = all)
__device__ __forceinline__ void stage_table(const AdamTensor* tab, int count, AdamTensor* s_tab, int64_t* s_first) {
  __shared__ int64_t s_sum[kThreads];
  const int t = threadIdx.x;
  const int words = count * (int)(sizeof(AdamTensor) / 4);
  const uint32_t* src = reinterpret_cast<const uint32_t*>(tab);
  uint32_t* dst = reinterpret_cast<uint32_t*>(s_tab);
  for (int i = t; i < words; i += kThreads) dst[i] = src[i];
  __syncthreads();
  // thread t counts the chunks of tensors 4 t .. 4 t + 3
  int64_t c[4], local = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int i = 4 * t + j;
    const int64_t n = i < count ? s_tab[i].n : 0;
    c[j] = n > 0 ? (n + kChunk - 1) / kChunk : 0;
    local += c[j];
  }
  s_sum[t] = local;
  __syncthreads();
  for (int d = 1; d < kThreads; d <<= 1) {
    const int64_t v = t >= d ? s_sum[t - d] : 0;
    __syncthreads();
    s_sum[t] += v;
    __syncthreads();
  }
  int64_t run = s_sum[t] - local;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int i = 4 * t + j;
    if (i < count) s_first[i] = run;
    run += c[j];
  }
  if (t == 0) s_first[count] = s_sum[kThreads - 1];
  __syncthreads();
}

// f(T, first element, elements) for every chunk of this block
template <typename F>
__device__ __forceinline__ void for_my_chunks(const AdamTensor* s_tab, const int64_t* s_first, int count, F&& f) {
  const int64_t total = s_first[count];
  const int64_t per = (total + gridDim.x - 1) / gridDim.x;
  int64_t k = (int64_t)blockIdx.x * per;
  const int64_t kend = k + per < total ? k + per : total;
  if (k >= kend) return;
  int lo = 0, hi = count - 1;  // the last tensor whose first chunk is at or before k
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (s_first[mid] <= k) lo = mid;
    else hi = mid - 1;
  }
  for (int t = lo; k < kend; ++k) {
    while (s_first[t + 1] <= k) ++t;  // (tensors without elements have no chunks)
    const AdamTensor& T = s_tab[t];
    const int64_t off = (k - s_first[t]) * kChunk;
    f(T, off, (int)(T.n - off < kChunk ? T.n - off : kChunk));
  }
}

__device__ __forceinline__ bool aligned(const void* p, int bytes) {
  return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0;
}

// four gradients from element i of a tensor of which `left` elements remain from there
__device__ __forceinline__ void load_grad(const AdamTensor& T, int64_t i, int left, float (&g)[4]) {
  if (T.g_type == 0) {  // bf16
    const bf16_t* p = static_cast<const bf16_t*>(T.g) + i;
    if (left >= 4 && aligned(p, 8)) {
      const uint2 v = *reinterpret_cast<const uint2*>(p);
      g[0] = bf2f(v.x & 0xffffu); g[1] = bf2f(v.x >> 16);
      g[2] = bf2f(v.y & 0xffffu); g[3] = bf2f(v.y >> 16);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) g[e] = e < left ? bf2f(p[e]) : 0.f;
    }
  } else {
    const float* p = static_cast<const float*>(T.g) + i;
    if (left >= 4 && aligned(p, 16)) {
      const float4 v = *reinterpret_cast<const float4*>(p);
      g[0] = v.x; g[1] = v.y; g[2] = v.z; g[3] = v.w;
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) g[e] = e < left ? p[e] : 0.f;
    }
  }
}
__device__ __forceinline__ void load4(const float* p, int left, float (&f)[4]) {
  if (left >= 4 && aligned(p, 16)) {
    const float4 v = *reinterpret_cast<const float4*>(p);
    f[0] = v.x; f[1] = v.y; f[2] = v.z; f[3] = v.w;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) f[e] = e < left ? p[e] : 0.f;
  }
}
__device__ __forceinline__ void store4(float* p, int left, const float (&f)[4]) {
  if (left >= 4 && aligned(p, 16)) {
    *reinterpret_cast<float4*>(p) = make_float4(f[0], f[1], f[2], f[3]);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < left) p[e] = f[e];
  }
}
__device__ __forceinline__ void store4(bf16_t* p, int left, const float (&f)[4]) {
  if (left >= 4 && aligned(p, 8)) {
    *reinterpret_cast<uint2*>(p) = make_uint2(pack2(f[0], f[1]), pack2(f[2], f[3]));
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < left) p[e] = (bf16_t)f2bf(f[e]);
  }
}
__device__ __forceinline__ uint32_t load_codes(const void* q, int64_t i, int left) {
  const uint8_t* p = static_cast<const uint8_t*>(q) + i;
  if (left >= 4 && aligned(p, 4)) return *reinterpret_cast<const uint32_t*>(p);
  uint32_t v = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (e < left) v |= (uint32_t)p[e] << (8 * e);
  return v;
}
__device__ __forceinline__ void store_codes(void* q, int64_t i, int left, uint32_t v) {
  uint8_t* p = static_cast<uint8_t*>(q) + i;
  if (left >= 4 && aligned(p, 4)) {
    *reinterpret_cast<uint32_t*>(p) = v;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < left) p[e] = (uint8_t)(v >> (8 * e));
  }
}

__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) x = fmaxf(x, __shfl_xor(x, d));
  return x;
}

// a block's unit (zero where it would not be a normal number: the block is stored as zeros) and
// its reciprocal
__device__ __forceinline__ void unit_of(float largest, float scale, float& u, float& inv) {
  u = largest * scale;
  if (u < 1.17549435e-38f) u = 0.f;
  inv = u > 0.f ? 1.0f / u : 0.f;
}

// the value of code q of a first moment / of the root of a second one
__device__ __forceinline__ float m_value(float u, float q) { return u * (q * fabsf(q)); }
__device__ __forceinline__ float r_value(float u, float q) { return u * (q * q); }

__global__ __launch_bounds__(kThreads) void adamw_norm_kernel(AdamArgs a) {
  extern __shared__ unsigned char s_dyn[];
  AdamTensor* s_tab = reinterpret_cast<AdamTensor*>(s_dyn);
  int64_t* s_first = reinterpret_cast<int64_t*>(s_dyn + (size_t)a.count * sizeof(AdamTensor));
  __shared__ double s_w[kThreads / 64];
  stage_table(a.tab, a.count, s_tab, s_first);
  double acc = 0.0;
  for_my_chunks(s_tab, s_first, a.count, [&](const AdamTensor& T, int64_t off, int len) {
#pragma unroll
    for (int r = 0; r < kChunk / (4 * kThreads); ++r) {
      const int i = 4 * ((int)threadIdx.x + r * kThreads);
      if (i < len) {
        float g[4];
        load_grad(T, off + i, len - i, g);
        acc += (double)g[0] * g[0] + (double)g[1] * g[1] + (double)g[2] * g[2] + (double)g[3] * g[3];
      }
    }
  });
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) acc += __shfl_xor(acc, d);
  if ((threadIdx.x & 63) == 0) s_w[threadIdx.x >> 6] = acc;
  __syncthreads();
  if (threadIdx.x == 0) a.part[blockIdx.x] = (s_w[0] + s_w[1]) + (s_w[2] + s_w[3]);
}

template <int BITS>
__global__ __launch_bounds__(kThreads) void adamw_kernel(AdamArgs a) {
#pragma clang fp contract(off)
  extern __shared__ unsigned char s_dyn[];
  AdamTensor* s_tab = reinterpret_cast<AdamTensor*>(s_dyn);
  int64_t* s_first = reinterpret_cast<int64_t*>(s_dyn + (size_t)a.count * sizeof(AdamTensor));
  __shared__ float s_coef;
  if (threadIdx.x < 64) {
    float coef = 1.f;
    if (a.max_norm > 0.f) {
      // lane l sums partials l, l + 64, ..., then a fixed butterfly over the wave
      double s = 0.0;
      for (int i = threadIdx.x; i < kAdamBlocks; i += 64) s += a.part[i];
#pragma unroll
      for (int d = 32; d >= 1; d >>= 1) s += __shfl_xor(s, d);
      const double total = sqrt(s), c = (double)a.max_norm / (total + 1e-6);
      coef = (float)(c < 1.0 ? c : 1.0);
      if (blockIdx.x == 0 && threadIdx.x == 0 && a.total_norm != nullptr) *a.total_norm = (float)total;
    }
    if (threadIdx.x == 0) s_coef = coef;
  }
  stage_table(a.tab, a.count, s_tab, s_first);  // (its barriers also publish s_coef)
  const float coef = s_coef;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  for_my_chunks(s_tab, s_first, a.count, [&](const AdamTensor& T, int64_t off, int len) {
#pragma clang fp contract(off)
    if (T.group < 0 || T.group >= a.ngroups) return;  // outside the given groups: left unchanged
    const float lr = a.lr[T.group], keep = a.keep[T.group];
#pragma unroll 1
    for (int r = 0; r < kChunk / (4 * kThreads); ++r) {
      const int b = (r * (kThreads / 64) + wave) * kAdamBlock;  // this wave's block within the chunk
      if (b >= len) break;
      const int i = b + 4 * lane, left = len - i;
      const int64_t at = off + i;
      float w[4], g[4], m[4], v[4];
      load4(T.w + at, left, w);
      load_grad(T, at, left, g);
      if constexpr (BITS == 32) {
        load4(static_cast<float*>(T.m) + at, left, m);
        load4(static_cast<float*>(T.v) + at, left, v);
      } else {
        const int64_t blk = (off + b) / kAdamBlock;
        const float um = T.m_unit[blk], uv = T.v_unit[blk];
        const uint32_t qm = load_codes(T.m, at, left), qv = load_codes(T.v, at, left);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          m[e] = m_value(um, (float)(int8_t)(qm >> (8 * e)));
          const float root = r_value(uv, (float)((qv >> (8 * e)) & 255u));
          v[e] = root * root;
        }
      }
      float root[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float d = a.max_norm > 0.f ? g[e] * coef : g[e];
        m[e] = m[e] * a.b1 + d * a.omb1;
        v[e] = v[e] * a.b2 + (d * d) * a.omb2;
        root[e] = sqrtf(v[e]);
        w[e] = w[e] * keep - lr * (m[e] / (root[e] * a.rsqrt_bc2 + a.eps));
      }
      store4(T.w + at, left, w);
      if (T.w_copy != nullptr) store4(T.w_copy + at, left, w);
      if constexpr (BITS == 32) {
        store4(static_cast<float*>(T.m) + at, left, m);
        store4(static_cast<float*>(T.v) + at, left, v);
      } else {
        // (elements past the end hold zeros: they change neither maximum; a moment that is not finite
        // takes the largest code and leaves the block's unit to the others)
        float lm = 0.f, lv = 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          lm = fabsf(m[e]) < INFINITY ? fmaxf(lm, fabsf(m[e])) : lm;
          lv = root[e] < INFINITY ? fmaxf(lv, root[e]) : lv;
        }
        float um, im, uv, iv;
        unit_of(wave_max(lm), 1.0f / (127.0f * 127.0f), um, im);
        unit_of(wave_max(lv), 1.0f / (255.0f * 255.0f), uv, iv);
        uint32_t qm = 0, qv = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float s = fminf(rintf(sqrtf(fabsf(m[e]) * im)), 127.f);
          const int q = (int)s;
          qm |= ((uint32_t)(m[e] < 0.f ? -q : q) & 255u) << (8 * e);
          float t = fminf(rintf(sqrtf(root[e] * iv)), 255.f);
          if (root[e] > 0.f) t = fmaxf(t, 1.f);
          qv |= (uint32_t)(int)t << (8 * e);
        }
        store_codes(T.m, at, left, qm);
        store_codes(T.v, at, left, qv);
        if (lane == 0) {
          const int64_t blk = (off + b) / kAdamBlock;
          T.m_unit[blk] = um;
          T.v_unit[blk] = uv;
        }
      }
    }
  });
}

__global__ __launch_bounds__(256) void adamw_values_kernel(int64_t n, const int8_t* m, const float* m_unit,
                                                           const uint8_t* v, const float* v_unit, float* mo, float* vo) {
  for (int64_t i = 4 * (blockIdx.x * 256ll + threadIdx.x); i < n; i += 4 * 256ll * gridDim.x) {
    const int left = n - i < 4 ? (int)(n - i) : 4;
    const float um = m_unit[i / kAdamBlock], uv = v_unit[i / kAdamBlock];
    const uint32_t qm = load_codes(m, i, left), qv = load_codes(v, i, left);
    float a[4], b[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      a[e] = m_value(um, (float)(int8_t)(qm >> (8 * e)));
      const float root = r_value(uv, (float)((qv >> (8 * e)) & 255u));
      b[e] = root * root;
    }
    store4(mo + i, left, a);
    store4(vo + i, left, b);
  }
}

}  // namespace

hipError_t adamw_launch(const AdamArgs& a, int bits, hipStream_t s) {
  const size_t smem = (size_t)a.count * sizeof(AdamTensor) + (size_t)(a.count + 1) * sizeof(int64_t);
  if (a.max_norm > 0.f) {
    trace_begin(KC_ADAMW_NORM);
    NUMBAT_LAUNCH(adamw_norm_kernel, dim3(kAdamBlocks), dim3(kThreads), smem, s, a);
    trace_end(KC_ADAMW_NORM);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  trace_begin(KC_ADAMW);
  if (bits == 8) NUMBAT_LAUNCH(adamw_kernel<8>, dim3(kAdamBlocks), dim3(kThreads), smem, s, a);
  else NUMBAT_LAUNCH(adamw_kernel<32>, dim3(kAdamBlocks), dim3(kThreads), smem, s, a);
  trace_end(KC_ADAMW);
  return hipGetLastError();
}

hipError_t adamw_values_launch(int64_t n, const int8_t* m, const float* m_unit, const uint8_t* v, const float* v_unit,
                               float* mo, float* vo, hipStream_t s) {
  const int64_t blocks = (n + 1023) / 1024;
  trace_begin(KC_ADAMW);
  NUMBAT_LAUNCH(adamw_values_kernel, dim3((unsigned)(blocks < 8192 ? blocks : 8192)), dim3(256), 0, s, n, m, m_unit, v,
                v_unit, mo, vo);
  trace_end(KC_ADAMW);
  return hipGetLastError();
}

}  // namespace numbat
