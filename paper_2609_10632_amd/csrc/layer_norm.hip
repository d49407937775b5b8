// Layer norm over the features of each row, forward and backward, on gfx950.
//   forward   y = gamma xh + beta,  xh = (x - mean) rstd,  rstd = (var + eps)^-1/2
//   backward  h = gamma dy;  dx = rstd (h - mean_c(h) - xh mean_c(h xh)) [+ the residual's gradient]
//             dgamma = sum_rows dy xh,  dbeta = sum_rows dy
// A row belongs to a group of G lanes (part of a wave, a wave, or a block of waves) which keeps
// it in registers: one pass over memory, the mean first and the variance from the centred values
// (no cancellation).  (The backward of 8193 to 16384 features, whose 1024 threads have 128 registers
// each, spills 60 to 188 bytes a lane in its loop; of 4097 to 8192 those of bf16 x with fp32 y, 28, and of
// fp32 x with odd rows, 8 or 16.)  Lanes hold 16-byte vectors where the rows allow them and single elements
// otherwise; a lane's columns are the same for every row, so the backward adds dgamma and dbeta in
// registers over all rows of a block and writes one partial per block, which a second kernel sums
// in a fixed order.  Everything is bound by the bytes of the rows: gradients of 102400 x 192 bf16 with the
// residual's 35 us (4.5 TB/s), of 16384 x 8192 fp32 346 us (5.4 TB/s); 16 x 4096 forward 3.4 us, a launch.
#include <algorithm>

#include "mlp_kernels.h"

namespace numbat {

namespace {

__device__ __forceinline__ void load8(const bf16_t* p, float (&f)[8]) { unpack8(*reinterpret_cast<const uint4*>(p), f); }
__device__ __forceinline__ void load8(const float* p, float (&f)[8]) {
  const float4 lo = reinterpret_cast<const float4*>(p)[0], hi = reinterpret_cast<const float4*>(p)[1];
  f[0] = lo.x; f[1] = lo.y; f[2] = lo.z; f[3] = lo.w;
  f[4] = hi.x; f[5] = hi.y; f[6] = hi.z; f[7] = hi.w;
}
__device__ __forceinline__ float load1(const bf16_t* p) { return bf2f(*p); }
__device__ __forceinline__ float load1(const float* p) { return *p; }
__device__ __forceinline__ void store8(bf16_t* p, const float (&f)[8]) { *reinterpret_cast<uint4*>(p) = pack8(f); }
__device__ __forceinline__ void store8(float* p, const float (&f)[8]) {
  reinterpret_cast<float4*>(p)[0] = make_float4(f[0], f[1], f[2], f[3]);
  reinterpret_cast<float4*>(p)[1] = make_float4(f[4], f[5], f[6], f[7]);
}
__device__ __forceinline__ void store1(bf16_t* p, float f) { *p = (bf16_t)f2bf(f); }
__device__ __forceinline__ void store1(float* p, float f) { *p = f; }

// The part of a row that one lane of a group of G holds: V vectors of 8 elements, element e of
// vector v at column (v G + lane) 8 + e (VEC) or (8 v + e) G + lane.  Columns past c read `past`.
template <int G, int V, bool VEC, typename T>
__device__ __forceinline__ void load_row(const T* row, int c, int gl, float past, float (&f)[V][8]) {
#pragma unroll
  for (int v = 0; v < V; ++v) {
    if constexpr (VEC) {
      const int col = (v * G + gl) * 8;
      if (col < c) load8(row + col, f[v]);
      else {
#pragma unroll
        for (int e = 0; e < 8; ++e) f[v][e] = past;
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int col = (8 * v + e) * G + gl;
        f[v][e] = col < c ? load1(row + col) : past;
      }
    }
  }
}
template <int G, int V, bool VEC, typename T>
__device__ __forceinline__ void store_row(T* row, int c, int gl, const float (&f)[V][8]) {
#pragma unroll
  for (int v = 0; v < V; ++v) {
    if constexpr (VEC) {
      const int col = (v * G + gl) * 8;
      if (col < c) store8(row + col, f[v]);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int col = (8 * v + e) * G + gl;
        if (col < c) store1(row + col, f[v][e]);
      }
    }
  }
}
// The same part of a row as it lies in memory, for loads that are issued long before their use.
template <int G, int V, bool VEC, typename T>
struct Row {
  static constexpr int Q = sizeof(T) / 2;  // 16-byte vectors per 8 elements
  uint4 q[VEC ? V * Q : 1];
  float f[VEC ? 1 : V][8];
  __device__ __forceinline__ void load(const T* row, int c, int gl) {
    if constexpr (VEC) {
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const int col = (v * G + gl) * 8;
#pragma unroll
        for (int i = 0; i < Q; ++i)
          q[v * Q + i] = col < c ? reinterpret_cast<const uint4*>(row + col)[i] : make_uint4(0, 0, 0, 0);
      }
    } else {
      load_row<G, V, false>(row, c, gl, 0.f, f);
    }
  }
  __device__ __forceinline__ void values(float (&o)[V][8]) const {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      if constexpr (!VEC) {
#pragma unroll
        for (int e = 0; e < 8; ++e) o[v][e] = f[v][e];
      } else if constexpr (Q == 1) {
        unpack8(q[v], o[v]);
      } else {
        const uint4 a = q[v * Q], b = q[v * Q + Q - 1];
        const uint32_t u[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
        for (int e = 0; e < 8; ++e) o[v][e] = __uint_as_float(u[e]);
      }
    }
  }
};

// whether the lane's element (v, e) is inside the row
template <int G, bool VEC>
__device__ __forceinline__ bool inside(int v, int e, int c, int gl) {
  return VEC ? (v * G + gl) * 8 < c : (8 * v + e) * G + gl < c;
}

// sums over the group of two values; groups wider than a wave add their waves' sums through LDS
// (s: 2 values for each wave of the block)
template <int G>
__device__ __forceinline__ float2 group_sum(float a, float b, float2* s) {
#pragma unroll
  for (int d = (G < 64 ? G : 64) / 2; d >= 1; d >>= 1) {
    a += __shfl_xor(a, d);
    b += __shfl_xor(b, d);
  }
  if constexpr (G > 64) {
    const int wave = threadIdx.x >> 6;
    __syncthreads();  // the last sums have been read
    if ((threadIdx.x & 63) == 0) s[wave] = make_float2(a, b);
    __syncthreads();
    a = b = 0.f;
#pragma unroll
    for (int w = 0; w < G / 64; ++w) {
      const float2 t = s[wave / (G / 64) * (G / 64) + w];
      a += t.x;
      b += t.y;
    }
  }
  return make_float2(a, b);
}

template <int G>
constexpr int ln_threads() { return G > 256 ? G : 256; }

template <int G, int V, bool VEC, typename TX, typename TY>
__global__ __launch_bounds__(ln_threads<G>()) void ln_fwd_kernel(LnArgs a, const TX* x, const float* gamma,
                                                                 const float* beta, TY* y, float* mean, float* rstd) {
  constexpr int RPB = ln_threads<G>() / G;
  __shared__ float2 s_sum[G > 64 ? ln_threads<G>() / 64 : 1];
  const int gl = threadIdx.x % G;
  const float inv_c = 1.0f / (float)a.c;
  const int64_t row = (int64_t)blockIdx.x * RPB + threadIdx.x / G;
  const bool live = row < a.m;
  float f[V][8], g[V][8], b[V][8];
  load_row<G, V, VEC>(x + (live ? row : 0) * a.ldx, a.c, gl, 0.f, f);
  float s = 0.f;
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int e = 0; e < 8; ++e) s += f[v][e];
  const float mu = group_sum<G>(s, 0.f, s_sum).x * inv_c;
  s = 0.f;
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      f[v][e] -= mu;
      s += inside<G, VEC>(v, e, a.c, gl) ? f[v][e] * f[v][e] : 0.f;
    }
  const float rs = 1.0f / sqrtf(group_sum<G>(s, 0.f, s_sum).x * inv_c + a.eps);
  if (!live) return;
  if (gl == 0) {
    if (mean != nullptr) mean[row] = mu;
    if (rstd != nullptr) rstd[row] = rs;
  }
  if (gamma != nullptr) load_row<G, V, VEC>(gamma, a.c, gl, 0.f, g);
  if (beta != nullptr) load_row<G, V, VEC>(beta, a.c, gl, 0.f, b);
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int e = 0; e < 8; ++e)
      f[v][e] = __builtin_fmaf(f[v][e] * rs, gamma != nullptr ? g[v][e] : 1.f, beta != nullptr ? b[v][e] : 0.f);
  store_row<G, V, VEC>(y + row * a.ldy, a.c, gl, f);
}

// part: [blocks][2][c] sums of dy xh and of dy
template <int G, int V, bool VEC, typename TX, typename TY>
__global__ __launch_bounds__(ln_threads<G>()) void ln_bwd_kernel(LnArgs a, const TY* dy, const TX* x,
                                                                 const float* mean, const float* rstd,
                                                                 const float* gamma, const TX* res, TX* dx,
                                                                 float* part) {
  constexpr int NT = ln_threads<G>(), RPB = NT / G;
  __shared__ float2 s_sum[G > 64 ? NT / 64 : 1];
  const int gl = threadIdx.x % G, grp = threadIdx.x / G;
  const float inv_c = 1.0f / (float)a.c;
  float g[V][8], dg[V][8], db[V][8];
  if (gamma != nullptr) load_row<G, V, VEC>(gamma, a.c, gl, 0.f, g);
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (gamma == nullptr) g[v][e] = 1.f;
      dg[v][e] = db[v][e] = 0.f;
    }
  // every group of the block takes the same number of rounds (the sums of wide groups hold barriers);
  // a round's rows are loaded a round ahead where registers allow
  constexpr bool AHEAD = G * V < 2048;
  const int64_t rounds = (a.m + RPB - 1) / RPB;
  struct Rows {
    Row<G, V, VEC, TX> x, res;
    Row<G, V, VEC, TY> dy;
    float mu, rs;
  };
  auto fetch = [&](int64_t k, Rows& r) __attribute__((always_inline)) {
    const int64_t row = k * RPB + grp, rr = row < a.m ? row : 0;
    r.x.load(x + rr * a.ldx, a.c, gl);
    r.dy.load(dy + rr * a.ldy, a.c, gl);
    if (res != nullptr) r.res.load(res + rr * a.ldr, a.c, gl);
    r.mu = mean[rr];
    r.rs = rstd[rr];
  };
  auto work = [&](int64_t k, const Rows& r) __attribute__((always_inline)) {
    const int64_t row = k * RPB + grp;
    const bool live = row < a.m;
    float f[V][8], h[V][8];
    r.x.values(f);
    r.dy.values(h);
    const float mu = r.mu, rs = r.rs;
    float s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const bool in = live && inside<G, VEC>(v, e, a.c, gl);
        const float d = in ? h[v][e] : 0.f, xh = in ? (f[v][e] - mu) * rs : 0.f;
        db[v][e] += d;
        dg[v][e] = __builtin_fmaf(d, xh, dg[v][e]);
        f[v][e] = xh;
        h[v][e] = in ? d * g[v][e] : 0.f;
        s1 += h[v][e];
        s2 = __builtin_fmaf(h[v][e], xh, s2);
      }
    const float2 t = group_sum<G>(s1, s2, s_sum);
    const float c1 = t.x * inv_c, c2 = t.y * inv_c;
    if (live && dx != nullptr) {
      float o[V][8];
      if (res != nullptr) r.res.values(o);
#pragma unroll
      for (int v = 0; v < V; ++v)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float d = rs * (h[v][e] - c1 - f[v][e] * c2);
          f[v][e] = res != nullptr ? d + o[v][e] : d;
        }
      store_row<G, V, VEC>(dx + row * a.lddx, a.c, gl, f);
    }
  };
  if constexpr (AHEAD) {
    Rows now, next;
    if (blockIdx.x < rounds) fetch(blockIdx.x, now);
    for (int64_t k = blockIdx.x; k < rounds; k += gridDim.x) {
      if (k + gridDim.x < rounds) fetch(k + gridDim.x, next);
      work(k, now);
      now = next;
    }
  } else {
    for (int64_t k = blockIdx.x; k < rounds; k += gridDim.x) {
      Rows now;
      fetch(k, now);
      work(k, now);
    }
  }
  if (part == nullptr) return;
  // the groups' sums, added in order by the first group
  float* p = part + (int64_t)blockIdx.x * 2 * a.c;
  if constexpr (RPB == 1) {
    store_row<G, V, VEC>(p, a.c, gl, dg);
    store_row<G, V, VEC>(p + a.c, a.c, gl, db);
  } else {
    __shared__ float s_col[RPB][G * V * 8 + G];
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      __syncthreads();
#pragma unroll
      for (int v = 0; v < V; ++v)
#pragma unroll
        for (int e = 0; e < 8; ++e) s_col[grp][(v * 8 + e) * G + gl] = which ? db[v][e] : dg[v][e];
      __syncthreads();
      for (int i = threadIdx.x; i < G * V * 8; i += NT) {
        const int gi = i % G, ve = i / G;
        const int col = VEC ? ((ve / 8) * G + gi) * 8 + ve % 8 : i;
        float s = 0.f;
#pragma unroll
        for (int r = 0; r < RPB; ++r) s += s_col[r][i];
        if (col < a.c) p[which * a.c + col] = s;
      }
    }
  }
}

// rows longer than the registers of a block hold: a block per row, in passes over memory
template <typename TX, typename TY>
__global__ __launch_bounds__(1024) void ln_fwd_long_kernel(LnArgs a, const TX* x, const float* gamma,
                                                           const float* beta, TY* y, float* mean, float* rstd) {
  __shared__ float2 s_sum[16];
  const float inv_c = 1.0f / (float)a.c;
  for (int64_t row = blockIdx.x; row < a.m; row += gridDim.x) {
    const TX* r = x + row * a.ldx;
    float s = 0.f;
    for (int i = threadIdx.x; i < a.c; i += 1024) s += load1(r + i);
    const float mu = group_sum<1024>(s, 0.f, s_sum).x * inv_c;
    s = 0.f;
    for (int i = threadIdx.x; i < a.c; i += 1024) {
      const float d = load1(r + i) - mu;
      s = __builtin_fmaf(d, d, s);
    }
    const float rs = 1.0f / sqrtf(group_sum<1024>(s, 0.f, s_sum).x * inv_c + a.eps);
    if (threadIdx.x == 0) {
      if (mean != nullptr) mean[row] = mu;
      if (rstd != nullptr) rstd[row] = rs;
    }
    for (int i = threadIdx.x; i < a.c; i += 1024)
      store1(y + row * a.ldy + i, __builtin_fmaf((load1(r + i) - mu) * rs, gamma != nullptr ? gamma[i] : 1.f,
                                                 beta != nullptr ? beta[i] : 0.f));
  }
}

template <typename TX, typename TY>
__global__ __launch_bounds__(1024) void ln_bwd_long_kernel(LnArgs a, const TY* dy, const TX* x, const float* mean,
                                                           const float* rstd, const float* gamma, const TX* res,
                                                           TX* dx) {
  __shared__ float2 s_sum[16];
  const float inv_c = 1.0f / (float)a.c;
  for (int64_t row = blockIdx.x; row < a.m; row += gridDim.x) {
    const TX* r = x + row * a.ldx;
    const TY* d = dy + row * a.ldy;
    const float mu = mean[row], rs = rstd[row];
    float s1 = 0.f, s2 = 0.f;
    for (int i = threadIdx.x; i < a.c; i += 1024) {
      const float h = load1(d + i) * (gamma != nullptr ? gamma[i] : 1.f);
      s1 += h;
      s2 = __builtin_fmaf(h, (load1(r + i) - mu) * rs, s2);
    }
    const float2 t = group_sum<1024>(s1, s2, s_sum);
    const float c1 = t.x * inv_c, c2 = t.y * inv_c;
    for (int i = threadIdx.x; i < a.c; i += 1024) {
      const float h = load1(d + i) * (gamma != nullptr ? gamma[i] : 1.f);
      const float o = rs * (h - c1 - (load1(r + i) - mu) * rs * c2);
      store1(dx + row * a.lddx + i, res != nullptr ? o + load1(res + row * a.ldr + i) : o);
    }
  }
}
// and their dgamma and dbeta partials: blocks of 256 columns x a range of rows
template <typename TX, typename TY>
__global__ __launch_bounds__(256) void ln_bwd_cols_kernel(LnArgs a, const TY* dy, const TX* x, const float* mean,
                                                          const float* rstd, int64_t rows_per, float* part) {
  const int c = blockIdx.x * 256 + threadIdx.x;
  if (c >= a.c) return;
  const int64_t r0 = blockIdx.y * rows_per, r1 = r0 + rows_per < a.m ? r0 + rows_per : a.m;
  float dg = 0.f, db = 0.f;
  for (int64_t r = r0; r < r1; ++r) {
    const float d = load1(dy + r * a.ldy + c);
    db += d;
    dg = __builtin_fmaf(d, (load1(x + r * a.ldx + c) - mean[r]) * rstd[r], dg);
  }
  float* p = part + (int64_t)blockIdx.y * 2 * a.c;
  p[c] = dg;
  p[a.c + c] = db;
}

constexpr int kLongest = 16384;  // the longest row that is held in registers
constexpr int kLongRanges = 64;

int group_lanes(int c) {
  int g = 16;
  while (g < 1024 && g * 8 < c) g *= 2;
  return g;
}
int bwd_blocks(const LnArgs& a) {
  if (a.c > kLongest) return (int)std::min<int64_t>(kLongRanges, a.m);
  const int g = group_lanes(a.c), rpb = (g > 256 ? g : 256) / g;
  // four blocks to a CU of short rows; a partial is as long as two rows, so long ones take fewer (us on
  // 512, 1024 and 2048 blocks: 102400 x 192 37.2, 29.6, 34.1; 16384 x 1024 30.3, 31.0, 38.8; 16384 x 8192
  // 346, 366, 399)
  return (int)std::min<int64_t>(g <= 128 ? 1024 : 512, (a.m + rpb - 1) / rpb);
}

// f.template operator()<G, V>() for the narrowest group that holds c elements
template <typename F>
void with_group(int c, F&& f) {
  switch (group_lanes(c)) {
    case 16: f(std::integral_constant<int, 16>{}, std::integral_constant<int, 1>{}); break;
    case 32: f(std::integral_constant<int, 32>{}, std::integral_constant<int, 1>{}); break;
    case 64: f(std::integral_constant<int, 64>{}, std::integral_constant<int, 1>{}); break;
    case 128: f(std::integral_constant<int, 128>{}, std::integral_constant<int, 1>{}); break;
    case 256: f(std::integral_constant<int, 256>{}, std::integral_constant<int, 1>{}); break;
    case 512: f(std::integral_constant<int, 512>{}, std::integral_constant<int, 1>{}); break;
    default:
      if (c <= 8192) f(std::integral_constant<int, 1024>{}, std::integral_constant<int, 1>{});
      else f(std::integral_constant<int, 1024>{}, std::integral_constant<int, 2>{});
  }
}

template <typename TX, typename TY>
void fwd_typed(const LnArgs& a, const void* x, const float* gamma, const float* beta, void* y, float* mean,
               float* rstd, hipStream_t s) {
  const TX* xp = static_cast<const TX*>(x);
  TY* yp = static_cast<TY*>(y);
  if (a.c > kLongest) {
    NUMBAT_LAUNCH((ln_fwd_long_kernel<TX, TY>), dim3((unsigned)std::min<int64_t>(a.m, 1 << 20)), dim3(1024), 0, s, a, xp,
                  gamma, beta, yp, mean, rstd);
    return;
  }
  with_group(a.c, [&](auto gc, auto vc) {
    constexpr int G = decltype(gc)::value, V = decltype(vc)::value, NT = ln_threads<G>();
    // a launch takes fewer than 2^32 threads: more rows than that in several
    constexpr int64_t RPB = NT / G, MOST = ((1ll << 31) / NT) * RPB;
    for (int64_t r = 0; r < a.m; r += MOST) {
      LnArgs b = a;
      b.m = std::min(a.m - r, MOST);
      const dim3 grid((unsigned)((b.m + RPB - 1) / RPB));
      const TX* xr = xp + r * a.ldx;
      TY* yr = yp + r * a.ldy;
      float *mr = mean != nullptr ? mean + r : nullptr, *sr = rstd != nullptr ? rstd + r : nullptr;
      if (a.vec) NUMBAT_LAUNCH((ln_fwd_kernel<G, V, true, TX, TY>), grid, dim3(NT), 0, s, b, xr, gamma, beta, yr, mr, sr);
      else NUMBAT_LAUNCH((ln_fwd_kernel<G, V, false, TX, TY>), grid, dim3(NT), 0, s, b, xr, gamma, beta, yr, mr, sr);
    }
  });
}

template <typename TX, typename TY>
void bwd_typed(const LnArgs& a, const void* dy, const void* x, const float* mean, const float* rstd,
               const float* gamma, const void* res, void* dx, float* part, hipStream_t s) {
  const TX *xp = static_cast<const TX*>(x), *rp = static_cast<const TX*>(res);
  const TY* dp = static_cast<const TY*>(dy);
  TX* op = static_cast<TX*>(dx);
  const int blocks = bwd_blocks(a);
  if (a.c > kLongest) {
    if (dx != nullptr)
      NUMBAT_LAUNCH((ln_bwd_long_kernel<TX, TY>), dim3((unsigned)std::min<int64_t>(a.m, 1 << 20)), dim3(1024), 0, s, a,
                    dp, xp, mean, rstd, gamma, rp, op);
    if (part != nullptr)
      NUMBAT_LAUNCH((ln_bwd_cols_kernel<TX, TY>), dim3((unsigned)((a.c + 255) / 256), (unsigned)blocks), dim3(256), 0, s,
                    a, dp, xp, mean, rstd, (a.m + blocks - 1) / blocks, part);
    return;
  }
  with_group(a.c, [&](auto gc, auto vc) {
    constexpr int G = decltype(gc)::value, V = decltype(vc)::value, NT = ln_threads<G>();
    const dim3 grid((unsigned)blocks);
    if (a.vec)
      NUMBAT_LAUNCH((ln_bwd_kernel<G, V, true, TX, TY>), grid, dim3(NT), 0, s, a, dp, xp, mean, rstd, gamma, rp, op, part);
    else
      NUMBAT_LAUNCH((ln_bwd_kernel<G, V, false, TX, TY>), grid, dim3(NT), 0, s, a, dp, xp, mean, rstd, gamma, rp, op, part);
  });
}

}  // namespace

hipError_t ln_fwd_launch(const LnArgs& a, const void* x, const float* gamma, const float* beta, void* y, float* mean,
                         float* rstd, hipStream_t s) {
  trace_begin(KC_LN_FWD);
  if (a.x_f32) {
    if (a.y_f32) fwd_typed<float, float>(a, x, gamma, beta, y, mean, rstd, s);
    else fwd_typed<float, bf16_t>(a, x, gamma, beta, y, mean, rstd, s);
  } else {
    if (a.y_f32) fwd_typed<bf16_t, float>(a, x, gamma, beta, y, mean, rstd, s);
    else fwd_typed<bf16_t, bf16_t>(a, x, gamma, beta, y, mean, rstd, s);
  }
  trace_end(KC_LN_FWD);
  return hipGetLastError();
}

size_t ln_bwd_part_bytes(const LnArgs& a) { return (size_t)bwd_blocks(a) * 2 * a.c * sizeof(float); }

hipError_t ln_bwd_launch(const LnArgs& a, const void* dy, const void* x, const float* mean, const float* rstd,
                         const float* gamma, const void* res, void* dx, float* dgamma, float* dbeta, int accumulate,
                         float* part, hipStream_t s) {
  float* pt = dgamma != nullptr || dbeta != nullptr ? part : nullptr;
  trace_begin(KC_LN_BWD);
  if (a.x_f32) {
    if (a.y_f32) bwd_typed<float, float>(a, dy, x, mean, rstd, gamma, res, dx, pt, s);
    else bwd_typed<float, bf16_t>(a, dy, x, mean, rstd, gamma, res, dx, pt, s);
  } else {
    if (a.y_f32) bwd_typed<bf16_t, float>(a, dy, x, mean, rstd, gamma, res, dx, pt, s);
    else bwd_typed<bf16_t, bf16_t>(a, dy, x, mean, rstd, gamma, res, dx, pt, s);
  }
  trace_end(KC_LN_BWD);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || pt == nullptr) return e;
  trace_begin(KC_LN_BWD_FINISH);
  column_sum_launch(pt, bwd_blocks(a), 2 * (int64_t)a.c, 2 * a.c, a.c, dgamma, dbeta, accumulate, s);
  trace_end(KC_LN_BWD_FINISH);
  return hipGetLastError();
}

}  // namespace numbat
