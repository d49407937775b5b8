// Group norm with an activation over NHWC maps, forward and backward, on gfx950.
//   forward   t = gamma xh + beta,  y = act(t),  xh = (x - mean) rstd,  rstd = (var + eps)^-1/2
//   backward  dt = dy act'(t),  h = gamma dt;  dx = rstd (h - mean(h) - xh mean(h xh))
//             dgamma = sum dt xh,  dbeta = sum dt
// the means over the rows and channels of an image's group.
//
// A thread owns eight neighbouring channels and walks down rows, so that a block covers whole rows of a slab
// of channels.  Two ways:
//   held      a block's slab is whole groups of one image and its threads hold it in registers: every value
//             is read once and written once, in one launch.
//   passes    larger maps: a pass over ranges of rows leaves each group's sums of each range, and the pass
//             that writes the result joins them first, every block for the groups of its slab; the second
//             read of a map is mostly from the caches.
// Squares are added after a value within the data's range is taken off (`shift`), so that a mean far from
// zero costs nothing; threads, ranges and channels are joined by counts, means and centred squares.  All in
// a fixed order.
//
// HBM bounds the large maps and the steps of one block the small ones: loads, six barriers of sums, stores.  Held: one
// image of 20x20 x 576 with SiLU 8.6 us, 16 of 40x40 x 384 15.0 (2.6 TB/s of x and y), their gradients 20.5 and 4
// for the sums over images (2.4 TB/s).  Passes: 16 of 80x80 x 192 28.6 us (statistics 10.5, writing 18.4: 4.1 TB/s of
// the three reads and writes), 5 of 53x97 x 327 in fp32 with GELU, gradients: 44 us.
#include <algorithm>

#include "act.h"
#include "attention_kernels.h"
#include "mlp_kernels.h"
#include "vec_io.h"

namespace numbat {

namespace {

constexpr int V = 8;            // channels of a thread
constexpr int kThreads = 256;   // of the passes
constexpr int kSlab = 2048;     // channels of a block of the passes at most
constexpr int kAhead = 8;       // rows a thread of the statistics pass loads before it works on them, and of the
constexpr int kHalf = kAhead / 2;  // others, which hold two turns or two operands

__device__ __forceinline__ void act8(float (&t)[V], int act) {
  auto each = [&](auto f) __attribute__((always_inline)) {
#pragma unroll
    for (int e = 0; e < V; ++e) t[e] = f(t[e]);
  };
  switch (act) {
    case kActRelu: each([](float z) { return act_apply(z, kActRelu); }); break;
    case kActGelu: each([](float z) { return act_apply(z, kActGelu); }); break;
    case kActGeluTanh: each([](float z) { return act_apply(z, kActGeluTanh); }); break;
    case kActSilu: each([](float z) { return act_apply(z, kActSilu); }); break;
    default: break;
  }
}
// d *= act'(t)
__device__ __forceinline__ void slope8(const float (&t)[V], float (&d)[V], int act) {
  auto each = [&](auto f) __attribute__((always_inline)) {
#pragma unroll
    for (int e = 0; e < V; ++e) d[e] *= f(t[e]);
  };
  switch (act) {
    case kActRelu: each([](float z) { return act_slope(z, kActRelu); }); break;
    case kActGelu: each([](float z) { return act_slope(z, kActGelu); }); break;
    case kActGeluTanh: each([](float z) { return act_slope(z, kActGeluTanh); }); break;
    case kActSilu: each([](float z) { return act_slope(z, kActSilu); }); break;
    default: break;
  }
}

// The work on one row ends: left to itself the compiler unpacks every row that a thread holds at once
__device__ __forceinline__ void row_done() { __builtin_amdgcn_sched_barrier(0); }

// How vectors are loaded.  Whole ones stand in no branch: one that some lanes leave out makes the next wait for it.
// (Moving vectors that a row ends in down from the row's last V channels, to load those without a branch too, costs
// odd rows of fp32 more than the branch: 5 x 5141 x 327 with GELU 58 us against 32.)
enum {
  kWhole,    // whole vectors at 16-byte aligned addresses
  kAnywhere  // at any address; a vector that the row ends in by elements
};
// A vector as it was loaded: bf16 stays packed until it is worked on.  Values behind `count` are not the thread's.
template <typename T>
struct Raw;
template <>
struct Raw<bf16_t> {
  u32x4 u;
  template <int HOW>
  __device__ __forceinline__ void get(const bf16_t* p, int count) {
    if constexpr (HOW == kWhole) {
      u = *reinterpret_cast<const u32x4*>(p);
    } else if (count >= V) {
      const uint4 v = get16<false>(p);
      u = u32x4{v.x, v.y, v.z, v.w};
    } else {
      float f[V];
      get_some<false>(p, count, f);
      const uint4 v = pack8(f);
      u = u32x4{v.x, v.y, v.z, v.w};
    }
  }
  __device__ __forceinline__ void values(float (&f)[V]) const { unpack8(make_uint4(u.x, u.y, u.z, u.w), f); }
  __device__ __forceinline__ void zero() { u = u32x4{0, 0, 0, 0}; }
  // (the compiler would otherwise keep what it has unpacked, twice the registers)
  __device__ __forceinline__ void keep() { asm volatile("" : "+v"(u)); }
};
template <>
struct Raw<float> {
  float v[V];
  template <int HOW>
  __device__ __forceinline__ void get(const float* p, int count) {
    if constexpr (HOW == kWhole) get_vec<true>(p, v);
    else get_some<false>(p, count, v);
  }
  __device__ __forceinline__ void values(float (&f)[V]) const {
#pragma unroll
    for (int e = 0; e < V; ++e) f[e] = v[e];
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = 0.f;
  }
  __device__ __forceinline__ void keep() {}
};
template <int HOW, typename T>
__device__ __forceinline__ void put_row(T* p, int count, const float (&f)[V]) {
  if constexpr (HOW == kWhole) put_vec<true>(p, f);
  else put_some<false>(p, count, f);
}

// what a thread knows of its channels
struct Gain {
  float gamma[V], beta[V];
  __device__ __forceinline__ Gain(const float* ga, const float* be, int col, int count) {
    if (ga != nullptr) {
      get_some<false>(ga + col, count, gamma);
    } else {
#pragma unroll
      for (int e = 0; e < V; ++e) gamma[e] = 1.f;
    }
    if (be != nullptr) {
      get_some<false>(be + col, count, beta);
    } else {
#pragma unroll
      for (int e = 0; e < V; ++e) beta[e] = 0.f;
    }
  }
};

// f(e, group) of a vector's channels; behind the last that counts its group again
template <typename F>
__device__ __forceinline__ void each_channel(int col, int count, int per_group, F&& f) {
  int grp = col / per_group, left = (grp + 1) * per_group - col;
#pragma unroll
  for (int e = 0; e < V; ++e) {
    f(e, grp);
    if (--left == 0 && e + 1 < count) {
      left = per_group;
      ++grp;
    }
  }
}

// xh, and dt in dy's place, of a vector
__device__ __forceinline__ void grads8(float (&x)[V], float (&d)[V], const float (&mean)[V], const float (&rstd)[V],
                                       const Gain& g, int act) {
  float t[V];
#pragma unroll
  for (int e = 0; e < V; ++e) {
    x[e] = (x[e] - mean[e]) * rstd[e];
    t[e] = __builtin_fmaf(x[e], g.gamma[e], g.beta[e]);
  }
  slope8(t, d, act);
}

// A thread's values of its channels in LDS, 16 bytes at a time
__device__ __forceinline__ void lds_put(float* p, const float (&f)[V]) {
  *reinterpret_cast<float4*>(p) = make_float4(f[0], f[1], f[2], f[3]);
  *reinterpret_cast<float4*>(p + 4) = make_float4(f[4], f[5], f[6], f[7]);
}
__device__ __forceinline__ void lds_get(const float* p, float (&f)[V]) {
  const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
  f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w;
  f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
}

// A thread's sums go into LDS, there added to those of before, and begin anew
__device__ __forceinline__ void lds_close(float* p, float (&f)[V], bool first) {
  if (!first) {
    float t[V];
    lds_get(p, t);
#pragma unroll
    for (int e = 0; e < V; ++e) f[e] += t[e];
  }
  lds_put(p, f);
#pragma unroll
  for (int e = 0; e < V; ++e) f[e] = 0.f;
}

// Sums two values of every channel over the `side` threads down a slab of `width` channels (rounded up to whole
// vectors): in a[c] and b[c] of a[side][width], b[side][width] afterwards.  Called by all T threads, after a
// barrier.
template <int T>
__device__ __forceinline__ void slab_sums(float* a, float* b, int width, int side) {
  const int parts = max(1, min(side, T / width));
  float ta = 0.f, tb = 0.f;
  const int c = threadIdx.x % width, part = threadIdx.x / width;
  if (parts > 1) {
    if (part < parts)
      for (int i = part; i < side; i += parts) {
        ta += a[i * width + c];
        tb += b[i * width + c];
      }
    __syncthreads();
    if (part < parts) {
      a[part * width + c] = ta;
      b[part * width + c] = tb;
    }
    __syncthreads();
    side = parts;
  }
  for (int k = threadIdx.x; k < width; k += T) {  // (a column belongs to one thread)
    ta = tb = 0.f;
    for (int i = 0; i < side; ++i) {
      ta += a[i * width + k];
      tb += b[i * width + k];
    }
    a[k] = ta;
    b[k] = tb;
  }
  __syncthreads();
}

// f(group number of the slab, its channels lo .. hi of the slab, lane, lanes) by a power of two of lanes for each
// group that overlaps channels c0 .. c0 + width - 1; whole waves stay together, so f may exchange values among a
// group's lanes.  Groups past the last have lo >= hi.
template <int T, typename F>
__device__ __forceinline__ void each_group(int c0, int width, int per_group, F&& f) {
  int lanes = 1;
  while (lanes < 64 && lanes < per_group) lanes *= 2;
  const int g0 = c0 / per_group, g1 = (c0 + width - 1) / per_group;
  for (int first = g0; first <= g1; first += T / lanes) {
    const int grp = first + threadIdx.x / lanes;
    const int lo = max(grp * per_group - c0, 0), hi = grp <= g1 ? min((grp + 1) * per_group - c0, width) : 0;
    f(grp, lo, hi, (int)threadIdx.x % lanes, lanes);
  }
}
// (what is no number stays that)
__device__ __forceinline__ float not_below_zero(float t) { return t < 0.f ? 0.f : t; }
__device__ __forceinline__ float lane_sum(float t, int lanes) {
  for (int o = lanes / 2; o > 0; o /= 2) t += __shfl_xor(t, o);
  return t;
}

// Mean and centred squares of a group's channels lo .. hi out of the channels' own (each of `rows` values)
__device__ __forceinline__ float2 join_channels(const float* mean, const float* sq, float rows, int lo, int hi, int lane,
                                                int lanes) {
  float m = 0.f, s = 0.f;
  for (int c = lo + lane; c < hi; c += lanes) m += mean[c];
  m = lane_sum(m, lanes);
  m = hi > lo ? m / (float)(hi - lo) : 0.f;
  for (int c = lo + lane; c < hi; c += lanes) {
    const float d = mean[c] - m;
    s += __builtin_fmaf(rows * d, d, sq[c]);
  }
  return make_float2(m, lane_sum(s, lanes));
}

// ---------------------------------------------------------------------------
// Held: a block of T threads for `width` channels of an image, whole groups, NV rows of each thread.

struct GnHeld {
  int32_t width, slabs, cols, side;  // channels of a block, blocks of an image, threads across and down
  int32_t rows;                      // of a thread
  int32_t per_group;
};

template <int T>
struct HeldPlace {
  int img, c0, at, col, count, lane_row;  // col: the thread's first channel; at: within the slab
  __device__ __forceinline__ HeldPlace(const GnHeld& g) {
    // an XCD's L2 sees neighbouring slabs of an image: their rows share cache lines
    const uint32_t t = xcd_remap(blockIdx.x, gridDim.x);
    img = t / g.slabs;
    c0 = (t - img * g.slabs) * g.width;
    lane_row = threadIdx.x / g.cols;
    at = (threadIdx.x - lane_row * g.cols) * V;
    if (lane_row >= g.side) at = lane_row = 0;  // (threads left over load what the first does, and are done)
    col = c0 + at;
    count = threadIdx.x < (unsigned)(g.side * g.cols) ? min(V, g.width - at) : 0;
  }
};

template <typename TX, typename TY, int HOW, int NV, int T>
__global__ __launch_bounds__(T) void gn_fwd_held_kernel(GnArgs a, GnHeld g, const TX* x, const float* gamma,
                                                        const float* beta, TY* y, float* mean, float* rstd) {
  extern __shared__ __attribute__((aligned(16))) float lds[];
  const int span = g.cols * V;
  float *s_a = lds, *s_b = s_a + g.side * span, *s_shift = s_b + g.side * span, *s_mean = s_shift + span,
        *s_rstd = s_mean + span;
  const HeldPlace<T> p(g);
  const int m = (int)a.m;
  Raw<TX> v[NV];
  const TX* xp = x + (int64_t)p.img * a.m * a.ldx + p.col;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    v[i].zero();
    // (rows past the last are the last again)
    if (i < g.rows) v[i].template get<HOW>(xp + (int64_t)min(p.lane_row + i * g.side, m - 1) * a.ldx, p.count);
  }
  const Gain gain(gamma, beta, p.count > 0 ? p.col : 0, p.count);
  // the first thread's mean of a channel is every thread's shift
  if (p.lane_row == 0 && p.count > 0) {
    float t[V] = {};
    int rows = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (i * g.side < m) {
        float f[V];
        v[i].values(f);
        ++rows;
#pragma unroll
        for (int e = 0; e < V; ++e) t[e] += f[e];
      }
    const float inv = 1.0f / (float)rows;
#pragma unroll
    for (int e = 0; e < V; ++e) t[e] *= inv;
    lds_put(s_shift + p.at, t);
  }
#pragma unroll
  for (int i = 0; i < NV; ++i) v[i].keep();
  __syncthreads();
  if (p.count > 0) {
    float shift[V], s1[V] = {}, s2[V] = {};
    lds_get(s_shift + p.at, shift);
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (p.lane_row + i * g.side < m) {
        float f[V];
        v[i].values(f);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const float d = f[e] - shift[e];
          s1[e] += d;
          s2[e] = __builtin_fmaf(d, d, s2[e]);
        }
        row_done();
      }
    lds_put(s_a + p.lane_row * span + p.at, s1);
    lds_put(s_b + p.lane_row * span + p.at, s2);
  }
#pragma unroll
  for (int i = 0; i < NV; ++i) v[i].keep();
  __syncthreads();
  slab_sums<T>(s_a, s_b, span, g.side);
  const float rows = (float)m;
  for (int c = threadIdx.x; c < g.width; c += T) {  // each channel's mean and centred squares
    const float d = s_a[c] / rows;
    s_b[c] = not_below_zero(__builtin_fmaf(-s_a[c], d, s_b[c]));
    s_a[c] = s_shift[c] + d;
  }
  __syncthreads();
  each_group<T>(p.c0, g.width, g.per_group, [&](int grp, int lo, int hi, int lane, int lanes) __attribute__((always_inline)) {
    const float2 t = join_channels(s_a, s_b, rows, lo, hi, lane, lanes);
    const float r = 1.0f / sqrtf(t.y / (rows * (float)g.per_group) + a.eps);
    for (int c = lo + lane; c < hi; c += lanes) {
      s_mean[c] = t.x;
      s_rstd[c] = r;
    }
    if (lane == 0 && hi > lo) {
      if (mean != nullptr) mean[(int64_t)p.img * a.groups + grp] = t.x;
      if (rstd != nullptr) rstd[(int64_t)p.img * a.groups + grp] = r;
    }
  });
  __syncthreads();
  if (p.count <= 0) return;
  float mu[V], scale[V];
  lds_get(s_mean + p.at, mu);
  lds_get(s_rstd + p.at, scale);
#pragma unroll
  for (int e = 0; e < V; ++e) scale[e] *= gain.gamma[e];
  TY* yp = y + (int64_t)p.img * a.m * a.ldy + p.col;
#pragma unroll
  for (int i = 0; i < NV; ++i)
    if (p.lane_row + i * g.side < m) {
      float f[V];
      v[i].values(f);
#pragma unroll
      for (int e = 0; e < V; ++e) f[e] = __builtin_fmaf(f[e] - mu[e], scale[e], gain.beta[e]);
      act8(f, a.act);
      put_row<HOW>(yp + (int64_t)(p.lane_row + i * g.side) * a.ldy, p.count, f);
      row_done();
    }
}

// sums: each image's sums of dt and dt xh, [img][2][c], or nullptr
template <typename TX, typename TY, int HOW, int NV, int T>
__global__ __launch_bounds__(T) void gn_bwd_held_kernel(GnArgs a, GnHeld g, const TY* dy, const TX* x, const float* mean,
                                                        const float* rstd, const float* gamma, const float* beta,
                                                        const TX* res, TX* dx, float* sums) {
  extern __shared__ __attribute__((aligned(16))) float lds[];
  const int span = g.cols * V;
  float *s_a = lds, *s_b = s_a + g.side * span, *s_h1 = s_b + g.side * span, *s_h2 = s_h1 + span;
  const HeldPlace<T> p(g);
  const int m = (int)a.m;
  Raw<TX> v[NV];
  Raw<TY> d[NV];
  const TX* xp = x + (int64_t)p.img * a.m * a.ldx + p.col;
  const TY* dp = dy + (int64_t)p.img * a.m * a.ldy + p.col;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    v[i].zero();
    d[i].zero();
    if (i < g.rows) {  // (rows past the last are the last again)
      const int64_t r = min(p.lane_row + i * g.side, m - 1);
      v[i].template get<HOW>(xp + r * a.ldx, p.count);
      d[i].template get<HOW>(dp + r * a.ldy, p.count);
    }
  }
  const Gain gain(gamma, beta, p.count > 0 ? p.col : 0, p.count);
  float mu[V], rs[V];
  each_channel(p.count > 0 ? p.col : 0, p.count, g.per_group, [&](int e, int grp) __attribute__((always_inline)) {
    mu[e] = mean[(int64_t)p.img * a.groups + grp];
    rs[e] = rstd[(int64_t)p.img * a.groups + grp];
  });
  float dt[NV][V];
  if (p.count > 0) {
    float s1[V] = {}, s2[V] = {};
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (p.lane_row + i * g.side < m) {
        float f[V];
        v[i].values(f);
        d[i].values(dt[i]);
        grads8(f, dt[i], mu, rs, gain, a.act);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          s1[e] += dt[i][e];
          s2[e] = __builtin_fmaf(dt[i][e], f[e], s2[e]);
        }
        row_done();
      }
    lds_put(s_a + p.lane_row * span + p.at, s1);
    lds_put(s_b + p.lane_row * span + p.at, s2);
  }
#pragma unroll
  for (int i = 0; i < NV; ++i) v[i].keep();
  __syncthreads();
  slab_sums<T>(s_a, s_b, span, g.side);
  if (sums != nullptr)
    for (int c = threadIdx.x; c < g.width; c += T) {
      sums[(int64_t)p.img * 2 * a.c + p.c0 + c] = s_a[c];
      sums[(int64_t)p.img * 2 * a.c + a.c + p.c0 + c] = s_b[c];
    }
  if (dx == nullptr) return;
  const float inv = 1.0f / ((float)m * (float)g.per_group);
  each_group<T>(p.c0, g.width, g.per_group, [&](int, int lo, int hi, int lane, int lanes) __attribute__((always_inline)) {
    float h1 = 0.f, h2 = 0.f;
    for (int c = lo + lane; c < hi; c += lanes) {
      const float ga = gamma != nullptr ? gamma[p.c0 + c] : 1.f;
      h1 = __builtin_fmaf(ga, s_a[c], h1);
      h2 = __builtin_fmaf(ga, s_b[c], h2);
    }
    h1 = lane_sum(h1, lanes) * inv;
    h2 = lane_sum(h2, lanes) * inv;
    for (int c = lo + lane; c < hi; c += lanes) {
      s_h1[c] = h1;
      s_h2[c] = h2;
    }
  });
  __syncthreads();
  if (p.count <= 0) return;
  float h1[V], h2[V];
  lds_get(s_h1 + p.at, h1);
  lds_get(s_h2 + p.at, h2);
  TX* op = dx + (int64_t)p.img * a.m * a.lddx + p.col;
  const TX* rp = res != nullptr ? res + (int64_t)p.img * a.m * a.ldr + p.col : nullptr;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int64_t r = p.lane_row + i * g.side;
    if (r < m) {
      float f[V], q[V] = {};
      if (rp != nullptr) {
        Raw<TX> w;
        w.template get<HOW>(rp + r * a.ldr, p.count);
        w.values(q);
      }
      v[i].values(f);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float xh = (f[e] - mu[e]) * rs[e];
        f[e] = __builtin_fmaf(rs[e], __builtin_fmaf(dt[i][e], gain.gamma[e], -h1[e]) - xh * h2[e], q[e]);
      }
      put_row<HOW>(op + r * a.lddx, p.count, f);
      row_done();
    }
  }
}

// ---------------------------------------------------------------------------
// Passes over ranges of rows

// how an image's values are dealt to blocks of one pass
struct GnGrid {
  int32_t slabs, slab;        // slabs of channels, and their channels (the last may have fewer), a multiple of V
  int32_t cols, side;         // threads across a slab and down
  int32_t chunks;             // ranges of rows
  int64_t rows;               // of a range (the last may have fewer)
  int32_t run;                // rows whose sums a thread adds one after another, before it adds what they come to
  int32_t per_group;          // channels of a group
};

// ranges of rows, the same number for each thread, that make up to `blocks` blocks
GnGrid make_grid(const GnArgs& a, int64_t blocks, int64_t most) {
  GnGrid g;
  const int vecs = (a.c + V - 1) / V;
  g.slabs = (a.c + kSlab - 1) / kSlab;
  g.cols = (vecs + g.slabs - 1) / g.slabs;
  g.slab = g.cols * V;
  g.slabs = (a.c + g.slab - 1) / g.slab;
  g.side = kThreads / g.cols;
  const int64_t least = (int64_t)g.side * kHalf;
  const int64_t chunks = std::clamp<int64_t>(blocks / ((int64_t)a.n * g.slabs), 1, most);
  g.rows = std::max(least, (a.m + g.side * chunks - 1) / (g.side * chunks) * g.side);
  g.chunks = (int32_t)((a.m + g.rows - 1) / g.rows);
  // 64 rows, or the root of a thread's where that is more: sums of few additions in a row, however long a range is
  g.run = 64;
  while ((int64_t)g.run * g.run < g.rows / g.side) g.run += 64;
  g.per_group = a.c / a.groups;
  return g;
}
dim3 blocks_of(const GnArgs& a, const GnGrid& g) { return dim3((unsigned)g.chunks, (unsigned)g.slabs, (unsigned)a.n); }

// A (slab, group) pair that overlaps is entry slab + group of a list: along the channels one of them
// advances at every entry.
__host__ __device__ __forceinline__ int entries(const GnArgs& a, const GnGrid& g) { return a.groups + g.slabs; }

// this thread's part of the block's rows and channels
struct Place {
  int img, c0, width, at, col, count;  // the slab's first channel and channels; the thread's, how many lie inside
  int64_t row, end;                    // first row within the image, and the range's end
  int lane_row;
  __device__ __forceinline__ Place(const GnArgs& a, const GnGrid& g) {
    img = blockIdx.z;
    c0 = blockIdx.y * g.slab;
    width = min(g.slab, a.c - c0);
    lane_row = threadIdx.x / g.cols;
    at = (threadIdx.x - lane_row * g.cols) * V;
    col = c0 + at;
    count = lane_row < g.side ? min(V, a.c - col) : 0;
    row = blockIdx.x * g.rows + lane_row;
    end = min(a.m, (int64_t)(blockIdx.x + 1) * g.rows);
  }
};

// N rows of a thread, row, row + side, ... (past the range's end the last one again, or none)
template <int HOW, int N, typename T>
__device__ __forceinline__ void get_rows(const T* base, int64_t ld, int64_t row, const Place& p, int side, Raw<T> (&v)[N]) {
  if (row >= p.end) return;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int64_t r = row + i * side;
    if constexpr (HOW == kWhole) v[i].template get<HOW>(base + min(r, p.end - 1) * ld, p.count);
    else if (r < p.end) v[i].template get<HOW>(base + r * ld, p.count);  // (there are branches anyhow)
  }
}

// mean and centred squares of every entry of a block: part[img][chunk][entry]
template <typename T, int HOW>
__global__ __launch_bounds__(kThreads) void gn_stats_kernel(GnArgs a, GnGrid g, const T* x, float2* part) {
  __shared__ __attribute__((aligned(16))) float s_a[kThreads * V], s_b[kThreads * V], s_shift[kSlab];
  const Place p(a, g);
  const T* xp = x + (int64_t)p.img * a.m * a.ldx + p.col;
  const int64_t first = (int64_t)blockIdx.x * g.rows;
  float shift[V], s1[V] = {}, s2[V] = {};
  Raw<T> v[kAhead];
  if (p.count > 0) get_rows<HOW>(xp, a.ldx, p.row, p, g.side, v);
  // the first thread's mean of a channel is every thread's shift
  if (p.lane_row == 0 && p.count > 0) {
    float t[V] = {};
    int rows = 0;
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
      if (p.row + i * g.side < p.end) {
        float f[V];
        v[i].values(f);
        ++rows;
#pragma unroll
        for (int e = 0; e < V; ++e) t[e] += f[e];
      }
    const float inv = 1.0f / (float)rows;
#pragma unroll
    for (int e = 0; e < V; ++e) t[e] *= inv;
    lds_put(s_shift + p.at, t);
  }
  __syncthreads();
  if (p.count > 0) {
    lds_get(s_shift + p.at, shift);
    float *at_a = s_a + p.lane_row * g.slab + p.at, *at_b = s_b + p.lane_row * g.slab + p.at;
    int run = 0;
    bool first_run = true;
    for (int64_t r = p.row; r < p.end; r += (int64_t)kAhead * g.side) {
#pragma unroll
      for (int i = 0; i < kAhead; ++i)
        if (r + i * g.side < p.end) {
          float f[V];
          v[i].values(f);
#pragma unroll
          for (int e = 0; e < V; ++e) {
            const float d = f[e] - shift[e];
            s1[e] += d;
            s2[e] = __builtin_fmaf(d, d, s2[e]);
          }
          row_done();
        }
      get_rows<HOW>(xp, a.ldx, r + (int64_t)kAhead * g.side, p, g.side, v);
      run += kAhead;
      if (run == g.run) {
        lds_close(at_a, s1, first_run);
        lds_close(at_b, s2, first_run);
        run = 0;
        first_run = false;
      }
    }
    lds_close(at_a, s1, first_run);
    lds_close(at_b, s2, first_run);
  }
  __syncthreads();
  slab_sums<kThreads>(s_a, s_b, g.slab, g.side);
  const float rows = (float)(p.end - first);
  for (int c = threadIdx.x; c < p.width; c += kThreads) {
    const float d = s_a[c] / rows;
    s_b[c] = not_below_zero(__builtin_fmaf(-s_a[c], d, s_b[c]));
    s_a[c] = s_shift[c] + d;
  }
  __syncthreads();
  float2* out = part + ((int64_t)p.img * g.chunks + blockIdx.x) * entries(a, g) + blockIdx.y;
  each_group<kThreads>(p.c0, p.width, g.per_group, [&](int grp, int lo, int hi, int lane, int lanes) __attribute__((always_inline)) {
    const float2 t = join_channels(s_a, s_b, rows, lo, hi, lane, lanes);
    if (lane == 0 && hi > lo) out[grp] = t;
  });
}

// f(range, its entry) of every lane's share of the ranges, eight loads in flight
template <typename F>
__device__ __forceinline__ void each_chunk(const float2* at, int step, int chunks, int lane, int lanes, F&& f) {
  for (int i = lane; i < chunks; i += 8 * lanes) {
    float2 v[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = at[(int64_t)min(i + k * lanes, chunks - 1) * step];
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (i + k * lanes < chunks) f(i + k * lanes, v[k]);
  }
}

// The entries of an image's group, joined by a power of two of lanes: mean and centred squares.  The first
// entry's mean is the shift of the others' (of E ranges at most 1 + E of cancellation).
__device__ __forceinline__ float2 join_stats(const GnArgs& a, const GnGrid& g, const float2* part, int img, int grp,
                                             int lane, int lanes) {
  const int s0 = grp * g.per_group / g.slab, s1 = ((grp + 1) * g.per_group - 1) / g.slab;
  const float2* at = part + (int64_t)img * g.chunks * entries(a, g) + grp;
  const float shift = at[s0].x;
  float t1 = 0.f, t2 = 0.f;
  for (int s = s0; s <= s1; ++s) {
    const int wide = min((grp + 1) * g.per_group, (s + 1) * g.slab) - max(grp * g.per_group, s * g.slab);
    each_chunk(at + s, entries(a, g), g.chunks, lane, lanes, [&](int i, float2 v) __attribute__((always_inline)) {
      const float count = (float)(min(a.m, (int64_t)(i + 1) * g.rows) - i * g.rows) * (float)wide, d = v.x - shift;
      t1 = __builtin_fmaf(count, d, t1);
      t2 += __builtin_fmaf(count * d, d, v.y);
    });
  }
  t1 = lane_sum(t1, lanes);
  t2 = lane_sum(t2, lanes);
  const float inv = 1.0f / ((float)a.m * (float)g.per_group), d = t1 * inv;
  return make_float2(shift + d, 1.0f / sqrtf(not_below_zero(__builtin_fmaf(-t1, d, t2)) * inv + a.eps));
}
// the entries' sums, times what makes them means
__device__ __forceinline__ float2 join_sums(const GnArgs& a, const GnGrid& g, const float2* part, int img, int grp,
                                            int lane, int lanes) {
  const int s0 = grp * g.per_group / g.slab, s1 = ((grp + 1) * g.per_group - 1) / g.slab;
  const float2* at = part + (int64_t)img * g.chunks * entries(a, g) + grp;
  float t1 = 0.f, t2 = 0.f;
  for (int s = s0; s <= s1; ++s)
    each_chunk(at + s, entries(a, g), g.chunks, lane, lanes, [&](int, float2 v) __attribute__((always_inline)) {
      t1 += v.x;
      t2 += v.y;
    });
  const float inv = 1.0f / ((float)a.m * (float)g.per_group);
  return make_float2(lane_sum(t1, lanes) * inv, lane_sum(t2, lanes) * inv);
}

// A block of the writing pass joins the groups of its slab, or, where they have too many entries for that, a
// kernel of its own has joined every group: which of the two, and the lanes of a group
constexpr int kJoinInBlock = 4096;
bool joins_in_block(const GnArgs& a, const GnGrid& g) {
  const int64_t groups = std::min<int64_t>(a.groups, g.slab / g.per_group + 2);
  return groups * g.chunks <= kJoinInBlock && groups <= kThreads;
}

// Joins every group, a wave for each.  (Groups of all images may be more than the waves of a launch, which end at 2^32
// threads.)
template <bool STATS>
__global__ __launch_bounds__(kThreads) void gn_join_kernel(GnArgs a, GnGrid g, const float2* part, float2* joined) {
  constexpr int kWaves = kThreads / 64;
  for (int64_t i = (int64_t)blockIdx.x * kWaves + threadIdx.x / 64; i < (int64_t)a.n * a.groups; i += (int64_t)gridDim.x * kWaves) {
    const int img = (int)(i / a.groups), grp = (int)(i - (int64_t)img * a.groups), lane = threadIdx.x % 64;
    const float2 t = STATS ? join_stats(a, g, part, img, grp, lane, 64) : join_sums(a, g, part, img, grp, lane, 64);
    if (lane == 0) joined[i] = t;
  }
}
template <bool STATS>
void join_launch(const GnArgs& a, const GnGrid& g, const float2* part, float2* joined, hipStream_t s) {
  const int64_t joins = ((int64_t)a.n * a.groups + kThreads / 64 - 1) / (kThreads / 64);
  NUMBAT_LAUNCH((gn_join_kernel<STATS>), dim3((unsigned)std::min<int64_t>(joins, 1 << 20)), dim3(kThreads), 0, s, a, g, part,
                joined);
}

// s_join[group of the slab]: from the entries (joined == nullptr), or from what was joined before
template <bool STATS>
__device__ __forceinline__ void block_join(const GnArgs& a, const GnGrid& src, const Place& p, const float2* part,
                                           const float2* joined, float2* s_join) {
  const int g0 = p.c0 / src.per_group, count = (p.c0 + p.width - 1) / src.per_group - g0 + 1;
  int lanes = 1;
  while (lanes < 64 && lanes * 2 * count <= kThreads) lanes *= 2;
  const int i = threadIdx.x / lanes, lane = threadIdx.x % lanes, grp = g0 + min(i, count - 1);
  const float2 t = STATS ? join_stats(a, src, part, p.img, grp, lane, lanes) : join_sums(a, src, part, p.img, grp, lane, lanes);
  if (lane == 0 && i < count) s_join[i] = t;
  __syncthreads();
}

template <typename TX, typename TY, int HOW>
__global__ __launch_bounds__(kThreads, sizeof(TX) == 2 ? 4 : 3) void gn_fwd_kernel(GnArgs a, GnGrid g, GnGrid src, const TX* x, const float* gamma,
                                                          const float* beta, const float2* part, const float2* joined,
                                                          TY* y, float* mean, float* rstd) {
  __shared__ float2 s_join[kThreads];
  const Place p(a, g);
  const TX* xp = x + (int64_t)p.img * a.m * a.ldx + p.col;
  TY* yp = y + (int64_t)p.img * a.m * a.ldy + p.col;
  Raw<TX> v[kHalf], w[kHalf];
  const int64_t turn = (int64_t)kHalf * g.side;
  if (p.count > 0) {
    get_rows<HOW>(xp, a.ldx, p.row, p, g.side, v);
    get_rows<HOW>(xp, a.ldx, p.row + turn, p, g.side, w);
  }
  const Gain gain(gamma, beta, p.count > 0 ? p.col : 0, p.count);
  if (joined == nullptr) block_join<true>(a, src, p, part, joined, s_join);
  const int g0 = p.c0 / g.per_group;
  // the first range's blocks write the statistics of the groups that start in their slab
  if (blockIdx.x == 0)
    for (int grp = (p.c0 + g.per_group - 1) / g.per_group + threadIdx.x; grp * g.per_group < p.c0 + p.width; grp += kThreads) {
      const int64_t i = (int64_t)p.img * a.groups + grp;
      const float2 t = joined == nullptr ? s_join[grp - g0] : joined[i];
      if (mean != nullptr) mean[i] = t.x;
      if (rstd != nullptr) rstd[i] = t.y;
    }
  if (p.count <= 0) return;
  float mu[V], scale[V];
  each_channel(p.col, p.count, g.per_group, [&](int e, int grp) __attribute__((always_inline)) {
    const float2 t = joined == nullptr ? s_join[grp - g0] : joined[(int64_t)p.img * a.groups + grp];
    mu[e] = t.x;
    scale[e] = t.y * gain.gamma[e];
  });
  auto write = [&](int64_t r, const Raw<TX>(&u)[kHalf]) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < kHalf; ++i)
      if (r + i * g.side < p.end) {
        float f[V];
        u[i].values(f);
#pragma unroll
        for (int e = 0; e < V; ++e) f[e] = __builtin_fmaf(f[e] - mu[e], scale[e], gain.beta[e]);
        act8(f, a.act);
        put_row<HOW>(yp + (r + i * g.side) * a.ldy, p.count, f);
        row_done();
      }
  };
  for (int64_t r = p.row; r < p.end; r += 2 * turn) {
    write(r, v);
    get_rows<HOW>(xp, a.ldx, r + 2 * turn, p, g.side, v);
    write(r + turn, w);
    get_rows<HOW>(xp, a.ldx, r + 3 * turn, p, g.side, w);
  }
}

// Sums over a block's rows: of dt and of dt xh for each channel, sums[img][chunk][2][c], and of h and h xh for
// each entry, part[img][chunk][entry]
template <typename TX, typename TY, int HOW>
__global__ __launch_bounds__(kThreads) void gn_bwd_sums_kernel(GnArgs a, GnGrid g, const TY* dy, const TX* x,
                                                               const float* mean, const float* rstd, const float* gamma,
                                                               const float* beta, float* sums, float2* part) {
  __shared__ __attribute__((aligned(16))) float s_a[kThreads * V], s_b[kThreads * V];
  const Place p(a, g);
  if (p.count > 0) {
    constexpr int N = kHalf;
    const TX* xp = x + (int64_t)p.img * a.m * a.ldx + p.col;
    const TY* dp = dy + (int64_t)p.img * a.m * a.ldy + p.col;
    Raw<TX> v[N];
    Raw<TY> d[N];
    get_rows<HOW>(xp, a.ldx, p.row, p, g.side, v);
    get_rows<HOW>(dp, a.ldy, p.row, p, g.side, d);
    const Gain gain(gamma, beta, p.col, p.count);
    float mu[V], rs[V], s1[V] = {}, s2[V] = {};
    each_channel(p.col, p.count, g.per_group, [&](int e, int grp) __attribute__((always_inline)) {
      mu[e] = mean[(int64_t)p.img * a.groups + grp];
      rs[e] = rstd[(int64_t)p.img * a.groups + grp];
    });
    float *at_a = s_a + p.lane_row * g.slab + p.at, *at_b = s_b + p.lane_row * g.slab + p.at;
    int run = 0;
    bool first_run = true;
    for (int64_t r = p.row; r < p.end; r += (int64_t)N * g.side) {
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (r + i * g.side < p.end) {
          float f[V], t[V];
          v[i].values(f);
          d[i].values(t);
          grads8(f, t, mu, rs, gain, a.act);
#pragma unroll
          for (int e = 0; e < V; ++e) {
            s1[e] += t[e];
            s2[e] = __builtin_fmaf(t[e], f[e], s2[e]);
          }
          row_done();
        }
      get_rows<HOW>(xp, a.ldx, r + (int64_t)N * g.side, p, g.side, v);
      get_rows<HOW>(dp, a.ldy, r + (int64_t)N * g.side, p, g.side, d);
      run += N;
      if (run == g.run) {
        lds_close(at_a, s1, first_run);
        lds_close(at_b, s2, first_run);
        run = 0;
        first_run = false;
      }
    }
    lds_close(at_a, s1, first_run);
    lds_close(at_b, s2, first_run);
  }
  __syncthreads();
  slab_sums<kThreads>(s_a, s_b, g.slab, g.side);
  float* out = sums + ((int64_t)p.img * g.chunks + blockIdx.x) * 2 * a.c + p.c0;
  for (int c = threadIdx.x; c < p.width; c += kThreads) {
    out[c] = s_a[c];
    out[a.c + c] = s_b[c];
  }
  float2* pt = part + ((int64_t)p.img * g.chunks + blockIdx.x) * entries(a, g) + blockIdx.y;
  each_group<kThreads>(p.c0, p.width, g.per_group, [&](int grp, int lo, int hi, int lane, int lanes) __attribute__((always_inline)) {
    float h1 = 0.f, h2 = 0.f;
    for (int c = lo + lane; c < hi; c += lanes) {
      const float ga = gamma != nullptr ? gamma[p.c0 + c] : 1.f;
      h1 = __builtin_fmaf(ga, s_a[c], h1);
      h2 = __builtin_fmaf(ga, s_b[c], h2);
    }
    h1 = lane_sum(h1, lanes);
    h2 = lane_sum(h2, lanes);
    if (lane == 0 && hi > lo) pt[grp] = make_float2(h1, h2);
  });
}

template <typename TX, typename TY, int HOW>
__global__ __launch_bounds__(kThreads, sizeof(TX) < sizeof(TY) || (sizeof(TX) == 4 && HOW == kWhole) ? 2 : 3) void gn_bwd_kernel(GnArgs a, GnGrid g, GnGrid src, const TY* dy, const TX* x,
                                                          const float* mean, const float* rstd, const float* gamma,
                                                          const float* beta, const TX* res, const float2* part,
                                                          const float2* joined, TX* dx) {
  __shared__ float2 s_join[kThreads];
  constexpr int N = kHalf;
  const Place p(a, g);
  const TX* xp = x + (int64_t)p.img * a.m * a.ldx + p.col;
  const TY* dp = dy + (int64_t)p.img * a.m * a.ldy + p.col;
  const TX* rp = res != nullptr ? res + (int64_t)p.img * a.m * a.ldr + p.col : nullptr;
  TX* op = dx + (int64_t)p.img * a.m * a.lddx + p.col;
  Raw<TX> v[N];
  Raw<TY> d[N];
  if (p.count > 0) {
    get_rows<HOW>(xp, a.ldx, p.row, p, g.side, v);
    get_rows<HOW>(dp, a.ldy, p.row, p, g.side, d);
  }
  const Gain gain(gamma, beta, p.count > 0 ? p.col : 0, p.count);
  if (joined == nullptr) block_join<false>(a, src, p, part, joined, s_join);
  if (p.count <= 0) return;
  const int g0 = p.c0 / g.per_group;
  float mu[V], rs[V], h1[V], h2[V];
  each_channel(p.col, p.count, g.per_group, [&](int e, int grp) __attribute__((always_inline)) {
    const int64_t at = (int64_t)p.img * a.groups + grp;
    mu[e] = mean[at];
    rs[e] = rstd[at];
    const float2 t = joined == nullptr ? s_join[grp - g0] : joined[at];
    h1[e] = t.x;
    h2[e] = t.y;
  });
  for (int64_t r = p.row; r < p.end; r += (int64_t)N * g.side) {
    if (r != p.row) {
      get_rows<HOW>(xp, a.ldx, r, p, g.side, v);
      get_rows<HOW>(dp, a.ldy, r, p, g.side, d);
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (r + i * g.side < p.end) {
        float f[V], t[V], q[V] = {};
        if (rp != nullptr) {
          Raw<TX> w;
          w.template get<HOW>(rp + (r + i * g.side) * a.ldr, p.count);
          w.values(q);
        }
        v[i].values(f);
        d[i].values(t);
        grads8(f, t, mu, rs, gain, a.act);
#pragma unroll
        for (int e = 0; e < V; ++e)
          t[e] = __builtin_fmaf(rs[e], __builtin_fmaf(t[e], gain.gamma[e], -h1[e]) - f[e] * h2[e], q[e]);
        put_row<HOW>(op + (r + i * g.side) * a.lddx, p.count, t);
        row_done();
      }
  }
}

// ---------------------------------------------------------------------------
// f(TX, TY, how vectors are loaded)
template <typename F>
void with_types(const GnArgs& a, bool whole, F&& f) {
  auto typed = [&](auto x, auto y) {
    if (whole) f(x, y, std::integral_constant<int, kWhole>{});
    else f(x, y, std::integral_constant<int, kAnywhere>{});
  };
  if (a.x_f32 && a.y_f32) typed(0.f, 0.f);
  else if (a.x_f32) typed(0.f, bf16_t{});
  else if (a.y_f32) typed(bf16_t{}, 0.f);
  else typed(bf16_t{}, bf16_t{});
}

constexpr int kHeldThreads = 512;

// Whether an image's groups are held, and by which blocks: the fewest whole groups that are whole vectors, more of
// them while rows of a slab are short of a cache line and there are blocks enough.  held_rows: rows that a thread's
// registers hold.
bool make_held(const GnArgs& a, int held_rows, GnHeld* g) {
  const int per = a.c / a.groups;
  int width = per;
  while (width % V != 0 && width < a.c) width += per;
  if (width % V != 0 || a.c % width != 0) width = per;  // (the last vector of a slab is then a part of one)
  auto rows = [&](int w) {
    const int cols = (w + V - 1) / V;
    return cols > kHeldThreads / 2 ? INT64_MAX : (a.m + kHeldThreads / cols - 1) / (kHeldThreads / cols);
  };
  const int bytes = a.x_f32 ? 4 : 2;
  if (rows(width) > held_rows) return false;
  while (width * bytes < 128 && a.c % (2 * width) == 0 && rows(2 * width) <= held_rows &&
         (int64_t)a.n * a.c / (2 * width) >= 512)
    width *= 2;
  if ((int64_t)a.n * (a.c / width) > ((1ll << 32) - 1) / kHeldThreads) return false;  // (threads of a launch)
  g->width = width;
  g->slabs = a.c / width;
  g->cols = (width + V - 1) / V;
  g->side = (int)std::min<int64_t>(kHeldThreads / g->cols, a.m);
  g->rows = (int)((a.m + g->side - 1) / g->side);
  g->per_group = per;
  return true;
}
size_t held_lds(const GnHeld& g, int arrays) { return (size_t)(2 * g.side + arrays) * g.cols * V * sizeof(float); }

// Rows that a thread of the held kernels holds at most: a row takes 4 registers of bf16 and 8 of fp32, the
// backward two of them
int held_fwd_rows(const GnArgs& a) { return a.x_f32 ? 8 : 16; }
int held_bwd_rows(const GnArgs& a) { return a.x_f32 || a.y_f32 ? 6 : 10; }
// f(rows) for the fewest of ROWS... that are enough
template <int FIRST, int... REST, typename F>
void with_rows(int rows, F&& f) {
  if constexpr (sizeof...(REST) == 0) f(std::integral_constant<int, FIRST>{});
  else if (rows <= FIRST) f(std::integral_constant<int, FIRST>{});
  else with_rows<REST...>(rows, f);
}

// Blocks of the passes: as many as run at a time (four to a CU of the forward's, three of the backward's), so that
// no part of a round is left for the end
GnGrid stats_grid(const GnArgs& a) { return make_grid(a, 1024, 256); }
GnGrid fwd_grid(const GnArgs& a) { return make_grid(a, 1024, 1 << 20); }
GnGrid sums_grid(const GnArgs& a) { return make_grid(a, 768, 256); }
GnGrid bwd_grid(const GnArgs& a) { return make_grid(a, 768, 1 << 20); }

}  // namespace

size_t gn_fwd_ws(const GnArgs& a) {
  GnHeld h;
  if (make_held(a, held_fwd_rows(a), &h)) return 0;
  const GnGrid g = stats_grid(a);
  return ((size_t)a.n * a.groups + (size_t)a.n * g.chunks * entries(a, g)) * sizeof(float2);
}

hipError_t gn_fwd_launch(const GnArgs& a, const void* x, const float* gamma, const float* beta, void* y, float* mean,
                         float* rstd, void* ws, hipStream_t s) {
  GnHeld h;
  const bool held = make_held(a, held_fwd_rows(a), &h);
  const bool whole = a.c % V == 0 && a.ldx % V == 0 && a.ldy % V == 0 && (!held || h.width % V == 0);
  with_types(a, whole, [&](auto tx, auto ty, auto how) {
    using TX = decltype(tx);
    using TY = decltype(ty);
    constexpr int HOW = decltype(how)::value;
    const TX* xp = static_cast<const TX*>(x);
    TY* yp = static_cast<TY*>(y);
    if (held) {
      trace_begin(KC_GN_FWD);
      auto go = [&](auto nv) {
        NUMBAT_LAUNCH((gn_fwd_held_kernel<TX, TY, HOW, decltype(nv)::value, kHeldThreads>), dim3((unsigned)(a.n * h.slabs)),
                      dim3(kHeldThreads), held_lds(h, 3), s, a, h, xp, gamma, beta, yp, mean, rstd);
      };
      if constexpr (sizeof(TX) == 4) with_rows<2, 8>(h.rows, go);
      else with_rows<2, 8, 16>(h.rows, go);
      trace_end(KC_GN_FWD);
      return;
    }
    const GnGrid g = stats_grid(a), ga = fwd_grid(a);
    float2* joined = static_cast<float2*>(ws);
    float2* part = joined + (size_t)a.n * a.groups;
    trace_begin(KC_GN_STATS);
    NUMBAT_LAUNCH((gn_stats_kernel<TX, HOW>), blocks_of(a, g), dim3(kThreads), 0, s, a, g, xp, part);
    if (joins_in_block(a, g)) {
      joined = nullptr;
    } else {
      join_launch<true>(a, g, part, joined, s);
    }
    trace_end(KC_GN_STATS);
    trace_begin(KC_GN_FWD);
    NUMBAT_LAUNCH((gn_fwd_kernel<TX, TY, HOW>), blocks_of(a, ga), dim3(kThreads), 0, s, a, ga, g, xp, gamma, beta, part,
                  joined, yp, mean, rstd);
    trace_end(KC_GN_FWD);
  });
  return hipGetLastError();
}

size_t gn_bwd_ws(const GnArgs& a) {
  GnHeld h;
  if (make_held(a, held_bwd_rows(a), &h)) return (size_t)a.n * 2 * a.c * sizeof(float);
  const GnGrid g = sums_grid(a);
  return (size_t)a.n * (a.groups + (size_t)g.chunks * entries(a, g)) * sizeof(float2) +
         (size_t)a.n * g.chunks * 2 * a.c * sizeof(float);
}

hipError_t gn_bwd_launch(const GnArgs& a, const void* dy, const void* x, const float* mean, const float* rstd,
                         const float* gamma, const float* beta, const void* res, void* dx, float* dgamma, float* dbeta,
                         int accumulate, void* ws, hipStream_t s) {
  GnHeld h;
  const bool held = make_held(a, held_bwd_rows(a), &h);
  const bool whole = a.c % V == 0 && a.ldx % V == 0 && a.ldy % V == 0 && (dx == nullptr || a.lddx % V == 0) &&
                     (res == nullptr || a.ldr % V == 0) && (!held || h.width % V == 0);
  const bool vectors = dgamma != nullptr || dbeta != nullptr;
  float* sums = static_cast<float*>(ws);
  int ranges = a.n;  // rows of sums
  with_types(a, whole, [&](auto tx, auto ty, auto how) {
    using TX = decltype(tx);
    using TY = decltype(ty);
    constexpr int HOW = decltype(how)::value;
    const TX *xp = static_cast<const TX*>(x), *rp = static_cast<const TX*>(res);
    const TY* dp = static_cast<const TY*>(dy);
    TX* op = static_cast<TX*>(dx);
    if (held) {
      trace_begin(KC_GN_BWD);
      auto go = [&](auto nv) {
        NUMBAT_LAUNCH((gn_bwd_held_kernel<TX, TY, HOW, decltype(nv)::value, kHeldThreads>), dim3((unsigned)(a.n * h.slabs)),
                      dim3(kHeldThreads), held_lds(h, 2), s, a, h, dp, xp, mean, rstd, gamma, beta, rp, op,
                      vectors ? sums : nullptr);
      };
      if constexpr (sizeof(TX) == 4 || sizeof(TY) == 4) with_rows<2, 6>(h.rows, go);
      else with_rows<2, 6, 10>(h.rows, go);
      trace_end(KC_GN_BWD);
      return;
    }
    const GnGrid g = sums_grid(a), ga = bwd_grid(a);
    ranges = a.n * g.chunks;
    float2* joined = reinterpret_cast<float2*>(sums + (size_t)ranges * 2 * a.c);
    float2* part = joined + (size_t)a.n * a.groups;
    trace_begin(KC_GN_BWD_SUMS);
    NUMBAT_LAUNCH((gn_bwd_sums_kernel<TX, TY, HOW>), blocks_of(a, g), dim3(kThreads), 0, s, a, g, dp, xp, mean, rstd, gamma,
                  beta, sums, part);
    if (joins_in_block(a, g)) {
      joined = nullptr;
    } else if (dx != nullptr) {
      join_launch<false>(a, g, part, joined, s);
    }
    trace_end(KC_GN_BWD_SUMS);
    if (dx != nullptr) {
      trace_begin(KC_GN_BWD);
      NUMBAT_LAUNCH((gn_bwd_kernel<TX, TY, HOW>), blocks_of(a, ga), dim3(kThreads), 0, s, a, ga, g, dp, xp, mean, rstd, gamma,
                    beta, rp, part, joined, op);
      trace_end(KC_GN_BWD);
    }
  });
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !vectors) return e;
  trace_begin(KC_GN_BWD_FINISH);
  column_sum_launch(sums, ranges, 2 * (int64_t)a.c, 2 * a.c, a.c, dbeta, dgamma, accumulate, s);
  trace_end(KC_GN_BWD_FINISH);
  return hipGetLastError();
}

}  // namespace numbat
