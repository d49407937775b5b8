// Group norm with an activation over NHWC maps, forward and backward, on gfx950.
//   forward   t = gamma xh + beta,  y = act(t),  xh = (x - mean) rstd,  rstd = (var + eps)^-1/2
//   backward  dt = dy act'(t),  h = gamma dt;  dx = rstd (h - mean(h) - xh mean(h xh))
//             dgamma = sum dt xh,  dbeta = sum dt
// the means over the rows and channels of an image's group.
//
// A thread owns eight neighbouring channels and walks down rows, so that a block reads whole rows of a
// slab of channels.  Values are added after the mean of the thread's first rows is taken off them
// (`shift`): a thread of n rows then loses at most a factor n / 4 + 1 of cancellation in its sum of squares,
// whatever the mean.  Threads, blocks and channels are joined by their counts, means and centred
// squares, in a fixed order.
#include <algorithm>

#include "act.h"
#include "attention_kernels.h"
#include "mlp_kernels.h"
#include "vec_io.h"

namespace numbat {

namespace {

constexpr int V = 8;            // channels of a thread
constexpr int kThreads = 256;
constexpr int kSlab = 2048;     // channels of a block at most
constexpr int kAhead = 4;       // rows a thread loads before it works on them

// how an image's values are dealt to blocks of one pass
struct GnGrid {
  int32_t slabs, slab;        // slabs of channels, and their channels (the last may have fewer), a multiple of V
  int32_t cols, side;         // threads across a slab and down
  int32_t chunks;             // ranges of rows
  int64_t rows;               // of a range (the last may have fewer)
  int32_t per_group;          // channels of a group
};

GnGrid make_grid(const GnArgs& a, int64_t blocks, int most) {
  GnGrid g;
  const int vecs = (a.c + V - 1) / V;
  g.slabs = (a.c + kSlab - 1) / kSlab;
  g.cols = (vecs + g.slabs - 1) / g.slabs;
  g.slab = g.cols * V;
  g.slabs = (a.c + g.slab - 1) / g.slab;
  g.side = kThreads / g.cols;
  const int64_t least = (int64_t)g.side * kAhead;
  int64_t chunks = std::clamp<int64_t>(blocks / ((int64_t)a.n * g.slabs), 1, most);
  chunks = std::min(chunks, (a.m + least - 1) / least);
  g.rows = (a.m + chunks - 1) / chunks;
  g.chunks = (int32_t)((a.m + g.rows - 1) / g.rows);
  g.per_group = a.c / a.groups;
  return g;
}
dim3 blocks_of(const GnArgs& a, const GnGrid& g) { return dim3((unsigned)g.chunks, (unsigned)g.slabs, (unsigned)a.n); }

// A (slab, group) pair that overlaps is entry slab + group of a list: along the channels one of them
// advances at every entry.
__host__ __device__ __forceinline__ int entries(const GnArgs& a, const GnGrid& g) { return a.groups + g.slabs; }

// this thread's part of the block's rows and channels
struct Place {
  int img, col, count;  // first channel and how many of its V lie inside
  int64_t row, end;     // first row within the image, and the range's end
  int lane_row;
  __device__ __forceinline__ Place(const GnArgs& a, const GnGrid& g) {
    img = blockIdx.z;
    const int across = threadIdx.x % g.cols;
    lane_row = threadIdx.x / g.cols;
    col = blockIdx.y * g.slab + across * V;
    count = lane_row < g.side ? min(V, a.c - col) : 0;
    row = blockIdx.x * g.rows + lane_row;
    end = min(a.m, (int64_t)(blockIdx.x + 1) * g.rows);
  }
};

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

// rows row, row + side, ... of a thread: f(row number, vectors of one or two operands), kAhead loaded at a time
template <typename F>
__device__ __forceinline__ void walk(const Place& p, int side, F&& f) {
  int64_t r = p.row;
  for (; r + (kAhead - 1) * side < p.end; r += kAhead * side) f(r, std::integral_constant<int, kAhead>{});
  for (; r < p.end; r += side) f(r, std::integral_constant<int, 1>{});
}

// ---------------------------------------------------------------------------
// count, mean and centred squares of every entry of a block: part[img][chunk][entry]
template <typename T, bool ALIGNED>
__global__ __launch_bounds__(kThreads) void gn_stats_kernel(GnArgs a, GnGrid g, const T* x, float2* part) {
  __shared__ float s_mean[kThreads * V], s_sq[kThreads * V];
  const Place p(a, g);
  const T* xp = x + (int64_t)p.img * a.m * a.ldx + p.col;
  const int64_t rows = p.end - (int64_t)blockIdx.x * g.rows;
  if (p.count > 0) {
    float shift[V], s1[V], s2[V];
#pragma unroll
    for (int e = 0; e < V; ++e) shift[e] = s1[e] = s2[e] = 0.f;
    bool first = true;
    walk(p, g.side, [&](int64_t r, auto nc) __attribute__((always_inline)) {
      constexpr int N = decltype(nc)::value;
      float f[N][V];
#pragma unroll
      for (int i = 0; i < N; ++i) get_some<ALIGNED>(xp + (r + (int64_t)i * g.side) * a.ldx, p.count, f[i]);
      if (first) {
        first = false;
#pragma unroll
        for (int e = 0; e < V; ++e) {
          float t = 0.f;
#pragma unroll
          for (int i = 0; i < N; ++i) t += f[i][e];
          shift[e] = t * (1.0f / N);
        }
      }
#pragma unroll
      for (int i = 0; i < N; ++i)
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const float d = f[i][e] - shift[e];
          s1[e] += d;
          s2[e] = __builtin_fmaf(d, d, s2[e]);
        }
    });
    const int64_t mine = p.row < p.end ? (p.end - p.row + g.side - 1) / g.side : 0;
    const float inv = mine > 0 ? 1.0f / (float)mine : 0.f;
    const int at = p.lane_row * g.slab + (p.col - (int)blockIdx.y * g.slab);
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const float d = s1[e] * inv;
      s_mean[at + e] = shift[e] + d;
      s_sq[at + e] = fmaxf(__builtin_fmaf(-s1[e], d, s2[e]), 0.f);
    }
  }
  __syncthreads();
  // each channel's over the threads of its column
  const int c0 = blockIdx.y * g.slab, width = min(g.slab, a.c - c0);
  const int side = (int)min<int64_t>(g.side, rows);  // (threads further down had no row)
  const float inv_rows = 1.0f / (float)rows;
  for (int c = threadIdx.x; c < width; c += kThreads) {
    float mean = 0.f, sq = 0.f;
    for (int i = 0; i < side; ++i) mean = __builtin_fmaf((float)((rows - i + g.side - 1) / g.side), s_mean[i * g.slab + c], mean);
    mean *= inv_rows;
    for (int i = 0; i < side; ++i) {
      const float d = s_mean[i * g.slab + c] - mean;
      sq += __builtin_fmaf((float)((rows - i + g.side - 1) / g.side) * d, d, s_sq[i * g.slab + c]);
    }
    s_mean[c] = mean;
    s_sq[c] = sq;
  }
  __syncthreads();
  // each group's over its channels of the slab, by a power of two of lanes
  int lanes = 1;
  while (lanes < 64 && lanes < g.per_group) lanes *= 2;
  const int lane = threadIdx.x % lanes;
  const int g0 = c0 / g.per_group, g1 = (c0 + width - 1) / g.per_group;
  float2* out = part + ((int64_t)p.img * g.chunks + blockIdx.x) * entries(a, g) + blockIdx.y;
  for (int first = g0; first <= g1; first += kThreads / lanes) {  // (whole waves stay together)
    const int grp = first + threadIdx.x / lanes;
    const int lo = max(grp * g.per_group - c0, 0), hi = min((grp + 1) * g.per_group - c0, width);
    float mean = 0.f, sq = 0.f;
    for (int c = lo + lane; c < hi; c += lanes) mean += s_mean[c];
    for (int o = lanes / 2; o > 0; o /= 2) mean += __shfl_xor(mean, o);
    mean = hi > lo ? mean / (float)(hi - lo) : 0.f;
    for (int c = lo + lane; c < hi; c += lanes) {
      const float d = s_mean[c] - mean;
      sq += __builtin_fmaf((float)rows * d, d, s_sq[c]);
    }
    for (int o = lanes / 2; o > 0; o /= 2) sq += __shfl_xor(sq, o);
    if (lane == 0 && grp <= g1) out[grp] = make_float2(mean, sq);
  }
}

// the entries of an image's group, joined by one wave
__device__ __forceinline__ float2 join_group(const GnArgs& a, const GnGrid& g, const float2* part, int img, int grp,
                                             int lane) {
  const int s0 = grp * g.per_group / g.slab, s1 = ((grp + 1) * g.per_group - 1) / g.slab, parts = s1 - s0 + 1;
  const float2* at = part + (int64_t)img * g.chunks * entries(a, g) + grp + s0;
  // values of entry i: its rows times its channels of the group
  auto count = [&](int i) __attribute__((always_inline)) {
    const int chunk = i / parts, slab = s0 + i % parts;
    const int64_t rows = min(a.m, (int64_t)(chunk + 1) * g.rows) - chunk * g.rows;
    const int lo = max(grp * g.per_group, slab * g.slab), hi = min((grp + 1) * g.per_group, (slab + 1) * g.slab);
    return (float)rows * (float)(hi - lo);
  };
  auto entry = [&](int i) __attribute__((always_inline)) { return at[(int64_t)(i / parts) * entries(a, g) + i % parts]; };
  const int total = g.chunks * parts;
  const float inv = 1.0f / ((float)a.m * (float)g.per_group);
  float mean = 0.f, sq = 0.f;
  for (int i = lane; i < total; i += 64) mean = __builtin_fmaf(count(i), entry(i).x, mean);
  for (int o = 32; o > 0; o /= 2) mean += __shfl_xor(mean, o);
  mean *= inv;
  for (int i = lane; i < total; i += 64) {
    const float2 v = entry(i);
    const float d = v.x - mean;
    sq += __builtin_fmaf(count(i) * d, d, v.y);
  }
  for (int o = 32; o > 0; o /= 2) sq += __shfl_xor(sq, o);
  return make_float2(mean, 1.0f / sqrtf(sq * inv + a.eps));
}

__global__ __launch_bounds__(kThreads) void gn_join_kernel(GnArgs a, GnGrid g, const float2* part, float2* stats,
                                                           float* mean, float* rstd) {
  const int64_t i = (int64_t)blockIdx.x * (kThreads / 64) + threadIdx.x / 64;
  if (i >= (int64_t)a.n * a.groups) return;
  const float2 t = join_group(a, g, part, (int)(i / a.groups), (int)(i % a.groups), threadIdx.x % 64);
  if (threadIdx.x % 64 != 0) return;
  stats[i] = t;
  if (mean != nullptr) mean[i] = t.x;
  if (rstd != nullptr) rstd[i] = t.y;
}

template <typename TX, typename TY, bool ALIGNED>
__global__ __launch_bounds__(kThreads) void gn_fwd_kernel(GnArgs a, GnGrid g, const TX* x, const float* gamma,
                                                          const float* beta, const float2* stats, TY* y) {
  const Place p(a, g);
  if (p.count <= 0) return;
  float mean[V], scale[V], shift[V];
#pragma unroll
  for (int e = 0; e < V; ++e) {
    const int c = p.col + (e < p.count ? e : 0);
    const float2 t = stats[(int64_t)p.img * a.groups + c / g.per_group];
    mean[e] = t.x;
    scale[e] = t.y * (gamma != nullptr ? gamma[c] : 1.f);
    shift[e] = beta != nullptr ? beta[c] : 0.f;
  }
  const TX* xp = x + (int64_t)p.img * a.m * a.ldx + p.col;
  TY* yp = y + (int64_t)p.img * a.m * a.ldy + p.col;
  walk(p, g.side, [&](int64_t r, auto nc) __attribute__((always_inline)) {
    constexpr int N = decltype(nc)::value;
    float f[N][V];
#pragma unroll
    for (int i = 0; i < N; ++i) get_some<ALIGNED>(xp + (r + (int64_t)i * g.side) * a.ldx, p.count, f[i]);
#pragma unroll
    for (int i = 0; i < N; ++i) {
#pragma unroll
      for (int e = 0; e < V; ++e) f[i][e] = __builtin_fmaf(f[i][e] - mean[e], scale[e], shift[e]);
      act8(f[i], a.act);
      put_some<ALIGNED>(yp + (r + (int64_t)i * g.side) * a.ldy, p.count, f[i]);
    }
  });
}

// ---------------------------------------------------------------------------
// sums over a block's rows: part[img][chunk][2][c] of dt and of dt xh
template <typename TX, typename TY, bool ALIGNED>
__global__ __launch_bounds__(kThreads) void gn_bwd_sums_kernel(GnArgs a, GnGrid g, const TY* dy, const TX* x,
                                                               const float* mean, const float* rstd,
                                                               const float* gamma, const float* beta, float* part) {
  __shared__ float s_sum[2][kThreads * V];
  const Place p(a, g);
  if (p.count > 0) {
    float mu[V], rs[V], ga[V], be[V], s1[V], s2[V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const int c = p.col + (e < p.count ? e : 0);
      const int64_t at = (int64_t)p.img * a.groups + c / g.per_group;
      mu[e] = mean[at];
      rs[e] = rstd[at];
      ga[e] = gamma != nullptr ? gamma[c] : 1.f;
      be[e] = beta != nullptr ? beta[c] : 0.f;
      s1[e] = s2[e] = 0.f;
    }
    const TX* xp = x + (int64_t)p.img * a.m * a.ldx + p.col;
    const TY* dp = dy + (int64_t)p.img * a.m * a.ldy + p.col;
    walk(p, g.side, [&](int64_t r, auto nc) __attribute__((always_inline)) {
      constexpr int N = decltype(nc)::value;
      float f[N][V], d[N][V];
#pragma unroll
      for (int i = 0; i < N; ++i) {
        get_some<ALIGNED>(xp + (r + (int64_t)i * g.side) * a.ldx, p.count, f[i]);
        get_some<ALIGNED>(dp + (r + (int64_t)i * g.side) * a.ldy, p.count, d[i]);
      }
#pragma unroll
      for (int i = 0; i < N; ++i) {
        float t[V];
#pragma unroll
        for (int e = 0; e < V; ++e) {
          f[i][e] = (f[i][e] - mu[e]) * rs[e];
          t[e] = __builtin_fmaf(f[i][e], ga[e], be[e]);
        }
        slope8(t, d[i], a.act);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          s1[e] += d[i][e];
          s2[e] = __builtin_fmaf(d[i][e], f[i][e], s2[e]);
        }
      }
    });
    const int at = p.lane_row * g.slab + (p.col - (int)blockIdx.y * g.slab);
#pragma unroll
    for (int e = 0; e < V; ++e) {
      s_sum[0][at + e] = s1[e];
      s_sum[1][at + e] = s2[e];
    }
  }
  __syncthreads();
  const int c0 = blockIdx.y * g.slab, width = min(g.slab, a.c - c0);
  float* out = part + ((int64_t)p.img * g.chunks + blockIdx.x) * 2 * a.c + c0;
  for (int i = threadIdx.x; i < 2 * width; i += kThreads) {
    const int k = i >= width, c = i - k * width;
    float t = 0.f;
    for (int j = 0; j < g.side; ++j) t += s_sum[k][j * g.slab + c];
    out[(int64_t)k * a.c + c] = t;
  }
}

// a block for each image's group: the chunks' sums added for each channel (sums[img][2][c]) and the
// group's means of h and h xh (means[img][group])
__global__ __launch_bounds__(kThreads) void gn_bwd_join_kernel(GnArgs a, GnGrid g, const float* part,
                                                               const float* gamma, float* sums, float2* means) {
  __shared__ float2 s_sum[kThreads];
  const int img = blockIdx.y, grp = blockIdx.x, tid = threadIdx.x;
  int lanes = 1;
  while (lanes < kThreads && lanes < g.per_group) lanes *= 2;
  const int lane = tid % lanes, side = kThreads / lanes;
  float h1 = 0.f, h2 = 0.f;
  for (int first = 0; first < g.per_group; first += lanes) {
    const int c = first + lane;
    float2 t = make_float2(0.f, 0.f);
    if (c < g.per_group) {
      const float* at = part + (int64_t)img * g.chunks * 2 * a.c + grp * g.per_group + c;
      for (int j = tid / lanes; j < g.chunks; j += side) {
        t.x += at[(int64_t)j * 2 * a.c];
        t.y += at[(int64_t)j * 2 * a.c + a.c];
      }
    }
    s_sum[tid] = t;
    __syncthreads();
    if (tid < lanes && c < g.per_group) {
      for (int j = 1; j < side; ++j) {
        t.x += s_sum[j * lanes + lane].x;
        t.y += s_sum[j * lanes + lane].y;
      }
      const int ch = grp * g.per_group + c;
      sums[(int64_t)img * 2 * a.c + ch] = t.x;
      sums[(int64_t)img * 2 * a.c + a.c + ch] = t.y;
      const float ga = gamma != nullptr ? gamma[ch] : 1.f;
      h1 = __builtin_fmaf(ga, t.x, h1);
      h2 = __builtin_fmaf(ga, t.y, h2);
    }
    __syncthreads();
  }
  s_sum[tid] = make_float2(h1, h2);
  __syncthreads();
  for (int o = lanes / 2; o > 0; o /= 2) {
    if (tid < o) {
      s_sum[tid].x += s_sum[tid + o].x;
      s_sum[tid].y += s_sum[tid + o].y;
    }
    __syncthreads();
  }
  if (tid == 0) {
    const float inv = 1.0f / ((float)a.m * (float)g.per_group);
    means[(int64_t)img * a.groups + grp] = make_float2(s_sum[0].x * inv, s_sum[0].y * inv);
  }
}

template <typename TX, typename TY, bool ALIGNED>
__global__ __launch_bounds__(kThreads) void gn_bwd_kernel(GnArgs a, GnGrid g, const TY* dy, const TX* x,
                                                          const float* mean, const float* rstd, const float* gamma,
                                                          const float* beta, const float2* means, TX* dx) {
  const Place p(a, g);
  if (p.count <= 0) return;
  float mu[V], rs[V], ga[V], be[V], h1[V], h2[V];
#pragma unroll
  for (int e = 0; e < V; ++e) {
    const int c = p.col + (e < p.count ? e : 0);
    const int64_t at = (int64_t)p.img * a.groups + c / g.per_group;
    mu[e] = mean[at];
    rs[e] = rstd[at];
    ga[e] = gamma != nullptr ? gamma[c] : 1.f;
    be[e] = beta != nullptr ? beta[c] : 0.f;
    h1[e] = means[at].x;
    h2[e] = means[at].y;
  }
  const TX* xp = x + (int64_t)p.img * a.m * a.ldx + p.col;
  const TY* dp = dy + (int64_t)p.img * a.m * a.ldy + p.col;
  TX* op = dx + (int64_t)p.img * a.m * a.lddx + p.col;
  walk(p, g.side, [&](int64_t r, auto nc) __attribute__((always_inline)) {
    constexpr int N = decltype(nc)::value;
    float f[N][V], d[N][V];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      get_some<ALIGNED>(xp + (r + (int64_t)i * g.side) * a.ldx, p.count, f[i]);
      get_some<ALIGNED>(dp + (r + (int64_t)i * g.side) * a.ldy, p.count, d[i]);
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float t[V];
#pragma unroll
      for (int e = 0; e < V; ++e) {
        f[i][e] = (f[i][e] - mu[e]) * rs[e];
        t[e] = __builtin_fmaf(f[i][e], ga[e], be[e]);
      }
      slope8(t, d[i], a.act);
#pragma unroll
      for (int e = 0; e < V; ++e) t[e] = rs[e] * (__builtin_fmaf(d[i][e], ga[e], -h1[e]) - f[i][e] * h2[e]);
      put_some<ALIGNED>(op + (r + (int64_t)i * g.side) * a.lddx, p.count, t);
    }
  });
}

// f(TX, TY, ALIGNED)
template <typename F>
void with_types(const GnArgs& a, bool aligned, F&& f) {
  auto typed = [&](auto x, auto y) {
    if (aligned) f(x, y, std::true_type{});
    else f(x, y, std::false_type{});
  };
  if (a.x_f32 && a.y_f32) typed(0.f, 0.f);
  else if (a.x_f32) typed(0.f, bf16_t{});
  else if (a.y_f32) typed(bf16_t{}, 0.f);
  else typed(bf16_t{}, bf16_t{});
}

// blocks of the passes: what they read is bound for HBM
GnGrid sums_grid(const GnArgs& a) { return make_grid(a, 2048, 256); }
GnGrid apply_grid(const GnArgs& a) { return make_grid(a, 4096, 1 << 20); }

bool rows_aligned(const GnArgs& a) { return a.ldx % V == 0 && a.ldy % V == 0; }

}  // namespace

size_t gn_fwd_ws(const GnArgs& a) {
  const GnGrid g = sums_grid(a);
  return ((size_t)a.n * a.groups + (size_t)a.n * g.chunks * entries(a, g)) * sizeof(float2);
}

hipError_t gn_fwd_launch(const GnArgs& a, const void* x, const float* gamma, const float* beta, void* y, float* mean,
                         float* rstd, void* ws, hipStream_t s) {
  const GnGrid g = sums_grid(a), ga = apply_grid(a);
  float2* stats = static_cast<float2*>(ws);
  float2* part = stats + (size_t)a.n * a.groups;
  with_types(a, rows_aligned(a), [&](auto tx, auto ty, auto al) {
    using TX = decltype(tx);
    using TY = decltype(ty);
    constexpr bool AL = decltype(al)::value;
    trace_begin(KC_GN_STATS);
    NUMBAT_LAUNCH((gn_stats_kernel<TX, AL>), blocks_of(a, g), dim3(kThreads), 0, s, a, g, static_cast<const TX*>(x), part);
    const unsigned joins = (unsigned)(((int64_t)a.n * a.groups + kThreads / 64 - 1) / (kThreads / 64));
    NUMBAT_LAUNCH(gn_join_kernel, dim3(joins), dim3(kThreads), 0, s, a, g, part, stats, mean, rstd);
    trace_end(KC_GN_STATS);
    trace_begin(KC_GN_FWD);
    NUMBAT_LAUNCH((gn_fwd_kernel<TX, TY, AL>), blocks_of(a, ga), dim3(kThreads), 0, s, a, ga, static_cast<const TX*>(x),
                  gamma, beta, stats, static_cast<TY*>(y));
    trace_end(KC_GN_FWD);
  });
  return hipGetLastError();
}

size_t gn_bwd_ws(const GnArgs& a) {
  const GnGrid g = sums_grid(a);
  return (size_t)a.n * a.groups * sizeof(float2) + (size_t)a.n * (g.chunks + 1) * 2 * a.c * sizeof(float);
}

hipError_t gn_bwd_launch(const GnArgs& a, const void* dy, const void* x, const float* mean, const float* rstd,
                         const float* gamma, const float* beta, void* dx, float* dgamma, float* dbeta, int accumulate,
                         void* ws, hipStream_t s) {
  const GnGrid g = sums_grid(a), ga = apply_grid(a);
  float2* means = static_cast<float2*>(ws);
  float* sums = reinterpret_cast<float*>(means + (size_t)a.n * a.groups);
  float* part = sums + (size_t)a.n * 2 * a.c;
  with_types(a, rows_aligned(a) && a.lddx % V == 0, [&](auto tx, auto ty, auto al) {
    using TX = decltype(tx);
    using TY = decltype(ty);
    constexpr bool AL = decltype(al)::value;
    const TX* xp = static_cast<const TX*>(x);
    const TY* dp = static_cast<const TY*>(dy);
    trace_begin(KC_GN_BWD_SUMS);
    NUMBAT_LAUNCH((gn_bwd_sums_kernel<TX, TY, AL>), blocks_of(a, g), dim3(kThreads), 0, s, a, g, dp, xp, mean, rstd, gamma,
                  beta, part);
    NUMBAT_LAUNCH(gn_bwd_join_kernel, dim3((unsigned)a.groups, (unsigned)a.n), dim3(kThreads), 0, s, a, g, part, gamma,
                  sums, means);
    trace_end(KC_GN_BWD_SUMS);
    if (dx != nullptr) {
      trace_begin(KC_GN_BWD);
      NUMBAT_LAUNCH((gn_bwd_kernel<TX, TY, AL>), blocks_of(a, ga), dim3(kThreads), 0, s, a, ga, dp, xp, mean, rstd, gamma,
                    beta, means, static_cast<TX*>(dx));
      trace_end(KC_GN_BWD);
    }
  });
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || (dgamma == nullptr && dbeta == nullptr)) return e;
  trace_begin(KC_GN_BWD_FINISH);
  column_sum_launch(sums, a.n, 2 * (int64_t)a.c, 2 * a.c, a.c, dbeta, dgamma, accumulate, s);
  trace_end(KC_GN_BWD_FINISH);
  return hipGetLastError();
}

}  // namespace numbat
