// Rotary positions on gfx950: every pair (a, b) of a head's features turned by its row's angle,
//   a' = a cos t - b sin t,  b' = b cos t + a sin t,  t = position * frequency
// Every head of a row turns by the same angles.  A block takes whole rows (or a part of a long one), forms each
// row's cosines and sines once, in LDS, and a thread goes through some of a row's heads with 16 bytes' worth of
// pairs: no table is read, and the angles cost little beside the rows' bytes, which bound the kernel (formed by
// every thread for itself they took 12 of 19 us of 25600 rows of 12 heads of 64 features).  Angles are counted in
// full turns in 64 bits, where whole turns fall away exactly: in 32 bits position 10^6 would be off by 0.06 of a
// radian.  Cosine and sine of what is left are fp32's, within 2 units of the last place.
#include <algorithm>

#include "attention_kernels.h"
#include "vec_io.h"

namespace numbat {

namespace {

struct RotaryGrid {
  int32_t pair_slots, slots;  // threads on a head's pairs, and on all its features
  int32_t head_step;          // heads that a row's threads take side by side
  int32_t unit;               // threads of a row: slots * head_step
  int32_t rows;               // rows of a block, 0 where a row takes several blocks
  int64_t row_blocks;
  FastDiv div_slots, div_unit, div_pairs;
};

constexpr int kThreads = 256;

template <typename T, bool HALVES, bool ALIGNED>
__global__ __launch_bounds__(kThreads) void rotary_kernel(RotaryArgs a, RotaryGrid g, const T* x, T* y) {
  constexpr int V = kVec<T>, NP = HALVES ? V : V / 2;  // pairs a thread turns: 16 bytes on each side, or of both
  constexpr int N = HALVES ? 2 : 4;                    // heads at a time: four loads in flight
  __shared__ float2 s_turn[kThreads * 8];              // (a row's threads hold all its pairs, 8 each at most)
  const uint32_t in_row = g.rows > 0 ? threadIdx.x : blockIdx.y * kThreads + threadIdx.x;
  const uint32_t sub = g.rows > 0 ? fdiv(in_row, g.div_unit) : 0;
  const uint32_t u = in_row - sub * g.unit;
  const int head0 = (int)fdiv(u, g.div_slots), slot = (int)(u - head0 * g.slots);
  const int rows = g.rows > 0 ? g.rows : 1;
  const bool mine = g.rows > 0 ? (int)sub < g.rows : (int)in_row < g.unit;
  const bool turns = slot < g.pair_slots;
  const int j0 = slot * NP, count = a.pairs - j0;
  for (int64_t rb = blockIdx.x; rb < g.row_blocks; rb += gridDim.x) {
    const int64_t row0 = rb * rows, row = row0 + sub;
    const bool work = mine && row < a.m;
    const T* xr = x + row * a.ldx;
    T* yr = y + row * a.ldy;
    float p[N][V], q[HALVES ? N : 1][V];
    auto load = [&](int h) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int at = min(h + i * g.head_step, a.heads - 1) * a.d;
        if constexpr (HALVES) {
          get_some<ALIGNED>(xr + at + j0, count, p[i]);
          get_some<ALIGNED>(xr + at + j0 + a.pairs, count, q[i]);
        } else {
          get_some<ALIGNED>(xr + at + 2 * j0, 2 * count, p[i]);
        }
      }
    };
    if (work && turns) load(head0);
    // the rows' angles
    const int angles = (int)min<int64_t>(rows, a.m - row0) * a.pairs;
    for (int i = threadIdx.x; i < angles; i += kThreads) {
      const uint32_t r = fdiv((uint32_t)i, g.div_pairs);
      const int j = i - r * a.pairs;
      const int axis = (j >= a.first[1]) + (j >= a.first[2]) + (j >= a.first[3]);
      int32_t pos = 0;
      if (a.pos != nullptr) {
        pos = a.pos[(row0 + r) * a.axes + axis];
      } else {
        uint32_t left = (uint32_t)(row0 + r);
#pragma unroll
        for (int k = kRotaryAxes - 1; k >= 0; --k)
          if (k < a.axes && k >= axis) {
            const uint32_t w = fdiv(left, a.extent[k]);
            pos = (int32_t)(left - w * a.extent[k].d);
            left = w;
          }
      }
      const double t = (double)pos * a.turns[j];
      float2 cs;
      sincospif(2.0f * (float)(t - rint(t)), &cs.y, &cs.x);
      s_turn[i] = cs;
    }
    __syncthreads();
    if (work && turns) {
      float c[NP], s[NP];
#pragma unroll
      for (int e = 0; e < NP; ++e) {
        const float2 cs = s_turn[sub * a.pairs + j0 + (e < count ? e : 0)];
        c[e] = cs.x;
        s[e] = cs.y;
      }
      for (int h = head0; h < a.heads; h += N * g.head_step) {
        if (h != head0) load(h);
#pragma unroll
        for (int i = 0; i < N; ++i) {
          if (h + i * g.head_step >= a.heads) break;
          const int at = (h + i * g.head_step) * a.d;
          float f[NP], o[HALVES ? NP : V];
          if constexpr (HALVES) {
#pragma unroll
            for (int e = 0; e < NP; ++e) {
              f[e] = __builtin_fmaf(p[i][e], c[e], -(q[i][e] * s[e]));
              o[e] = __builtin_fmaf(q[i][e], c[e], p[i][e] * s[e]);
            }
            put_some<ALIGNED>(yr + at + j0, count, f);
            put_some<ALIGNED>(yr + at + j0 + a.pairs, count, o);
          } else {
#pragma unroll
            for (int e = 0; e < NP; ++e) {
              o[2 * e] = __builtin_fmaf(p[i][2 * e], c[e], -(p[i][2 * e + 1] * s[e]));
              o[2 * e + 1] = __builtin_fmaf(p[i][2 * e + 1], c[e], p[i][2 * e] * s[e]);
            }
            put_some<ALIGNED>(yr + at + 2 * j0, 2 * count, o);
          }
        }
      }
    } else if (work) {  // features that do not turn
      const int first = 2 * a.pairs + (slot - g.pair_slots) * V, left = a.d - first;
      for (int h = head0; h < a.heads; h += g.head_step) {
        float f[V];
        get_some<ALIGNED>(xr + h * a.d + first, left, f);
        put_some<ALIGNED>(yr + h * a.d + first, left, f);
      }
    }
    __syncthreads();
  }
}

template <typename T>
void launch_typed(const RotaryArgs& a, const void* x, void* y, hipStream_t s) {
  constexpr int V = kVec<T>;
  RotaryGrid g;
  const int np = a.halves ? V : V / 2, rest = x == y ? 0 : a.d - 2 * a.pairs;
  g.pair_slots = (a.pairs + np - 1) / np;
  g.slots = g.pair_slots + (rest + V - 1) / V;
  // threads enough to fill the card twice, where there are heads for them
  constexpr int64_t kFill = 1 << 20;
  g.head_step = (int)std::clamp<int64_t>((kFill + a.m * g.slots - 1) / (a.m * g.slots), 1, a.heads);
  const int each = (a.heads + g.head_step - 1) / g.head_step;  // heads of a thread; as evenly as can be
  g.head_step = (a.heads + each - 1) / each;
  g.unit = g.slots * g.head_step;
  g.rows = g.unit <= kThreads ? kThreads / g.unit : 0;
  g.row_blocks = g.rows > 0 ? (a.m + g.rows - 1) / g.rows : a.m;
  g.div_slots = make_fastdiv((uint32_t)g.slots);
  g.div_unit = make_fastdiv((uint32_t)g.unit);
  g.div_pairs = make_fastdiv((uint32_t)a.pairs);
  const unsigned per_row = g.rows > 0 ? 1 : (unsigned)((g.unit + kThreads - 1) / kThreads);
  const dim3 grid((unsigned)std::min<int64_t>(g.row_blocks, std::max(1u, (1u << 20) / per_row)), per_row);
  // every access of 16 bytes starts at a multiple of them
  const bool aligned = a.d % V == 0 && a.ldx % V == 0 && a.ldy % V == 0 && (a.halves ? a.pairs % V == 0 : true) &&
                       (rest == 0 || 2 * a.pairs % V == 0);
  const T* xp = static_cast<const T*>(x);
  T* yp = static_cast<T*>(y);
  if (a.halves && aligned) NUMBAT_LAUNCH((rotary_kernel<T, true, true>), grid, dim3(kThreads), 0, s, a, g, xp, yp);
  else if (a.halves) NUMBAT_LAUNCH((rotary_kernel<T, true, false>), grid, dim3(kThreads), 0, s, a, g, xp, yp);
  else if (aligned) NUMBAT_LAUNCH((rotary_kernel<T, false, true>), grid, dim3(kThreads), 0, s, a, g, xp, yp);
  else NUMBAT_LAUNCH((rotary_kernel<T, false, false>), grid, dim3(kThreads), 0, s, a, g, xp, yp);
}

}  // namespace

hipError_t rotary_launch(const RotaryArgs& a, const void* x, void* y, hipStream_t s) {
  trace_begin(KC_ROTARY);
  if (a.f32) launch_typed<float>(a, x, y, s);
  else launch_typed<bf16_t>(a, x, y, s);
  trace_end(KC_ROTARY);
  return hipGetLastError();
}

}  // namespace numbat
