// Rotary positions on gfx950: every pair (a, b) of a head's features turned by its row's angle,
//   a' = a cos t - b sin t,  b' = b cos t + a sin t,  t = position * frequency
// Every head of a row turns by the same angles.  A thread owns 16 bytes' worth of pairs, forms their
// cosines and sines once and goes through heads of its row with them, so that no table is read and the
// angles cost little beside the rows' bytes, which bound the kernel.  Angles are counted in full
// turns in 64 bits, where whole turns fall away exactly: in 32 bits position 10^6 would be off by
// 0.06 of a radian.  Cosine and sine of what is left are fp32's, within 2 units of the last place.
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
  FastDiv div_slots, div_unit;
};

template <typename T, bool HALVES, bool ALIGNED>
__global__ __launch_bounds__(256) void rotary_kernel(RotaryArgs a, RotaryGrid g, const T* x, T* y) {
  constexpr int V = kVec<T>, NP = HALVES ? V : V / 2;  // pairs a thread turns: 16 bytes on each side, or of both
  for (int64_t rb = blockIdx.x; rb < g.row_blocks; rb += gridDim.x) {
    const uint32_t in_row = g.rows > 0 ? threadIdx.x : blockIdx.y * 256 + threadIdx.x;
    const uint32_t sub = g.rows > 0 ? fdiv(in_row, g.div_unit) : 0;
    const uint32_t u = in_row - sub * g.unit;
    const int64_t row = g.rows > 0 ? rb * g.rows + sub : rb;
    if (row >= a.m || (g.rows > 0 ? (int)sub >= g.rows : (int)in_row >= g.unit)) continue;
    const int head0 = (int)fdiv(u, g.div_slots), slot = (int)(u - head0 * g.slots);
    const T* xr = x + row * a.ldx;
    T* yr = y + row * a.ldy;
    if (slot >= g.pair_slots) {  // features that do not turn
      const int at = 2 * a.pairs + (slot - g.pair_slots) * V, count = a.d - at;
      for (int h = head0; h < a.heads; h += g.head_step) {
        float f[V];
        get_some<ALIGNED>(xr + h * a.d + at, count, f);
        put_some<ALIGNED>(yr + h * a.d + at, count, f);
      }
      continue;
    }
    const int j0 = slot * NP, count = a.pairs - j0;
    int32_t pos[kRotaryAxes];
    uint32_t left = (uint32_t)row;
#pragma unroll
    for (int i = kRotaryAxes - 1; i >= 0; --i) {
      pos[i] = 0;
      if (i >= a.axes) continue;
      if (a.pos != nullptr) {
        pos[i] = a.pos[row * a.axes + i];
      } else {
        const uint32_t q = fdiv(left, a.extent[i]);
        pos[i] = (int32_t)(left - q * a.extent[i].d);
        left = q;
      }
    }
    float c[NP], s[NP];
#pragma unroll
    for (int e = 0; e < NP; ++e) {
      const int j = j0 + (e < count ? e : 0);
      const int32_t p = j < a.first[1] ? pos[0] : j < a.first[2] ? pos[1] : j < a.first[3] ? pos[2] : pos[3];
      const double t = (double)p * a.turns[j];
      sincospif(2.0f * (float)(t - rint(t)), &s[e], &c[e]);
    }
    for (int h = head0; h < a.heads; h += g.head_step) {
      if constexpr (HALVES) {
        const int at = h * a.d + j0;
        float u[NP], v[NP], p[NP], q[NP];
        get_some<ALIGNED>(xr + at, count, u);
        get_some<ALIGNED>(xr + at + a.pairs, count, v);
#pragma unroll
        for (int e = 0; e < NP; ++e) {
          p[e] = __builtin_fmaf(u[e], c[e], -(v[e] * s[e]));
          q[e] = __builtin_fmaf(v[e], c[e], u[e] * s[e]);
        }
        put_some<ALIGNED>(yr + at, count, p);
        put_some<ALIGNED>(yr + at + a.pairs, count, q);
      } else {
        const int at = h * a.d + 2 * j0;
        float u[V], p[V];
        get_some<ALIGNED>(xr + at, 2 * count, u);
#pragma unroll
        for (int e = 0; e < NP; ++e) {
          p[2 * e] = __builtin_fmaf(u[2 * e], c[e], -(u[2 * e + 1] * s[e]));
          p[2 * e + 1] = __builtin_fmaf(u[2 * e + 1], c[e], u[2 * e] * s[e]);
        }
        put_some<ALIGNED>(yr + at, 2 * count, p);
      }
    }
  }
}

template <typename T>
void launch_typed(const RotaryArgs& a, const void* x, void* y, hipStream_t s) {
  constexpr int V = kVec<T>;
  RotaryGrid g;
  const int np = a.halves ? V : V / 2, rest = x == y ? 0 : a.d - 2 * a.pairs;
  g.pair_slots = (a.pairs + np - 1) / np;
  g.slots = g.pair_slots + (rest + V - 1) / V;
  // as few threads to a row as fill the card, so that each forms its angles for as many heads as can be
  constexpr int64_t kThreads = 1 << 19;
  g.head_step = (int)std::clamp<int64_t>((kThreads + a.m * g.slots - 1) / (a.m * g.slots), 1, a.heads);
  g.unit = g.slots * g.head_step;
  g.rows = g.unit <= 256 ? 256 / g.unit : 0;
  g.row_blocks = g.rows > 0 ? (a.m + g.rows - 1) / g.rows : a.m;
  g.div_slots = make_fastdiv((uint32_t)g.slots);
  g.div_unit = make_fastdiv((uint32_t)g.unit);
  const unsigned per_row = g.rows > 0 ? 1 : (unsigned)((g.unit + 255) / 256);
  const dim3 grid((unsigned)std::min<int64_t>(g.row_blocks, std::max(1u, (1u << 20) / per_row)), per_row);
  // every access of 16 bytes starts at a multiple of them
  const bool aligned = a.d % V == 0 && a.ldx % V == 0 && a.ldy % V == 0 && (a.halves ? a.pairs % V == 0 : true) &&
                       (rest == 0 || 2 * a.pairs % V == 0);
  const T* xp = static_cast<const T*>(x);
  T* yp = static_cast<T*>(y);
  if (a.halves && aligned) NUMBAT_LAUNCH((rotary_kernel<T, true, true>), grid, dim3(256), 0, s, a, g, xp, yp);
  else if (a.halves) NUMBAT_LAUNCH((rotary_kernel<T, true, false>), grid, dim3(256), 0, s, a, g, xp, yp);
  else if (aligned) NUMBAT_LAUNCH((rotary_kernel<T, false, true>), grid, dim3(256), 0, s, a, g, xp, yp);
  else NUMBAT_LAUNCH((rotary_kernel<T, false, false>), grid, dim3(256), 0, s, a, g, xp, yp);
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
