// Attention on gfx950: y_i = sum_j exp(s_ij - lse_i) v_j, s_ij = scale q_i k_j, one pass over the keys with the
// running maximum and sum of each query.
//
// A wave owns 32 columns (queries of the heads that share a head of k and v) and walks the keys in tiles
// of 64.  It forms the scores transposed, s^T = k q^T, so that a lane has 32 keys of one column: maximum
// and sum are the lane's own work and one exchange between the half waves, and the weights are the
// second product's operand as they lie (attention_tile.h): y^T += v^T p^T.  k and v come by direct-to-LDS
// loads into one of two stages while the other is worked on; q stays in registers.
// The maximum is only raised where a score has passed it by 2^8: until then weights up to 2^8 do as well,
// and the accumulators need no scaling.  Weights are exp2(s scale log2(e) - unit) with the maximum's product
// rounded once into unit, which all of a column's weights share; where that rounding could be more than a
// small factor (scores past 10^4) the maximum is taken off the scores first, so that the largest key's weight
// is one at any score.  Few columns over many keys (one new token) are split into ranges
// of keys, whose results a second kernel joins.
//
// A tile's 64 x 32 scores cost a wave 128 d multiply-adds on the matrix unit, 32 cycles for each 32 x 32 x 16 of them,
// and 160 vector instructions, 32 of them exponentials at a quarter of the rate: at d = 64 twice the matrix unit's
// time, at d = 128 as much.  Two to four waves a SIMD cover one with the other.  2 x 32 heads on 2 x 8 of 8192 x 8192
// causal, d = 128: 1.00 to 1.13 ms, 1098 TFLOP/s at best, of the 1218 that the largest library product reached on that
// card (both are held by the card's power rather than by the matrix unit, which is busy 56 to 60% of the time at 1.65
// to 1.7 GHz).  16 x 9 heads of 400 x 400, d = 64: 15 us, of which the first loads, the last stores and the launch are
// half.  One query of each of 8 x 32 heads over up to 8192 keys of 8 x 8: 48 us, 3.9 TB/s, with 4 us of the join.
#include <algorithm>

#include "attention_tile.h"

namespace numbat {

namespace {

constexpr float kRaise = 8.f;    // (log2)
constexpr float kFar = 16384.f;  // a unit's rounding, and a range's logarithm's, is at most 2^-11 up to here

template <int DP, int NW>
__global__ __launch_bounds__(NW * 64, DP <= 64 || NW == 4 ? 2 : 1) void attn_fwd_kernel(AttnArgs a, AttnGrid g, float* part, float2* part_lse) {
  using H = Head<DP>;
  // a wave on its own reads operands ahead; waves that share a SIMD cover each other's reads (in either order within
  // 1%, but for d = 64: 4 x 8 heads, 4096 x 4096 168 us in the compiler's order, 177 pinned)
  constexpr int KS = H::KS, FB = H::FB, AHEAD = NW == 1 ? 2 : 0;
  // one object per stage: the compiler then knows that a stage's reads do not wait for the loads in
  // flight into the other
  __shared__ __attribute__((aligned(1024))) unsigned char st0[2 * H::TILE];
  __shared__ __attribute__((aligned(1024))) unsigned char st1[2 * H::TILE];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int half = lane >> 5;
  AttnPlace p(a, g, NW > 1);
  if (a.causal) p.tile = g.tiles - 1 - p.tile;  // the longest first
  const Lengths n(a, p.b);
  const int cols = a.q_len * a.group, c0 = p.tile * NW * 32;
  const int col = c0 + wave * 32 + (lane & 31);
  const int row = (int)fdiv((uint32_t)col, a.div_group), head = p.h * a.group + col - row * a.group;
  const bool inside = col < cols, valid = inside && row < n.q;
  const int keys = valid ? n.keys(a, row) : 0;
  // keys that the wave's and the block's columns see at most, and that all of the wave's see
  auto seen = [&](int c, int last) __attribute__((always_inline)) {
    const int r = (int)fdiv((uint32_t)c, a.div_group);
    return r < n.q ? n.keys(a, min((int)fdiv((uint32_t)last, a.div_group), n.q - 1)) : 0;
  };
  const int w0 = c0 + wave * 32;
  const int block_end = min(seen(c0, c0 + NW * 32 - 1), (p.split + 1) * g.per_split);
  const int wave_end = seen(w0, w0 + 31);
  const int r0 = (int)fdiv((uint32_t)w0, a.div_group);
  const int wave_all = r0 < n.q ? n.keys(a, r0) : 0;
  const int key_first = p.split * g.per_split;

  const bf16_t* qrow = a.q + ((int64_t)p.b * a.q_len + row) * a.ldq + head * a.d;
  u32x4 qf[KS];
#pragma unroll
  for (int k = 0; k < KS; ++k) qf[k] = row_chunk(qrow, valid, a.d, k, half);

  const bf16_t* kbase = a.k + (int64_t)p.b * a.kv_len * a.ldk + p.h * a.d;
  const bf16_t* vbase = a.v + (int64_t)p.b * a.kv_len * a.ldv + p.h * a.d;
  TileLoad<DP, NW> kl, vl;
  kl.init(a.ldk, a.d, wave, lane);
  vl.init(a.ldv, a.d, wave, lane);
  auto load = [&](unsigned char* st, int key) __attribute__((always_inline)) {
    kl.load(st, kbase + (int64_t)key * a.ldk, n.kv - key, wave, lane);
    vl.load(st + H::TILE, vbase + (int64_t)key * a.ldv, n.kv - key, wave, lane);
  };
  Along<DP> along;
  Across<DP> across;
  along.init(lane);
  across.init(lane);

  f32x16 o[FB];
#pragma unroll
  for (int f = 0; f < FB; ++f) o[f] = zeros16();
  // A score's weight is exp2((s - base) scale_log2 - unit), base = 0 up to kFar; this half's sum of weights
  float base = 0.f, unit = -INFINITY, sum = 0.f;
  float limit = -INFINITY;  // the score from which on the maximum is raised
  bool far = false;         // whether a column of the wave has a base
  const float per_log2 = 1.0f / a.scale_log2;

  auto tile = [&](const unsigned char* st, int key) __attribute__((always_inline)) {
    f32x16 s[2];
    u32x4 vf[2][FB];  // v's operands of two slices of 16 keys
    auto read_v = [&](int u) __attribute__((always_inline)) {
#pragma unroll
      for (int f = 0; f < FB; ++f) vf[u & 1][f] = across.read(st + H::TILE, f, u);
    };
    along_pair<DP, AHEAD>(along, st, 0, st, 1, qf, qf, s[0], s[1], [&] { read_v(0); });
    if (key + kTile > wave_all) {
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (key + 32 * i + 8 * (r / 4) + 4 * half + r % 4 >= keys) s[i][r] = -INFINITY;
    }
    float top = s[0][0];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) top = fmaxf(top, s[i][r]);
    top = half_max(top);
    if (far || __any(top > limit)) {
      const float was = base, had = unit, at = top * a.scale_log2;
      if (__builtin_fmaf(top - base, a.scale_log2, -unit) > 0.f) {  // (its weight would be above one)
        const bool past = !(fabsf(at) <= kFar);
        base = past ? top : 0.f;
        unit = past ? 0.f : at;
        limit = __builtin_fmaf(unit + kRaise, per_log2, base);
      }
      // (a column that has seen no key yet has nothing to scale)
      const float by = had == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(__builtin_fmaf(was - base, a.scale_log2, had - unit));
      sum *= by;
#pragma unroll
      for (int f = 0; f < FB; ++f)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[f][r] *= by;
      far = __any(base != 0.f);
      if (far)
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int r = 0; r < 16; ++r) s[i][r] -= base;
    }
    const float less = unit == -INFINITY ? 0.f : unit;  // (a column that has seen no key yet)
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        s[i][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i][r], a.scale_log2, -less));
        sum += s[i][r];
      }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (AHEAD == 0) read_v(u);
      else if (u < 3) read_v(u + 1);
      const u32x4 w = operand(s[u / 2], u % 2);
      if (AHEAD > 0) pin();
#pragma unroll
      for (int f = 0; f < FB; ++f) o[f] = mfma32x32x16(vf[u & 1][f], w, o[f]);
      if (AHEAD > 0) pin();
    }
  };
  auto step = [&](unsigned char* st, unsigned char* next, int key) __attribute__((always_inline)) {
    stage_ready();  // this stage has landed, and every wave is done with the other
    if (key + kTile < block_end) load(next, key + kTile);
    if (key < wave_end) tile(st, key);
  };
  if (key_first < block_end) load(st0, key_first);
  for (int key = key_first; key < block_end; key += 2 * kTile) {
    step(st0, st1, key);
    if (key + kTile < block_end) step(st1, st0, key + kTile);
  }

  sum = half_sum(sum);
  const bool any = valid && !(sum == 0.f);  // (a sum that is no number stays one)
  const float inv = any ? 1.0f / sum : 0.f;
  const float lse = any ? unit + __builtin_amdgcn_logf(sum) : -INFINITY;  // (log2, beside base)
  if (!any) base = 0.f;
  if (!any)  // (what columns that count for nothing have added up)
#pragma unroll
    for (int f = 0; f < FB; ++f) o[f] = zeros16();
  if (g.splits == 1) {
    store_row<FB>(a.out + ((int64_t)p.b * a.q_len + row) * a.ldy + head * a.d, inside, a.d, o, inv, half);
    if (a.lse != nullptr && inside && half == 0)
      a.lse[((int64_t)p.b * a.kv_heads * a.group + head) * a.q_len + row] = __builtin_fmaf(base, a.scale, lse * kLn2);
  } else {
    const int64_t at = (((int64_t)p.split * a.batch + p.b) * a.kv_heads + p.h) * cols + col;
    store_part<FB>(part + at * a.d, inside, a.d, o, inv, half);
    if (inside && half == 0) part_lse[at] = make_float2(base, lse);
  }
}

// the ranges' results weighted by their sums: a thread for 4 features of a column
__global__ __launch_bounds__(64) void attn_join_kernel(AttnArgs a, int splits, const float* part, const float2* part_lse) {
  const int per = a.d / 4, cols = a.q_len * a.group;
  const int64_t total = (int64_t)a.batch * a.kv_heads * cols;
  for (int64_t i = blockIdx.x * 64ll + threadIdx.x; i < total * per; i += gridDim.x * 64ll) {
    const int64_t c = i / per;
    const int f = (int)(i - c * per) * 4;
    // (eight ranges' loads in flight)
    constexpr int N = 8;
    float base = 0.f, unit = -INFINITY, sum = 0.f;  // the largest range's
    f32x4 y = {0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < splits; s += N) {
      float2 lse[N];
#pragma unroll
      for (int e = 0; e < N; ++e) lse[e] = part_lse[min(s + e, splits - 1) * total + c];
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (__builtin_fmaf(lse[e].x - base, a.scale_log2, lse[e].y - unit) > 0.f) {
          base = lse[e].x;
          unit = lse[e].y;
        }
    }
    if (unit == -INFINITY) unit = 0.f;
    for (int s = 0; s < splits; s += N) {
      float2 lse[N];
      f32x4 v[N];
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const int64_t at = min(s + e, splits - 1) * total + c;
        lse[e] = part_lse[at];
        v[e] = *reinterpret_cast<const f32x4*>(part + at * a.d + f);
      }
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const float w = s + e < splits
                            ? __builtin_amdgcn_exp2f(__builtin_fmaf(lse[e].x - base, a.scale_log2, lse[e].y - unit))
                            : 0.f;
        sum += w;
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = __builtin_fmaf(w, v[e][i], y[i]);
      }
    }
    const float inv = sum == 0.f ? 0.f : 1.0f / sum;
    const int64_t bh = c / cols;
    const int col = (int)(c - bh * cols), row = (int)fdiv((uint32_t)col, a.div_group);
    const int b = (int)(bh / a.kv_heads), head = (int)(bh - (int64_t)b * a.kv_heads) * a.group + col - row * a.group;
    uint2 out;
    out.x = pack2(y.x * inv, y.y * inv);
    out.y = pack2(y.z * inv, y.w * inv);
    *reinterpret_cast<uint2*>(a.out + ((int64_t)b * a.q_len + row) * a.ldy + head * a.d + f) = out;
    if (a.lse != nullptr && f == 0)
      a.lse[((int64_t)b * a.kv_heads * a.group + head) * a.q_len + row] =
          sum == 0.f ? -INFINITY : __builtin_fmaf(base, a.scale, (unit + __builtin_amdgcn_logf(sum)) * kLn2);
  }
}

int fwd_waves(const AttnArgs& a) { return attn_waves(a, (int64_t)a.q_len * a.group, a.kv_len, true); }

AttnGrid fwd_grid(const AttnArgs& a) {
  const int64_t columns = fwd_waves(a) * 32, tiles = ((int64_t)a.q_len * a.group + columns - 1) / columns;
  return make_attn_grid(a, tiles, a.kv_len, fwd_waves(a));
}

size_t columns_of(const AttnArgs& a) { return (size_t)a.batch * a.kv_heads * a.q_len * a.group; }

}  // namespace

bool attn_fits(const AttnArgs& a) {
  const int64_t columns = (int64_t)a.q_len * a.group, heads = (int64_t)a.batch * a.kv_heads;
  return heads * std::max((columns + 31) / 32, ((int64_t)a.kv_len + 31) / 32) <= kMaxBlocks &&
         fwd_grid(a).blocks <= kMaxBlocks;
}

size_t attn_fwd_ws(const AttnArgs& a) {
  const AttnGrid g = fwd_grid(a);
  return g.splits > 1 ? g.splits * columns_of(a) * (a.d + 2) * sizeof(float) : 0;
}

hipError_t attn_fwd_launch(const AttnArgs& a, void* ws, hipStream_t s) {
  const AttnGrid g = fwd_grid(a);
  float* part = static_cast<float*>(ws);
  float2* part_lse = reinterpret_cast<float2*>(part + (g.splits > 1 ? g.splits * columns_of(a) * a.d : 0));
  trace_begin(KC_ATTN_FWD);
  with_head(a.d, [&](auto dc) {
    constexpr int DP = decltype(dc)::value;
    const int nw = fwd_waves(a);
    if (nw == 1) NUMBAT_LAUNCH((attn_fwd_kernel<DP, 1>), dim3(g.blocks), dim3(64), 0, s, a, g, part, part_lse);
    else if (nw == 2) NUMBAT_LAUNCH((attn_fwd_kernel<DP, 2>), dim3(g.blocks), dim3(128), 0, s, a, g, part, part_lse);
    else NUMBAT_LAUNCH((attn_fwd_kernel<DP, 4>), dim3(g.blocks), dim3(256), 0, s, a, g, part, part_lse);
  });
  trace_end(KC_ATTN_FWD);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || g.splits == 1) return e;
  trace_begin(KC_ATTN_JOIN);
  const int64_t threads = (int64_t)columns_of(a) * (a.d / 4);
  NUMBAT_LAUNCH(attn_join_kernel, dim3((unsigned)std::min<int64_t>((threads + 63) / 64, 1 << 18)), dim3(64), 0, s, a,
                g.splits, part, part_lse);
  trace_end(KC_ATTN_JOIN);
  return hipGetLastError();
}

}  // namespace numbat
