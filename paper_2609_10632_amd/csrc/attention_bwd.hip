// The backward of attention on gfx950, with P = exp(s - lse) and ds = P (dy v^T - delta):
//   dq = scale ds k,  dk = scale ds^T q,  dv = P^T dy
// as two kernels that each form P and ds anew, since a single one would have to add dq over blocks of
// keys in an order that changes from run to run (or keep a copy of dq for each): seven products
// where five would do.
//   dq    first delta = sum dy y of each column, which it leaves for the other; a wave owns 32 columns and walks the
//         keys, as in the forward: s^T = k q^T, dp^T = v dy^T, dq^T += k^T ds^T; k and v in LDS, q and dy in registers
//   dkv   a wave owns 32 keys and walks the columns: s = q k^T, dp = dy v^T, dv^T += dy^T P, dk^T += q^T ds;
//         q and dy in LDS, k and v in registers.  The heads that share a head of k and v are columns of one
//         product, so their gradients are added in its sums.
// Few columns, or few keys, are split into ranges of the other, whose sums a third kernel adds in order.
//
// Seven products of 2 d operations a pair and two exponentials.  2 x 16 heads on 2 x 8 of 8192 x 8192 causal, d = 128:
// dq 0.72 ms (1140 TFLOP/s of its six d operations a pair), dkv 1.18 to 1.22 ms (900 to 930 of its eight), 1.83 to
// 1.96 together, against 1218 TFLOP/s of the largest library product.  dkv's accumulators, k and v take 192 registers
// of a lane at d = 128, so that it runs one wave to a SIMD, its operands read two slices ahead; up to d = 96 two fit,
// which takes 4 x 8 heads of 4096 x 4096 x 96 from 516 to 395 us.  16 padded maps of up to 1600 pixels, 6 heads, d =
// 64: 66 to 70 and 85 to 94 us; there the vector work is more than the products, and the last blocks of long maps run
// alone.
#include <algorithm>
#include <type_traits>

#include "attention_tile.h"

namespace numbat {

namespace {

template <int DP, int NW>
__global__ __launch_bounds__(NW * 64, DP <= 64 || NW == 4 ? 2 : 1) void attn_dq_kernel(AttnArgs a, AttnGrid g, float2* rows, float* part) {
  using H = Head<DP>;
  constexpr int KS = H::KS, FB = H::FB;
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
  const bf16_t* drow = a.dy + ((int64_t)p.b * a.q_len + row) * a.ldy + head * a.d;
  u32x4 qf[KS], df[KS];
#pragma unroll
  for (int k = 0; k < KS; ++k) {
    qf[k] = row_chunk(qrow, valid, a.d, k, half);
    df[k] = row_chunk(drow, valid, a.d, k, half);
  }
  // lse in base 2 and delta of the lane's column, which the other kernel reads too; a column that counts for
  // nothing, or sees no key, gets an lse of plus infinity, hence weights of zero, and no delta, whatever it holds
  float2 stat = make_float2(INFINITY, 0.f);
  {
    const bf16_t* yrow = a.y + ((int64_t)p.b * a.q_len + row) * a.ldy + head * a.d;
    float t = 0.f;
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      const u32x4 yf = row_chunk(yrow, valid, a.d, k, half);
      float y[8], g8[8];
      unpack8(make_uint4(yf.x, yf.y, yf.z, yf.w), y);
      unpack8(make_uint4(df[k].x, df[k].y, df[k].z, df[k].w), g8);
#pragma unroll
      for (int e = 0; e < 8; ++e) t = __builtin_fmaf(y[e], g8[e], t);
    }
    t = half_sum(t);
    if (keys > 0) {
      const float lse = a.lse[((int64_t)p.b * a.kv_heads * a.group + head) * a.q_len + row];
      if (lse != -INFINITY) stat = make_float2(lse * kLog2e, t);
    }
    if (inside && half == 0 && p.split == 0) rows[((int64_t)p.b * a.kv_heads + p.h) * cols + col] = stat;
  }

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
  f32x16 dq[FB];
#pragma unroll
  for (int f = 0; f < FB; ++f) dq[f] = zeros16();

  auto tile = [&](const unsigned char* st, int key) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      f32x16 s, dp;
      u32x4 kf[2][FB];  // k's operands of two slices of 16 keys
      auto read_k = [&](int u) __attribute__((always_inline)) {
#pragma unroll
        for (int f = 0; f < FB; ++f) kf[u][f] = across.read(st, f, 2 * i + u);
      };
      along_pair<DP, 2>(along, st, i, st + H::TILE, i, qf, df, s, dp, [&] { read_k(0); });
#pragma unroll
      for (int r = 0; r < 16; ++r)
        s[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], a.scale_log2, -stat.x)) * (dp[r] - stat.y);
      if (key + kTile > wave_all) {
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (key + 32 * i + 8 * (r / 4) + 4 * half + r % 4 >= keys) s[r] = 0.f;
      }
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        if (u == 0) read_k(1);
        const u32x4 w = operand(s, u);
        pin();
#pragma unroll
        for (int f = 0; f < FB; ++f) dq[f] = mfma32x32x16(kf[u][f], w, dq[f]);
        pin();
      }
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
  if (keys == 0)
#pragma unroll
    for (int f = 0; f < FB; ++f) dq[f] = zeros16();
  if (g.splits == 1) {
    store_row<FB>(a.dq + ((int64_t)p.b * a.q_len + row) * a.ldq + head * a.d, inside, a.d, dq, a.scale, half);
  } else {
    const int64_t at = (((int64_t)p.split * a.batch + p.b) * a.kv_heads + p.h) * cols + col;
    store_part<FB>(part + at * a.d, inside, a.d, dq, a.scale, half);
  }
}

template <int DP, int NW>
__global__ __launch_bounds__(NW * 64, DP <= 64 || (NW == 4 && DP <= 96) ? 2 : 1) void attn_dkv_kernel(AttnArgs a, AttnGrid g, const float2* rows,
                                                                             float* part) {
  using H = Head<DP>;
  constexpr int KS = H::KS, FB = H::FB;
  __shared__ __attribute__((aligned(1024))) unsigned char st0[2 * H::TILE];
  __shared__ __attribute__((aligned(1024))) unsigned char st1[2 * H::TILE];
  // of each column: lse in base 2, delta, and the keys it sees
  __shared__ __attribute__((aligned(16))) float s_lse[2][kTile], s_delta[2][kTile];
  __shared__ __attribute__((aligned(16))) int s_keys[2][kTile];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int half = lane >> 5;
  const AttnPlace p(a, g, NW > 1);
  const Lengths n(a, p.b);
  const int cols = a.q_len * a.group;
  const int k0 = p.tile * NW * 32, key = k0 + wave * 32 + (lane & 31);
  const bool inside = key < a.kv_len, valid = key < n.kv;

  const int64_t krow = (int64_t)p.b * a.kv_len + key;
  u32x4 kf[KS], vf[KS];
#pragma unroll
  for (int k = 0; k < KS; ++k) {
    kf[k] = row_chunk(a.k + krow * a.ldk + p.h * a.d, valid, a.d, k, half);
    vf[k] = row_chunk(a.v + krow * a.ldv + p.h * a.d, valid, a.d, k, half);
  }

  // columns that see a key of the block: all that count, or those from the first row that sees key k0 on.  (The
  // others of its tile are zeros, like those behind the end.)
  const int end = k0 < n.kv ? (int)min((int64_t)n.q * a.group, (int64_t)(p.split + 1) * g.per_split) : 0;
  const int first = (int)min(a.causal ? (int64_t)max(k0 - (n.kv - n.q), 0) * a.group : 0, (int64_t)end);
  const int begin = (int)min(max((int64_t)(first / kTile * kTile), (int64_t)p.split * g.per_split), (int64_t)end);
  auto sees = [&](int c) __attribute__((always_inline)) { return (uint32_t)(c - first) < (uint32_t)(end - first); };

  // Rows of q and dy of a tile of columns: bytes from the tile's first row
  using L = TileLoad<DP, NW>;
  const bf16_t* qbase = a.q + (int64_t)p.b * a.q_len * a.ldq + p.h * a.group * a.d;
  const bf16_t* dbase = a.dy + (int64_t)p.b * a.q_len * a.ldy + p.h * a.group * a.d;
  auto load = [&](unsigned char* st, int c) __attribute__((always_inline)) {
    const int r0 = (int)fdiv((uint32_t)c, a.div_group);
    const auto rq = rsrc(qbase + (int64_t)r0 * a.ldq), rd = rsrc(dbase + (int64_t)r0 * a.ldy);
#pragma unroll
    for (int q = 0; q < L::N; ++q) {
      const int col = c + L::row(q, wave, lane), chunk = L::chunk(q, wave, lane);
      const int r = (int)fdiv((uint32_t)col, a.div_group), at = (col - r * a.group) * a.d + chunk * 8;
      const bool counts = sees(col) && chunk * 8 < a.d;
      const uint32_t vq = counts ? (uint32_t)((r - r0) * a.ldq + at) * 2 : kOob;
      const uint32_t vd = counts ? (uint32_t)((r - r0) * a.ldy + at) * 2 : kOob;
      lds_void_t* to = (lds_void_t*)(st + (q * NW + wave) * 1024);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rq, to, 16, vq, 0, 0, 0);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rd, (lds_void_t*)(st + H::TILE + (q * NW + wave) * 1024), 16, vd, 0, 0, 0);
    }
  };
  const float2* stats = rows + ((int64_t)p.b * a.kv_heads + p.h) * cols;
  auto stat_of = [&](int c) __attribute__((always_inline)) {
    return tid < kTile && sees(c + tid) ? stats[c + tid] : make_float2(INFINITY, 0.f);
  };
  auto put_stats = [&](int u, int c, float2 v) __attribute__((always_inline)) {
    if (tid < kTile) {
      s_lse[u][tid] = v.x;
      s_delta[u][tid] = v.y;
      s_keys[u][tid] = n.keys(a, (int)fdiv((uint32_t)(c + tid), a.div_group));
    }
  };
  constexpr int AHEAD = 2;  // slices of operands read ahead
  Along<DP> along;
  Across<DP> across;
  along.init(lane);
  across.init(lane);
  f32x16 dk[FB], dv[FB];
#pragma unroll
  for (int f = 0; f < FB; ++f) dk[f] = dv[f] = zeros16();

  auto tile = [&](const unsigned char* st, int u, auto maskedc) __attribute__((always_inline)) {
    constexpr bool masked = decltype(maskedc)::value;
    const unsigned char *tq = st, *td = st + H::TILE;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      f32x16 s, dp;
      along_pair<DP, AHEAD>(along, tq, i, td, i, kf, vf, s, dp, [] {});
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int at = 32 * i + 8 * j + 4 * half;
        const f32x4 lse = *reinterpret_cast<const f32x4*>(&s_lse[u][at]);
        const f32x4 delta = *reinterpret_cast<const f32x4*>(&s_delta[u][at]);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int r = 4 * j + e;
          s[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], a.scale_log2, -lse[e]));
        }
        if constexpr (masked) {
          const int4 last = *reinterpret_cast<const int4*>(&s_keys[u][at]);
          const int l[4] = {last.x, last.y, last.z, last.w};
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (key >= l[e]) s[4 * j + e] = 0.f;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) dp[4 * j + e] = (dp[4 * j + e] - delta[e]) * s[4 * j + e];
      }
      // operands read one product ahead
      u32x4 x[2], y[2], pw, dw;
      x[0] = across.read(td, 0, 2 * i);
      y[0] = across.read(tq, 0, 2 * i);
#pragma unroll
      for (int t = 0; t < 2 * FB; ++t) {
        if (t % FB == 0) {
          pw = operand(s, t / FB);
          dw = operand(dp, t / FB);
        }
        if (t + 1 < 2 * FB) {
          x[(t + 1) & 1] = across.read(td, (t + 1) % FB, 2 * i + (t + 1) / FB);
          y[(t + 1) & 1] = across.read(tq, (t + 1) % FB, 2 * i + (t + 1) / FB);
        }
        pin();
        dv[t % FB] = mfma32x32x16(x[t & 1], pw, dv[t % FB]);
        dk[t % FB] = mfma32x32x16(y[t & 1], dw, dk[t % FB]);
        pin();
      }
    }
  };
  auto step = [&](unsigned char* st, unsigned char* next, int u, int c, auto maskedc) __attribute__((always_inline)) {
    stage_ready();  // this stage has landed, and every wave is done with the other
    float2 v = make_float2(INFINITY, 0.f);
    if (c + kTile < end) {
      load(next, c + kTile);
      v = stat_of(c + kTile);
    }
    tile(st, u, maskedc);
    if (c + kTile < end) put_stats(u ^ 1, c + kTile, v);
  };
  if (begin < end) {
    load(st0, begin);
    put_stats(0, begin, stat_of(begin));
  }
  // Pairs of tiles, first those with a column that does not see every key of the block.  (Loops of their own: one
  // with both kinds in it would move its accumulators from register to register.)
  auto pairs = [&](int c, int to, auto maskedc) __attribute__((always_inline)) {
    for (; c < to; c += 2 * kTile) {
      step(st0, st1, 0, c, maskedc);
      if (c + kTile < end) step(st1, st0, 1, c + kTile, maskedc);
    }
    return c;
  };
  const int64_t all = a.causal ? (int64_t)max(k0 + NW * 32 - 1 - (n.kv - n.q), 0) * a.group : 0;  // the first that sees all
  const int from = pairs(begin, (int)min(all, (int64_t)end), std::true_type{});
  pairs(from, end, std::false_type{});

  if (!valid)  // (rows behind the sequence's end)
#pragma unroll
    for (int f = 0; f < FB; ++f) dk[f] = dv[f] = zeros16();
  if (g.splits == 1) {
    store_row<FB>(a.dk + krow * a.ldk + p.h * a.d, inside, a.d, dk, a.scale, half);
    store_row<FB>(a.dv + krow * a.ldv + p.h * a.d, inside, a.d, dv, 1.f, half);
  } else {
    float* at = part + (((((int64_t)p.split * a.batch + p.b) * a.kv_heads + p.h) * a.kv_len + key) * 2) * a.d;
    store_part<FB>(at, inside, a.d, dk, a.scale, half);
    store_part<FB>(at + a.d, inside, a.d, dv, 1.f, half);
  }
}

// the ranges' sums added in order, a thread for 4 features: of columns (dq), or of keys (dk and dv beside it)
template <bool KEYS>
__global__ __launch_bounds__(64) void attn_bwd_join_kernel(AttnArgs a, int splits, const float* part) {
  const int per = a.d / 4, len = KEYS ? 2 * a.kv_len : a.q_len * a.group;
  const int64_t total = (int64_t)a.batch * a.kv_heads * len;
  for (int64_t i = blockIdx.x * 64ll + threadIdx.x; i < total * per; i += gridDim.x * 64ll) {
    const int64_t c = i / per;
    const int f = (int)(i - c * per) * 4;
    constexpr int N = 8;  // ranges' loads in flight
    f32x4 y = {0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < splits; s += N) {
      f32x4 v[N];
#pragma unroll
      for (int e = 0; e < N; ++e) v[e] = *reinterpret_cast<const f32x4*>(part + (min(s + e, splits - 1) * total + c) * a.d + f);
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (s + e < splits) y += v[e];
    }
    const int64_t bh = c / len;
    const int at = (int)(c - bh * len), b = (int)(bh / a.kv_heads), h = (int)(bh - (int64_t)b * a.kv_heads);
    bf16_t* to;
    if constexpr (KEYS) {
      const int64_t row = (int64_t)b * a.kv_len + at / 2;
      to = at % 2 == 0 ? a.dk + row * a.ldk : a.dv + row * a.ldv;
      to += h * a.d;
    } else {
      const int row = (int)fdiv((uint32_t)at, a.div_group);
      to = a.dq + ((int64_t)b * a.q_len + row) * a.ldq + (h * a.group + at - row * a.group) * a.d;
    }
    uint2 out;
    out.x = pack2(y.x, y.y);
    out.y = pack2(y.z, y.w);
    *reinterpret_cast<uint2*>(to + f) = out;
  }
}

int dq_waves(const AttnArgs& a) { return attn_waves(a, (int64_t)a.q_len * a.group, a.kv_len, false); }
int dkv_waves(const AttnArgs& a) { return attn_waves(a, a.kv_len, (int64_t)a.q_len * a.group, false); }

size_t columns_of(const AttnArgs& a) { return (size_t)a.batch * a.kv_heads * a.q_len * a.group; }
size_t keys_of(const AttnArgs& a) { return (size_t)a.batch * a.kv_heads * a.kv_len; }

AttnGrid dq_grid(const AttnArgs& a) {
  const int64_t side = dq_waves(a) * 32;
  return make_attn_grid(a, ((int64_t)a.q_len * a.group + side - 1) / side, a.kv_len, dq_waves(a));
}
AttnGrid dkv_grid(const AttnArgs& a) {
  const int64_t side = dkv_waves(a) * 32;
  return make_attn_grid(a, ((int64_t)a.kv_len + side - 1) / side, (int64_t)a.q_len * a.group, dkv_waves(a));
}
// dq and dkv run one after the other: their partials share their space
size_t part_floats(const AttnArgs& a) {
  const AttnGrid q = dq_grid(a), k = dkv_grid(a);
  return std::max(q.splits > 1 ? q.splits * columns_of(a) * a.d : 0, k.splits > 1 ? k.splits * keys_of(a) * 2 * a.d : 0);
}
size_t rows_bytes(const AttnArgs& a) { return (columns_of(a) * sizeof(float2) + 255) / 256 * 256; }

}  // namespace

size_t attn_bwd_ws(const AttnArgs& a) {
  if (a.batch == 0) return 0;
  return rows_bytes(a) + part_floats(a) * sizeof(float);
}

hipError_t attn_bwd_launch(const AttnArgs& a, void* ws, hipStream_t s) {
  float2* rows = static_cast<float2*>(ws);
  float* part = reinterpret_cast<float*>(static_cast<char*>(ws) + rows_bytes(a));
  const AttnGrid gq = dq_grid(a), gk = dkv_grid(a);
  auto join = [&](auto kc, const AttnGrid& g, size_t vectors) {
    trace_begin(KC_ATTN_JOIN);
    const int64_t threads = (int64_t)vectors * (a.d / 4);
    NUMBAT_LAUNCH((attn_bwd_join_kernel<decltype(kc)::value>), dim3((unsigned)std::min<int64_t>((threads + 63) / 64, 1 << 18)),
                  dim3(64), 0, s, a, g.splits, part);
    trace_end(KC_ATTN_JOIN);
  };
  hipError_t e = hipSuccess;
  with_head(a.d, [&](auto dc) {
    constexpr int DP = decltype(dc)::value;
    if (e == hipSuccess && a.q_len > 0) {
      trace_begin(KC_ATTN_DQ);
      if (dq_waves(a) == 4) NUMBAT_LAUNCH((attn_dq_kernel<DP, 4>), dim3(gq.blocks), dim3(256), 0, s, a, gq, rows, part);
      else NUMBAT_LAUNCH((attn_dq_kernel<DP, 2>), dim3(gq.blocks), dim3(128), 0, s, a, gq, rows, part);
      trace_end(KC_ATTN_DQ);
      if (gq.splits > 1) join(std::false_type{}, gq, columns_of(a));
      e = hipGetLastError();
    }
    if (e == hipSuccess && a.kv_len > 0) {
      trace_begin(KC_ATTN_DKV);
      if (dkv_waves(a) == 4) NUMBAT_LAUNCH((attn_dkv_kernel<DP, 4>), dim3(gk.blocks), dim3(256), 0, s, a, gk, rows, part);
      else NUMBAT_LAUNCH((attn_dkv_kernel<DP, 2>), dim3(gk.blocks), dim3(128), 0, s, a, gk, rows, part);
      trace_end(KC_ATTN_DKV);
      if (gk.splits > 1) join(std::true_type{}, gk, 2 * keys_of(a));
      e = hipGetLastError();
    }
  });
  return e;
}

}  // namespace numbat
