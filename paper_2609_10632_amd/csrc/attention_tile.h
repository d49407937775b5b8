// What the attention kernels share: tiles of rows of one head in LDS, the matrix instructions' operands
// out of them, and the stores of their results.
//
// A tile has 64 rows (keys, or queries) of DP features, d rounded up, zeros past d and past the rows that
// count.  It is loaded by direct-to-LDS loads and read in two ways: along the features, 16 bytes a lane
// (a product that sums over features), and across them, four rows of one feature a lane, by transposing
// reads (a product that sums over the rows).  The second kind meets the accumulators of a 32 x 32 product as
// they are: a lane holds rows 8 j + 4 h + 0..3 of its column, h = lane / 32, and so a slice of 16 rows
// of the next product takes rows 4 h + 0..3 and 8 + 4 h + 0..3 of both operands.  Weights never leave
// their registers.
#pragma once

#include "attention_kernels.h"

namespace numbat {

namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr uint32_t kOob = 0x80000000u;  // a buffer offset past every range: zeros are loaded
constexpr int kRecords = 0x7ffffff0;
constexpr int kTile = 64;               // rows of a tile

typedef __attribute__((address_space(3))) void lds_void_t;
typedef short v4s_t __attribute__((ext_vector_type(4)));
typedef unsigned v2u_t __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) v4s_t lds_v4s_t;

__device__ __forceinline__ __amdgpu_buffer_rsrc_t rsrc(const void* base) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), (short)0, kRecords, 0x00020000);
}

// A lane's 16-byte chunk c of row r lies in slot c ^ swizzle(r) of the row.  Reading along the features, 16
// consecutive rows take one chunk each: the swizzle (with the row's place in the 256 bytes of the
// banks) spreads them over all 16 chunk positions.  Reading across, 4 consecutive rows take four
// neighbouring chunks each: the swizzle's upper bits differ among them.
template <int DP>
struct Head {
  static constexpr int KS = DP / 16, FB = DP / 32;                   // slices of 16 and blocks of 32 features
  static constexpr int CPR = DP <= 32 ? 4 : DP <= 64 ? 8 : 16;       // chunks of a stored row
  static constexpr int ROW = CPR * 16, TILE = kTile * ROW;           // bytes
  static __device__ __forceinline__ int swizzle(int r) {
    if constexpr (CPR == 16) return (r & 3) << 2 | (r >> 2 & 3);
    else if constexpr (CPR == 8) return (r >> 1 & 1) << 2 | (r >> 2 & 3);
    else return r >> 2 & 3;
  }
};

// loads of a tile, shared by NW waves
template <int DP, int NW>
struct TileLoad {
  using H = Head<DP>;
  static constexpr int N = H::TILE / 1024 / NW;  // load instructions of a wave
  static_assert(H::TILE % (1024 * NW) == 0, "whole load instructions");
  uint32_t off[N];  // this lane's bytes from the tile's first row, kOob past d
  __device__ __forceinline__ static int row(int q, int wave, int lane) { return ((q * NW + wave) * 64 + lane) / H::CPR; }
  __device__ __forceinline__ static int chunk(int q, int wave, int lane) {
    return lane % H::CPR ^ H::swizzle(row(q, wave, lane));
  }
  __device__ __forceinline__ void init(int64_t ld, int d, int wave, int lane) {
#pragma unroll
    for (int q = 0; q < N; ++q) {
      const int c = chunk(q, wave, lane);
      off[q] = c * 8 < d ? (uint32_t)(row(q, wave, lane) * ld * 2) + c * 16 : kOob;
    }
  }
  // `left` rows of the tile count
  __device__ __forceinline__ void load(unsigned char* tile, const bf16_t* base, int left, int wave, int lane) const {
    const auto r = rsrc(base);
#pragma unroll
    for (int q = 0; q < N; ++q)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void_t*)(tile + (q * NW + wave) * 1024), 16,
                                               row(q, wave, lane) < left ? off[q] : kOob, 0, 0, 0);
  }
};

// The wave's loads have landed and its reads are done, and so are the block's other waves'.  (By builtins: the
// compiler does not see a wait inside assembly and would wait for the next stage's loads as well.)
__device__ __forceinline__ void stage_ready() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0x0070);  // vmcnt(0) lgkmcnt(0)
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// Operand rows of 32 along the features.  (Where a lane's chunks lie differs by exclusive-ors of constants: one
// address serves all.)
template <int DP>
struct Along {
  using H = Head<DP>;
  uint32_t at;
  __device__ __forceinline__ void init(int lane) {
    const int r = lane & 31;
    at = r * H::ROW + ((lane >> 5) ^ H::swizzle(r)) * 16;
  }
  __device__ __forceinline__ u32x4 read(const unsigned char* tile, int block, int k) const {
    return *reinterpret_cast<const u32x4*>(tile + (at ^ (uint32_t)(32 * k)) + block * 32 * H::ROW);
  }
};

// 32 features across 16 rows, in the accumulators' order of rows
template <int DP>
struct Across {
  using H = Head<DP>;
  uint32_t at;
  __device__ __forceinline__ void init(int lane) {
    // lanes of 16 read 4 rows x 16 features: lane 4 e + q of them 4 features of row e
    const int g = lane >> 4, e = lane >> 2 & 3, q = lane & 3;
    const int r = 4 * (g >> 1) + e, c = 2 * (g & 1) + (q >> 1);
    at = r * H::ROW + (c ^ H::swizzle(r)) * 16 + (q & 1) * 8;
  }
  // (8 rows further down the swizzle differs in bit 1)
  __device__ __forceinline__ u32x4 read(const unsigned char* tile, int f, int slice) const {
    const unsigned char* p = tile + slice * 16 * H::ROW;
    const v2u_t lo = __builtin_bit_cast(
        v2u_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s_t*)(p + (at ^ (uint32_t)(64 * f)))));
    const v2u_t hi = __builtin_bit_cast(
        v2u_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s_t*)(p + (at ^ (uint32_t)(64 * f + 32)) + 8 * H::ROW)));
    return u32x4{lo.x, lo.y, hi.x, hi.y};
  }
};

__device__ __forceinline__ f32x16 zeros16() {
  f32x16 x;
#pragma unroll
  for (int i = 0; i < 16; ++i) x[i] = 0.f;
  return x;
}

// Keeps what is written before it before, and what is written behind it behind.  The products' operands are
// read from LDS some instructions ahead of their use; left to itself the compiler moves each read to its
// use, where a wave waits out the LDS's latency.
__device__ __forceinline__ void pin() { __builtin_amdgcn_sched_barrier(0); }

// s[j] = sum over features of rows `block[j]` of tile[j] and the columns in f[j]: two products side by side.  AHEAD: their
// operands are read that many slices ahead; 0 leaves the order to the compiler.  behind(): reads for what follows,
// issued with the last slices.
template <int DP, int AHEAD, typename F>
__device__ __forceinline__ void along_pair(const Along<DP>& along, const unsigned char* t0, int b0, const unsigned char* t1,
                                           int b1, const u32x4 (&f0)[DP / 16], const u32x4 (&f1)[DP / 16], f32x16& s0,
                                           f32x16& s1, F&& behind) {
  constexpr int KS = DP / 16;
  s0 = zeros16();
  s1 = zeros16();
  if constexpr (AHEAD == 0) {
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      s0 = mfma32x32x16(along.read(t0, b0, k), f0[k], s0);
      s1 = mfma32x32x16(along.read(t1, b1, k), f1[k], s1);
    }
  } else {
    u32x4 x[AHEAD + 1], y[AHEAD + 1];
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      x[k] = along.read(t0, b0, k);
      y[k] = along.read(t1, b1, k);
    }
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      if (k + AHEAD < KS) {
        x[(k + AHEAD) % (AHEAD + 1)] = along.read(t0, b0, k + AHEAD);
        y[(k + AHEAD) % (AHEAD + 1)] = along.read(t1, b1, k + AHEAD);
      } else if (k + AHEAD == KS) {
        behind();
      }
      pin();
      s0 = mfma32x32x16(x[k % (AHEAD + 1)], f0[k], s0);
      s1 = mfma32x32x16(y[k % (AHEAD + 1)], f1[k], s1);
      pin();
    }
  }
}

// slice s (16 rows) of a 32 x 32 product's accumulators as an operand
__device__ __forceinline__ u32x4 operand(const f32x16& x, int s) {
  return u32x4{pack2(x[8 * s], x[8 * s + 1]), pack2(x[8 * s + 2], x[8 * s + 3]), pack2(x[8 * s + 4], x[8 * s + 5]),
               pack2(x[8 * s + 6], x[8 * s + 7])};
}

// a lane's 16 bytes of a row of d features in memory: features 16 k + 8 h .. + 7
__device__ __forceinline__ u32x4 row_chunk(const bf16_t* row, bool valid, int d, int k, int half) {
  const int c = 16 * k + 8 * half;
  return valid && c < d ? *reinterpret_cast<const u32x4*>(row + c) : u32x4{0, 0, 0, 0};
}

// the other half wave's value beside one's own, in the halves' order
__device__ __forceinline__ v2u_t both_halves(uint32_t x) {
  const auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
  return v2u_t{r[0], r[1]};
}
__device__ __forceinline__ float half_max(float x) {
  const v2u_t r = both_halves(__float_as_uint(x));
  return fmaxf(__uint_as_float(r.x), __uint_as_float(r.y));
}
__device__ __forceinline__ float half_sum(float x) {
  const v2u_t r = both_halves(__float_as_uint(x));
  return __uint_as_float(r.x) + __uint_as_float(r.y);
}

// Stores the lane's column of DP / 32 accumulators, times `by`, as a row of d bf16 features.  A lane has 4
// of every 8 features; the halves trade them so that each stores 8.
template <int FB>
__device__ __forceinline__ void store_row(bf16_t* row, bool valid, int d, const f32x16 (&x)[FB], float by, int half) {
#pragma unroll
  for (int f = 0; f < FB; ++f)
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int i = 8 * j;
      const uint32_t a0 = pack2(x[f][i] * by, x[f][i + 1] * by), a1 = pack2(x[f][i + 2] * by, x[f][i + 3] * by);
      const uint32_t b0 = pack2(x[f][i + 4] * by, x[f][i + 5] * by), b1 = pack2(x[f][i + 6] * by, x[f][i + 7] * by);
      const auto r0 = __builtin_amdgcn_permlane32_swap(a0, b0, false, false);
      const auto r1 = __builtin_amdgcn_permlane32_swap(a1, b1, false, false);
      const int c = 32 * f + 16 * j + 8 * half;
      if (valid && c < d) *reinterpret_cast<u32x4*>(row + c) = u32x4{r0[0], r1[0], r0[1], r1[1]};
    }
}
// the same as fp32 (dense rows of d, a multiple of 8)
template <int FB>
__device__ __forceinline__ void store_part(float* row, bool valid, int d, const f32x16 (&x)[FB], float by, int half) {
#pragma unroll
  for (int f = 0; f < FB; ++f)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int c = 32 * f + 8 * j + 4 * half;
      if (valid && c < d)
        *reinterpret_cast<f32x4*>(row + c) =
            f32x4{x[f][4 * j] * by, x[f][4 * j + 1] * by, x[f][4 * j + 2] * by, x[f][4 * j + 3] * by};
    }
}

constexpr int kCus = 256;
constexpr int64_t kMaxBlocks = (1ll << 32) / 256 - 1;  // of 256 threads in a launch

// A sequence's numbers of queries and keys that count
struct Lengths {
  int q, kv;
  __device__ __forceinline__ Lengths(const AttnArgs& a, int b) {
    q = a.q_lengths != nullptr ? min(max(a.q_lengths[b], 0), a.q_len) : a.q_len;
    kv = a.kv_lengths != nullptr ? min(max(a.kv_lengths[b], 0), a.kv_len) : a.kv_len;
  }
  // keys that query r sees
  __device__ __forceinline__ int keys(const AttnArgs& a, int r) const {
    return a.causal ? min(max(r + (kv - q) + 1, 0), kv) : kv;
  }
};

// The sequence with the b-th most work of a batch of up to 64: the blocks of long sequences come first, so that the
// last ones to run are short (gradients of 16 padded maps of 610 to 1600 pixels, 6 heads, d = 64: 176 us in the
// sequences' own order, 163 in this; forward 57 and 53).  Each wave ranks them for itself, which takes 1 to 3 us and is
// lost where a grid is one round of blocks (16 maps of up to 400 pixels, 9 heads: 13.5 us without, 14.5 with): blocks
// of one wave, whose work is a few columns over a range of keys, take the sequences as they come.
__device__ __forceinline__ int by_work(const AttnArgs& a, int b) {
  const int lane = threadIdx.x & 63;
  const Lengths n(a, min(lane, a.batch - 1));
  const float work = (float)n.q * (float)n.kv;
  int rank = 0;
  for (int j = 0; j < a.batch; ++j) {
    const float other = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(work), j));
    rank += other > work || (other == work && j < lane);
  }
  return __ffsll((unsigned long long)__ballot(lane < a.batch && rank == b)) - 1;
}

// a block's place: which sequence and head of k and v, which range (split), which tile
struct AttnGrid {
  int32_t tiles, splits, per_split;  // of columns, or of keys; per_split: rows of a range of the other, a multiple of kTile
  FastDiv div_tiles, div_splits, div_heads;
  uint32_t units, blocks;  // sequences, heads and ranges; times tiles
};
struct AttnPlace {
  int b, h, split, tile;
  __device__ __forceinline__ AttnPlace(const AttnArgs& a, const AttnGrid& g, bool order) {
    // The tiles of one head and range read the same k and v (or q and dy), so they share an XCD's L2.  Heads are
    // dealt to the XCDs in turn: sequences of different lengths then weigh on all of them alike.  (Those left
    // over are dealt by tiles.)
    const uint32_t x = blockIdx.x % kXcds, i = blockIdx.x / kXcds, dealt = g.units / kXcds * kXcds;
    uint32_t u = fdiv(i, g.div_tiles);
    tile = i - u * g.tiles;
    u = u * kXcds + x;
    if (u >= dealt) {
      const uint32_t left = blockIdx.x - dealt * g.tiles;
      u = fdiv(left, g.div_tiles);
      tile = left - u * g.tiles;
      u += dealt;
    }
    const uint32_t w = fdiv(u, g.div_splits);
    split = u - w * g.splits;
    b = fdiv(w, g.div_heads);
    h = w - b * a.kv_heads;
    if (order && (a.q_lengths != nullptr || a.kv_lengths != nullptr) && a.batch <= 64) b = by_work(a, b);
  }
};

// Ranges of `rows` rows where there would be fewer than 512 blocks (1024 of one wave), of 256 rows at least
inline int64_t attn_splits(int64_t blocks, int64_t rows, int waves) {
  return std::clamp<int64_t>((waves == 1 ? 1024 : 512) / std::max<int64_t>(1, blocks), 1, std::max<int64_t>(1, rows / 256));
}

// tiles * splits * sequences * heads
inline AttnGrid make_attn_grid(const AttnArgs& a, int64_t tiles, int64_t rows, int waves) {
  AttnGrid g;
  const int64_t splits = attn_splits((int64_t)a.batch * a.kv_heads * tiles, rows, waves);
  int64_t per = (rows + splits - 1) / splits;
  per = std::max<int64_t>(kTile, (per + kTile - 1) / kTile * kTile);
  g.per_split = (int32_t)std::min<int64_t>(per, 1 << 30);
  g.splits = (int32_t)std::max<int64_t>(1, (rows + per - 1) / per);
  g.tiles = (int32_t)tiles;
  g.div_tiles = make_fastdiv((uint32_t)std::max<int64_t>(1, tiles));
  g.div_splits = make_fastdiv((uint32_t)g.splits);
  g.div_heads = make_fastdiv((uint32_t)a.kv_heads);
  g.units = (uint32_t)std::min<int64_t>((int64_t)a.batch * a.kv_heads * g.splits, 0xffffffffll);
  g.blocks = (uint32_t)std::min<int64_t>((int64_t)a.batch * a.kv_heads * tiles * g.splits, 0xffffffffll);
  return g;
}

// Waves of a block: four share a tile's loads, but a grid of few blocks, or blocks of few columns, leave less of the
// card idle with two or one.  What counts is the waves' work on the fullest CU, ranges counted, times what it costs
// with fewer to share the loads (4 x 8 heads, 4096 x 4096, d = 64, dq: 1.2 to 1.4 times in twos; forward of 16 x 6
// heads of 1600 columns: 149 us in ones, 80 in fours; of 16 x 9 heads of 400: 19 us in fours, 16 in twos).
inline int attn_waves(const AttnArgs& a, int64_t columns, int64_t rows, bool one) {
  const int64_t heads = (int64_t)a.batch * a.kv_heads;
  int best = 4;
  double least = 1e300;
  for (int nw = 4; nw >= (one ? 1 : 2); nw /= 2) {
    const int64_t blocks = heads * ((columns + nw * 32 - 1) / (nw * 32)), splits = attn_splits(blocks, rows, nw);
    const double work = (double)((blocks * splits + kCus - 1) / kCus * nw) / (double)splits *
                        (nw == 4 ? 1.0 : nw == 2 ? 1.3 : 1.9);
    if (work < least) {
      least = work;
      best = nw;
    }
  }
  return best;
}

// f(DP) for the narrowest head that holds d features
template <typename F>
void with_head(int d, F&& f) {
  if (d <= 32) f(std::integral_constant<int, 32>{});
  else if (d <= 64) f(std::integral_constant<int, 64>{});
  else if (d <= 96) f(std::integral_constant<int, 96>{});
  else f(std::integral_constant<int, 128>{});
}


}  // namespace

}  // namespace numbat
