// The matrix products of a linear layer on gfx950: y = act(x w^T + b) + r, the data gradient
// (dy w) * act'(z) and the weight gradient dy^T x, as one tiled product
//   C[m][n] = sum_k A(m, k) B(n, k)
// whose operands either run along the reduction in memory ([m][k], [n][k]) or across it
// ([k][m], [k][n]), with the layer's element-wise work in its epilogue.
//
// A block owns a BM x BN tile of C and walks the reduction in steps of BK.  A step's two
// operand tiles are loaded by direct-to-LDS loads into one of S stages, in the operands' own
// layout; the MFMA fragments (8 consecutive k of one row per lane) come out by 16-byte reads
// where the operand runs along the reduction and by transposing reads (ds_read_b64_tr_b16)
// where it runs across it, so neither form costs a register transpose or a copy in memory.
// w's side is the MFMA's row operand: a lane's accumulators then hold 4 consecutive n of one
// m, which the epilogue stages through LDS with 16-byte writes and stores as rows.
//
// Per step a block reads (BM + BN) * BK * 2 bytes of operands and issues BM * BN * BK
// multiply-adds: a 256 x 256 tile needs 1/64 byte per multiply-add, which the L2s deliver at the
// matrix cores' rate; what bounds long reductions is the matrix cores, short ones (maps of
// few channels) the bytes of x, z and y.  8192 rows, 4096 -> 16384 with GELU and z: 973 us, 1130 TFLOP/s
// (without an epilogue's work 1195; dx 1130, dw 1340; the largest library product of this card reaches
// 1395); 102400 rows, 192 -> 768 with SiLU and z: 80 us, 4.4 TB/s of 5.1.
#include <algorithm>
#include <cmath>

#include "gemm_epilogue.h"

namespace numbat {

namespace {

constexpr uint32_t kOob = 0x80000000u;  // a buffer offset past every range
constexpr int kRecords = 0x7ffffff0;

typedef __attribute__((address_space(3))) void lds_void_t;
typedef short v4s_t __attribute__((ext_vector_type(4)));
typedef unsigned v2u_t __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) v4s_t lds_v4s_t;

template <int V>
using Ic = std::integral_constant<int, V>;
template <int I, int N, typename F>
__device__ __forceinline__ void static_for(F&& f) {
  if constexpr (I < N) {
    f(Ic<I>{});
    static_for<I + 1, N>(f);
  }
}

__device__ __forceinline__ __amdgpu_buffer_rsrc_t rsrc(const void* base) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), (short)0, kRecords, 0x00020000);
}

// the sum of 8 bf16 values
__device__ __forceinline__ float sum8(u32x4 v) {
  float f[8];
  unpack8(make_uint4(v.x, v.y, v.z, v.w), f);
  return ((f[0] + f[1]) + (f[2] + f[3])) + ((f[4] + f[5]) + (f[6] + f[7]));
}

// ---------------------------------------------------------------------------
// ANY_: operands' rows may start at any element (they pass through registers to LDS)
template <int BM_, int BN_, int BK_, int S_, int WM_, int WN_, bool ANY_ = false>
struct Tile {
  static constexpr bool ANY = ANY_;
  static constexpr int BM = BM_, BN = BN_, BK = BK_, S = S_, WM = WM_, WN = WN_, NW = WM * WN;
  static constexpr int TM = BM / WM / 32, TN = BN / WN / 32;   // 32 x 32 blocks per wave
  static constexpr int A_BYTES = BM * BK * 2, B_BYTES = BN * BK * 2, STAGE = A_BYTES + B_BYTES;
  static constexpr int AI = A_BYTES / 1024 / NW, BI = B_BYTES / 1024 / NW;  // load instructions per wave
  static constexpr int KS = BK / 16;
  static constexpr int OW = TN == 1 ? 32 : 64;                 // columns a wave stages at a time
  static constexpr int OLD = OW + 4;                           // fp32 per staged row
  static constexpr int OUT_BYTES = 32 * OLD * 4;               // per wave
  static constexpr int WPS = (NW + S - 1) / S;                 // waves that stage in one stage's space
  static_assert(A_BYTES % (1024 * NW) == 0 && B_BYTES % (1024 * NW) == 0, "whole load instructions");
  static_assert(WPS * OUT_BYTES <= STAGE, "the epilogue fits the stages");
  static_assert(KS % 2 == 0 && S >= 2 && S <= 4, "two fragment buffers, 2 to 4 stages");
  static_assert(TN == 1 || TN % 2 == 0, "whole staging strips");
  static_assert(!ANY || S == 2, "two stages, two steps in registers");
};

// An operand tile of SIDE rows of C (or columns) by BK of the reduction, as LDS holds it.
//  T false: [SIDE][BK], rows of 2 BK bytes; 16-byte chunk c of row r in slot c ^ (r / WIN % CPR),
//           WIN rows filling the 64 banks once, so that 16 rows' reads of one chunk spread over them
//  T true:  [BK][SIDE]; chunk c of row r in slot c ^ swz(r): a transposing read of 32 lanes covers
//           4 rows x 64 bytes, which the swizzle puts in different quarters of the banks
template <bool T, int SIDE, int BK, int NW, int NI>
struct Operand {
  static constexpr int CPR = BK / 8, WIN = 128 / BK;
  static __device__ __forceinline__ int swz(int r) { return SIDE == 64 ? 4 * ((r >> 1) & 1) : 4 * (r & 3); }

  const unsigned char* base;  // first element of the tile's rows, at the block's first k
  int64_t step;               // bytes to the next step
  uint32_t off[NI];           // this lane's part of each load instruction, kOob past the matrix
  int kpos[T ? NI : 1];       // its k within a step

  __device__ __forceinline__ void init(const bf16_t* p, int64_t ld, int64_t r0, int64_t rows, int64_t k0, int wave,
                                       int lane) {
    if constexpr (!T) {
      base = reinterpret_cast<const unsigned char*>(p + r0 * ld + k0);
      step = 2 * BK;
#pragma unroll
      for (int q = 0; q < NI; ++q) {
        const int row = (q * NW + wave) * (512 / BK) + lane / CPR;
        const int chunk = (lane % CPR) ^ (row / WIN % CPR);  // the same for every q: NW is even
        kpos[0] = chunk * 8;
        off[q] = r0 + row < rows ? (uint32_t)(row * ld * 2) + chunk * 16 : kOob;
      }
    } else {
      base = reinterpret_cast<const unsigned char*>(p + k0 * ld + r0);
      step = 2 * BK * ld;
#pragma unroll
      for (int q = 0; q < NI; ++q) {
        const int byte = (q * NW + wave) * 1024 + lane * 16;
        const int row = byte / (2 * SIDE), chunk = (byte % (2 * SIDE)) / 16 ^ swz(row);
        kpos[q] = row;
        off[q] = r0 + chunk * 8 < rows ? (uint32_t)(row * ld * 2) + chunk * 16 : kOob;
      }
    }
  }

  // load instruction q of the next step, of which `left` k remain (none or fewer: zeros)
  __device__ __forceinline__ void load(unsigned char* stage, int q, int64_t left, int wave) const {
    const uint32_t vo = kpos[T ? q : 0] < left ? off[q] : kOob;
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc(base), (lds_void_t*)(stage + (q * NW + wave) * 1024), 16, vo, 0, 0, 0);
  }
};

// The same tile from rows that start at any element: unaligned 16-byte loads into registers, two steps
// ahead, and 16-byte writes into LDS.  A vector that the row or the reduction ends in is read by
// elements, the rest of it zero.
template <bool T, int SIDE, int BK, int NW, int NI>
struct OperandAny {
  using Op = Operand<T, SIDE, BK, NW, NI>;
  const unsigned char* base;
  int64_t step;
  uint32_t off[NI];
  int kpos[T ? NI : 1];
  int whole[NI];  // elements of the lane's vector inside the matrix: T: columns left; else 8 or 0 by the row
  uint4 v[2][NI];

  __device__ __forceinline__ void init(const bf16_t* p, int64_t ld, int64_t r0, int64_t rows, int64_t k0, int wave,
                                       int lane) {
    base = reinterpret_cast<const unsigned char*>(T ? p + k0 * ld + r0 : p + r0 * ld + k0);
    step = T ? 2 * BK * ld : 2 * BK;
#pragma unroll
    for (int q = 0; q < NI; ++q) {
      const int byte = (q * NW + wave) * 1024 + lane * 16;
      if constexpr (!T) {
        const int row = byte / (2 * BK), chunk = (byte % (2 * BK)) / 16 ^ (row / Op::WIN % Op::CPR);
        kpos[0] = chunk * 8;  // the same for every q: NW is even
        off[q] = (uint32_t)(row * ld * 2) + chunk * 16;
        whole[q] = r0 + row < rows ? 8 : 0;
      } else {
        const int row = byte / (2 * SIDE), chunk = (byte % (2 * SIDE)) / 16 ^ Op::swz(row);
        const int64_t have = rows - r0 - chunk * 8;
        kpos[q] = row;
        off[q] = (uint32_t)(row * ld * 2) + chunk * 16;
        whole[q] = have < 8 ? (have > 0 ? (int)have : 0) : 8;
      }
    }
  }
  __device__ __forceinline__ void load(int b, int q, int64_t left) {
    const int64_t kleft = left - kpos[T ? q : 0];
    const int count = T ? (kleft > 0 ? whole[q] : 0) : (kleft < whole[q] ? (int)kleft : whole[q]);
    v[b][q] = make_uint4(0, 0, 0, 0);
    const bf16_t* p = reinterpret_cast<const bf16_t*>(base + off[q]);
    if (count >= 8) {
      v[b][q] = load16<false>(p);
    } else if (count > 0) {
      uint32_t h[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) h[e] = e < count ? p[e] : 0;
      v[b][q] = make_uint4(h[0] | h[1] << 16, h[2] | h[3] << 16, h[4] | h[5] << 16, h[6] | h[7] << 16);
    }
  }
  __device__ __forceinline__ void put(unsigned char* stage, int b, int wave, int lane) const {
#pragma unroll
    for (int q = 0; q < NI; ++q) *reinterpret_cast<uint4*>(stage + (q * NW + wave) * 1024 + lane * 16) = v[b][q];
  }
};

// fragment addresses of NB blocks of 32 rows from row `first` of an operand tile
template <bool T, int SIDE, int BK, int NB>
struct Frags {
  using Op = Operand<T, SIDE, BK, 2, 1>;
  uint32_t at[T ? NB : BK / 16];
  __device__ __forceinline__ void init(int first, int lane) {
    if constexpr (!T) {
      const int l32 = lane & 31, half = lane >> 5;
#pragma unroll
      for (int ks = 0; ks < BK / 16; ++ks)
        at[ks] = (uint32_t)((first + l32) * (BK * 2) + ((2 * ks + half) ^ (l32 / Op::WIN % Op::CPR)) * 16);
    } else {
      // lane 16 g + 4 e + q reads 4 columns (8 bytes) of rows 8 (g / 2) + e and that + 4 of a
      // 16-row slice; the read hands each lane 4 consecutive rows of one column
      const int g = lane >> 4, e = (lane & 15) >> 2, q = lane & 3, r0 = 8 * (g >> 1) + e;
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        const int c = first / 8 + 4 * i + 2 * (g & 1) + (q >> 1);
        at[i] = (uint32_t)(r0 * 2 * SIDE + (c ^ Op::swz(r0)) * 16 + (q & 1) * 8);
      }
    }
  }
  __device__ __forceinline__ u32x4 read(const unsigned char* tile, int i, int ks) const {
    if constexpr (!T) {
      return *reinterpret_cast<const u32x4*>(tile + at[ks] + i * 32 * BK * 2);
    } else {
      const unsigned char* p = tile + at[i] + ks * 16 * 2 * SIDE;
      const v2u_t lo = __builtin_bit_cast(v2u_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s_t*)p));
      const v2u_t hi =
          __builtin_bit_cast(v2u_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s_t*)(p + 4 * 2 * SIDE)));
      return u32x4{lo.x, lo.y, hi.x, hi.y};
    }
  }
};

template <int KIND, typename C>
__global__ __launch_bounds__(C::NW * 64) void gemm_kernel(GemmArgs a) {
  constexpr bool TA = KIND == kGemmWgrad, TB = KIND != kGemmFwd;
  constexpr int BM = C::BM, BN = C::BN, BK = C::BK, S = C::S, NW = C::NW, TM = C::TM, TN = C::TN, KS = C::KS;
  // one object per stage: the compiler then knows that a stage's reads do not wait for the
  // loads in flight into the others
  __shared__ __attribute__((aligned(1024))) unsigned char st0[C::STAGE];
  __shared__ __attribute__((aligned(1024))) unsigned char st1[C::STAGE];
  __shared__ __attribute__((aligned(1024))) unsigned char st2[S > 2 ? C::STAGE : 16];
  __shared__ __attribute__((aligned(1024))) unsigned char st3[S > 3 ? C::STAGE : 16];
  auto stage = [&](auto uc) __attribute__((always_inline)) -> unsigned char* {
    constexpr int u = decltype(uc)::value;
    if constexpr (u == 0) return st0;
    else if constexpr (u == 1) return st1;
    else if constexpr (u == 2) return st2;
    else return st3;
  };

  // tile of this block: each XCD takes a contiguous run of tiles, in columns of 8 tiles of m, so
  // that the blocks running on it at a time share operand rows in its L2
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const uint32_t tiles = (uint32_t)a.tiles_m * (uint32_t)a.tiles_n;
  uint32_t t = xcd_remap(blockIdx.x, gridDim.x);
  const uint32_t split = a.splits > 1 ? fdiv(t, a.div_tiles) : 0;
  t -= split * tiles;
  const uint32_t grp = fdiv(t, a.div_group), in_grp = t - grp * a.div_group.d;
  const uint32_t gsize = (uint32_t)a.tiles_m - grp * 8u;  // rows of tiles left: 8, or those of the last column
  const uint32_t tn = gsize >= 8u ? in_grp >> 3 : fdiv(in_grp, a.div_last);
  const uint32_t tm = grp * 8u + in_grp - tn * (gsize >= 8u ? 8u : gsize);
  const int64_t m0 = (int64_t)tm * BM;
  const int n0 = (int)tn * BN;
  const int64_t k0 = (int64_t)split * a.k_per_split;
  int64_t left = (a.k - k0 < a.k_per_split ? a.k - k0 : a.k_per_split);  // k not yet loaded
  const int nk = (int)((left + BK - 1) / BK);

  const int wm = wave / C::WN, wn = wave % C::WN;
  // The epilogue goes by strips of 32 rows x OW columns of the wave's sums, 16 bytes of results a lane
  // (8 columns of bf16 or 4 of fp32).  What it reads beside the sums for the first strips is loaded
  // before anything else, so that it is there when the sums are (and these loads, the oldest, disturb
  // no count of those in flight).
  constexpr int JS = C::OW / 32, STRIPS = TN / JS * TM;
  static_assert(TN == JS, "a lane's columns are the same in every strip");
  // strips loaded ahead: all of two, one of more, and of fp32 operands, which take twice the
  // registers, then none
  constexpr auto ahead = [](int nv) { return STRIPS <= 2 ? STRIPS : nv == 8 ? 1 : 0; };
  constexpr auto buffers = [](int nv) { return STRIPS <= 2 ? STRIPS : nv == 8 ? 2 : 1; };
  const EpiloguePtr ep = epilogue_at<KIND>(a.e, m0, n0);
  const int rows = (int)(a.m - m0 < BM ? a.m - m0 : BM), cols = a.n - n0;  // of the tile
  Aux x[STRIPS <= 2 && KIND != kGemmDgrad ? STRIPS * (C::OW / 8) : 2 * (C::OW / 16)];
  float bias[8];
  // row, column and passes of a strip with NV columns a lane
  auto row_of = [&](int s, int nv) __attribute__((always_inline)) { return (wm * TM + s % TM) * 32 + lane / (C::OW / nv); };
  auto col_of = [&](int s, int nv) __attribute__((always_inline)) {
    return (wn * TN + s / TM * JS) * 32 + lane % (C::OW / nv) * nv;
  };
  auto fetch = [&](auto nvc, auto sc) __attribute__((always_inline)) {
    constexpr int NV = decltype(nvc)::value, s = decltype(sc)::value, RPP = 64 * NV / C::OW;
    const int c = col_of(s, NV);
#pragma unroll
    for (int p = 0; p < 32 / RPP; ++p) {
      const int r = row_of(s, NV) + p * RPP;
      if (r < rows && c < cols) load_aux<NV>(ep, r, c, x[s % buffers(NV) * (32 / RPP) + p]);
    }
  };
  // f(columns a lane): 8 or 4 by the type of the results
  auto by_type = [&](auto&& f) __attribute__((always_inline)) {
    if constexpr (KIND == kGemmDgrad) f(Ic<8>{});
    else if constexpr (KIND == kGemmWgrad) f(Ic<4>{});
    else if (ep.out_f32) f(Ic<4>{});
    else f(Ic<8>{});
  };
  if (a.splits == 1)
    by_type([&](auto nvc) __attribute__((always_inline)) {
      constexpr int NV = decltype(nvc)::value;
      load_bias<KIND, NV>(a.e, n0 + col_of(0, NV), a.n, bias);
      if (a.e.vec) static_for<0, ahead(NV)>([&](auto sc) __attribute__((always_inline)) { fetch(nvc, sc); });
    });

  std::conditional_t<C::ANY, OperandAny<TA, BM, BK, NW, C::AI>, Operand<TA, BM, BK, NW, C::AI>> oa;
  std::conditional_t<C::ANY, OperandAny<TB, BN, BK, NW, C::BI>, Operand<TB, BN, BK, NW, C::BI>> ob;
  oa.init(a.a, a.lda, m0, a.m, k0, wave, lane);
  ob.init(a.b, a.ldb, n0, a.n, k0, wave, lane);
  // load instruction q of the step that `left` counts, A's first
  constexpr int L = C::AI + C::BI;
  auto load = [&](auto uc, int q) __attribute__((always_inline)) {
    if constexpr (C::ANY) {  // (into the registers of that parity)
      if (q < C::AI) oa.load(decltype(uc)::value, q, left);
      else ob.load(decltype(uc)::value, q - C::AI, left);
    } else {
      unsigned char* st = stage(uc);
      if (q < C::AI) oa.load(st, q, left, wave);
      else ob.load(st + C::A_BYTES, q - C::AI, left, wave);
    }
  };
  auto put_stage = [&](auto uc) __attribute__((always_inline)) {
    if constexpr (C::ANY) {
      oa.put(stage(uc), decltype(uc)::value, wave, lane);
      ob.put(stage(uc) + C::A_BYTES, decltype(uc)::value, wave, lane);
    }
  };
  auto advance = [&]() __attribute__((always_inline)) {
    oa.base += oa.step;
    ob.base += ob.step;
    left -= BK;
  };

  Frags<TA, BM, BK, TM> fa;
  Frags<TB, BN, BK, TN> fb;
  fa.init(wm * TM * 32, lane);
  fb.init(wn * TN * 32, lane);

  f32x16 acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;

  u32x4 af[2][TM], bf[2][TN];
  // The bias gradient is the sum of the weight gradient's first operand over the reduction: the blocks
  // of the first column of tiles add up the fragments that they multiply anyway, each of the waves that
  // share TM of them one.  (Not where a.db is left out: see gemm_sums_rows.)
  static_assert(TM <= C::WN, "a wave for each fragment");
  const bool sums = __builtin_amdgcn_readfirstlane(KIND == kGemmWgrad && a.db != nullptr && tn == 0 ? 1 : 0) != 0;
  float rowsum = 0.f;
  // fragment r of slice ks of a stage, A's first, into buffer b
  auto rd = [&](auto uc, int r, int ks, int b) __attribute__((always_inline)) {
    const unsigned char* st = stage(uc);
    if (r < TM) af[b][r] = fa.read(st, r, ks);
    else bf[b][r - TM] = fb.read(st + C::A_BYTES, r - TM, ks);
  };
  // The products of slice ks of stage u, with the reads of the next slice's fragments behind the
  // first half of them and a share of the step's loads spread over them.  Pinned: left to itself the
  // compiler sinks each read to its use, and a SIMD with one wave then waits out the LDS's latency
  // in every slice.
  constexpr int LOADING = S == 2 ? KS - 1 : KS;  // slices that carry loads
  auto slice = [&](auto uc, auto kc, auto sumc) __attribute__((always_inline)) {
    constexpr int u = decltype(uc)::value, ks = decltype(kc)::value, b = ks & 1;
    constexpr bool last = ks == KS - 1;
    constexpr int L0 = ks < LOADING ? ks * L / LOADING : L, L1 = ks < LOADING ? (ks + 1) * L / LOADING : L;
    constexpr int NM = TM * TN, NR = TM + TN, RW = NM >= 2 * NR ? NM / 2 : NM;
    static_for<0, NM>([&](auto tc) __attribute__((always_inline)) {
      constexpr int t = decltype(tc)::value;
      constexpr int r0 = t < RW ? t * NR / RW : NR, r1 = t < RW ? (t + 1) * NR / RW : NR;
      constexpr int l0 = L0 + t * (L1 - L0) / NM, l1 = L0 + (t + 1) * (L1 - L0) / NM;
#pragma unroll
      for (int r = r0; r < r1; ++r) rd(Ic<last ? (u + 1) % S : u>{}, r, last ? 0 : ks + 1, b ^ 1);
#pragma unroll
      for (int q = l0; q < l1; ++q) load(Ic<(u + S - 1) % S>{}, q);
      acc[t / TN][t % TN] = mfma32x32x16(bf[b][t % TN], af[b][t / TN], acc[t / TN][t % TN]);
      if constexpr (decltype(sumc)::value != 0 && t % TN == 0)
        if (wn == t / TN) rowsum += sum8(af[b][t / TN]);
      __builtin_amdgcn_sched_barrier(0);
    });
  };
  // Step kt multiplies out of stage u = kt mod S and loads step kt + S - 1 into the stage read last
  // step.  Before its last slice the wave's reads of the stage are done and the next step's loads
  // have landed (those of later steps stay in flight); past the barrier that holds for every wave,
  // so the last slice can read the next stage.
  constexpr int PENDING = S == 2 ? 0 : (S - 3) * L + (KS - 1) * L / KS;
  // (ANY: step kt + 1 goes from its registers to LDS first, and step kt + 3 is loaded into them)
  auto step = [&](auto uc, auto sumc) __attribute__((always_inline)) {
    constexpr int u = decltype(uc)::value;
    put_stage(Ic<(u + 1) % S>{});
    static_for<0, KS - 1>([&](auto kc) __attribute__((always_inline)) { slice(uc, kc, sumc); });
    if constexpr (C::ANY) __syncthreads();
    else asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(PENDING) : "memory");
    slice(uc, Ic<KS - 1>{}, sumc);
    advance();
  };
  static_for<0, S - 1>([&](auto uc) {
#pragma unroll
    for (int q = 0; q < L; ++q) load(uc, q);
    advance();
  });
  if constexpr (C::ANY) {
#pragma unroll
    for (int q = 0; q < L; ++q) load(Ic<1>{}, q);
    advance();
    put_stage(Ic<0>{});
#pragma unroll
    for (int q = 0; q < L; ++q) load(Ic<0>{}, q);
    advance();
    __syncthreads();
  } else {
    asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"((S - 2) * L) : "memory");
  }
#pragma unroll
  for (int r = 0; r < TM + TN; ++r) rd(Ic<0>{}, r, 0, 0);
  // (a loop of its own for the blocks that add up fragments: the branch in its slices would cost every
  // 256 x 256 tile 5%)
  auto walk = [&](auto sumc) __attribute__((always_inline)) {
    int kt = 0;
    for (; kt + S <= nk; kt += S) static_for<0, S>([&](auto uc) { step(uc, sumc); });
    static_for<0, S - 1>([&](auto uc) {
      if (kt + decltype(uc)::value < nk) step(uc, sumc);
    });
  };
  if constexpr (KIND == kGemmWgrad) {
    if (sums) walk(Ic<1>{});
    else walk(Ic<0>{});
  } else {
    walk(Ic<0>{});
  }
  // the loads issued past the last step land before the stages become staging space
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");

  // ---- epilogue: a wave stages 32 rows x OW columns of its sums as fp32 in LDS of its own and
  // takes them out again as rows
  const int ws = wave / C::WPS;
  unsigned char* mine = ws == 0 ? st0 : ws == 1 ? st1 : ws == 2 ? st2 : st3;
  float* out = reinterpret_cast<float*>(mine + (wave % C::WPS) * C::OUT_BYTES);
  const int l32 = lane & 31, half = lane >> 5;
  // accumulators of strip s (rows first, then columns) into the wave's LDS
  auto put = [&](auto sc) __attribute__((always_inline)) {
    constexpr int i = decltype(sc)::value % TM, js = decltype(sc)::value / TM * JS;
#pragma unroll
    for (int j = 0; j < JS; ++j)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const f32x16& x = acc[i][js + j];
        *reinterpret_cast<f32x4*>(out + l32 * C::OLD + j * 32 + 8 * g + 4 * half) =
            f32x4{x[4 * g], x[4 * g + 1], x[4 * g + 2], x[4 * g + 3]};
      }
    __builtin_amdgcn_wave_barrier();
  };
  // NV columns of the lane's row of pass p of the strip
  auto take = [&](int p, auto& f) __attribute__((always_inline)) {
    constexpr int NV = sizeof(f) / 4, VPR = C::OW / NV, RPP = 64 / VPR;
    const float4* at = reinterpret_cast<const float4*>(out + (p * RPP + lane / VPR) * C::OLD + lane % VPR * NV);
#pragma unroll
    for (int i = 0; i < NV / 4; ++i) {
      const float4 v = at[i];
      f[4 * i] = v.x;
      f[4 * i + 1] = v.y;
      f[4 * i + 2] = v.z;
      f[4 * i + 3] = v.w;
    }
  };
  if constexpr (KIND == kGemmWgrad) {
    if (sums && wn < TM) {
      float* db = (a.splits > 1 ? a.db_part + split * a.m : a.db) + m0;
      const float s = rowsum + __shfl_xor(rowsum, 32);  // (the halves hold different k)
      const int r = (wm * TM + wn) * 32 + l32;
      if (half == 0 && r < rows) db[r] = a.splits == 1 && a.e.accumulate ? db[r] + s : s;
    }
  }
  if (a.splits > 1) {
    constexpr int RPP = 256 / C::OW;
    float* part = a.part + ((int64_t)split * a.m + m0) * a.ldp + n0;
    static_for<0, STRIPS>([&](auto sc) __attribute__((always_inline)) {
      constexpr int s = decltype(sc)::value;
      put(sc);
      const int c = col_of(s, 4);
#pragma unroll
      for (int p = 0; p < 32 / RPP; ++p) {
        const int r = row_of(s, 4) + p * RPP;
        float f[4];
        take(p, f);
        // (the partials' rows are padded to whole lines)
        if (r < rows && c < cols) store_cols<4, kStoreStream>(part + (int64_t)r * a.ldp + c, f);
      }
      __builtin_amdgcn_wave_barrier();
    });
    return;
  }
  by_type([&](auto nvc) __attribute__((always_inline)) {
    constexpr int NV = decltype(nvc)::value, RPP = 64 * NV / C::OW;
    // the next strip's auxiliary loads are in flight while a strip is finished
    auto vectors = [&](auto howc) __attribute__((always_inline)) {
      static_for<0, STRIPS>([&](auto sc) __attribute__((always_inline)) {
        constexpr int s = decltype(sc)::value;
        const int c = col_of(s, NV);
        if constexpr (s + ahead(NV) < STRIPS) fetch(nvc, Ic<s + ahead(NV)>{});
        put(sc);
#pragma unroll
        for (int p = 0; p < 32 / RPP; ++p) {
          const int r = row_of(s, NV) + p * RPP;
          float f[NV];
          take(p, f);
          if (r < rows && c < cols)
            finish_cols<KIND, NV, decltype(howc)::value>(a.e, ep, r, c, f, bias, x[s % buffers(NV) * (32 / RPP) + p]);
        }
        __builtin_amdgcn_wave_barrier();
      });
    };
    if (a.e.vec && ep.stream) {
      vectors(Ic<kStoreStream>{});
    } else if (a.e.vec) {
      vectors(Ic<kStoreVec>{});
    } else {
      static_for<0, STRIPS>([&](auto sc) __attribute__((always_inline)) {
        constexpr int s = decltype(sc)::value;
        const int c = col_of(s, NV);
        put(sc);
#pragma unroll 1
        for (int p = 0; p < 32 / RPP; ++p) {
          const int r = row_of(s, NV) + p * RPP;
          float f[NV];
          take(p, f);
          if (r < rows) finish_any<KIND, NV>(a.e, ep, r, c, cols - c, f, bias);
        }
        __builtin_amdgcn_wave_barrier();
      });
    }
  });
}

// the sums of the reduction ranges, added in order (eight ranges' loads in flight), then the epilogue
template <int KIND, bool VEC>
__global__ __launch_bounds__(256) void gemm_finish_kernel(GemmArgs a) {
  const int per_row = (a.n + 3) / 4;
  const int64_t total = a.m * per_row, step = a.m * a.ldp;
  for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < total + (KIND == kGemmWgrad && a.db != nullptr ? a.m : 0);
       i += gridDim.x * 256ll) {
    if (KIND == kGemmWgrad && i >= total) {  // the bias gradient's ranges
      float t = 0.f;
      for (int s = 0; s < a.splits; ++s) t += a.db_part[s * a.m + i - total];
      a.db[i - total] = a.e.accumulate ? a.db[i - total] + t : t;
      continue;
    }
    const int64_t row = i / per_row;
    const int col = (int)(i - row * per_row) * 4;
    float f[4] = {}, b[4];
    const float* p = a.part + row * a.ldp + col;
    auto add = [&](auto countc) __attribute__((always_inline)) {
      constexpr int COUNT = decltype(countc)::value;
      float v[COUNT][4];
#pragma unroll
      for (int s = 0; s < COUNT; ++s) load_cols<4>(p + s * step, v[s]);
#pragma unroll
      for (int s = 0; s < COUNT; ++s)
#pragma unroll
        for (int e = 0; e < 4; ++e) f[e] += v[s][e];
      p += COUNT * step;
    };
    int s = 0;
    for (; s + 8 <= a.splits; s += 8) add(Ic<8>{});
    for (; s + 2 <= a.splits; s += 2) add(Ic<2>{});
    if (s < a.splits) add(Ic<1>{});
    const EpiloguePtr ep = epilogue_at<KIND>(a.e, row, col);
    load_bias<KIND, 4>(a.e, col, a.n, b);
    if constexpr (VEC) {
      Aux x;
      load_aux<4>(ep, 0, 0, x);
      finish_cols<KIND, 4>(a.e, ep, 0, 0, f, b, x);
    } else {
      finish_any<KIND, 4>(a.e, ep, 0, 0, a.n - col, f, b);
    }
  }
}

// Operands whose rows are not whole aligned vectors, copied with rows padded by zeros; both of a
// product in one launch, a thread a vector.
__global__ __launch_bounds__(256) void gemm_pack_kernel(GemmPack a, GemmPack b) {
  const int64_t na = a.rows * (a.ldd / 8), total = na + b.rows * (b.ldd / 8);
  for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < total; i += gridDim.x * 256ll) {
    const GemmPack& o = i < na ? a : b;
    const int64_t j = i < na ? i : i - na;
    const int per_row = (int)(o.ldd / 8);
    const int64_t row = j / per_row;
    const int c = (int)(j - row * per_row) * 8;
    const bf16_t* s = o.src + row * o.lds + c;
    uint4 v;
    if (c + 8 <= o.cols) {
      v = load16<false>(s);
    } else {
      uint32_t h[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) h[e] = c + e < o.cols ? s[e] : 0;
      v = make_uint4(h[0] | h[1] << 16, h[2] | h[3] << 16, h[4] | h[5] << 16, h[6] | h[7] << 16);
    }
    *reinterpret_cast<uint4*>(o.dst + row * o.ldd + c) = v;
  }
}

// Bias gradient: a block of 16 waves sums a range of rows of 512 columns, a wave every sixteenth row of
// it with 8 columns per lane and four rows' loads in flight; column_sum_kernel adds the ranges' sums.
template <bool VEC>
__global__ __launch_bounds__(1024) void colsum_kernel(const bf16_t* src, int64_t lds, int64_t rows, int cols,
                                                      int64_t rows_per, float* part) {
  __shared__ float s_sum[16][512];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = blockIdx.x * 512 + lane * 8;
  const int64_t r0 = blockIdx.y * rows_per, r1 = r0 + rows_per < rows ? r0 + rows_per : rows;
  float s[8] = {};
  auto add = [&](const uint4& v) __attribute__((always_inline)) {
    float f[8];
    unpack8(v, f);
#pragma unroll
    for (int e = 0; e < 8; ++e) s[e] += f[e];
  };
  auto get = [&](int64_t r) __attribute__((always_inline)) -> uint4 {
    const bf16_t* p = src + r * lds + c;
    if (VEC || c + 8 <= cols) return load16<VEC>(p);
    uint32_t h[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) h[e] = c + e < cols ? p[e] : 0;
    return make_uint4(h[0] | h[1] << 16, h[2] | h[3] << 16, h[4] | h[5] << 16, h[6] | h[7] << 16);
  };
  if (c < cols) {
    int64_t r = r0 + wave;
    for (; r + 48 < r1; r += 64) {
      const uint4 v0 = get(r), v1 = get(r + 16), v2 = get(r + 32), v3 = get(r + 48);
      add(v0);
      add(v1);
      add(v2);
      add(v3);
    }
    for (; r < r1; r += 16) add(get(r));
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) s_sum[wave][lane * 8 + e] = s[e];
  __syncthreads();
  const int i = threadIdx.x, col = blockIdx.x * 512 + i;
  if (i < 512 && col < cols) {
    float t = s_sum[0][i];
#pragma unroll
    for (int w = 1; w < 16; ++w) t += s_sum[w][i];
    part[(int64_t)blockIdx.y * cols + col] = t;
  }
}

// The sums of the columns of a [rows][ld] matrix of partials, in a fixed order: the first cols0 go to
// out0, the others to out1 (each may be nullptr).  A block takes CW columns; its waves' lanes in groups
// of CW take every (1024 / CW)th row, eight loads in flight.  16 columns a block spread few columns
// over more CUs (1024 x 384 partials 4.9 us with 64).
template <int CW>
__global__ __launch_bounds__(1024) void column_sum_kernel(const float* part, int rows, int64_t ld, int cols, int cols0,
                                                          float* out0, float* out1, int accumulate) {
  constexpr int G = 1024 / CW;
  __shared__ float s_sum[G][CW + 1];
  const int i = threadIdx.x % CW, g = threadIdx.x / CW, c = blockIdx.x * CW + i;
  float s = 0.f;
  if (c < cols) {
    int r = g;
    for (; r + 7 * G < rows; r += 8 * G) {
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = part[(int64_t)(r + G * e) * ld + c];
#pragma unroll
      for (int e = 0; e < 8; ++e) s += v[e];
    }
    for (; r < rows; r += G) s += part[(int64_t)r * ld + c];
  }
  s_sum[g][i] = s;
  __syncthreads();
  // 16 groups at a time, then the 16 (or fewer) sums of those
  if (G > 16 && g < 16) {
    s = s_sum[g][i];
#pragma unroll
    for (int k = 1; k < G / 16; ++k) s += s_sum[g + 16 * k][i];
  }
  if (G > 16) {
    __syncthreads();
    if (g < 16) s_sum[g][i] = s;
    __syncthreads();
  }
  if (g == 0 && c < cols) {
    s = s_sum[0][i];
#pragma unroll
    for (int w = 1; w < 16; ++w) s += s_sum[w][i];
    float* out = c < cols0 ? out0 : out1;
    if (out != nullptr) {
      out += c < cols0 ? c : c - cols0;
      *out = accumulate ? *out + s : s;
    }
  }
}

// ranges of rows: enough blocks for the chip
int64_t colsum_rows_per(int64_t rows, int cols) {
  const int64_t blocks = (cols + 511) / 512;
  const int64_t ranges = std::max<int64_t>(1, std::min<int64_t>((2048 + blocks - 1) / blocks, rows / 64));
  return (rows + ranges - 1) / ranges;
}

__global__ __launch_bounds__(256) void fill_zero_kernel(float* p, int64_t n) {
  for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < n; i += gridDim.x * 256ll) p[i] = 0.f;
}

unsigned grid_for(int64_t threads) { return (unsigned)std::min<int64_t>(4096, std::max<int64_t>(1, (threads + 255) / 256)); }

// The tiles, largest first (us of each where its neighbours were measured too; m x k -> n, forward):
//   256 x 256   the least operand bytes per flop: 8192 x 4096 -> 16384 920 (128 x 256: 968, 128 x 128: 1110)
//   128 x 256   the same where 256 x 256 leaves CUs idle: 2048 x 4096 -> 4096 56.6 (75.0, 60.5)
//   128 x 128, four stages, one block to a CU: few blocks with long reductions, whose latency the
//               stages hide: 4096 x 2048 -> 1024 18.9 (128 x 256: 23.3, two stages: 25.1)
//   128 x 128, two stages, two blocks to a CU: short reductions, where one block's epilogue runs
//               beside the other's products: 102400 x 192 -> 768 59.9 (four stages: 75.8)
//   64 x 64     little work: 1024 x 512 -> 768 4.8 (128 x 128: 6.5); 64 x 1024 -> 1024 5.7 (8.3)
//   64 x 64 of any rows, through registers: 334 x 441 -> 329 7.7 (copies and the above: 8.1); larger
//               products of odd rows are faster from copies: 1531 x 1003 -> 2049 23.2 (29.8)
// Split reductions add blocks where there are few: 24 x 8192 -> 4096 16 us on 64 tiles of 4 ranges.
using T256 = Tile<256, 256, 32, 4, 2, 4>;
using T128W = Tile<128, 256, 64, 3, 2, 4>;
using T128D = Tile<128, 128, 64, 4, 2, 4>;
using T128 = Tile<128, 128, 64, 2, 2, 4>;
using T64 = Tile<64, 64, 64, 4, 2, 2>;
using T64Any = Tile<64, 64, 64, 2, 2, 2, true>;

enum { kTile256, kTile128W, kTile128D, kTile128, kTile64, kTile64Any, kTileRows };

template <int KIND, typename C>
hipError_t launch_tile(const GemmArgs& a, hipStream_t s) {
  NUMBAT_LAUNCH((gemm_kernel<KIND, C>), dim3((unsigned)(a.tiles_m * a.tiles_n * a.splits)), dim3(C::NW * 64), 0, s, a);
  return hipGetLastError();
}

template <int KIND>
hipError_t launch_kind(const GemmArgs& a, int tile, hipStream_t s) {
  trace_begin(KC_LINEAR);
  hipError_t e = tile == kTile256    ? launch_tile<KIND, T256>(a, s)
                 : tile == kTile128W ? launch_tile<KIND, T128W>(a, s)
                 : tile == kTile128D ? launch_tile<KIND, T128D>(a, s)
                 : tile == kTile128  ? launch_tile<KIND, T128>(a, s)
                 : tile == kTile64   ? launch_tile<KIND, T64>(a, s)
                                     : launch_tile<KIND, T64Any>(a, s);
  trace_end(KC_LINEAR);
  if (e != hipSuccess || a.splits == 1) return e;
  trace_begin(KC_LINEAR_FINISH);
  const dim3 grid(grid_for(a.m * ((a.n + 3) / 4) + (a.db != nullptr ? a.m : 0)));
  if (a.e.vec) NUMBAT_LAUNCH((gemm_finish_kernel<KIND, true>), grid, dim3(256), 0, s, a);
  else NUMBAT_LAUNCH((gemm_finish_kernel<KIND, false>), grid, dim3(256), 0, s, a);
  trace_end(KC_LINEAR_FINISH);
  return hipGetLastError();
}

struct TileSize {
  int m, n;
};
constexpr TileSize kTiles[] = {{T256::BM, T256::BN}, {T128W::BM, T128W::BN}, {T128D::BM, T128D::BN}, {T128::BM, T128::BN}, {T64::BM, T64::BN}, {T64Any::BM, T64Any::BN}};
int64_t tile_count(int tile, int64_t m, int n) {
  const TileSize t = kTiles[tile];
  return ((m + t.m - 1) / t.m) * ((n + t.n - 1) / t.n);
}

// What a product takes on a tile, in us, as measured: the blocks that fall to one of the 256 CUs (one,
// two or four at a time), each a fixed part (first loads, epilogue: out_bytes for each element of C)
// and a part per k.
double tile_time(GemmKind kind, int tile, int64_t blocks, int64_t k, int out_bytes) {
  // small tiles of operands that run across the reduction: twice the LDS reads, shorter rows
  const double across = kind == kGemmFwd ? 1.0 : kind == kGemmDgrad ? 1.35 : tile == kTile64Any ? 2.0 : 1.4;
  const double b = (double)blocks, per_cu = std::ceil(b / 256);
  switch (tile) {
    case kTile256: return per_cu * (1.5 + 2.75 * out_bytes + 0.0255 * k);
    case kTile128W: return per_cu * (1.4 + 1.5 * out_bytes + (blocks <= 256 ? 0.012 : 0.0135) * k);
    case kTile128D: return per_cu * (1.2 + 0.65 * out_bytes + 0.0079 * k);
    case kTile128:
      return std::floor(per_cu / 2) * (2.5 + 0.75 * out_bytes + 0.015 * k) + std::fmod(per_cu, 2) * (3.0 + 0.0115 * k);
    case kTile64Any:
      return std::max(1.0, b / 1024 + 0.25) * (2.0 + 0.4 * out_bytes + (0.009 * across + 0.002 * std::min(4.0, b / 256)) * k);
    default:
      return blocks <= 256 ? 2.5 + 0.0031 * across * k
                           : std::max(1.0, b / 512 + 0.25) * (1.7 + 0.4 * out_bytes + 0.0058 * across * k);
  }
}

// and on the kernel for few rows: a block streams 16 rows of w past its rows of x; odd rows (unaligned
// loads) make x the longer part (us there and on the best tile; m x k -> n): 16 x 2048 -> 2048 5.9 and 7.7,
// 4 x 4096 -> 4096 8.4 and 10.7, 16 x 8192 -> 1024 16.4 and 11.9, 16 x 4096 -> 16384 37 and 31,
// 16 x 5441 -> 345 36 and 12
double rows_time(int64_t m, int n, int64_t k, bool odd) {
  const double per_cu = std::ceil(n / 4096.0);
  return 3.0 + per_cu * k * (odd ? 2.5 + 0.22 * m : 1.0 + 0.04 * m + 0.3 * std::min(1.0, n / 4096.0)) / 1000;
}

// and the second launch that adds the sums of the splits
double finish_time(int splits, int64_t m, int n) { return splits == 1 ? 0.0 : 4.0 + 0.1 * splits + (double)splits * m * n * 8 / 6e6; }

}  // namespace

GemmPlan gemm_pick(GemmKind kind, int64_t m, int n, int64_t k, int out_bytes, double pack_bytes) {
  GemmPlan p{kTile64, 1, 0};
  const int64_t steps = (k + 63) / 64;
  double best = 1e30;
  for (int tile = kTile256; tile <= (pack_bytes > 0 ? kTile64Any : kTile64); ++tile) {
    const int64_t tiles = tile_count(tile, m, n);
    const double pack = pack_bytes > 0 && tile != kTile64Any ? 3.5 + 2 * pack_bytes / 4e6 : 0.0;
    for (int s : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64}) {
      if (s > 1 && (steps / s < 4 || tiles * s > 1024)) break;
      const int64_t kps = (steps + s - 1) / s;
      const double t = tile_time(kind, tile, tiles * s, kps * 64, s > 1 ? 4 : out_bytes) + finish_time(s, m, n) + pack;
      if (t < best) {
        best = t;
        p.tile = tile;
        p.splits = (int)((steps + kps - 1) / kps);
        p.k_per_split = kps * 64;
      }
    }
  }
  // no tile is faster than w's bytes come
  if (kind == kGemmFwd && m <= kLinearRows && rows_time(m, n, k, pack_bytes > 0) <= std::max(best, 2.5 + 2.0 * n * k / 5e6))
    return GemmPlan{kTileRows, 1, k};
  return p;
}

// a launch takes fewer than 2^32 threads
bool gemm_fits(const GemmPlan& p, int64_t m, int n) {
  return p.tile == kTileRows || tile_count(p.tile, m, n) * p.splits < (1ll << 32) / (p.tile >= kTile64 ? 256 : 512);
}

bool gemm_any_rows(const GemmPlan& p) { return p.tile == kTileRows || p.tile == kTile64Any; }

// Adding up fragments slows a long block of 256 columns by a tenth, and a block's time grows with its
// range, where a pass over A of its own takes about 10 us: 20000 x 4096 x 2048's gradients 302 us with
// the pass and 328 without, 1000 x 2048 x 2048's 21 and 18.  Narrower tiles never lose by it (20000 x
// 4096 x 2048 on 128 x 128: 368 and 346).
bool gemm_sums_rows(const GemmPlan& p) { return kTiles[p.tile].n < 256 || p.k_per_split <= 4096; }

size_t gemm_part_bytes(const GemmPlan& p, int64_t m, int n) {
  return p.splits > 1 ? (size_t)p.splits * (size_t)m * ((n + 31) / 32 * 32) * sizeof(float) : 0;
}

hipError_t gemm_launch(GemmKind kind, GemmArgs a, const GemmPlan& p, hipStream_t s) {
  if (p.tile == kTileRows) return linear_rows_launch(a, s);
  const TileSize t = kTiles[p.tile];
  a.tiles_m = (int32_t)((a.m + t.m - 1) / t.m);
  a.tiles_n = (a.n + t.n - 1) / t.n;
  a.splits = p.splits;
  a.div_tiles = make_fastdiv((uint32_t)a.tiles_m * (uint32_t)a.tiles_n);
  a.div_group = make_fastdiv(8u * (uint32_t)a.tiles_n);
  a.div_last = make_fastdiv(a.tiles_m % 8 ? a.tiles_m % 8 : 8);
  a.k_per_split = p.k_per_split;
  a.ldp = (a.n + 31) / 32 * 32;
  return kind == kGemmFwd     ? launch_kind<kGemmFwd>(a, p.tile, s)
         : kind == kGemmDgrad ? launch_kind<kGemmDgrad>(a, p.tile, s)
                              : launch_kind<kGemmWgrad>(a, p.tile, s);
}

hipError_t gemm_pack_launch(const GemmPack& a, const GemmPack& b, hipStream_t s) {
  trace_begin(KC_LINEAR_PACK);
  NUMBAT_LAUNCH(gemm_pack_kernel, dim3(grid_for(a.rows * (a.ldd / 8) + b.rows * (b.ldd / 8))), dim3(256), 0, s, a, b);
  trace_end(KC_LINEAR_PACK);
  return hipGetLastError();
}

size_t colsum_part_bytes(int64_t rows, int32_t cols) {
  const int64_t per = colsum_rows_per(rows, cols);
  return (size_t)((rows + per - 1) / per) * cols * sizeof(float);
}

hipError_t colsum_launch(const bf16_t* src, int64_t lds, int64_t rows, int32_t cols, float* part, float* out,
                         int accumulate, hipStream_t s) {
  const int64_t per = colsum_rows_per(rows, cols);
  const unsigned ranges = (unsigned)((rows + per - 1) / per);
  const dim3 grid((unsigned)((cols + 511) / 512), ranges);
  trace_begin(KC_LINEAR_BIAS_GRAD);
  if (cols % 8 == 0 && lds % 8 == 0) NUMBAT_LAUNCH(colsum_kernel<true>, grid, dim3(1024), 0, s, src, lds, rows, cols, per, part);
  else NUMBAT_LAUNCH(colsum_kernel<false>, grid, dim3(1024), 0, s, src, lds, rows, cols, per, part);
  const hipError_t e = hipGetLastError();
  if (e == hipSuccess) column_sum_launch(part, (int)ranges, cols, cols, cols, out, nullptr, accumulate, s);
  trace_end(KC_LINEAR_BIAS_GRAD);
  return e != hipSuccess ? e : hipGetLastError();
}

void column_sum_launch(const float* part, int rows, int64_t ld, int cols, int cols0, float* out0, float* out1,
                       int accumulate, hipStream_t s) {
  if (cols <= 4096) {
    NUMBAT_LAUNCH(column_sum_kernel<16>, dim3((unsigned)((cols + 15) / 16)), dim3(1024), 0, s, part, rows, ld, cols, cols0,
                  out0, out1, accumulate);
  } else {
    NUMBAT_LAUNCH(column_sum_kernel<64>, dim3((unsigned)((cols + 63) / 64)), dim3(1024), 0, s, part, rows, ld, cols, cols0,
                  out0, out1, accumulate);
  }
}

hipError_t fill_zero_launch(float* p, int64_t n, hipStream_t s) {
  trace_begin(KC_LINEAR_FINISH);
  NUMBAT_LAUNCH(fill_zero_kernel, dim3(grid_for(n)), dim3(256), 0, s, p, n);
  trace_end(KC_LINEAR_FINISH);
  return hipGetLastError();
}

}  // namespace numbat
