// The forward of a linear layer for few rows (one token, a decode batch) on gfx950:
//   y[m][n] = epilogue(sum_k x[m][k] w[n][k]),  m at most 16.
// Bound by the bytes of w, which every launch reads once (one row of 2048 -> 8192 in 8.0 us: 34 MB at
// 4.2 TB/s with the launch in it, where a large copy moves 5.1 TB/s).  A block takes 16 rows of w and its waves
// split the reduction, each with 4 x 2 KiB of it in flight.  Layers below 4096 outputs have fewer
// blocks than there are CUs and fall short of that (one row of 8192 -> 1024 on 64 blocks 11.1 us, 3.3
// us of bytes); the reduction is not split over blocks.  The matrix core multiplies 16 rows of w by 16 rows of x per
// instruction (a 16 x 16 x 32 product, most of it idle for one token: the arithmetic is free here).
// The reduction's order within a 64-element step is chosen for the loads: a lane takes 16
// consecutive k of its row, so a step reads whole 128-byte lines.  x comes from the L2 straight into
// registers.  The waves' sums meet in LDS and are added in wave order; the epilogue's other operands
// are loaded before the loop.  Rows may start at any element (odd lengths and strides): loads are
// then unaligned 16-byte ones, which cost a second request for some lines but no copy of w.
#include "gemm_epilogue.h"

namespace numbat {

namespace {

constexpr int kStep = 64;  // k per step

struct __attribute__((packed, aligned(2))) Unaligned {
  uint32_t u[4];
};

// 8 elements from k of a row of length n (zeros past it)
template <bool ALIGNED, bool WHOLE>
__device__ __forceinline__ u32x4 load_k(const bf16_t* row, int k, int n) {
  if (WHOLE || k + 8 <= n) {
    if constexpr (ALIGNED) return *reinterpret_cast<const u32x4*>(row + k);
    const Unaligned v = *reinterpret_cast<const Unaligned*>(row + k);
    return u32x4{v.u[0], v.u[1], v.u[2], v.u[3]};
  }
  uint32_t h[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) h[e] = k + e < n ? row[k + e] : 0;
  return u32x4{h[0] | h[1] << 16, h[2] | h[3] << 16, h[4] | h[5] << 16, h[6] | h[7] << 16};
}

template <int NW, bool ALIGNED>
__global__ __launch_bounds__(NW * 64) void linear_rows_kernel(GemmArgs a) {
  constexpr int U = 4;  // steps in flight
  __shared__ float s_sum[NW][16][17];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l16 = lane & 15, kg = (lane >> 4) * 16;
  const int n0 = blockIdx.x * 16, K = (int)a.k, M = (int)a.m;

  // this thread's output (the first 256 threads'), and what the epilogue adds to it
  const int oc = n0 + (tid & 15), orow = tid >> 4;
  const bool mine = orow < M && oc < a.n;
  float bias[1];
  Aux aux;
  load_bias<kGemmFwd, 1>(a.e, oc, a.n, bias);
  const EpiloguePtr ep = epilogue_at<kGemmFwd>(a.e, 0, n0);
  if (mine) load_aux<1>(ep, orow, tid & 15, aux);

  // (rows past the end read the last one: their sums are not stored)
  const bf16_t* wrow = a.b + (int64_t)(n0 + l16 < a.n ? n0 + l16 : a.n - 1) * a.ldb;
  const bf16_t* xrow = a.a + (int64_t)(l16 < M ? l16 : M - 1) * a.lda;
  const int per = ((K + kStep - 1) / kStep + NW - 1) / NW * kStep;
  const int kbeg = wave * per, kend = kbeg + per < K ? kbeg + per : K;
  f32x4 acc = f32x4{0.f, 0.f, 0.f, 0.f};
  u32x4 wf[U][2], xf[U][2];
  auto mma = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int h = 0; h < 2; ++h) acc = mfma16x16x32(wf[u][h], xf[u][h], acc);
  };
  auto fetch = [&](auto whole, int k) __attribute__((always_inline)) {
    constexpr bool W = decltype(whole)::value;
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int at = k + u * kStep + kg + 8 * h;
        wf[u][h] = load_k<ALIGNED, W>(wrow, at, kend);
        xf[u][h] = load_k<ALIGNED, W>(xrow, at, kend);
      }
  };
  int k = kbeg;
  for (; k + U * kStep <= kend; k += U * kStep) {
    fetch(std::true_type{}, k);
    mma();
  }
  if (k < kend) {
    fetch(std::false_type{}, k);
    mma();
  }
  // lane holds columns 4 (lane / 16) .. + 3 of row lane % 16
#pragma unroll
  for (int r = 0; r < 4; ++r) s_sum[wave][l16][4 * (lane >> 4) + r] = acc[r];
  __syncthreads();
  if (!mine) return;
  float f[1] = {s_sum[0][orow][tid & 15]};
#pragma unroll
  for (int w = 1; w < NW; ++w) f[0] += s_sum[w][orow][tid & 15];
  finish_cols<kGemmFwd, 1>(a.e, ep, orow, tid & 15, f, bias, aux);
}

template <int NW>
void launch_rows(const GemmArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)((a.n + 15) / 16)), block(NW * 64);
  if (a.lda % 8 == 0 && a.ldb % 8 == 0) NUMBAT_LAUNCH((linear_rows_kernel<NW, true>), grid, block, 0, s, a);
  else NUMBAT_LAUNCH((linear_rows_kernel<NW, false>), grid, block, 0, s, a);
}

}  // namespace

hipError_t linear_rows_launch(const GemmArgs& a, hipStream_t s) {
  trace_begin(KC_LINEAR);
  // More waves to a block hide more of w's latency where there are few blocks and their share of k is
  // long, and cost more sums (us for one row on 4, 8 and 16 waves; k -> n): 512 -> 4096 4.5, 5.4, 5.5;
  // 2048 -> 4096 5.2, 5.2, 7.7; 8192 -> 1024 13.3, 11.9, 11.1; 8192 -> 4096 14.7, 13.6, 14.7;
  // 2048 -> 16384 12.3, 14.8, 24.8.
  if (a.k < 2048 || a.n >= 8192) launch_rows<4>(a, s);
  else if (a.k < 4096 || a.n >= 4096) launch_rows<8>(a, s);
  else launch_rows<16>(a, s);
  trace_end(KC_LINEAR);
  return hipGetLastError();
}

}  // namespace numbat
