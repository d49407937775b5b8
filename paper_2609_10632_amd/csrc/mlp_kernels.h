// Host-side launch interface of the residual MLP block's kernels: linear layers, layer norm
// and the AdamW step.
#pragma once

#include "kernels.h"

namespace numbat {

// Kernel classes of numbat_mlp.h's functions for the launch timing, numbered apart from the others.
// (Here and not with those: the committed HBM traffic of the convolutions is tied to a hash of the
// convolutions' sources, kernels.h among them.)
enum MlpKernelClass {
  KC_MLP_FIRST = 64,
  KC_LINEAR = KC_MLP_FIRST,  // linear layers: matrix products with their epilogues
  KC_LINEAR_PACK,       // linear layers: operands with odd rows, padded
  KC_LINEAR_FINISH,     // linear layers: sums of reduction ranges
  KC_LINEAR_BIAS_GRAD,  // linear layers: bias gradient
  KC_LN_FWD,            // layer norm forward
  KC_LN_BWD,            // layer norm backward
  KC_LN_BWD_FINISH,     // layer norm backward: gain and shift gradients
  KC_ADAMW_NORM,        // AdamW: squared-norm partials of the gradients
  KC_ADAMW,             // AdamW: update, and the values of 8-bit moments
  KC_MLP_END
};

// ---------------------------------------------------------------------------
// Linear layers.  One matrix product C[m][n] = sum_k A(m, k) B(n, k) in three orientations:
//   forward          A = x  [m][k],  B = w [n][k]    (both run along the reduction)
//   data gradient    A = dy [m][k'], B = w [k'][n']  (B runs across the reduction)
//   weight gradient  A = dy [k'][m'], B = x [k'][n'] (both run across it)
enum GemmKind { kGemmFwd = 0, kGemmDgrad = 1, kGemmWgrad = 2 };

// What happens to the fp32 sums t before they are stored.
//   kGemmFwd:   z = t + bias (stored as bf16 if asked for), out = act(z) + res
//   kGemmDgrad: out = t * act'(z) [+ out]
//   kGemmWgrad: out = t [+ out], fp32
struct GemmEpilogue {
  int32_t act;
  int32_t out_f32;      // out (and res) are fp32, otherwise bf16
  int32_t accumulate;
  int32_t vec;          // every pointer and stride below allows 16-byte access, n is a multiple of 8
  const float* bias;    // [n] or nullptr
  const void* res;      // [m][n] or nullptr, out's type
  bf16_t* z;            // [m][n] or nullptr: written by the forward, read by the data gradient
  void* out;
  int64_t ldr, ldz, ldo;
};

struct GemmArgs {
  const bf16_t *a, *b;
  int64_t lda, ldb;     // elements between rows of the stored matrices, multiples of 8 (or see gemm_any_rows)
  int64_t m, k;
  int32_t n;
  int32_t tiles_m, tiles_n;
  FastDiv div_tiles, div_group, div_last;  // by the tiles, by 8 rows of them, by the last rows (set by gemm_launch)
  int32_t splits;       // reduction ranges; above 1 the sums go to part
  int64_t k_per_split;  // a multiple of the reduction step
  float* part;          // [splits][m][ldp] fp32
  int64_t ldp;
  float *db, *db_part;  // weight gradient: sums of A over the reduction [m] or nullptr, their ranges' [splits][m]
  GemmEpilogue e;
};

// tile and reduction split of a product
struct GemmPlan {
  int tile;    // instantiation id
  int splits;
  int64_t k_per_split;
};
// out_bytes: what the epilogue reads and writes for each element; pack_bytes: size of the operands that
// would have to be padded (0: none)
GemmPlan gemm_pick(GemmKind kind, int64_t m, int n, int64_t k, int out_bytes, double pack_bytes);
// whether the plan's grid is one that a launch takes
bool gemm_fits(const GemmPlan& p, int64_t m, int n);
// whether the plan's kernel takes operands whose rows start at any element
bool gemm_any_rows(const GemmPlan& p);
// whether a weight gradient's plan adds up its first operand on the way (GemmArgs::db)
bool gemm_sums_rows(const GemmPlan& p);
size_t gemm_part_bytes(const GemmPlan& p, int64_t m, int n);
// a.part holds gemm_part_bytes; every dimension is at least 1
hipError_t gemm_launch(GemmKind kind, GemmArgs a, const GemmPlan& p, hipStream_t s);

// the forward of few rows (linear_rows.hip), m at most kLinearRows
constexpr int kLinearRows = 16;
hipError_t linear_rows_launch(const GemmArgs& a, hipStream_t s);

// rows x cols of src (row stride lds) into dst with row stride ldd = cols rounded up to 8, the
// padding zero; rows = 0 for none
struct GemmPack {
  const bf16_t* src;
  int64_t lds, rows;
  int32_t cols;
  bf16_t* dst;
  int64_t ldd;
};
hipError_t gemm_pack_launch(const GemmPack& a, const GemmPack& b, hipStream_t s);

// out[c] (+)= sum over rows of src[r][c], fp32: per-block partials, then their sum in a fixed order
size_t colsum_part_bytes(int64_t rows, int32_t cols);
hipError_t colsum_launch(const bf16_t* src, int64_t lds, int64_t rows, int32_t cols, float* part, float* out,
                         int accumulate, hipStream_t s);

// the column sums of rows x cols partials (row stride ld), in a fixed order: the first cols0 (+)= to
// out0, the others to out1 (each may be nullptr); the caller opens the timing class and reads the
// launch status
void column_sum_launch(const float* part, int rows, int64_t ld, int cols, int cols0, float* out0, float* out1,
                       int accumulate, hipStream_t s);

hipError_t fill_zero_launch(float* p, int64_t n, hipStream_t s);

// ---------------------------------------------------------------------------
// Layer norm over c features of m rows
struct LnArgs {
  int32_t c;
  int64_t m;
  float eps;
  int32_t x_f32, y_f32;  // type of x, dx, residual grad / of y, dy
  int64_t ldx, ldy, ldr, lddx;
  int32_t vec;           // rows allow 16-byte access and c is a multiple of 8
};
hipError_t ln_fwd_launch(const LnArgs& a, const void* x, const float* gamma, const float* beta, void* y, float* mean,
                         float* rstd, hipStream_t s);
size_t ln_bwd_part_bytes(const LnArgs& a);
hipError_t ln_bwd_launch(const LnArgs& a, const void* dy, const void* x, const float* mean, const float* rstd,
                         const float* gamma, const void* res, void* dx, float* dgamma, float* dbeta, int accumulate,
                         float* part, hipStream_t s);

// ---------------------------------------------------------------------------
// AdamW.  AdamTensor has the layout of numbat_adamw_tensor.
struct AdamTensor {
  float* w;
  const void* g;
  void* m;
  void* v;
  float* m_unit;
  float* v_unit;
  bf16_t* w_copy;
  int64_t n;
  int32_t group;
  int32_t g_type;  // numbat_type
};
constexpr int kAdamBlock = 256;        // elements that share the units of 8-bit moments
constexpr int kAdamMaxTensors = 1024;  // a block's threads count four tensors each
constexpr int kAdamBlocks = 1024;      // blocks of the update
constexpr int kAdamNormBlocks = 2048;  // blocks of the norm's sum, and its partials
struct AdamArgs {
  const AdamTensor* tab;
  int32_t count;
  int32_t ngroups;
  float lr[kOptMaxGroups], keep[kOptMaxGroups];  // lr / (1 - beta1^step), 1 - lr * weight decay
  float b1, omb1, b2, omb2, eps, rsqrt_bc2;      // omb = 1 - beta, rsqrt_bc2 = (1 - beta2^step)^-1/2
  float max_norm;                                // 0: no clipping
  float* total_norm;
  double* part;
};
hipError_t adamw_launch(const AdamArgs& a, int bits, hipStream_t s);
hipError_t adamw_values_launch(int64_t n, const int8_t* m, const float* m_unit, const uint8_t* v, const float* v_unit,
                               float* m_value, float* v_value, hipStream_t s);

}  // namespace numbat
