/*
 * numbat_attention.h -- C ABI of the residual attention block's operators for AMD Instinct MI355X
 * (gfx950): group norm with an activation over NHWC maps, rotary positions along one to four axes,
 * and attention over the pixels of maps or over tokens, each with its gradients.
 *
 * The functions live in the same library as those of numbat_conv.h and keep its conventions:
 * descriptors with their struct_size, status codes with thread-local detail text
 * (numbat_last_error), caller-owned memory sized by numbat_workspace_size, refusal before any
 * launch, everything enqueued on `stream`, results that are bitwise the same from run to run.
 *
 * Rows are the pixels of NHWC maps or tokens, as in numbat_mlp.h; they may be further apart than
 * they are long (a channel slice of a wider tensor, or q, k and v side by side in one matrix).
 * Strides are in elements; 0 means dense.  Pointers to matrices of bf16 or fp32 activations are
 * 16-byte aligned, other pointers aligned to their elements.  Operands may not overlap outputs
 * unless a function says so.
 */
#ifndef NUMBAT_ATTENTION_H
#define NUMBAT_ATTENTION_H

#include "numbat_mlp.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Kernel classes of numbat_kernel_class_name and numbat_timing_read for these functions' kernels. */
#define NUMBAT_ATTENTION_KERNEL_CLASS_FIRST 96
#define NUMBAT_ATTENTION_KERNEL_CLASS_COUNT 10

/* Group norm over n images of m rows (pixels) of c channels, in `groups` groups of neighbouring channels. */
typedef struct {
  uint32_t struct_size;  /* = sizeof(numbat_group_norm_problem) */
  int32_t n;             /* images */
  int64_t m;             /* rows of each image; image i starts at row i m */
  int32_t c;             /* channels, at most 65536 */
  int32_t groups;        /* divides c */
  int32_t act;           /* numbat_act, applied to the norm's result */
  float eps;             /* added to the variance inside the square root */
  int32_t x_type;        /* numbat_type of x and dx */
  int32_t y_type;        /* numbat_type of y and dy */
  int64_t x_row_stride;  /* x; at most 2^21, like the others */
  int64_t y_row_stride;  /* y and dy */
  int64_t r_row_stride;  /* residual_grad */
  int64_t dx_row_stride; /* dx */
} numbat_group_norm_problem;

typedef enum {
  NUMBAT_ROTARY_HALVES = 0, /* pair j is features j and j + P, P the number of pairs */
  NUMBAT_ROTARY_PAIRS = 1   /* pair j is features 2 j and 2 j + 1 */
} numbat_rotary_layout;

/* Rotary positions of m rows of `heads` heads of d features each, the heads of a row next to each other. */
typedef struct {
  uint32_t struct_size;  /* = sizeof(numbat_rotary_problem) */
  int32_t heads, d;      /* heads * d at most 2^21 */
  int32_t axes;          /* 1 .. 4 */
  int64_t m;             /* rows */
  int32_t pairs[4];      /* pairs that each axis turns, at least 1 for each of the axes and 0 past them; P,
                          * their sum, is at most 256 and 2 P at most d; features from 2 P on pass unchanged */
  int32_t extents[4];    /* grid of the rows where no positions are given, the last axis the fastest; at least 1
                          * for each of the axes (not read otherwise) */
  int32_t layout;        /* numbat_rotary_layout */
  int32_t shared;        /* 0: each axis has its own frequencies; 1: one ladder runs through all pairs */
  int32_t inverse;       /* 1: turn back, which is also the gradient */
  int32_t type;          /* numbat_type of x and y */
  double base;           /* above 1, at most 1e30 */
  int64_t x_row_stride;
  int64_t y_row_stride;
} numbat_rotary_problem;

/* Attention of `batch` sequences (images): queries of row r of sequence b are row b q_len + r of q, and so on. */
typedef struct {
  uint32_t struct_size;    /* = sizeof(numbat_attention_problem) */
  int32_t batch;           /* sequences, at most 65535 */
  int32_t q_len, kv_len;   /* rows of each sequence: queries, keys and values */
  int32_t q_heads;         /* heads of q and y */
  int32_t kv_heads;        /* heads of k and v; divides q_heads: head h of q reads head h / (q_heads / kv_heads) */
  int32_t d;               /* features of a head: a multiple of 8, at most 128 */
  int32_t causal;          /* 1: query i sees keys j <= i + (keys - queries), each sequence's own numbers */
  float scale;             /* of the scores, above 0 and at most 1e38; what q_i k_j is has to be finite in fp32 */
  int32_t reserved;        /* 0 */
  int64_t q_row_stride;    /* q and dq; a multiple of 8, like the others */
  int64_t k_row_stride;    /* k and dk */
  int64_t v_row_stride;    /* v and dv */
  int64_t y_row_stride;    /* y and dy */
} numbat_attention_problem;

/* Group norm and activation, the statistics over the rows and channels of each image's group:
 *   mean = sum x / N,  var = sum (x - mean)^2 / N,  rstd = 1 / sqrt(var + eps),  N = m c / groups
 *   y = act(gamma (x - mean) rstd + beta)
 * gamma, beta: fp32 [c], NULL for 1 and 0; mean, rstd: fp32 [n][groups], each NULL where it is not
 * wanted (the backward reads both).  y may be x's buffer if types and strides agree
 * (NUMBAT_ERR_BAD_DESC otherwise).  Activations as in numbat_linear_fwd.
 * ws: numbat_workspace_size(NUMBAT_OP_GROUP_NORM_FWD), which may be 0. */
numbat_status numbat_group_norm_fwd(const numbat_group_norm_problem* p, const void* x, const float* gamma,
                                    const float* beta, void* y, float* mean, float* rstd, void* ws, size_t ws_bytes,
                                    void* stream);

/* Backward of group norm and activation, with xh = (x - mean) rstd, t = gamma xh + beta, dt = dy act'(t)
 * and h = gamma dt:
 *   dx = rstd (h - sum h / N - xh sum(h xh) / N) + residual_grad   (sums over the image's group)
 *   dgamma = sum_rows dt xh,  dbeta = sum_rows dt                   (fp32 [c], over all images; accumulate: added)
 * gamma, beta NULL: 1 and 0.  residual_grad [n m][c] of x's type or NULL: the gradient that reaches x around the
 * norm.  Each of dx, dgamma, dbeta may be NULL where it is not wanted; the workspace is required all the
 * same.  dx may be the buffer of dy, of x or of residual_grad, if types and strides agree
 * (NUMBAT_ERR_BAD_DESC otherwise).
 * ws: numbat_workspace_size(NUMBAT_OP_GROUP_NORM_BWD). */
numbat_status numbat_group_norm_bwd(const numbat_group_norm_problem* p, const void* dy, const void* x,
                                    const float* mean, const float* rstd, const float* gamma, const float* beta,
                                    const void* residual_grad, void* dx, float* dgamma, float* dbeta, int accumulate,
                                    void* ws, size_t ws_bytes, void* stream);

/* Turns pair (a, b) number j of every head by the angle of its axis' position:
 *   y_a = a cos(t) - b sin(t),  y_b = b cos(t) + a sin(t),  t = position * base^-e   (inverse: -t)
 * Pairs belong to the axes in order.  For pair i of an axis of p pairs, e = i / p; with `shared`, e = j / P
 * for pair j of all P.  positions: int32 [m][axes], or NULL: row r lies at the grid point r mod (product of
 * the extents) of the extents (an image's pixels: extents = height, width).  Angles are formed in 64 bits.
 * y may be x's buffer if strides agree (NUMBAT_ERR_BAD_DESC otherwise); features beyond the heads of a row
 * (v's beside q and k) are neither read nor written. */
numbat_status numbat_rotary(const numbat_rotary_problem* p, const void* x, const int32_t* positions, void* y,
                            void* stream);

/* Attention:  s_ij = scale q_i k_j,  p_ij = exp(s_ij - lse_i),  y_i = sum_j p_ij v_j,  lse_i = log sum_j exp s_ij
 * over the keys j that query i sees.  q, k, v, y: bf16.  q_lengths, kv_lengths: int32 [batch] on the device, or
 * NULL: the queries and keys of each sequence that count (taken into 0 .. q_len and 0 .. kv_len); rows of k and v
 * behind them are not read.  y is zero, and lse minus infinity, for queries behind a sequence's length and for
 * queries that see no key.  lse: fp32 [batch][q_heads][q_len] or NULL (the backward reads it).
 * Scores, their exponentials' sums and the sums of products are fp32; the weights exp(s - max) are rounded to bf16
 * for their product with v.  The value of a key that only some queries of a tile see (causal) has to be
 * finite for those that do not: what is no number there is multiplied by a weight of zero and reaches queries up to
 * 127 rows before the key.
 * y or lse at the address of an operand or of each other: NUMBAT_ERR_BAD_DESC.
 * ws: numbat_workspace_size(NUMBAT_OP_ATTENTION_FWD), which may be 0. */
numbat_status numbat_attention_fwd(const numbat_attention_problem* p, const void* q, const void* k, const void* v,
                                   const int32_t* q_lengths, const int32_t* kv_lengths, void* y, float* lse, void* ws,
                                   size_t ws_bytes, void* stream);

/* Backward of attention, with y and lse of the forward, P = exp(s - lse) and delta_i = dy_i y_i:
 *   dv_j = sum_i P_ij dy_i,  ds_ij = P_ij (dy_i v_j - delta_i),  dq_i = scale sum_j ds_ij k_j,
 *   dk_j = scale sum_i ds_ij q_i          (sums over the heads of q that share a head of k and v)
 * dq, dk, dv: bf16, with the strides of q, k and v; zero behind the sequences' lengths, where q, k, v, y, dy and
 * lse are not read.  P and ds are rounded to bf16 for their products, sums are fp32.  P comes from lse as fp32 holds
 * it: its exponent is off by up to 2^-21 |lse|, so that P is off by as much as bf16's rounding where lse is 8192 and
 * by a factor of 1.6 where it is 10^6.  The forward has no such bound.
 * Queries that see no key (causal, more queries than keys) are not taken in, whatever they hold.  Of the others q, k, v
 * and dy have to be finite as in the forward: between a query and a key of the same tile that it does not see (causal;
 * up to 128 rows apart) what is no number is multiplied by zero and reaches the gradients of both.
 * dq, dk or dv at the address of an operand or of each other: NUMBAT_ERR_BAD_DESC (dk and dv are formed from q and dy
 * after dq is written).
 * ws: numbat_workspace_size(NUMBAT_OP_ATTENTION_BWD). */
numbat_status numbat_attention_bwd(const numbat_attention_problem* p, const void* dy, const void* q, const void* k,
                                   const void* v, const void* y, const float* lse, const int32_t* q_lengths,
                                   const int32_t* kv_lengths, void* dq, void* dk, void* dv, void* ws, size_t ws_bytes,
                                   void* stream);

#ifdef __cplusplus
}
#endif

#endif /* NUMBAT_ATTENTION_H */
