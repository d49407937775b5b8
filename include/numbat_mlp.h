/*
 * numbat_mlp.h -- C ABI of the residual MLP block's operators for AMD Instinct MI355X
 * (gfx950): linear layers with bias, activation and residual in their epilogue, layer norm,
 * and the AdamW step over many tensors, each with what training and serving need of it.
 *
 * The functions live in the same library as those of numbat_conv.h and keep its conventions:
 * descriptors with their struct_size, status codes with thread-local detail text
 * (numbat_last_error), caller-owned memory sized by numbat_workspace_size, refusal before any
 * launch, everything enqueued on `stream`, results that are bitwise the same from run to run.
 *
 * A matrix has `m` rows: the pixels of an NHWC map (an activation tensor of numbat_conv.h is
 * such a matrix, its pixel stride the row stride) or tokens.  Rows may be further apart than
 * they are long (a channel slice of a wider tensor); sizes and strides may be odd.  Pointers to
 * matrices of bf16 or fp32 activations and of weights are 16-byte aligned, other pointers
 * aligned to their elements.  m may be 0: results that sum over rows are then zeros, others
 * empty.  Operands may not overlap outputs unless a function says so.
 */
#ifndef NUMBAT_MLP_H
#define NUMBAT_MLP_H

#include "numbat_conv.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Kernel classes of numbat_kernel_class_name and numbat_timing_read for these functions' kernels. */
#define NUMBAT_MLP_KERNEL_CLASS_FIRST 64
#define NUMBAT_MLP_KERNEL_CLASS_COUNT 9

typedef enum { NUMBAT_TYPE_BF16 = 0, NUMBAT_TYPE_F32 = 1 } numbat_type;

typedef enum {
  NUMBAT_ACT_NONE = 0,
  NUMBAT_ACT_RELU = 1,
  NUMBAT_ACT_GELU = 2,      /* t Phi(t), Phi the normal distribution function (erf) */
  NUMBAT_ACT_GELU_TANH = 3, /* t/2 (1 + tanh(sqrt(2/pi) (t + 0.044715 t^3))) */
  NUMBAT_ACT_SILU = 4       /* t sigmoid(t) */
} numbat_act;

/* One linear layer: x [m][k], w [n][k] (dense, out features first), y [m][n].  n, k and row
 * strides are at most 2^21; products of more tiles than one launch takes (past 2^38 outputs, or
 * 2^30 rows of a narrow layer) are NUMBAT_ERR_UNSUPPORTED.  Strides are in elements; 0 means dense. */
typedef struct {
  uint32_t struct_size;  /* = sizeof(numbat_linear_problem) */
  int32_t n, k;          /* output and input features */
  int32_t act;           /* numbat_act; see each function for whose activation it is */
  int64_t m;             /* rows */
  int32_t y_type;        /* numbat_type of y and residual (forward); dy is bf16 */
  int32_t reserved;      /* 0 */
  int64_t x_row_stride;  /* x and dx */
  int64_t y_row_stride;  /* y and dy */
  int64_t r_row_stride;  /* residual */
  int64_t z_row_stride;  /* z: at least n in the forward, k in the data gradient (also where no z is given);
                          * the weight gradient takes either's descriptor */
} numbat_linear_problem;

/* Layer norm over the c features of each of m rows. */
typedef struct {
  uint32_t struct_size;   /* = sizeof(numbat_layer_norm_problem) */
  int32_t c;              /* features, at most 2^21 */
  int64_t m;              /* rows */
  float eps;              /* added to the variance inside the square root */
  int32_t x_type;         /* numbat_type of x, dx and residual_grad */
  int32_t y_type;         /* numbat_type of y and dy */
  int32_t reserved;       /* 0 */
  int64_t x_row_stride;   /* x */
  int64_t y_row_stride;   /* y and dy */
  int64_t r_row_stride;   /* residual_grad */
  int64_t dx_row_stride;  /* dx */
} numbat_layer_norm_problem;

/* Forward of a linear layer, everything on the fp32 sums, each output rounded once:
 *   t = x w^T + bias;  z = t;  y = act(t) + residual
 * x, w: bf16; bias: fp32 [n] or NULL; residual: [m][n] of y's type or NULL; z: bf16 [m][n] or
 * NULL (what the backward of act reads); y: y_type.  y may be the residual's buffer if their strides
 * agree (NUMBAT_ERR_BAD_DESC otherwise).
 * Activations take the hardware's reciprocal and exponential, and GELU a polynomial for erf: within
 * 2^-20 of |t|.  Relative to y, GELU's tail is off by up to 5e-4 below t = -3, 4e-3 at t = -6 and 3e-2
 * at t = -12 (y of -4e-3, -6e-9 and -2e-32).
 * ws: numbat_workspace_size(NUMBAT_OP_LINEAR_FWD), which may be 0. */
numbat_status numbat_linear_fwd(const numbat_linear_problem* p, const void* x, const void* w, const float* bias,
                                const void* residual, void* z, void* y, void* ws, size_t ws_bytes, void* stream);

/* Data gradient of a linear layer, through the activation that made its input:
 *   dx[r][c] = act'(z[r][c]) * sum_o dy[r][o] w[o][c]    (accumulate: added to dx in fp32)
 * where x = act(z), so `act` is here that of the layer before (NUMBAT_ACT_NONE: z is not read
 * and may be NULL) and z [m][k] what that layer's forward kept; dx is then the gradient with
 * respect to z.  dy: bf16 [m][n]; dx: bf16 [m][k] (x_row_stride).
 * ws: numbat_workspace_size(NUMBAT_OP_LINEAR_BWD_DATA). */
numbat_status numbat_linear_bwd_data(const numbat_linear_problem* p, const void* dy, const void* w, const void* z,
                                     void* dx, int accumulate, void* ws, size_t ws_bytes, void* stream);

/* Weight and bias gradients of a linear layer, fp32 (act plays no part):
 *   dw[o][c] = sum_r dy[r][o] x[r][c],  db[o] = sum_r dy[r][o]    (accumulate: added)
 * x, dy: bf16; dw: [n][k] dense; db: [n] or NULL.
 * ws: numbat_workspace_size(NUMBAT_OP_LINEAR_BWD_WEIGHT). */
numbat_status numbat_linear_bwd_weight(const numbat_linear_problem* p, const void* x, const void* dy, float* dw,
                                       float* db, int accumulate, void* ws, size_t ws_bytes, void* stream);

/* Layer norm:
 *   mean = sum_c x / c,  var = sum_c (x - mean)^2 / c,  rstd = 1 / sqrt(var + eps)
 *   y = gamma (x - mean) rstd + beta
 * gamma, beta: fp32 [c], NULL for 1 and 0; mean, rstd: fp32 [m], each NULL where it is not
 * wanted (the backward reads both).  y may be x's buffer if types and strides agree
 * (NUMBAT_ERR_BAD_DESC otherwise). */
numbat_status numbat_layer_norm_fwd(const numbat_layer_norm_problem* p, const void* x, const float* gamma,
                                    const float* beta, void* y, float* mean, float* rstd, void* stream);

/* Backward of layer norm, with xh = (x - mean) rstd and h = gamma dy:
 *   dx = rstd (h - sum_c h / c - xh sum_c(h xh) / c) + residual_grad
 *   dgamma = sum_rows dy xh,  dbeta = sum_rows dy          (fp32 [c]; accumulate: added)
 * gamma NULL: 1.  residual_grad [m][c] or NULL: the gradient that reaches x around the norm; dx
 * may be its buffer if their strides agree (NUMBAT_ERR_BAD_DESC otherwise).  Each of dx, dgamma,
 * dbeta may be NULL where it is not wanted; the workspace is required all the same.
 * ws: numbat_workspace_size(NUMBAT_OP_LAYER_NORM_BWD). */
numbat_status numbat_layer_norm_bwd(const numbat_layer_norm_problem* p, const void* dy, const void* x,
                                    const float* mean, const float* rstd, const float* gamma,
                                    const void* residual_grad, void* dx, float* dgamma, float* dbeta, int accumulate,
                                    void* ws, size_t ws_bytes, void* stream);

/* One parameter tensor of the AdamW step (device pointers, n elements each unless stated).
 * With 32-bit state m and v are fp32 and the units are not read.  With 8-bit state each block of
 * 256 elements from the tensor's start (the last one partial) has one fp32 unit in m_unit and
 * v_unit, m holds int8 codes q of the value u q|q|, and v uint8 codes q of the value (u q^2)^2.
 * Moments, and units, are zeros before the first step. */
typedef struct {
  float* w;           /* parameters, updated in place */
  const void* grad;   /* gradient, grad_type */
  void *m, *v;        /* first and second moments, updated in place */
  float *m_unit, *v_unit;
  void* w_copy;       /* NULL, or bf16: receives the updated parameters, rounded */
  int64_t n;
  int32_t group;      /* 0 .. ngroups-1 (a tensor outside them is left unchanged) */
  int32_t grad_type;  /* numbat_type */
} numbat_adamw_tensor;

/* The AdamW step (the paper's optimisers are SGD and Adam(W) in parameter groups with one fused
 * update over every tensor, Sec. 3.2) at step number `step` (1 for the first):
 *   c = 1, or with max_norm > 0:  min(1, max_norm / (norm + 1e-6)), norm the L2 norm of every gradient
 *   g = c grad;  m = beta1 m + (1 - beta1) g;  v = beta2 v + (1 - beta2) g^2
 *   w = w (1 - lr weight_decay) - lr / (1 - beta1^step) * m / (sqrt(v / (1 - beta2^step)) + eps)
 * beta1, beta2: 0 or more, below 1; eps, and max_norm unless it is 0: at least 2^-126 (fp32's smallest
 * normal number) and below 3e38.
 * tensors: DEVICE array of count (1 .. 1024) entries; groups: HOST array of ngroups (1 .. 8).
 * state_bits: 32 or 8.  In 8 bits the update uses the new moments before they are rounded; a
 * block whose unit would be below the smallest normal number is stored as zeros, and a v above
 * zero never rounds to zero within its block; a moment that is not finite takes the largest code.
 * The step's reciprocal, and with 32-bit state its root, are the hardware's, good to one unit in the
 * last place each; moments, units and codes are formed by IEEE operations.
 * total_norm: NULL, or a device float that receives the norm (only with max_norm > 0).  Of a
 * gradient that is not finite: a NaN norm does not clip, an infinite one gives c = 0 (its infinite
 * elements then become NaN).
 * ws: numbat_workspace_size(NUMBAT_OP_ADAMW), problem ignored. */
numbat_status numbat_adamw_step(const numbat_adamw_tensor* tensors, int32_t count, const numbat_sgd_group* groups,
                                int32_t ngroups, int32_t state_bits, double beta1, double beta2, double eps,
                                int64_t step, double max_norm, float* total_norm, void* ws, size_t ws_bytes,
                                void* stream);

/* The values that n elements of 8-bit state stand for, from the start of a tensor (or of tensors
 * whose blocks follow each other): m_value and v_value, fp32 [n] (a checkpoint's form). */
numbat_status numbat_adamw_state_values(int64_t n, const void* m, const float* m_unit, const void* v,
                                        const float* v_unit, float* m_value, float* v_value, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* NUMBAT_MLP_H */
