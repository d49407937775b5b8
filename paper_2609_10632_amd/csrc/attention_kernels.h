// Host-side launch interface of the residual attention block's kernels: group norm, rotary positions,
// attention.
#pragma once

#include "kernels.h"

namespace numbat {

// Kernel classes of numbat_attention.h's functions for the launch timing, numbered apart from the others
enum AttentionKernelClass {
  KC_ATTENTION_FIRST = 96,
  KC_GN_STATS = KC_ATTENTION_FIRST,  // group norm: statistics, where they are passes of their own
  KC_GN_FWD,                         // group norm forward
  KC_GN_BWD_SUMS,                    // group norm backward: sums, where they are passes of their own
  KC_GN_BWD,                         // group norm backward
  KC_GN_BWD_FINISH,                  // group norm backward: gain and shift gradients
  KC_ROTARY,
  KC_ATTN_FWD,                       // attention forward
  KC_ATTN_JOIN,                      // results of ranges of keys or queries, joined
  KC_ATTN_DQ,                        // attention backward: gradient of q
  KC_ATTN_DKV,                       // attention backward: gradients of k and v
  KC_ATTENTION_END
};

// ---------------------------------------------------------------------------
// Group norm over m rows of c channels of each of n images
struct GnArgs {
  int32_t n, c, groups, act;
  int64_t m;
  float eps;
  int32_t x_f32, y_f32;  // type of x, dx / of y, dy
  int64_t ldx, ldy, ldr, lddx;
};
size_t gn_fwd_ws(const GnArgs& a);
hipError_t gn_fwd_launch(const GnArgs& a, const void* x, const float* gamma, const float* beta, void* y, float* mean,
                         float* rstd, void* ws, hipStream_t s);
size_t gn_bwd_ws(const GnArgs& a);
hipError_t gn_bwd_launch(const GnArgs& a, const void* dy, const void* x, const float* mean, const float* rstd,
                         const float* gamma, const float* beta, const void* res, void* dx, float* dgamma, float* dbeta,
                         int accumulate, void* ws, hipStream_t s);

// ---------------------------------------------------------------------------
// Rotary positions
constexpr int kRotaryPairs = 256, kRotaryAxes = 4;
struct RotaryArgs {
  int64_t m;
  int32_t heads, d, axes, pairs;  // pairs: of all axes
  int32_t halves, f32;
  int64_t ldx, ldy;
  const int32_t* pos;             // [m][axes] or nullptr
  int32_t first[kRotaryAxes + 1]; // an axis' first pair, and the end
  FastDiv extent[kRotaryAxes];
  double turns[kRotaryPairs];     // full turns by one step of the pair's axis (negative: back)
};
hipError_t rotary_launch(const RotaryArgs& a, const void* x, void* y, hipStream_t s);

// ---------------------------------------------------------------------------
// Attention.  The queries of the heads that share a head of k and v are the columns of one product:
// column c is row c / group, head c % group of the group.
struct AttnArgs {
  const bf16_t *q, *k, *v, *y, *dy;
  bf16_t *out, *dq, *dk, *dv;
  float* lse;
  const int32_t *q_lengths, *kv_lengths;
  int32_t batch, q_len, kv_len, kv_heads, group, d, causal;
  int64_t ldq, ldk, ldv, ldy;
  float scale, scale_log2;  // scale, scale log2(e)
  FastDiv div_group;
};
// whether every grid is one that a launch takes
bool attn_fits(const AttnArgs& a);
size_t attn_fwd_ws(const AttnArgs& a);
hipError_t attn_fwd_launch(const AttnArgs& a, void* ws, hipStream_t s);
size_t attn_bwd_ws(const AttnArgs& a);
hipError_t attn_bwd_launch(const AttnArgs& a, void* ws, hipStream_t s);

}  // namespace numbat
