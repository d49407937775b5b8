// C ABI of the residual attention block's operators (numbat_attention.h): descriptor validation,
// workspace sizes and dispatch.  Every check runs before anything is enqueued.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <initializer_list>

#include "../../include/numbat_attention.h"
#include "abi_util.h"
#include "attention_kernels.h"
#include "mlp_kernels.h"

using namespace numbat;

namespace {

constexpr int64_t kMaxStride = 1 << 21;  // a tile's rows stay within 31-bit byte offsets

bool stride_ok(int64_t stride, int64_t width) { return stride == 0 || (stride >= width && stride <= kMaxStride); }
int64_t dense(int64_t stride, int64_t width) { return stride != 0 ? stride : width; }
bool known_type(int32_t t) { return t == NUMBAT_TYPE_BF16 || t == NUMBAT_TYPE_F32; }
// Launches report by hipGetLastError: an error that another caller's call has left there is not one of theirs, and would
// keep the later kernels of an operator from being launched
void drop_old_error() { (void)hipGetLastError(); }
bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

template <typename P>
numbat_status check_size(const P* p, const char* name) {
  if (p == nullptr) return fail(NUMBAT_ERR_NULL, "problem descriptor is NULL");
  if (p->struct_size != sizeof(P))
    return fail(NUMBAT_ERR_VERSION, "%s.struct_size is %u, this library expects %zu", name, p->struct_size, sizeof(P));
  return NUMBAT_OK;
}

numbat_status check_gn(const numbat_group_norm_problem* p, GnArgs* a) {
  const numbat_status st = check_size(p, "numbat_group_norm_problem");
  if (st != NUMBAT_OK) return st;
  if (p->n < 0 || p->m < 0 || p->c < 1 || p->groups < 1)
    return fail(NUMBAT_ERR_BAD_DESC, "n and m must be >= 0, c and groups >= 1 (n=%d m=%lld c=%d groups=%d)", p->n,
                (long long)p->m, p->c, p->groups);
  if (p->c % p->groups != 0) return fail(NUMBAT_ERR_BAD_DESC, "%d groups do not divide c = %d", p->groups, p->c);
  if (p->act < NUMBAT_ACT_NONE || p->act > NUMBAT_ACT_SILU) return fail(NUMBAT_ERR_BAD_DESC, "unknown act %d", p->act);
  if (!(p->eps >= 0.0f && p->eps < 3.0e38f)) return fail(NUMBAT_ERR_BAD_DESC, "eps must be finite and >= 0");
  for (int32_t t : {p->x_type, p->y_type})
    if (!known_type(t)) return fail(NUMBAT_ERR_BAD_DESC, "unknown type %d", t);
  if (p->n > 65535 || p->c > 65536 || p->m > kMaxIndex)
    return fail(NUMBAT_ERR_UNSUPPORTED, "at most 65535 images, 65536 channels and 2^31-1 rows (n=%d c=%d m=%lld)", p->n,
                p->c, (long long)p->m);
  for (int64_t s : {p->x_row_stride, p->y_row_stride, p->r_row_stride, p->dx_row_stride})
    if (!stride_ok(s, p->c))
      return fail(NUMBAT_ERR_BAD_DESC, "row stride %lld is smaller than c = %d or above 2^21", (long long)s, p->c);
  std::memset(a, 0, sizeof *a);
  a->n = p->n;
  a->m = p->m;
  a->c = p->c;
  a->groups = p->groups;
  a->act = p->act;
  a->eps = p->eps;
  a->x_f32 = p->x_type == NUMBAT_TYPE_F32;
  a->y_f32 = p->y_type == NUMBAT_TYPE_F32;
  a->ldx = dense(p->x_row_stride, p->c);
  a->ldy = dense(p->y_row_stride, p->c);
  a->ldr = dense(p->r_row_stride, p->c);
  a->lddx = dense(p->dx_row_stride, p->c);
  return NUMBAT_OK;
}

bool gn_empty(const GnArgs& a) { return a.n == 0 || a.m == 0; }

numbat_status check_rotary(const numbat_rotary_problem* p, bool grid, RotaryArgs* a) {
  const numbat_status st = check_size(p, "numbat_rotary_problem");
  if (st != NUMBAT_OK) return st;
  if (p->m < 0 || p->heads < 1 || p->d < 2)
    return fail(NUMBAT_ERR_BAD_DESC, "m must be >= 0, heads >= 1 and d >= 2 (m=%lld heads=%d d=%d)", (long long)p->m,
                p->heads, p->d);
  if (p->axes < 1 || p->axes > kRotaryAxes) return fail(NUMBAT_ERR_BAD_DESC, "axes = %d: 1 .. 4", p->axes);
  if (p->layout != NUMBAT_ROTARY_HALVES && p->layout != NUMBAT_ROTARY_PAIRS)
    return fail(NUMBAT_ERR_BAD_DESC, "unknown layout %d", p->layout);
  if ((p->shared != 0 && p->shared != 1) || (p->inverse != 0 && p->inverse != 1))
    return fail(NUMBAT_ERR_BAD_DESC, "shared and inverse are 0 or 1");
  if (!known_type(p->type)) return fail(NUMBAT_ERR_BAD_DESC, "unknown type %d", p->type);
  if (!(p->base > 1.0 && p->base <= 1e30)) return fail(NUMBAT_ERR_BAD_DESC, "base must be above 1 and at most 1e30");
  std::memset(a, 0, sizeof *a);
  int64_t total = 0;
  for (int i = 0; i < kRotaryAxes; ++i) {
    if (i < p->axes ? p->pairs[i] < 1 : p->pairs[i] != 0)
      return fail(NUMBAT_ERR_BAD_DESC, "pairs[%d] = %d: at least 1 for each axis, 0 past them", i, p->pairs[i]);
    if (grid && i < p->axes && p->extents[i] < 1)
      return fail(NUMBAT_ERR_BAD_DESC, "extents[%d] = %d: at least 1 for each axis without positions", i, p->extents[i]);
    a->first[i] = (int32_t)std::min<int64_t>(total, kRotaryPairs);
    total += p->pairs[i];
  }
  a->first[kRotaryAxes] = (int32_t)std::min<int64_t>(total, kRotaryPairs);
  if (2 * total > p->d) return fail(NUMBAT_ERR_BAD_DESC, "%lld pairs take more than d = %d features", (long long)total, p->d);
  const int64_t width = (int64_t)p->heads * p->d;
  if (total > kRotaryPairs || width > kMaxStride || p->m > kMaxIndex)
    return fail(NUMBAT_ERR_UNSUPPORTED, "at most 256 pairs, heads * d up to 2^21 and 2^31-1 rows (%lld, %lld, %lld)",
                (long long)total, (long long)width, (long long)p->m);
  for (int64_t s : {p->x_row_stride, p->y_row_stride})
    if (!stride_ok(s, width))
      return fail(NUMBAT_ERR_BAD_DESC, "row stride %lld is smaller than heads * d = %lld or above 2^21", (long long)s,
                  (long long)width);
  a->m = p->m;
  a->heads = p->heads;
  a->d = p->d;
  a->axes = p->axes;
  a->pairs = (int32_t)total;
  a->halves = p->layout == NUMBAT_ROTARY_HALVES;
  a->f32 = p->type == NUMBAT_TYPE_F32;
  a->ldx = dense(p->x_row_stride, width);
  a->ldy = dense(p->y_row_stride, width);
  const double way = (p->inverse ? -1.0 : 1.0) / 6.283185307179586476925286766559;
  for (int i = 0, j = 0; i < p->axes; ++i) {
    if (grid) a->extent[i] = make_fastdiv((uint32_t)p->extents[i]);
    for (int k = 0; k < p->pairs[i]; ++k, ++j)
      a->turns[j] = way * std::pow(p->base, p->shared ? -(double)j / (double)total : -(double)k / (double)p->pairs[i]);
  }
  return NUMBAT_OK;
}

// A result at the address of an operand, or of another result, that is there
numbat_status check_apart(std::initializer_list<const void*> results, std::initializer_list<const void*> operands) {
  for (auto r = results.begin(); r != results.end(); ++r) {
    if (*r == nullptr) continue;
    for (const void* o : operands)
      if (*r == o) return fail(NUMBAT_ERR_BAD_DESC, "a result lies in an operand's buffer, which others still read");
    for (auto q = results.begin(); q != r; ++q)
      if (*r == *q) return fail(NUMBAT_ERR_BAD_DESC, "two results lie in one buffer");
  }
  return NUMBAT_OK;
}

numbat_status check_attention(const numbat_attention_problem* p, AttnArgs* a) {
  const numbat_status st = check_size(p, "numbat_attention_problem");
  if (st != NUMBAT_OK) return st;
  if (p->batch < 0 || p->q_len < 0 || p->kv_len < 0 || p->q_heads < 1 || p->kv_heads < 1 || p->d < 1)
    return fail(NUMBAT_ERR_BAD_DESC,
                "batch, q_len and kv_len must be >= 0, heads and d >= 1 (batch=%d q_len=%d kv_len=%d q_heads=%d "
                "kv_heads=%d d=%d)",
                p->batch, p->q_len, p->kv_len, p->q_heads, p->kv_heads, p->d);
  if (p->q_heads % p->kv_heads != 0)
    return fail(NUMBAT_ERR_BAD_DESC, "kv_heads = %d does not divide q_heads = %d", p->kv_heads, p->q_heads);
  if (p->causal != 0 && p->causal != 1) return fail(NUMBAT_ERR_BAD_DESC, "causal is 0 or 1");
  // (the kernels multiply it by log2(e))
  if (!(p->scale > 0.0f && p->scale <= 1.0e38f)) return fail(NUMBAT_ERR_BAD_DESC, "scale must be above 0 and at most 1e38");
  if (p->reserved != 0) return fail(NUMBAT_ERR_BAD_DESC, "reserved must be 0");
  const int64_t qw = (int64_t)p->q_heads * p->d, kw = (int64_t)p->kv_heads * p->d;
  const int32_t group = p->q_heads / p->kv_heads;
  if (p->d % 8 != 0 || p->d > 128)
    return fail(NUMBAT_ERR_UNSUPPORTED, "d = %d: a multiple of 8, at most 128", p->d);
  if (p->batch > 65535 || qw > kMaxStride || (int64_t)p->q_len * group > (1 << 30) || p->kv_len > (1 << 30))
    return fail(NUMBAT_ERR_UNSUPPORTED,
                "at most 65535 sequences, heads * d up to 2^21, 2^30 keys, and queries times heads that share them");
  for (int64_t s : {p->q_row_stride, p->y_row_stride})
    if (!stride_ok(s, qw))
      return fail(NUMBAT_ERR_BAD_DESC, "row stride %lld is smaller than q_heads * d = %lld or above 2^21", (long long)s,
                  (long long)qw);
  for (int64_t s : {p->k_row_stride, p->v_row_stride})
    if (!stride_ok(s, kw))
      return fail(NUMBAT_ERR_BAD_DESC, "row stride %lld is smaller than kv_heads * d = %lld or above 2^21", (long long)s,
                  (long long)kw);
  for (int64_t s : {p->q_row_stride, p->k_row_stride, p->v_row_stride, p->y_row_stride})
    if (s % 8 != 0) return fail(NUMBAT_ERR_ALIGN, "row stride %lld is no multiple of 8", (long long)s);
  std::memset(a, 0, sizeof *a);
  a->batch = p->batch;
  a->q_len = p->q_len;
  a->kv_len = p->kv_len;
  a->kv_heads = p->kv_heads;
  a->group = group;
  a->d = p->d;
  a->causal = p->causal;
  a->ldq = dense(p->q_row_stride, qw);
  a->ldk = dense(p->k_row_stride, kw);
  a->ldv = dense(p->v_row_stride, kw);
  a->ldy = dense(p->y_row_stride, qw);
  a->scale = p->scale;
  a->scale_log2 = p->scale * 1.4426950408889634f;
  a->div_group = make_fastdiv((uint32_t)group);
  return attn_fits(*a) ? NUMBAT_OK
                       : fail(NUMBAT_ERR_UNSUPPORTED, "more tiles of queries or keys than one launch takes");
}

}  // namespace

namespace numbat {

bool attention_workspace_size(int op, const void* problem, size_t* bytes, numbat_status* st) {
  switch (op) {
    case NUMBAT_OP_GROUP_NORM_FWD:
    case NUMBAT_OP_GROUP_NORM_BWD: {
      GnArgs a;
      *st = check_gn(static_cast<const numbat_group_norm_problem*>(problem), &a);
      if (*st != NUMBAT_OK) return true;
      *bytes = gn_empty(a) ? 0 : with_header(op == NUMBAT_OP_GROUP_NORM_FWD ? gn_fwd_ws(a) : gn_bwd_ws(a));
      break;
    }
    case NUMBAT_OP_ATTENTION_FWD:
    case NUMBAT_OP_ATTENTION_BWD: {
      AttnArgs a;
      *st = check_attention(static_cast<const numbat_attention_problem*>(problem), &a);
      if (*st != NUMBAT_OK) return true;
      *bytes = with_header(op == NUMBAT_OP_ATTENTION_FWD ? attn_fwd_ws(a) : attn_bwd_ws(a));
      break;
    }
    default: return false;
  }
  *st = ok();
  return true;
}

}  // namespace numbat

extern "C" {

numbat_status numbat_group_norm_fwd(const numbat_group_norm_problem* p, const void* x, const float* gamma,
                                    const float* beta, void* y, float* mean, float* rstd, void* ws, size_t ws_bytes,
                                    void* stream) {
  GnArgs a;
  numbat_status st = check_gn(p, &a);
  if (st != NUMBAT_OK) return st;
  if (gn_empty(a)) return ok();
  if (x == nullptr || y == nullptr) return fail(NUMBAT_ERR_NULL, "x and y are required");
  if (!aligned16(x) || !aligned16(y)) return fail(NUMBAT_ERR_ALIGN, "x and y must be 16-byte aligned");
  for (const float* f : {gamma, beta, (const float*)mean, (const float*)rstd})
    if (!aligned4(f)) return fail(NUMBAT_ERR_ALIGN, "gamma, beta, mean and rstd must be 4-byte aligned");
  if (x == y && (a.x_f32 != a.y_f32 || a.ldx != a.ldy))
    return fail(NUMBAT_ERR_BAD_DESC, "y in x's buffer needs its type and row stride (y %lld, x %lld)", (long long)a.ldy,
                (long long)a.ldx);
  st = check_ws(ws, ws_bytes, with_header(gn_fwd_ws(a)));
  if (st != NUMBAT_OK) return st;
  drop_old_error();
  const hipError_t e = gn_fwd_launch(a, x, gamma, beta, y, mean, rstd, ws_body(ws), static_cast<hipStream_t>(stream));
  return e == hipSuccess ? ok() : hip_fail(e, "group norm forward launch");
}

numbat_status numbat_group_norm_bwd(const numbat_group_norm_problem* p, const void* dy, const void* x,
                                    const float* mean, const float* rstd, const float* gamma, const float* beta,
                                    const void* residual_grad, void* dx, float* dgamma, float* dbeta, int accumulate,
                                    void* ws, size_t ws_bytes, void* stream) {
  GnArgs a;
  numbat_status st = check_gn(p, &a);
  if (st != NUMBAT_OK) return st;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  hipError_t e = hipSuccess;
  for (const float* f : {mean, rstd, gamma, beta, (const float*)dgamma, (const float*)dbeta})
    if (!aligned4(f)) return fail(NUMBAT_ERR_ALIGN, "mean, rstd, gamma, beta, dgamma and dbeta must be 4-byte aligned");
  if (gn_empty(a)) {  // empty sums
    drop_old_error();
    if (!accumulate && dgamma != nullptr) e = fill_zero_launch(dgamma, a.c, s);
    if (!accumulate && dbeta != nullptr && e == hipSuccess) e = fill_zero_launch(dbeta, a.c, s);
    return e == hipSuccess ? ok() : hip_fail(e, "group norm backward launch");
  }
  if (dy == nullptr || x == nullptr || mean == nullptr || rstd == nullptr)
    return fail(NUMBAT_ERR_NULL, "dy, x, mean and rstd are required");
  if (dx == nullptr && dgamma == nullptr && dbeta == nullptr)
    return fail(NUMBAT_ERR_NULL, "at least one of dx, dgamma and dbeta is required");
  if (dx == nullptr && residual_grad != nullptr) return fail(NUMBAT_ERR_NULL, "residual_grad needs dx");
  if (!aligned16(dy) || !aligned16(x) || !aligned16(residual_grad) || !aligned16(dx))
    return fail(NUMBAT_ERR_ALIGN, "dy, x, residual_grad and dx must be 16-byte aligned");
  if (dx != nullptr && dx == residual_grad && a.ldr != a.lddx)
    return fail(NUMBAT_ERR_BAD_DESC, "dx in residual_grad's buffer needs its row stride (dx %lld, residual_grad %lld)",
                (long long)a.lddx, (long long)a.ldr);
  if (dx == x && a.ldx != a.lddx)
    return fail(NUMBAT_ERR_BAD_DESC, "dx in x's buffer needs its row stride (dx %lld, x %lld)", (long long)a.lddx,
                (long long)a.ldx);
  if (dx == dy && (a.x_f32 != a.y_f32 || a.ldy != a.lddx))
    return fail(NUMBAT_ERR_BAD_DESC, "dx in dy's buffer needs its type and row stride (dx %lld, dy %lld)",
                (long long)a.lddx, (long long)a.ldy);
  st = check_ws(ws, ws_bytes, with_header(gn_bwd_ws(a)));
  if (st != NUMBAT_OK) return st;
  drop_old_error();
  e = gn_bwd_launch(a, dy, x, mean, rstd, gamma, beta, residual_grad, dx, dgamma, dbeta, accumulate != 0, ws_body(ws), s);
  return e == hipSuccess ? ok() : hip_fail(e, "group norm backward launch");
}

numbat_status numbat_rotary(const numbat_rotary_problem* p, const void* x, const int32_t* positions, void* y,
                            void* stream) {
  RotaryArgs a;
  const numbat_status st = check_rotary(p, positions == nullptr, &a);
  if (st != NUMBAT_OK) return st;
  if (a.m == 0) return ok();
  if (x == nullptr || y == nullptr) return fail(NUMBAT_ERR_NULL, "x and y are required");
  if (!aligned16(x) || !aligned16(y) || !aligned4(positions))
    return fail(NUMBAT_ERR_ALIGN, "x and y must be 16-byte aligned, positions 4-byte aligned");
  if (x == y && a.m > 1 && a.ldx != a.ldy)
    return fail(NUMBAT_ERR_BAD_DESC, "y in x's buffer needs its row stride (y %lld, x %lld)", (long long)a.ldy,
                (long long)a.ldx);
  a.pos = positions;
  drop_old_error();
  const hipError_t e = rotary_launch(a, x, y, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? ok() : hip_fail(e, "rotary launch");
}

numbat_status numbat_attention_fwd(const numbat_attention_problem* p, const void* q, const void* k, const void* v,
                                   const int32_t* q_lengths, const int32_t* kv_lengths, void* y, float* lse, void* ws,
                                   size_t ws_bytes, void* stream) {
  AttnArgs a;
  numbat_status st = check_attention(p, &a);
  if (st != NUMBAT_OK) return st;
  if (a.batch == 0 || a.q_len == 0) return ok();
  if (q == nullptr || y == nullptr || (a.kv_len > 0 && (k == nullptr || v == nullptr)))
    return fail(NUMBAT_ERR_NULL, "q, k, v and y are required");
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(y))
    return fail(NUMBAT_ERR_ALIGN, "q, k, v and y must be 16-byte aligned");
  if (!aligned4(q_lengths) || !aligned4(kv_lengths) || !aligned4(lse))
    return fail(NUMBAT_ERR_ALIGN, "q_lengths, kv_lengths and lse must be 4-byte aligned");
  st = check_ws(ws, ws_bytes, with_header(attn_fwd_ws(a)));
  if (st != NUMBAT_OK) return st;
  st = check_apart({y, lse}, {q, k, v, q_lengths, kv_lengths});
  if (st != NUMBAT_OK) return st;
  a.q = static_cast<const bf16_t*>(q);
  a.k = static_cast<const bf16_t*>(k);
  a.v = static_cast<const bf16_t*>(v);
  a.q_lengths = q_lengths;
  a.kv_lengths = kv_lengths;
  a.out = static_cast<bf16_t*>(y);
  a.lse = lse;
  drop_old_error();
  const hipError_t e = attn_fwd_launch(a, ws_body(ws), static_cast<hipStream_t>(stream));
  return e == hipSuccess ? ok() : hip_fail(e, "attention forward launch");
}

numbat_status numbat_attention_bwd(const numbat_attention_problem* p, const void* dy, const void* q, const void* k,
                                   const void* v, const void* y, const float* lse, const int32_t* q_lengths,
                                   const int32_t* kv_lengths, void* dq, void* dk, void* dv, void* ws, size_t ws_bytes,
                                   void* stream) {
  AttnArgs a;
  numbat_status st = check_attention(p, &a);
  if (st != NUMBAT_OK) return st;
  if (a.batch == 0 || (a.q_len == 0 && a.kv_len == 0)) return ok();
  if (a.q_len > 0 && (q == nullptr || y == nullptr || dy == nullptr || lse == nullptr || dq == nullptr))
    return fail(NUMBAT_ERR_NULL, "dy, q, y, lse and dq are required");
  if (a.kv_len > 0 && (k == nullptr || v == nullptr || dk == nullptr || dv == nullptr))
    return fail(NUMBAT_ERR_NULL, "k, v, dk and dv are required");
  for (const void* t : {dy, q, k, v, y, (const void*)dq, (const void*)dk, (const void*)dv})
    if (!aligned16(t)) return fail(NUMBAT_ERR_ALIGN, "dy, q, k, v, y, dq, dk and dv must be 16-byte aligned");
  if (!aligned4(q_lengths) || !aligned4(kv_lengths) || !aligned4(lse))
    return fail(NUMBAT_ERR_ALIGN, "q_lengths, kv_lengths and lse must be 4-byte aligned");
  st = check_ws(ws, ws_bytes, with_header(attn_bwd_ws(a)));
  if (st != NUMBAT_OK) return st;
  st = check_apart({dq, dk, dv}, {dy, q, k, v, y, lse, q_lengths, kv_lengths});
  if (st != NUMBAT_OK) return st;
  a.q = static_cast<const bf16_t*>(q);
  a.k = static_cast<const bf16_t*>(k);
  a.v = static_cast<const bf16_t*>(v);
  a.y = static_cast<const bf16_t*>(y);
  a.dy = static_cast<const bf16_t*>(dy);
  a.lse = const_cast<float*>(lse);
  a.q_lengths = q_lengths;
  a.kv_lengths = kv_lengths;
  a.dq = static_cast<bf16_t*>(dq);
  a.dk = static_cast<bf16_t*>(dk);
  a.dv = static_cast<bf16_t*>(dv);
  drop_old_error();
  const hipError_t e = attn_bwd_launch(a, ws_body(ws), static_cast<hipStream_t>(stream));
  return e == hipSuccess ? ok() : hip_fail(e, "attention backward launch");
}

}  // extern "C"
