// C ABI of the residual MLP block's operators (numbat_mlp.h): descriptor validation, workspace
// layout and dispatch.  Every check runs before anything is enqueued.
#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstddef>
#include <cstring>

#include "../../include/numbat_mlp.h"
#include "abi_util.h"
#include "mlp_kernels.h"

using namespace numbat;

namespace {

constexpr int64_t kMaxFeatures = 1 << 21;  // a tile's rows stay within 31-bit byte offsets

struct LinearDesc {
  int64_t m;
  int32_t n, k, act;
  bool y_f32;
  int64_t ldx, ldy, ldr, ldz;  // z is n wide in the forward, k in the data gradient
};

bool stride_ok(int64_t stride, int64_t width) { return stride == 0 || (stride >= width && stride <= kMaxFeatures); }

// A result in an operand's buffer lies where the operand does, element for element; otherwise one
// block's rows would overwrite what another has yet to read.
bool in_place_ok(const void* operand, const void* result, int64_t rows, int64_t ld_operand, int64_t ld_result) {
  return operand == nullptr || operand != result || rows <= 1 || ld_operand == ld_result;
}

numbat_status check_linear(const numbat_linear_problem* p, GemmKind kind, LinearDesc* d) {
  if (p == nullptr) return fail(NUMBAT_ERR_NULL, "problem descriptor is NULL");
  if (p->struct_size != sizeof(numbat_linear_problem))
    return fail(NUMBAT_ERR_VERSION, "numbat_linear_problem.struct_size is %u, this library expects %zu", p->struct_size,
                sizeof(numbat_linear_problem));
  if (p->m < 0 || p->n < 1 || p->k < 1)
    return fail(NUMBAT_ERR_BAD_DESC, "m must be >= 0, n and k >= 1 (m=%lld n=%d k=%d)", (long long)p->m, p->n, p->k);
  if (p->act < NUMBAT_ACT_NONE || p->act > NUMBAT_ACT_SILU) return fail(NUMBAT_ERR_BAD_DESC, "unknown act %d", p->act);
  if (p->y_type != NUMBAT_TYPE_BF16 && p->y_type != NUMBAT_TYPE_F32)
    return fail(NUMBAT_ERR_BAD_DESC, "unknown y_type %d", p->y_type);
  if (p->reserved != 0) return fail(NUMBAT_ERR_BAD_DESC, "reserved must be 0");
  if (p->m > kMaxIndex || p->n > kMaxFeatures || p->k > kMaxFeatures)
    return fail(NUMBAT_ERR_UNSUPPORTED, "at most 2^31-1 rows and 2^21 features (m=%lld n=%d k=%d)", (long long)p->m, p->n,
                p->k);
  // (the weight gradient has no z: it takes the forward's descriptor and the data gradient's)
  const int64_t zw = kind == kGemmFwd ? p->n : kind == kGemmDgrad ? p->k : std::min(p->n, p->k);
  if (!stride_ok(p->x_row_stride, p->k) || !stride_ok(p->y_row_stride, p->n) || !stride_ok(p->r_row_stride, p->n) ||
      !stride_ok(p->z_row_stride, zw))
    return fail(NUMBAT_ERR_BAD_DESC, "a row stride is smaller than its row or above 2^21 (x %lld y %lld r %lld z %lld)",
                (long long)p->x_row_stride, (long long)p->y_row_stride, (long long)p->r_row_stride,
                (long long)p->z_row_stride);
  d->m = p->m;
  d->n = p->n;
  d->k = p->k;
  d->act = p->act;
  d->y_f32 = p->y_type == NUMBAT_TYPE_F32;
  d->ldx = p->x_row_stride ? p->x_row_stride : p->k;
  d->ldy = p->y_row_stride ? p->y_row_stride : p->n;
  d->ldr = p->r_row_stride ? p->r_row_stride : p->n;
  d->ldz = p->z_row_stride ? p->z_row_stride : zw;
  return NUMBAT_OK;
}

// One matrix product of a layer: its operands as stored, and where in the workspace their padded
// copies (operands whose rows are not whole 16-byte vectors) and the partial sums go.
struct Product {
  GemmKind kind;
  int64_t m, k;
  int32_t n;
  struct Op {
    int64_t rows;
    int32_t cols;
    int64_t ld;
    bool pack;
    int64_t ldp;
    size_t at;
  } a, b;
  GemmPlan plan;
  bool sums_rows;  // the bias gradient comes with the weight gradient
  size_t part_at, db_at, bytes;  // db: the bias gradient's partials
};

size_t place(size_t* at, size_t bytes) {
  const size_t here = *at;
  *at += round_up(bytes, 256);
  return here;
}

// pack: its rows are not whole aligned vectors
Product::Op operand(int64_t rows, int32_t cols, int64_t ld) {
  return Product::Op{rows, cols, ld, cols % 8 != 0 || ld % 8 != 0, (int64_t)round_up((size_t)cols, 8), 0};
}
double pack_bytes(const Product::Op& o) { return o.pack ? (double)o.rows * o.ldp * sizeof(bf16_t) : 0.0; }

Product product(const LinearDesc& d, GemmKind kind) {
  Product p;
  std::memset(&p, 0, sizeof p);
  p.kind = kind;
  size_t at = 0;
  if (d.m == 0) return p;
  if (kind == kGemmFwd) p.m = d.m, p.n = d.n, p.k = d.k;
  else if (kind == kGemmDgrad) p.m = d.m, p.n = d.k, p.k = d.n;
  else p.m = d.n, p.n = d.k, p.k = d.m;
  p.a = kind == kGemmFwd ? operand(d.m, d.k, d.ldx) : operand(d.m, d.n, d.ldy);
  p.b = kind == kGemmWgrad ? operand(d.m, d.k, d.ldx) : operand(d.n, d.k, d.k);
  // (the workspace depends on the problem alone, so that z is kept and read where there is an
  // activation is taken for granted here)
  const int z = d.act != NUMBAT_ACT_NONE ? 2 : 0;
  p.plan = gemm_pick(kind, p.m, p.n, p.k, kind == kGemmFwd ? (d.y_f32 ? 4 : 2) + z : kind == kGemmDgrad ? 2 + z : 4,
                     pack_bytes(p.a) + pack_bytes(p.b));
  for (Product::Op* o : {&p.a, &p.b}) {
    o->pack = o->pack && !gemm_any_rows(p.plan);
    if (o->pack) o->at = place(&at, (size_t)pack_bytes(*o));
  }
  p.part_at = place(&at, gemm_part_bytes(p.plan, p.m, p.n));
  if (kind == kGemmWgrad) {
    p.sums_rows = gemm_sums_rows(p.plan);
    if (!p.sums_rows) p.db_at = place(&at, colsum_part_bytes(d.m, d.n));
    else if (p.plan.splits > 1) p.db_at = place(&at, (size_t)p.plan.splits * (size_t)p.m * sizeof(float));
  }
  p.bytes = at;
  return p;
}

numbat_status check_grid(const Product& p) {
  if (p.m > 0 && !gemm_fits(p.plan, p.m, p.n))
    return fail(NUMBAT_ERR_UNSUPPORTED, "the product has more tiles than one launch takes (%lld x %d)", (long long)p.m, p.n);
  return NUMBAT_OK;
}

// the operand as the product reads it: where it lies, or its padded copy to be made
GemmPack packed(const Product::Op& o, const void* src, char* ws, const bf16_t** out, int64_t* ld) {
  const bf16_t* s = static_cast<const bf16_t*>(src);
  bf16_t* dst = o.pack ? reinterpret_cast<bf16_t*>(ws + o.at) : nullptr;
  *out = o.pack ? dst : s;
  *ld = o.pack ? o.ldp : o.ld;
  return GemmPack{s, o.ld, o.pack ? o.rows : 0, o.cols, dst, o.ldp};
}

hipError_t run_product(const Product& p, const void* a, const void* b, const GemmEpilogue& e, float* db, void* ws,
                       hipStream_t s) {
  GemmArgs g;
  std::memset(&g, 0, sizeof g);
  char* body = static_cast<char*>(ws);
  const GemmPack pa = packed(p.a, a, body, &g.a, &g.lda), pb = packed(p.b, b, body, &g.b, &g.ldb);
  if (pa.rows > 0 || pb.rows > 0) {
    const hipError_t err = gemm_pack_launch(pa, pb, s);
    if (err != hipSuccess) return err;
  }
  g.m = p.m;
  g.n = p.n;
  g.k = p.k;
  g.part = reinterpret_cast<float*>(body + p.part_at);
  g.db = db;
  g.db_part = reinterpret_cast<float*>(body + p.db_at);
  g.e = e;
  return gemm_launch(p.kind, g, p.plan, s);
}

numbat_status check_ln(const numbat_layer_norm_problem* p, LnArgs* a) {
  if (p == nullptr) return fail(NUMBAT_ERR_NULL, "problem descriptor is NULL");
  if (p->struct_size != sizeof(numbat_layer_norm_problem))
    return fail(NUMBAT_ERR_VERSION, "numbat_layer_norm_problem.struct_size is %u, this library expects %zu",
                p->struct_size, sizeof(numbat_layer_norm_problem));
  if (p->m < 0 || p->c < 1)
    return fail(NUMBAT_ERR_BAD_DESC, "m must be >= 0 and c >= 1 (m=%lld c=%d)", (long long)p->m, p->c);
  if (!(p->eps >= 0.0f && p->eps < 3.0e38f)) return fail(NUMBAT_ERR_BAD_DESC, "eps must be finite and >= 0");
  for (int32_t t : {p->x_type, p->y_type})
    if (t != NUMBAT_TYPE_BF16 && t != NUMBAT_TYPE_F32) return fail(NUMBAT_ERR_BAD_DESC, "unknown type %d", t);
  if (p->reserved != 0) return fail(NUMBAT_ERR_BAD_DESC, "reserved must be 0");
  if (p->m > kMaxIndex || p->c > kMaxFeatures)
    return fail(NUMBAT_ERR_UNSUPPORTED, "at most 2^31-1 rows and 2^21 features (m=%lld c=%d)", (long long)p->m, p->c);
  for (int64_t s : {p->x_row_stride, p->y_row_stride, p->r_row_stride, p->dx_row_stride})
    if (!stride_ok(s, p->c))
      return fail(NUMBAT_ERR_BAD_DESC, "row stride %lld is smaller than c = %d or above 2^21", (long long)s, p->c);
  std::memset(a, 0, sizeof *a);
  a->c = p->c;
  a->m = p->m;
  a->eps = p->eps;
  a->x_f32 = p->x_type == NUMBAT_TYPE_F32;
  a->y_f32 = p->y_type == NUMBAT_TYPE_F32;
  a->ldx = p->x_row_stride ? p->x_row_stride : p->c;
  a->ldy = p->y_row_stride ? p->y_row_stride : p->c;
  a->ldr = p->r_row_stride ? p->r_row_stride : p->c;
  a->lddx = p->dx_row_stride ? p->dx_row_stride : p->c;
  return NUMBAT_OK;
}

size_t ln_bwd_ws(const LnArgs& a) { return a.m > 0 ? ln_bwd_part_bytes(a) : 0; }
constexpr size_t kAdamWs = kAdamNormBlocks * sizeof(double);

}  // namespace

namespace numbat {

bool mlp_workspace_size(int op, const void* problem, size_t* bytes, numbat_status* st) {
  switch (op) {
    case NUMBAT_OP_LINEAR_FWD:
    case NUMBAT_OP_LINEAR_BWD_DATA:
    case NUMBAT_OP_LINEAR_BWD_WEIGHT: {
      const GemmKind kind = op == NUMBAT_OP_LINEAR_FWD        ? kGemmFwd
                            : op == NUMBAT_OP_LINEAR_BWD_DATA ? kGemmDgrad
                                                              : kGemmWgrad;
      LinearDesc d;
      *st = check_linear(static_cast<const numbat_linear_problem*>(problem), kind, &d);
      if (*st != NUMBAT_OK) return true;
      const Product pr = product(d, kind);
      *st = check_grid(pr);
      if (*st != NUMBAT_OK) return true;
      *bytes = with_header(pr.bytes);
      break;
    }
    case NUMBAT_OP_LAYER_NORM_BWD: {
      LnArgs a;
      *st = check_ln(static_cast<const numbat_layer_norm_problem*>(problem), &a);
      if (*st != NUMBAT_OK) return true;
      *bytes = with_header(ln_bwd_ws(a));
      break;
    }
    case NUMBAT_OP_ADAMW: *bytes = with_header(kAdamWs); break;
    default: return false;
  }
  *st = ok();
  return true;
}

}  // namespace numbat

extern "C" {

numbat_status numbat_linear_fwd(const numbat_linear_problem* p, const void* x, const void* w, const float* bias,
                                const void* residual, void* z, void* y, void* ws, size_t ws_bytes, void* stream) {
  LinearDesc d;
  numbat_status st = check_linear(p, kGemmFwd, &d);
  if (st != NUMBAT_OK) return st;
  if (d.m == 0) return ok();
  if (x == nullptr || w == nullptr || y == nullptr) return fail(NUMBAT_ERR_NULL, "x, w and y are required");
  if (!aligned16(x) || !aligned16(w) || !aligned16(y) || !aligned16(residual) || !aligned16(z))
    return fail(NUMBAT_ERR_ALIGN, "x, w, y, residual and z must be 16-byte aligned");
  if (!in_place_ok(residual, y, d.m, d.ldr, d.ldy))
    return fail(NUMBAT_ERR_BAD_DESC, "y in the residual's buffer needs its row stride (y %lld, residual %lld)",
                (long long)d.ldy, (long long)d.ldr);
  const Product pr = product(d, kGemmFwd);
  st = check_grid(pr);
  if (st != NUMBAT_OK) return st;
  st = check_ws(ws, ws_bytes, with_header(pr.bytes));
  if (st != NUMBAT_OK) return st;
  GemmEpilogue e;
  std::memset(&e, 0, sizeof e);
  e.act = d.act;
  e.out_f32 = d.y_f32;
  e.bias = bias;
  e.res = residual;
  e.z = static_cast<bf16_t*>(z);
  e.out = y;
  e.ldr = d.ldr;
  e.ldz = d.ldz;
  e.ldo = d.ldy;
  e.vec = d.n % 8 == 0 && d.ldy % 8 == 0 && (residual == nullptr || d.ldr % 8 == 0) && (z == nullptr || d.ldz % 8 == 0);
  const hipError_t err = run_product(pr, x, w, e, nullptr, ws_body(ws), static_cast<hipStream_t>(stream));
  return err == hipSuccess ? ok() : hip_fail(err, "linear forward launch");
}

numbat_status numbat_linear_bwd_data(const numbat_linear_problem* p, const void* dy, const void* w, const void* z,
                                     void* dx, int accumulate, void* ws, size_t ws_bytes, void* stream) {
  LinearDesc d;
  numbat_status st = check_linear(p, kGemmDgrad, &d);
  if (st != NUMBAT_OK) return st;
  if (d.m == 0) return ok();
  if (dy == nullptr || w == nullptr || dx == nullptr) return fail(NUMBAT_ERR_NULL, "dy, w and dx are required");
  if (d.act != NUMBAT_ACT_NONE && z == nullptr)
    return fail(NUMBAT_ERR_NULL, "z is required for the gradient of an activation");
  if (!aligned16(dy) || !aligned16(w) || !aligned16(dx) || !aligned16(z))
    return fail(NUMBAT_ERR_ALIGN, "dy, w, dx and z must be 16-byte aligned");
  const Product pr = product(d, kGemmDgrad);
  st = check_grid(pr);
  if (st != NUMBAT_OK) return st;
  st = check_ws(ws, ws_bytes, with_header(pr.bytes));
  if (st != NUMBAT_OK) return st;
  GemmEpilogue e;
  std::memset(&e, 0, sizeof e);
  e.act = d.act;
  e.accumulate = accumulate != 0;
  e.z = static_cast<bf16_t*>(const_cast<void*>(z));
  e.out = dx;
  e.ldz = d.ldz;
  e.ldo = d.ldx;
  e.vec = d.k % 8 == 0 && d.ldx % 8 == 0 && (d.act == NUMBAT_ACT_NONE || d.ldz % 8 == 0);
  const hipError_t err = run_product(pr, dy, w, e, nullptr, ws_body(ws), static_cast<hipStream_t>(stream));
  return err == hipSuccess ? ok() : hip_fail(err, "linear data gradient launch");
}

numbat_status numbat_linear_bwd_weight(const numbat_linear_problem* p, const void* x, const void* dy, float* dw,
                                       float* db, int accumulate, void* ws, size_t ws_bytes, void* stream) {
  LinearDesc d;
  numbat_status st = check_linear(p, kGemmWgrad, &d);
  if (st != NUMBAT_OK) return st;
  if (dw == nullptr || (d.m > 0 && (x == nullptr || dy == nullptr)))
    return fail(NUMBAT_ERR_NULL, "x, dy and dw are required");
  if (!aligned16(x) || !aligned16(dy)) return fail(NUMBAT_ERR_ALIGN, "x and dy must be 16-byte aligned");
  const Product pr = product(d, kGemmWgrad);
  st = check_grid(pr);
  if (st != NUMBAT_OK) return st;
  st = check_ws(ws, ws_bytes, with_header(pr.bytes));
  if (st != NUMBAT_OK) return st;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  hipError_t err = hipSuccess;
  if (d.m == 0) {  // empty sums
    if (!accumulate) err = fill_zero_launch(dw, (int64_t)d.n * d.k, s);
    if (!accumulate && err == hipSuccess && db != nullptr) err = fill_zero_launch(db, d.n, s);
    return err == hipSuccess ? ok() : hip_fail(err, "linear weight gradient launch");
  }
  GemmEpilogue e;
  std::memset(&e, 0, sizeof e);
  e.out_f32 = 1;
  e.accumulate = accumulate != 0;
  e.out = dw;
  e.ldo = d.k;
  e.vec = d.k % 8 == 0 && aligned16(dw);
  err = run_product(pr, dy, x, e, pr.sums_rows ? db : nullptr, ws_body(ws), s);
  if (err == hipSuccess && db != nullptr && !pr.sums_rows)
    err = colsum_launch(static_cast<const bf16_t*>(dy), d.ldy, d.m, d.n,
                        reinterpret_cast<float*>(static_cast<char*>(ws_body(ws)) + pr.db_at), db, accumulate != 0, s);
  return err == hipSuccess ? ok() : hip_fail(err, "linear weight gradient launch");
}

numbat_status numbat_layer_norm_fwd(const numbat_layer_norm_problem* p, const void* x, const float* gamma,
                                    const float* beta, void* y, float* mean, float* rstd, void* stream) {
  LnArgs a;
  numbat_status st = check_ln(p, &a);
  if (st != NUMBAT_OK) return st;
  if (a.m == 0) return ok();
  if (x == nullptr || y == nullptr) return fail(NUMBAT_ERR_NULL, "x and y are required");
  if (!aligned16(x) || !aligned16(y)) return fail(NUMBAT_ERR_ALIGN, "x and y must be 16-byte aligned");
  if (x == y && (a.x_f32 != a.y_f32 || !in_place_ok(x, y, a.m, a.ldx, a.ldy)))
    return fail(NUMBAT_ERR_BAD_DESC, "y in x's buffer needs its type and row stride (y %lld, x %lld)", (long long)a.ldy,
                (long long)a.ldx);
  a.vec = a.c % 8 == 0 && a.ldx % 8 == 0 && a.ldy % 8 == 0 && aligned16(gamma) && aligned16(beta);
  const hipError_t e = ln_fwd_launch(a, x, gamma, beta, y, mean, rstd, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? ok() : hip_fail(e, "layer norm forward launch");
}

numbat_status numbat_layer_norm_bwd(const numbat_layer_norm_problem* p, const void* dy, const void* x,
                                    const float* mean, const float* rstd, const float* gamma,
                                    const void* residual_grad, void* dx, float* dgamma, float* dbeta, int accumulate,
                                    void* ws, size_t ws_bytes, void* stream) {
  LnArgs a;
  numbat_status st = check_ln(p, &a);
  if (st != NUMBAT_OK) return st;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  hipError_t e = hipSuccess;
  if (a.m == 0) {  // empty sums
    if (!accumulate && dgamma != nullptr) e = fill_zero_launch(dgamma, a.c, s);
    if (!accumulate && dbeta != nullptr && e == hipSuccess) e = fill_zero_launch(dbeta, a.c, s);
    return e == hipSuccess ? ok() : hip_fail(e, "layer norm backward launch");
  }
  if (dy == nullptr || x == nullptr || mean == nullptr || rstd == nullptr)
    return fail(NUMBAT_ERR_NULL, "dy, x, mean and rstd are required");
  if (dx == nullptr && dgamma == nullptr && dbeta == nullptr)
    return fail(NUMBAT_ERR_NULL, "at least one of dx, dgamma and dbeta is required");
  if (dx == nullptr && residual_grad != nullptr) return fail(NUMBAT_ERR_NULL, "residual_grad needs dx");
  if (!aligned16(dy) || !aligned16(x) || !aligned16(residual_grad) || !aligned16(dx))
    return fail(NUMBAT_ERR_ALIGN, "dy, x, residual_grad and dx must be 16-byte aligned");
  if (!in_place_ok(residual_grad, dx, a.m, a.ldr, a.lddx))
    return fail(NUMBAT_ERR_BAD_DESC, "dx in residual_grad's buffer needs its row stride (dx %lld, residual_grad %lld)",
                (long long)a.lddx, (long long)a.ldr);
  st = check_ws(ws, ws_bytes, with_header(ln_bwd_ws(a)));
  if (st != NUMBAT_OK) return st;
  a.vec = a.c % 8 == 0 && a.ldx % 8 == 0 && a.ldy % 8 == 0 && (residual_grad == nullptr || a.ldr % 8 == 0) &&
          (dx == nullptr || a.lddx % 8 == 0) && aligned16(gamma);
  e = ln_bwd_launch(a, dy, x, mean, rstd, gamma, residual_grad, dx, dgamma, dbeta, accumulate != 0,
                    static_cast<float*>(ws_body(ws)), s);
  return e == hipSuccess ? ok() : hip_fail(e, "layer norm backward launch");
}

static_assert(sizeof(numbat_adamw_tensor) == sizeof(AdamTensor) &&
                  offsetof(numbat_adamw_tensor, w_copy) == offsetof(AdamTensor, w_copy) &&
                  offsetof(numbat_adamw_tensor, n) == offsetof(AdamTensor, n) &&
                  offsetof(numbat_adamw_tensor, grad_type) == offsetof(AdamTensor, g_type),
              "numbat_adamw_tensor and AdamTensor share one layout");

numbat_status numbat_adamw_step(const numbat_adamw_tensor* tensors, int32_t count, const numbat_sgd_group* groups,
                                int32_t ngroups, int32_t state_bits, double beta1, double beta2, double eps,
                                int64_t step, double max_norm, float* total_norm, void* ws, size_t ws_bytes,
                                void* stream) {
  if (tensors == nullptr || groups == nullptr) return fail(NUMBAT_ERR_NULL, "tensors and groups are required");
  if (reinterpret_cast<uintptr_t>(tensors) & 7u) return fail(NUMBAT_ERR_ALIGN, "tensors must be 8-byte aligned");
  if (reinterpret_cast<uintptr_t>(total_norm) & 3u) return fail(NUMBAT_ERR_ALIGN, "total_norm must be 4-byte aligned");
  if (count < 1 || count > kAdamMaxTensors)
    return fail(NUMBAT_ERR_BAD_DESC, "count = %d: 1 .. %d tensors", count, kAdamMaxTensors);
  if (ngroups < 1 || ngroups > kOptMaxGroups)
    return fail(NUMBAT_ERR_BAD_DESC, "ngroups = %d: 1 .. %d groups", ngroups, kOptMaxGroups);
  if (state_bits != 32 && state_bits != 8) return fail(NUMBAT_ERR_UNSUPPORTED, "state_bits = %d: 32 or 8", state_bits);
  if (!(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0))
    return fail(NUMBAT_ERR_BAD_DESC, "beta1 and beta2 must be in [0, 1)");
  // (the kernels take both in fp32: an eps that is no normal number there has no finite reciprocal)
  if (!((float)eps >= FLT_MIN && eps < 3.0e38))
    return fail(NUMBAT_ERR_BAD_DESC, "eps must be at least 2^-126 and finite");
  if (step < 1) return fail(NUMBAT_ERR_BAD_DESC, "step = %lld: the first step is 1", (long long)step);
  if (!(max_norm == 0.0 || ((float)max_norm >= FLT_MIN && max_norm < 3.0e38)))
    return fail(NUMBAT_ERR_BAD_DESC, "max_norm must be at least 2^-126 and finite, or 0 for no clipping");
  if (total_norm != nullptr && max_norm == 0.0)
    return fail(NUMBAT_ERR_BAD_DESC, "total_norm is formed only with max_norm > 0");
  AdamArgs a;
  std::memset(&a, 0, sizeof a);
  for (int i = 0; i < ngroups; ++i) {
    const float lr = groups[i].lr, wd = groups[i].weight_decay;
    if (!(lr >= 0.0f && lr < 3.0e38f) || !(wd >= 0.0f && wd < 3.0e38f))
      return fail(NUMBAT_ERR_BAD_DESC, "group %d: lr and weight_decay must be finite and >= 0", i);
    a.lr[i] = (float)((double)lr / (1.0 - std::pow(beta1, (double)step)));
    a.keep[i] = (float)(1.0 - (double)lr * (double)wd);
  }
  numbat_status st = check_ws(ws, ws_bytes, with_header(kAdamWs));
  if (st != NUMBAT_OK) return st;
  a.tab = reinterpret_cast<const AdamTensor*>(tensors);
  a.count = count;
  a.ngroups = ngroups;
  a.b1 = (float)beta1;
  a.omb1 = (float)(1.0 - beta1);
  a.b2 = (float)beta2;
  a.omb2 = (float)(1.0 - beta2);
  a.eps = (float)eps;
  a.rsqrt_bc2 = (float)(1.0 / std::sqrt(1.0 - std::pow(beta2, (double)step)));
  a.max_norm = (float)max_norm;
  a.total_norm = total_norm;
  a.part = static_cast<double*>(ws_body(ws));
  const hipError_t e = adamw_launch(a, state_bits, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? ok() : hip_fail(e, "AdamW step launch");
}

numbat_status numbat_adamw_state_values(int64_t n, const void* m, const float* m_unit, const void* v,
                                        const float* v_unit, float* m_value, float* v_value, void* stream) {
  if (n < 0) return fail(NUMBAT_ERR_BAD_DESC, "n must be >= 0");
  if (n == 0) return ok();
  if (m == nullptr || m_unit == nullptr || v == nullptr || v_unit == nullptr || m_value == nullptr || v_value == nullptr)
    return fail(NUMBAT_ERR_NULL, "m, m_unit, v, v_unit, m_value and v_value are required");
  const hipError_t e = adamw_values_launch(n, static_cast<const int8_t*>(m), m_unit, static_cast<const uint8_t*>(v),
                                           v_unit, m_value, v_value, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? ok() : hip_fail(e, "AdamW state values launch");
}

}  // extern "C"
