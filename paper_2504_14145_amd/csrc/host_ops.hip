// host_ops.hip -- entry points of the stage operators: argument checks,
// workspaces and launches.  Nothing here allocates or throws.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "host_state.h"
#include "ops_internal.h"

namespace {

using namespace dipops;
using dipsim_host::g_last_hip;

int elem_bytes(int32_t t) { return t == DIP_F32 ? 4 : 2; }
bool known_type(int32_t t) { return t == DIP_F32 || t == DIP_F16 || t == DIP_BF16; }
bool known_act(int32_t a) { return a >= DIP_ACT_NONE && a <= DIP_ACT_GELU; }

constexpr int64_t kMaxRows = int64_t(1) << 31;     // rows of an array
constexpr int64_t kMaxCols = int64_t(1) << 22;     // columns and strides of a matrix: 256 rows of 2-byte elements stay below 2^31 bytes

int hip_code(hipError_t e) {
  if (e == hipSuccess) return DIP_OK;
  g_last_hip = e;
  return DIP_E_HIP;
}

// A row-major array that a call reads or writes: null only where nothing is
// accessed, aligned to its element, rows that do not overlap.
int check_matrix(const void *p, int64_t rows, int64_t cols, int64_t ld, int elem) {
  if (rows == 0 || cols == 0) return DIP_OK;
  if (!p || reinterpret_cast<uintptr_t>(p) % elem) return DIP_E_INVAL;
  if (ld < cols) return DIP_E_INVAL;
  if (ld > kMaxCols) return DIP_E_RANGE;
  return DIP_OK;
}
int check_vector(const void *p, int elem) {
  return p && reinterpret_cast<uintptr_t>(p) % elem ? DIP_E_INVAL : DIP_OK;
}
int check_drop(const dip_dropout &d, int64_t rows) {
  if (d.drop_of > 65535) return DIP_E_INVAL;
  if (d.drop_of && int64_t(d.row0) + rows > (int64_t(1) << 32)) return DIP_E_RANGE;
  return DIP_OK;
}
int check_sizes(int64_t m, int64_t n, int64_t k) {
  if (m < 0 || n < 0 || k < 0) return DIP_E_INVAL;
  if (m >= kMaxRows || n > kMaxCols || k > kMaxCols) return DIP_E_RANGE;
  // outputs are m x n, m x k and n x k: a launch's workgroups of 256 threads, each with
  // 256 x 256 elements of one, have fewer than 2^32 threads
  const int64_t tm = (m + 255) / 256, tn = (n + 255) / 256, tk = (k + 255) / 256;
  if (tm * std::max(tn, tk) >= kMaxTiles || tn * tk >= kMaxTiles) return DIP_E_RANGE;
  return DIP_OK;
}
int check_workspace(const void *p, int64_t have, int64_t need) {
  if (need == 0) return DIP_OK;
  if (have < need) return DIP_E_CAPACITY;
  return p && reinterpret_cast<uintptr_t>(p) % 16 == 0 ? DIP_OK : DIP_E_INVAL;
}

#define OPS_CHECK(expr)                 \
  do {                                  \
    const int rc_ = (expr);             \
    if (rc_ != DIP_OK) return rc_;      \
  } while (0)

int check_linear(const dip_linear_args *a) {
  if (!a || !known_type(a->dtype) || !known_act(a->act)) return DIP_E_INVAL;
  if (a->dtype == DIP_F32) return DIP_E_UNSUPPORTED;
  OPS_CHECK(check_sizes(a->m, a->n, a->k));
  OPS_CHECK(check_drop(a->drop, a->m));
  OPS_CHECK(check_matrix(a->x, a->m, a->k, a->ldx, 2));
  OPS_CHECK(check_matrix(a->w, a->n, a->k, a->ldw, 2));
  OPS_CHECK(check_matrix(a->y, a->m, a->n, a->ldy, 2));
  OPS_CHECK(check_vector(a->bias, 2));
  if (a->residual) OPS_CHECK(check_matrix(a->residual, a->m, a->n, a->ldr, 2));
  if (a->pre) OPS_CHECK(check_matrix(a->pre, a->m, a->n, a->ldp, 2));
  return DIP_OK;
}

// A matrix in 8 bits that a call reads or writes.
int check_packed(const dip_packed8 &p, int64_t rows, int64_t cols) {
  OPS_CHECK(check_matrix(p.values, rows, cols, p.ld, 1));
  return check_matrix(p.scales, rows, (cols + 31) / 32, p.lds, 1);
}

int check_linear_kept(const dip_linear_args *a, const dip_packed8 *pre) {
  if (!a || !pre) return DIP_E_INVAL;
  dip_linear_args b = *a;
  b.pre = nullptr;
  OPS_CHECK(check_linear(&b));
  return check_packed(*pre, a->m, a->n);
}

// x8 and pre8: what is read in the place of a->x and a->pre, or null
int check_linear_grad(const dip_linear_grad_args *a, const dip_packed8 *x8 = nullptr, const dip_packed8 *pre8 = nullptr,
                      int32_t x_act = DIP_ACT_NONE) {
  if (!a || !known_type(a->dtype) || !known_act(a->act)) return DIP_E_INVAL;
  if (a->dtype == DIP_F32) return DIP_E_UNSUPPORTED;
  if (a->grad_dtype != a->dtype && a->grad_dtype != DIP_F32) return DIP_E_INVAL;
  OPS_CHECK(check_sizes(a->m, a->n, a->k));
  OPS_CHECK(check_drop(a->drop, a->m));
  if (a->dx || a->dw || a->db) {
    OPS_CHECK(check_matrix(a->dy, a->m, a->n, a->ldy, 2));
    if (a->act != DIP_ACT_NONE)
      OPS_CHECK(pre8 ? check_packed(*pre8, a->m, a->n) : check_matrix(a->pre, a->m, a->n, a->ldp, 2));
  }
  if (x8 && !known_act(x_act)) return DIP_E_INVAL;
  const int ge = elem_bytes(a->grad_dtype);
  if (a->dx) {
    OPS_CHECK(check_matrix(a->w, a->n, a->k, a->ldw, 2));
    OPS_CHECK(check_matrix(a->dx, a->m, a->k, a->lddx, 2));
  }
  if (a->dw) {
    OPS_CHECK(x8 ? check_packed(*x8, a->m, a->k) : check_matrix(a->x, a->m, a->k, a->ldx, 2));
    OPS_CHECK(check_matrix(a->dw, a->n, a->k, a->lddw, ge));
  }
  return check_vector(a->db, ge);
}

int64_t up8(int64_t n) { return (n + 7) / 8 * 8; }

// Whether the products can read an array where it is: aligned rows, and along a
// contraction that ends inside 16 bytes the zeros that only a copy has.
bool direct(const void *p, int64_t ld, int64_t cols, bool contracted) {
  return aligned16(p, ld, 2) && !(contracted && cols % 8);
}

// The workspace: arrays one after another, 16-byte aligned.
struct Space {
  int64_t total = 0;
  int64_t take(int64_t bytes) {
    const int64_t at = total;
    total += up16(bytes);
    return at;
  }
};

struct LinearPlan {
  GemmPlan gemm;
  int64_t x_at = -1, w_at = -1, partial_at = 0, total = 0;   // -1: read in place
};
LinearPlan plan_linear(const dip_linear_args *a, bool kept = false) {
  LinearPlan p;
  if (a->m == 0 || a->n == 0 || (!kept && thin(a->m, a->n, a->k))) return p;
  Space s;
  p.gemm = plan_gemm(a->m, a->n, a->k, true);
  if (!direct(a->x, a->ldx, a->k, true)) p.x_at = s.take(a->m * up8(a->k) * 2);
  if (!direct(a->w, a->ldw, a->k, true)) p.w_at = s.take(a->n * up8(a->k) * 2);
  p.partial_at = s.take(p.gemm.bytes);
  p.total = s.total;
  return p;
}

// Whether an activation or its slope has values that the operands' type does not hold.
bool rounded(int32_t act) { return act == DIP_ACT_SILU || act == DIP_ACT_GELU; }

struct GradPlan {
  GemmPlan dx, dw;
  bool pair = false;
  // dw's rows of g and x: m, or twice as many, g again below itself and below x what
  // rounding it left off.  Where g comes through one activation and x through another both
  // are rounded, and dw would be sqrt(3) of its own rounding's error off in the place of
  // the sqrt(2) that any other product's gradient is; this takes x's part back for one more
  // product (gradients behind GELU, of an x without and behind SiLU, bf16: 1152 x 1792 x
  // 3840 54 and 79 us, 8192 x 3584 x 4096 408 and 616).
  int64_t rows = 0;
  int64_t g_at = -1, x_at = -1, w_at = -1, sums_at = -1, partial_at = 0, total = 0;
  int32_t chunks = 0;
};
GradPlan plan_grad(const dip_linear_grad_args *a, bool x8 = false, int32_t x_act = DIP_ACT_NONE) {
  GradPlan p;
  if (a->m == 0 || a->n == 0) return p;
  Space s;
  p.rows = a->dw && x8 && rounded(x_act) && rounded(a->act) ? 2 * a->m : a->m;
  // g needs an array of its own where it is not dy itself or dy cannot be read
  // in place
  if ((a->dx || a->dw) &&
      (a->act != DIP_ACT_NONE || a->drop.drop_of || !direct(a->dy, a->ldy, a->n, a->dx != nullptr)))
    p.g_at = s.take(p.rows * up8(a->n) * 2);
  if (a->db) {
    p.chunks = grad_row_chunks(a->m, a->n);
    p.sums_at = s.take(int64_t(p.chunks) * a->n * 4);
  }
  int64_t partial = 0;
  if (a->dx && a->k > 0) {
    if (!direct(a->w, a->ldw, a->k, false)) p.w_at = s.take(a->n * up8(a->k) * 2);
    p.dx = plan_gemm(a->m, a->k, a->n, true);
    partial = p.dx.bytes;
  }
  if (a->dw && a->k > 0) {
    if (x8 || !direct(a->x, a->ldx, a->k, false)) p.x_at = s.take(p.rows * up8(a->k) * 2);
    p.dw = plan_gemm(a->n, a->k, p.rows, false);
    partial = partial > p.dw.bytes ? partial : p.dw.bytes;
  }
  // the two products run one after the other, or in one launch
  p.pair = a->dx && a->dw && a->k > 0 && pair_gemms(a->m, a->k, p.dx, a->n, a->k, p.dw);
  p.partial_at = s.take(p.pair ? p.dx.bytes + p.dw.bytes : partial);
  p.total = s.total;
  return p;
}

// An operand of a product: in place, or the copy that `job` is to make.
Operand place(const void *p, int64_t rows, int64_t cols, int64_t ld, bool k_rows, char *ws, int64_t at, PackJob *job) {
  if (at < 0 || rows == 0 || cols == 0) return Operand{p, ld, k_rows};
  *job = PackJob{p, rows, cols, ld, ws + at, up8(cols)};
  return Operand{job->out, job->ldo, k_rows};
}
int pack(int dtype, const PackJob &a, const PackJob &b, hipStream_t st) {
  return a.rows || b.rows ? hip_code(launch_pack(dtype, a, b, st)) : int(DIP_OK);
}

// dip_linear's epilogue, pre aside
Epilogue epilogue(const dip_linear_args *a) {
  Epilogue e{};
  e.bias = a->bias;
  e.residual = a->residual;
  e.out = a->y;
  e.ldr = a->ldr;
  e.ldo = a->ldy;
  e.ldp = a->ldp;
  e.drop = make_drop(a->drop);
  e.scale = 1.f;
  e.act = a->act;
  return e;
}
// its operands, where the plan has them
int operands(const dip_linear_args *a, const LinearPlan &p, hipStream_t st, Operand *x, Operand *w) {
  char *ws = static_cast<char *>(a->workspace);
  PackJob px, pw;
  *x = place(a->x, a->m, a->k, a->ldx, false, ws, p.x_at, &px);
  *w = place(a->w, a->n, a->k, a->ldw, false, ws, p.w_at, &pw);
  return pack(a->dtype, px, pw, st);
}
float *partial_of(const dip_linear_args *a, const LinearPlan &p) {
  return reinterpret_cast<float *>(static_cast<char *>(a->workspace) + p.partial_at);
}

// dip_linear_grad; x8 and pre8, if given, in the place of a->x and a->pre
int linear_grad(const dip_linear_grad_args *a, const dip_packed8 *x8, int32_t x_act, const dip_packed8 *pre8, void *stream) {
  OPS_CHECK(check_linear_grad(a, x8, pre8, x_act));
  const GradPlan p = plan_grad(a, x8 != nullptr, x_act);
  const bool twice = p.rows > a->m;
  OPS_CHECK(check_workspace(a->workspace, a->workspace_bytes, p.total));
  const hipStream_t st = hipStream_t(stream);
  char *ws = static_cast<char *>(a->workspace);
  const Drop drop = make_drop(a->drop);
  const void *g = a->dy;
  int64_t ldg = a->ldy;
  float *partial = reinterpret_cast<float *>(ws + p.partial_at);
  PackJob px, pw;
  const Operand w = place(a->w, a->dx ? a->n : 0, a->k, a->ldw, true, ws, p.w_at, &pw);
  Operand x;
  Restore rx{};
  if (x8) {
    x = Operand{p.x_at >= 0 ? ws + p.x_at : nullptr, up8(a->k), true};
    if (p.x_at >= 0) {
      char *to = ws + p.x_at;
      rx = Restore{make_packed(*x8), a->m, int32_t(a->k), x_act, to, twice ? to + a->m * up8(a->k) * 2 : nullptr, up8(a->k)};
    }
  } else {
    x = place(a->x, a->dw ? a->m : 0, a->k, a->ldx, true, ws, p.x_at, &px);
  }
  if (p.g_at >= 0 || p.sums_at >= 0) {
    GradIn gi{};
    gi.m = a->m;
    gi.n = a->n;
    gi.dy = a->dy;
    gi.pre = a->act != DIP_ACT_NONE && !pre8 ? a->pre : nullptr;
    if (a->act != DIP_ACT_NONE && pre8) gi.kept = make_packed(*pre8);
    gi.ldy = a->ldy;
    gi.ldp = a->ldp;
    gi.drop = drop;
    gi.act = a->act;
    if (p.g_at >= 0) {
      g = gi.out = ws + p.g_at;
      ldg = gi.ldo = up8(a->n);
      if (twice) gi.again = ws + p.g_at + a->m * ldg * 2;
    }
    gi.row_chunks = p.chunks ? p.chunks : grad_row_chunks(a->m, a->n);
    gi.partial = a->db ? reinterpret_cast<float *>(ws + p.sums_at) : nullptr;
    if (rx.m && grad_in_kept_fits(gi, rx, pw)) {
      OPS_CHECK(hip_code(launch_grad_in_kept(a->dtype, gi, rx, pw, st)));
      rx.m = 0;
      pw = PackJob{};
    } else {
      OPS_CHECK(hip_code(launch_grad_in(a->dtype, gi, st)));
    }
  }
  if (a->db && a->n > 0 && !(a->m == 0 && a->accumulate))
    OPS_CHECK(hip_code(launch_sum_rows(SumRows{reinterpret_cast<const float *>(ws + p.sums_at), p.chunks, a->n, a->n,
                                               a->db, nullptr, a->accumulate},
                                       a->grad_dtype, st)));
  if (rx.m)
    OPS_CHECK(hip_code(launch_unpack8(a->dtype, rx.m, rx.n, rx.x, rx.act, rx.out, rx.ldo, rx.ldo, st, rx.low)));
  OPS_CHECK(pack(a->dtype, px, pw, st));
  Gemm gx{a->m, a->k, a->n, Operand{g, ldg, false}, w, {}, p.dx, partial};
  gx.e.out = a->dx;
  gx.e.ldo = a->lddx;
  gx.e.scale = drop.scale;
  Gemm gw{a->n, a->k, p.rows, Operand{g, ldg, true}, x, {}, p.dw, p.pair ? partial + p.dx.bytes / 4 : partial};
  gw.e.out = a->dw;
  gw.e.ldo = a->lddw;
  gw.e.scale = drop.scale;
  gw.e.out_f32 = a->grad_dtype == DIP_F32;
  gw.e.accumulate = a->accumulate != 0;
  if (p.pair) return hip_code(launch_gemm_pair(a->dtype, gx, gw, st));
  if (a->dx && a->m > 0 && a->k > 0)
    OPS_CHECK(hip_code(launch_gemm(a->dtype, gx.m, gx.n, gx.k, gx.a, gx.b, gx.e, gx.plan, gx.partial, st)));
  if (a->dw && a->n > 0 && a->k > 0)
    OPS_CHECK(hip_code(launch_gemm(a->dtype, gw.m, gw.n, gw.k, gw.a, gw.b, gw.e, gw.plan, gw.partial, st)));
  return DIP_OK;
}

int check_norm(int64_t b, int64_t s, int64_t c, int32_t groups, int32_t dtype, int32_t act) {
  if (!known_type(dtype) || !known_act(act)) return DIP_E_INVAL;
  if (b < 0 || s < 0 || c < 0 || groups < 1 || c % groups) return DIP_E_INVAL;
  if (b >= kMaxRows || s >= kMaxRows || c > kMaxCols) return DIP_E_RANGE;
  if (b * groups > INT32_MAX || s * (c / groups) > (int64_t(1) << 40)) return DIP_E_RANGE;
  return DIP_OK;
}
// [b][s][c] with the given strides: positions and samples that do not overlap, either
// of them the outer one; a stride that nothing steps over may be anything
int check_rows(const void *p, int64_t b, int64_t s, int64_t c, int64_t sb, int64_t ss, int elem) {
  if (b == 0 || s == 0 || c == 0) return DIP_OK;
  if (!p || reinterpret_cast<uintptr_t>(p) % elem) return DIP_E_INVAL;
  if ((s > 1 && ss < c) || (b > 1 && sb < c)) return DIP_E_INVAL;
  if ((s > 1 && ss > (int64_t(1) << 46)) || (b > 1 && sb > (int64_t(1) << 46))) return DIP_E_RANGE;
  if (b == 1 || s == 1) return DIP_OK;
  // outer >= (n - 1) inner + c, without the product
  const int64_t outer = std::max(sb, ss), inner = std::min(sb, ss), n = sb >= ss ? s : b;
  return (outer - c) / inner >= n - 1 ? DIP_OK : DIP_E_INVAL;
}

int check_group_norm(const dip_group_norm_args *a) {
  if (!a) return DIP_E_INVAL;
  OPS_CHECK(check_norm(a->b, a->s, a->c, a->groups, a->dtype, a->act));
  if (!(a->eps >= 0.f)) return DIP_E_INVAL;
  const int e = elem_bytes(a->dtype);
  OPS_CHECK(check_rows(a->x, a->b, a->s, a->c, a->x_sb, a->x_ss, e));
  OPS_CHECK(check_rows(a->y, a->b, a->s, a->c, a->y_sb, a->y_ss, e));
  OPS_CHECK(check_vector(a->gamma, e));
  OPS_CHECK(check_vector(a->beta, e));
  OPS_CHECK(check_vector(a->mean, 4));
  return check_vector(a->rstd, 4);
}

int check_group_norm_grad(const dip_group_norm_grad_args *a) {
  if (!a) return DIP_E_INVAL;
  OPS_CHECK(check_norm(a->b, a->s, a->c, a->groups, a->dtype, a->act));
  const int e = elem_bytes(a->dtype);
  OPS_CHECK(check_rows(a->dy, a->b, a->s, a->c, a->dy_sb, a->dy_ss, e));
  OPS_CHECK(check_rows(a->x, a->b, a->s, a->c, a->x_sb, a->x_ss, e));
  if (a->dx) OPS_CHECK(check_rows(a->dx, a->b, a->s, a->c, a->dx_sb, a->dx_ss, e));
  if (a->b * a->groups > 0 && a->s > 0 && a->c > 0 && (!a->mean || !a->rstd)) return DIP_E_INVAL;
  OPS_CHECK(check_vector(a->mean, 4));
  OPS_CHECK(check_vector(a->rstd, 4));
  OPS_CHECK(check_vector(a->gamma, e));
  OPS_CHECK(check_vector(a->beta, e));
  OPS_CHECK(check_vector(a->dgamma, a->accumulate ? 4 : e));
  return check_vector(a->dbeta, a->accumulate ? 4 : e);
}

int check_rms_norm(const dip_rms_norm_args *a) {
  if (!a || !known_type(a->dtype) || !(a->eps >= 0.f)) return DIP_E_INVAL;
  OPS_CHECK(check_sizes(a->m, a->c, 0));
  const int e = elem_bytes(a->dtype);
  OPS_CHECK(check_matrix(a->x, a->m, a->c, a->ldx, e));
  if (a->residual) OPS_CHECK(check_matrix(a->residual, a->m, a->c, a->ldr, e));
  if (a->total) OPS_CHECK(check_matrix(a->total, a->m, a->c, a->ldt, e));
  if (a->y) OPS_CHECK(check_matrix(a->y, a->m, a->c, a->ldy, e));
  if (a->packed.values || a->packed.scales) OPS_CHECK(check_packed(a->packed, a->m, a->c));
  OPS_CHECK(check_vector(a->gamma, e));
  return check_vector(a->rstd, 4);
}

int check_rms_norm_grad(const dip_rms_norm_grad_args *a) {
  if (!a || !known_type(a->dtype)) return DIP_E_INVAL;
  OPS_CHECK(check_sizes(a->m, a->c, 0));
  const int e = elem_bytes(a->dtype);
  if (a->dx || a->dgamma) {
    OPS_CHECK(check_matrix(a->dy, a->m, a->c, a->ldy, e));
    OPS_CHECK(check_matrix(a->total, a->m, a->c, a->ldt, e));
    if (a->m > 0 && a->c > 0 && !a->rstd) return DIP_E_INVAL;
  }
  if (a->dx) {
    OPS_CHECK(check_matrix(a->dx, a->m, a->c, a->lddx, e));
    if (a->dtotal) OPS_CHECK(check_matrix(a->dtotal, a->m, a->c, a->lddt, e));
  }
  OPS_CHECK(check_vector(a->rstd, 4));
  OPS_CHECK(check_vector(a->gamma, e));
  return check_vector(a->dgamma, a->accumulate ? 4 : e);
}

// [t][heads][dim] with the given strides, as check_rows
int check_heads(const void *p, const dip_rotary_args *a, int32_t heads, int64_t st, int64_t sh) {
  return check_rows(p, a->t, heads, a->dim, st, sh, elem_bytes(a->dtype));
}
int check_rotary(const dip_rotary_args *a) {
  if (!a || !known_type(a->dtype) || a->pos_type < DIP_POS_I32 || a->pos_type > DIP_POS_F32) return DIP_E_INVAL;
  if (a->t < 0 || a->heads < 0 || a->keys < 0 || a->dim < 0 || a->pairs < 0 || a->axes < 0 || 2 * int64_t(a->pairs) > a->dim)
    return DIP_E_INVAL;
  if (a->t >= kMaxRows || a->dim > 2048 || int64_t(a->heads) + a->keys > 65536) return DIP_E_RANGE;
  OPS_CHECK(check_heads(a->q, a, a->heads, a->q_st, a->q_sh));
  OPS_CHECK(check_heads(a->q_out, a, a->heads, a->qo_st, a->qo_sh));
  OPS_CHECK(check_heads(a->k, a, a->keys, a->k_st, a->k_sh));
  OPS_CHECK(check_heads(a->k_out, a, a->keys, a->ko_st, a->ko_sh));
  if (a->t == 0 || a->heads + a->keys == 0 || a->pairs == 0) return DIP_OK;
  if (!a->freq || reinterpret_cast<uintptr_t>(a->freq) % 8 || !a->axis || reinterpret_cast<uintptr_t>(a->axis) % 4)
    return DIP_E_INVAL;
  const int pe = a->pos_type == DIP_POS_I64 ? 8 : 4;
  if (a->axes > 0 && (!a->pos || reinterpret_cast<uintptr_t>(a->pos) % pe)) return DIP_E_INVAL;
  constexpr int64_t most = int64_t(1) << 46;   // positions may lie anyhow, also one for all tokens
  const int64_t st = a->p_st < 0 ? -a->p_st : a->p_st, sa = a->p_sa < 0 ? -a->p_sa : a->p_sa;
  return (a->t > 1 && st > most) || (a->axes > 1 && sa > most) ? DIP_E_RANGE : DIP_OK;
}

}  // namespace

extern "C" {

int64_t dip_linear_workspace(const dip_linear_args *a) {
  OPS_CHECK(check_linear(a));
  return plan_linear(a).total;
}

int dip_linear(const dip_linear_args *a, void *stream) {
  OPS_CHECK(check_linear(a));
  const LinearPlan p = plan_linear(a);
  OPS_CHECK(check_workspace(a->workspace, a->workspace_bytes, p.total));
  if (a->m == 0 || a->n == 0) return DIP_OK;
  const hipStream_t st = hipStream_t(stream);
  Epilogue e = epilogue(a);
  e.pre = a->pre;
  if (thin(a->m, a->n, a->k))
    return hip_code(launch_thin(a->dtype, a->m, a->n, a->k, a->x, a->ldx, a->w, a->ldw, e, st));
  Operand x, w;
  OPS_CHECK(operands(a, p, st, &x, &w));
  return hip_code(launch_gemm(a->dtype, a->m, a->n, a->k, x, w, e, p.gemm, partial_of(a, p), st));
}

int64_t dip_linear_kept_workspace(const dip_linear_args *a, const dip_packed8 *pre) {
  OPS_CHECK(check_linear_kept(a, pre));
  return plan_linear(a, true).total;
}

int dip_linear_kept(const dip_linear_args *a, const dip_packed8 *pre, void *stream) {
  OPS_CHECK(check_linear_kept(a, pre));
  const LinearPlan p = plan_linear(a, true);
  OPS_CHECK(check_workspace(a->workspace, a->workspace_bytes, p.total));
  if (a->m == 0 || a->n == 0) return DIP_OK;
  const hipStream_t st = hipStream_t(stream);
  KeptEpilogue e{epilogue(a), make_packed(*pre)};
  Operand x, w;
  OPS_CHECK(operands(a, p, st, &x, &w));
  return hip_code(launch_gemm_kept(a->dtype, a->m, a->n, a->k, x, w, e, p.gemm, partial_of(a, p), st));
}

int64_t dip_linear_grad_workspace(const dip_linear_grad_args *a) {
  OPS_CHECK(check_linear_grad(a));
  return plan_grad(a).total;
}

int dip_linear_grad(const dip_linear_grad_args *a, void *stream) {
  return linear_grad(a, nullptr, DIP_ACT_NONE, nullptr, stream);
}

int64_t dip_linear_grad_kept_workspace(const dip_linear_grad_args *a, const dip_packed8 *x, int32_t x_act,
                                       const dip_packed8 *pre) {
  OPS_CHECK(check_linear_grad(a, x, pre, x_act));
  return plan_grad(a, x != nullptr, x_act).total;
}

int dip_linear_grad_kept(const dip_linear_grad_args *a, const dip_packed8 *x, int32_t x_act, const dip_packed8 *pre,
                         void *stream) {
  return linear_grad(a, x, x_act, pre, stream);
}

int dip_pack8(int32_t dtype, int64_t m, int64_t n, const void *x, int64_t ldx, const dip_packed8 *out, void *stream) {
  if (!out || !known_type(dtype)) return DIP_E_INVAL;
  OPS_CHECK(check_sizes(m, n, 0));
  OPS_CHECK(check_matrix(x, m, n, ldx, elem_bytes(dtype)));
  OPS_CHECK(check_packed(*out, m, n));
  if (m == 0 || n == 0) return DIP_OK;
  return hip_code(launch_pack8(dtype, m, n, x, ldx, make_packed(*out), hipStream_t(stream)));
}

int dip_unpack8(int32_t dtype, int64_t m, int64_t n, const dip_packed8 *x, int32_t act, void *y, int64_t ldy,
                void *stream) {
  if (!x || !known_type(dtype) || !known_act(act)) return DIP_E_INVAL;
  OPS_CHECK(check_sizes(m, n, 0));
  OPS_CHECK(check_packed(*x, m, n));
  OPS_CHECK(check_matrix(y, m, n, ldy, elem_bytes(dtype)));
  if (m == 0 || n == 0) return DIP_OK;
  return hip_code(launch_unpack8(dtype, m, n, make_packed(*x), act, y, ldy, n, hipStream_t(stream)));
}

int dip_rms_norm(const dip_rms_norm_args *a, void *stream) {
  OPS_CHECK(check_rms_norm(a));
  return hip_code(launch_rms_norm(*a, hipStream_t(stream)));
}

int64_t dip_rms_norm_grad_workspace(const dip_rms_norm_grad_args *a) {
  OPS_CHECK(check_rms_norm_grad(a));
  return rms_norm_grad_workspace(*a);
}

int dip_rms_norm_grad(const dip_rms_norm_grad_args *a, void *stream) {
  OPS_CHECK(check_rms_norm_grad(a));
  OPS_CHECK(check_workspace(a->workspace, a->workspace_bytes, rms_norm_grad_workspace(*a)));
  return hip_code(launch_rms_norm_grad(*a, hipStream_t(stream)));
}

int dip_rotary(const dip_rotary_args *a, void *stream) {
  OPS_CHECK(check_rotary(a));
  if (a->t == 0 || a->heads + a->keys == 0 || a->dim == 0) return DIP_OK;
  return hip_code(launch_rotary(*a, hipStream_t(stream)));
}

int dip_dropout_add(int32_t dtype, int64_t m, int64_t n, const void *x, int64_t ldx,
                    const void *residual, int64_t ldr, const dip_dropout *drop, void *y,
                    int64_t ldy, void *stream) {
  if (!drop || !known_type(dtype)) return DIP_E_INVAL;
  OPS_CHECK(check_sizes(m, n, 0));
  OPS_CHECK(check_drop(*drop, m));
  const int e = elem_bytes(dtype);
  OPS_CHECK(check_matrix(x, m, n, ldx, e));
  OPS_CHECK(check_matrix(y, m, n, ldy, e));
  if (residual) OPS_CHECK(check_matrix(residual, m, n, ldr, e));
  if (m == 0 || n == 0) return DIP_OK;
  return hip_code(launch_dropout_add(dtype, m, n, x, ldx, residual, ldr, make_drop(*drop), y, ldy,
                                     hipStream_t(stream)));
}

int64_t dip_group_norm_workspace(const dip_group_norm_args *a) {
  OPS_CHECK(check_group_norm(a));
  return group_norm_workspace(*a);
}

int dip_group_norm(const dip_group_norm_args *a, void *stream) {
  OPS_CHECK(check_group_norm(a));
  OPS_CHECK(check_workspace(a->workspace, a->workspace_bytes, group_norm_workspace(*a)));
  if (a->b == 0) return DIP_OK;
  return hip_code(launch_group_norm(*a, hipStream_t(stream)));
}

int64_t dip_group_norm_grad_workspace(const dip_group_norm_grad_args *a) {
  OPS_CHECK(check_group_norm_grad(a));
  return group_norm_grad_workspace(*a);
}

int dip_group_norm_grad(const dip_group_norm_grad_args *a, void *stream) {
  OPS_CHECK(check_group_norm_grad(a));
  OPS_CHECK(check_workspace(a->workspace, a->workspace_bytes, group_norm_grad_workspace(*a)));
  if (a->c == 0) return DIP_OK;
  return hip_code(launch_group_norm_grad(*a, hipStream_t(stream)));
}

}  // extern "C"
