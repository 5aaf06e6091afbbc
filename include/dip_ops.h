/*
 * dip_ops.h -- the operators that a pipeline stage runs, as kernels for one GPU.
 *
 * The cost tables of dip_sim.h (DIP, arXiv 2504.14145, Sec. 6.1) price a stage
 * operator by operator: matrix products, norms and element-wise work, forward
 * and backward.  These are such operators, so that their efficiency factors can
 * be measured on the card that the schedule is planned for (Sec. 7.4), and run:
 *
 *   dip_linear       y = residual + D(act(x w^T + bias))
 *   dip_linear_grad  its gradients of x, w and bias
 *   dip_dropout_add  y = residual + D(x), and with no residual its own gradient
 *   dip_group_norm   y = act(gamma (x - mean) rstd + beta), channels last
 *   dip_group_norm_grad
 *   dip_rms_norm     t = x + residual, y = gamma t rstd, also in 8 bits
 *   dip_rms_norm_grad
 *   dip_rotary       queries and keys turned by positions along several axes
 *   dip_pack8        activations kept in 8 bits (between the memory strategies of
 *   dip_unpack8      Sec. 5.3, keeping and recomputing), restored, and
 *   dip_linear_kept  written and read by the products and their gradients
 *   dip_linear_grad_kept
 *
 * D is dropout whose mask is a function of (seed, offset, row, column), never
 * stored: forward, backward and a recomputed forward (Sec. 5.3) draw the same
 * mask, and a piece of a sample that starts at row0 draws the sample's (Sec. 4).
 *
 * Conventions of all calls
 *  - Matrices are row-major with a leading stride in elements; the last
 *    dimension is contiguous.  Pointers are device pointers aligned to their
 *    element; 16-byte aligned rows run at full speed, others cost the products a
 *    copy into the workspace and the other operators little.
 *  - Sums, statistics and everything between inputs and outputs are held in
 *    float32; an output is rounded once (to nearest even), save where a comment
 *    below says otherwise.
 *  - Calls only enqueue kernels on stream (a hipStream_t; null: the default
 *    stream): no allocation, no synchronisation, nothing kept from one call to
 *    the next; they may be captured into a HIP graph.  The workspace belongs to
 *    the call until the stream has passed it.  Results do not depend on timing:
 *    no atomics, and the same call gives the same bits.
 *  - Outputs must not overlap inputs, except that y may be the residual itself
 *    (same pointer and stride), and dip_dropout_add's y may be its x.
 *  - Return DIP_OK or a negative code of dip_sim.h; arguments are checked on
 *    the host before anything is launched: DIP_E_INVAL (null or misaligned
 *    pointers, negative sizes, strides below the row, unknown type or
 *    activation, overlapping shapes), DIP_E_RANGE (sizes beyond the kernels'
 *    index range: 2^31 rows, 2^22 columns and strides of a matrix, 2^24 tiles of
 *    256 x 256 of an output),
 *    DIP_E_UNSUPPORTED (float32 in dip_linear), DIP_E_CAPACITY (workspace too
 *    small; nothing has been done), DIP_E_HIP.  Sizes of zero are legal: nothing
 *    is read, sums over nothing are zero (and so a norm's mean and variance).
 */
#ifndef DIP_OPS_H
#define DIP_OPS_H

#include <stdint.h>

#include "dip_sim.h"

#ifdef __cplusplus
extern "C" {
#endif

/* element types */
#define DIP_F32 0
#define DIP_F16 1
#define DIP_BF16 2

/* activations: z; max(z, 0); z s(z); z s(2 u), u = sqrt(2/pi) (z + 0.044715 z^3)
 * (the tanh form of GELU), s the logistic function.  ReLU's slope at 0 is 0. */
#define DIP_ACT_NONE 0
#define DIP_ACT_RELU 1
#define DIP_ACT_SILU 2
#define DIP_ACT_GELU 3

/* Dropout.  Element (row, col) is dropped iff its 16-bit draw is below drop_of
 * (the probability in 65536ths; 0: no dropout, no draws).  Kept elements are
 * multiplied by 65536 / (65536 - drop_of) in float32; dropped ones are 0
 * whatever they held.  The draws are those of Philox4x32-10 (Salmon et al.,
 * SC'11) with key (seed low, seed high) and counter (col / 8, row0 + row,
 * offset low, offset high): word j holds the draws of columns 2 j (low half)
 * and 2 j + 1 (high half) of the eight. */
typedef struct {
  uint64_t seed;
  uint64_t offset;
  uint32_t row0;             /* row0 + rows <= 2^32                             */
  uint32_t drop_of;          /* 0 .. 65535                                      */
} dip_dropout;

/* y[m][n] = residual[m][n] + D(act(sum_k x[m][k] w[n][k] + bias[n])).
 * Types: DIP_F16 or DIP_BF16 for all arrays; products are summed in float32.
 * pre, if given, receives x w^T + bias before the activation, rounded to the
 * type: what dip_linear_grad needs where act is not DIP_ACT_NONE. */
typedef struct {
  int64_t m, n, k;           /* rows (tokens), output and input features        */
  int32_t dtype, act;
  const void *x;             /* [m][k], ldx                                     */
  int64_t ldx;
  const void *w;             /* [n][k], ldw                                     */
  int64_t ldw;
  const void *bias;          /* [n] or null                                     */
  const void *residual;      /* [m][n], ldr, or null                            */
  int64_t ldr;
  dip_dropout drop;
  void *y;                   /* [m][n], ldy                                     */
  int64_t ldy;
  void *pre;                 /* [m][n], ldp, or null                            */
  int64_t ldp;
  void *workspace;           /* 16-byte aligned, dip_linear_workspace() bytes   */
  int64_t workspace_bytes;
} dip_linear_args;

/* Bytes of workspace of a call with these arguments (its pointers count by
 * their alignment, the workspace itself does not), or a negative code. */
int64_t dip_linear_workspace(const dip_linear_args *a);
int dip_linear(const dip_linear_args *a, void *stream);

/* Gradients of dip_linear for the gradient dy of y:
 *   g = D(dy) act'(pre), dx = g w, dw = g^T x, db = sum_m g; the residual's
 *   gradient is dy itself.  The matrix instructions take g rounded to the type,
 *   and the factor of D's kept elements only after them: the rounding changes
 *   nothing where act is DIP_ACT_NONE or DIP_ACT_RELU.  db has g unrounded.
 * Each of dx, dw, db may be null.  dw and db are of type grad_dtype: the
 * operands' type or DIP_F32; with accumulate != 0 they are added to what the
 * arrays hold (gradients summed over sub-microbatches). */
typedef struct {
  int64_t m, n, k;
  int32_t dtype, act;
  const void *dy;            /* [m][n], ldy                                     */
  int64_t ldy;
  const void *x;             /* [m][k], ldx; may be null without dw             */
  int64_t ldx;
  const void *w;             /* [n][k], ldw; may be null without dx             */
  int64_t ldw;
  const void *pre;           /* [m][n], ldp; may be null for DIP_ACT_NONE       */
  int64_t ldp;
  dip_dropout drop;
  void *dx;                  /* [m][k], lddx                                    */
  int64_t lddx;
  void *dw;                  /* [n][k], lddw                                    */
  int64_t lddw;
  void *db;                  /* [n]                                             */
  int32_t grad_dtype, accumulate;
  void *workspace;           /* 16-byte aligned, dip_linear_grad_workspace()    */
  int64_t workspace_bytes;
} dip_linear_grad_args;

int64_t dip_linear_grad_workspace(const dip_linear_grad_args *a);
int dip_linear_grad(const dip_linear_grad_args *a, void *stream);

/* y[m][n] = residual[m][n] + D(x[m][n]); residual may be null.  The gradient of
 * x is the same call on dy without a residual; the residual's is dy. */
int dip_dropout_add(int32_t dtype, int64_t m, int64_t n, const void *x, int64_t ldx,
                    const void *residual, int64_t ldr, const dip_dropout *drop, void *y,
                    int64_t ldy, void *stream);

/* Group norm over channels-last arrays [b][s][c]: group g of sample i holds the
 * channels g c/groups .. of all s positions; mean and (biased) variance over
 * them, rstd = 1 / sqrt(var + eps), y = act(gamma[c] (x - mean) rstd + beta[c]).
 * With s = 1 and groups = 1 this is a layer norm of b rows.  gamma and beta may
 * be null (1 and 0).  mean and rstd: float32 [b][groups], outputs of the forward
 * and inputs of the gradient; null in the forward where no gradient follows.
 * Strides in elements, up to 2^46: sb between samples, ss between positions, in
 * either order ([b][s][c] or [s][b][c]). */
typedef struct {
  int64_t b, s, c;
  int32_t groups, dtype, act;
  float eps;                 /* >= 0                                            */
  const void *x;
  int64_t x_sb, x_ss;
  const void *gamma, *beta;  /* [c] of the type, or null                        */
  void *y;
  int64_t y_sb, y_ss;
  float *mean, *rstd;
  void *workspace;           /* 16-byte aligned, dip_group_norm_workspace()     */
  int64_t workspace_bytes;
} dip_group_norm_args;

int64_t dip_group_norm_workspace(const dip_group_norm_args *a);
int dip_group_norm(const dip_group_norm_args *a, void *stream);

/* Its gradients: g = dy act'(z), xh = (x - mean) rstd, dgamma = sum g xh and
 * dbeta = sum g over samples and positions, and with h = g gamma
 * dx = rstd (h - mean(h) - xh mean(h xh)), means over the group.  dx, dgamma,
 * dbeta may each be null; dx is of the inputs' type, dgamma and dbeta too or, for
 * gradients summed over sub-microbatches, float32. */
typedef struct {
  int64_t b, s, c;
  int32_t groups, dtype, act;
  int32_t accumulate;        /* 0: dgamma and dbeta are of the type; else float32 */
                             /* and added to what the arrays hold               */
  const void *dy;
  int64_t dy_sb, dy_ss;
  const void *x;
  int64_t x_sb, x_ss;
  const void *gamma, *beta;
  const float *mean, *rstd;
  void *dx;
  int64_t dx_sb, dx_ss;
  void *dgamma, *dbeta;      /* [c]                                             */
  void *workspace;           /* 16-byte aligned, dip_group_norm_grad_workspace() */
  int64_t workspace_bytes;
} dip_group_norm_grad_args;

int64_t dip_group_norm_grad_workspace(const dip_group_norm_grad_args *a);
int dip_group_norm_grad(const dip_group_norm_grad_args *a, void *stream);

/* A matrix in 8 bits.  32 consecutive columns of a row (the last ones: what is
 * left) share a scale 2^e, the smallest with e >= -126 by which the largest finite
 * magnitude of them divides to at most 448; its byte is e + 127.  Values are v / 2^e
 * rounded to nearest even with four significant bits and steps of at least 2^-9
 * (sign, 4 bits of exponent, 3 of mantissa; OCP FP8 E4M3).  Infinities and NaN are
 * kept as NaN.  What is read may have any bytes: scales 0 and 255 are 2^-127 and NaN.
 * Restored values are exact in float32, and in bfloat16 from 2^-126 on; one that
 * rounded up beyond the largest value of the type it is restored to becomes that
 * value (through an activation: beyond float32's, before it). */
typedef struct {
  void *values;              /* [m][n] bytes, ld; any alignment                 */
  int64_t ld;
  void *scales;              /* [m][(n + 31) / 32] bytes, lds                   */
  int64_t lds;
} dip_packed8;

/* x[m][n] in 8 bits, and y[m][n] = act(x) of a matrix in 8 bits, x exact and y
 * rounded to dtype. */
int dip_pack8(int32_t dtype, int64_t m, int64_t n, const void *x, int64_t ldx, const dip_packed8 *out, void *stream);
int dip_unpack8(int32_t dtype, int64_t m, int64_t n, const dip_packed8 *x, int32_t act, void *y, int64_t ldy,
                void *stream);

/* dip_linear with pre kept in 8 bits, from the float32 sums; a->pre is not used. */
int64_t dip_linear_kept_workspace(const dip_linear_args *a, const dip_packed8 *pre);
int dip_linear_kept(const dip_linear_args *a, const dip_packed8 *pre, void *stream);
/* dip_linear_grad from activations kept in 8 bits: x is x_act of the kept matrix,
 * rounded to the type (where act rounds g too, x_act's values are taken as two of the
 * type, so that one of dw's factors is rounded), and slopes are those at the kept pre.
 * Either may be null: then a->x (x_act not used) or a->pre is read. */
int64_t dip_linear_grad_kept_workspace(const dip_linear_grad_args *a, const dip_packed8 *x, int32_t x_act,
                                       const dip_packed8 *pre);
int dip_linear_grad_kept(const dip_linear_grad_args *a, const dip_packed8 *x, int32_t x_act, const dip_packed8 *pre,
                         void *stream);

/* Root-mean-square norm of m rows of c: t = x + residual rounded to the type (the
 * stream of residuals; x itself without one), rstd = 1 / sqrt(mean(t^2) + eps),
 * y = gamma t rstd.  Squares are summed in float64, and rstd is rounded once, also of
 * rows whose squares no float32 holds; one that float32 does not hold is infinite.  total
 * (t) may be the residual itself or null; y,
 * rstd and packed.values too, where they are not wanted.  packed has y in 8 bits, from
 * the float32 values.  gamma may be null (1). */
typedef struct {
  int64_t m, c;
  int32_t dtype;
  float eps;                 /* >= 0                                            */
  const void *x;             /* [m][c], ldx                                     */
  int64_t ldx;
  const void *residual;      /* [m][c], ldr, or null                            */
  int64_t ldr;
  const void *gamma;         /* [c] of the type, or null                        */
  void *total;               /* [m][c], ldt                                     */
  int64_t ldt;
  void *y;                   /* [m][c], ldy                                     */
  int64_t ldy;
  dip_packed8 packed;
  float *rstd;               /* [m]                                             */
} dip_rms_norm_args;

int dip_rms_norm(const dip_rms_norm_args *a, void *stream);

/* Its gradients for the gradients dy of y and dtotal of t (null: none): with
 * xh = t rstd and h = dy gamma, dx = dtotal + rstd (h - xh mean(h xh)), which is the
 * gradient of x and of the residual, and dgamma = sum over rows of dy xh.  Either may
 * be null.  dx may be dtotal itself.  dgamma is of the type; with accumulate != 0
 * float32 and added to. */
typedef struct {
  int64_t m, c;
  int32_t dtype, accumulate;
  const void *dy;            /* [m][c], ldy                                     */
  int64_t ldy;
  const void *total;         /* [m][c], ldt                                     */
  int64_t ldt;
  const void *gamma;
  const float *rstd;
  const void *dtotal;        /* [m][c], lddt, or null                           */
  int64_t lddt;
  void *dx;                  /* [m][c], lddx                                    */
  int64_t lddx;
  void *dgamma;              /* [c]                                             */
  void *workspace;           /* 16-byte aligned, dip_rms_norm_grad_workspace()  */
  int64_t workspace_bytes;
} dip_rms_norm_grad_args;

int64_t dip_rms_norm_grad_workspace(const dip_rms_norm_grad_args *a);
int dip_rms_norm_grad(const dip_rms_norm_grad_args *a, void *stream);

/* types of positions */
#define DIP_POS_I32 0
#define DIP_POS_I64 1
#define DIP_POS_F32 2

/* Rotary positions with several axes: pair j of every head of token i is turned by
 * the angle pos[i][axis[j]] freq[j] radians (inverse != 0: by its negative, which is
 * the gradient), (a, b) to (a cos - b sin, a sin + b cos).  Pair j is elements
 * j and pairs + j of the head, or with interleaved != 0 2 j and 2 j + 1; elements from
 * 2 pairs on are copied.  Angles are float64, and so their sines and cosines up to one
 * rounding to float32.  A pair whose axis is not one of the axes stays as it is.  k with
 * its heads goes along where keys > 0.  Strides in elements, up to 2^46: st between
 * tokens, sh between heads, in either order; pos st and sa between tokens and axes.  An
 * output may be its input itself (same pointer and strides). */
typedef struct {
  int64_t t;                 /* tokens                                          */
  int32_t heads, keys;       /* heads of q and of k, up to 65,536 together      */
  int32_t dim, pairs, axes;  /* elements a head, up to 2048; 2 pairs <= dim     */
  int32_t dtype, pos_type, interleaved, inverse;
  const void *q;             /* [t][heads][dim]                                 */
  int64_t q_st, q_sh;
  const void *k;             /* [t][keys][dim]                                  */
  int64_t k_st, k_sh;
  const void *pos;           /* [t][axes]                                       */
  int64_t p_st, p_sa;
  const double *freq;        /* [pairs]                                         */
  const int32_t *axis;       /* [pairs]                                         */
  void *q_out;
  int64_t qo_st, qo_sh;
  void *k_out;
  int64_t ko_st, ko_sh;
} dip_rotary_args;

int dip_rotary(const dip_rotary_args *a, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* DIP_OPS_H */
