// ops_internal.h -- launches of the stage operators' kernels, called by
// host_ops.hip after it has checked the arguments.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "ops_device.h"

namespace dipops {

// n / d for n below 2^31, d at least 1, by one high product.
struct Divide {
  uint32_t by, mul, shift;
  explicit Divide(uint32_t d) : by(d), mul(0), shift(0) {
    while ((uint64_t(1) << shift) < d) ++shift;
    // ceil(2^(32 + shift) / d) - 2^32, below 2^32
    mul = uint32_t(((uint64_t(1) << 32) * ((uint64_t(1) << shift) - d)) / d + 1);
  }
  __device__ __forceinline__ uint32_t operator()(uint32_t n) const { return (__umulhi(n, mul) + n) >> shift; }
};

// One operand of a matrix product: element (i, k), i the output's row or
// column, k the contraction, at p[i * ld + k], or with k_rows at p[k * ld + i].
struct Operand {
  const void *p;
  int64_t ld;
  bool k_rows;
};

// The epilogue whose pre goes out in 8 bits (e.pre is null).
struct KeptEpilogue : Epilogue {
  Packed kept;
};

// out[m][n] = epilogue(sum_k a(m, k) b(n, k)).  Operands are 16-byte aligned with
// strides that are multiples of 8; one whose contraction runs along its rows
// (k_rows false) has zeros, or k itself, up to the next multiple of 8 of k.
struct GemmPlan {
  int32_t tile = 0, splits = 1;
  int64_t steps = 0;           // contraction steps a split
  int64_t bytes = 0;           // of partial products
  double us = 0;               // expected, without the join
};
constexpr int64_t kMaxTiles = int64_t(1) << 24;   // 256-thread workgroups a launch
GemmPlan plan_gemm(int64_t m, int64_t n, int64_t k, bool a_rows);   // by sizes and a's layout (not k_rows)
hipError_t launch_gemm(int dtype, int64_t m, int64_t n, int64_t k, const Operand &a,
                       const Operand &b, const Epilogue &e, const GemmPlan &plan, float *partial,
                       hipStream_t stream);
// The products of dx (a along the contraction, b not) and of dw (neither) in one launch,
// where that is faster than one after the other; their partial products are apart.
struct Gemm {
  int64_t m, n, k;
  Operand a, b;
  Epilogue e;
  GemmPlan plan;
  float *partial;
};
bool pair_gemms(int64_t mx, int64_t nx, const GemmPlan &x, int64_t mw, int64_t nw, const GemmPlan &w);
hipError_t launch_gemm_pair(int dtype, const Gemm &x, const Gemm &w, hipStream_t stream);
// a and b along the contraction, pre kept in 8 bits
hipError_t launch_gemm_kept(int dtype, int64_t m, int64_t n, int64_t k, const Operand &a, const Operand &b,
                            const KeptEpilogue &e, const GemmPlan &plan, float *partial, hipStream_t stream);
// The same for few rows of an x that is read where it is, as w is: any alignment,
// no workspace.  Every 8 to 32 rows of w read x again, from the caches, so it pays
// for few rows, and for more where w is small.  bf16, w from memory, this way
// against tiles, us (k x n): 1 row 4096 x 3584 9.6 / 13.8, 4096 x 14336 26 / 28; 8
// rows 12.2 / 14.8 and 13696 x 1664 17.5 / 19.3; 16 rows 13.1 / 14.9, 32 / 29 and
// 14336 x 4096 33.6 / 32.4; 17 rows 2048 x 4096 9.1 / 12.9, 8192 x 4096 24 / 21; 32
// rows 1000 x 1000 5.8 / 10.3, 2048 x 4096 10.6 / 13.3, 4096 x 3584 17 / 15.4, 8192 x
// 4096 30 / 21.
inline bool thin(int64_t m, int64_t n, int64_t k) { return m <= 16 || (m <= 32 && n * k <= (int64_t(1) << 23)); }
hipError_t launch_thin(int dtype, int64_t m, int64_t n, int64_t k, const void *x, int64_t ldx, const void *w,
                       int64_t ldw, const Epilogue &e, hipStream_t stream);
// rows x cols from p to out (16-byte aligned, stride ldo a multiple of 8), zeros
// in columns cols .. ldo - 1; no rows: nothing
struct PackJob {
  const void *p = nullptr;
  int64_t rows = 0, cols = 0, ld = 0;
  void *out = nullptr;
  int64_t ldo = 8;
};
hipError_t launch_pack(int dtype, const PackJob &a, const PackJob &b, hipStream_t stream);
// vector i of a job, if it has that many
template <class T>
__device__ __forceinline__ void pack_item(const PackJob &j, int64_t i) {
  const uint32_t per = uint32_t(j.ldo / 8);
  if (i >= j.rows * per) return;
  const int64_t row = i / per, col = (i - row * per) * 8;
  float v[8];
  load8(static_cast<const T *>(j.p) + row * j.ld + col, int(min(int64_t(8), j.cols - col)), v);
  store8(static_cast<T *>(j.out) + row * j.ldo + col, 8, v);
}

// g = D(dy) act'(pre), without the factor of D's kept elements, to out (ld a
// multiple of 8, padding columns zero; null: not wanted), and its column sums with
// the factor and before rounding to partial[row_chunks][n] (null: not wanted).
struct GradIn {
  int64_t m, n;
  const void *dy, *pre;
  int64_t ldy, ldp;
  Drop drop;
  int32_t act;
  void *out, *again;         // again: the same once more, or null
  int64_t ldo;
  float *partial;
  int32_t row_chunks;
  Packed kept;               // pre in 8 bits, in the place of pre; q null: none
};
int32_t grad_row_chunks(int64_t m, int64_t n);
hipError_t launch_grad_in(int dtype, const GradIn &g, hipStream_t stream);
// act of x [m][n] in 8 bits to out (16-byte aligned, ldo a multiple of 8), zeros in
// columns n .. ldo - 1; what rounding it left off to low, laid out like out (null: not
// wanted)
struct Restore {
  Packed x;
  int64_t m;
  int32_t n, act;
  void *out, *low;
  int64_t ldo;
};
// All three in one launch, where that is faster and has the threads; w may have no rows.
bool grad_in_kept_fits(const GradIn &g, const Restore &x, const PackJob &w);
hipError_t launch_grad_in_kept(int dtype, const GradIn &g, const Restore &x, const PackJob &w, hipStream_t stream);
// out0[j] (+)= the sum over the rows of partial[rows][ld] of column j, and out1[j]
// of column c + j, j < c, in an order that depends on the sizes alone; either may
// be null.
struct SumRows {
  const float *partial;
  int64_t rows, ld, c;
  void *out0, *out1;
  int accumulate;
};
hipError_t launch_sum_rows(const SumRows &s, int out_dtype, hipStream_t stream);

hipError_t launch_dropout_add(int dtype, int64_t m, int64_t n, const void *x, int64_t ldx,
                              const void *residual, int64_t ldr, const Drop &drop, void *y,
                              int64_t ldy, hipStream_t stream);

hipError_t launch_pack8(int dtype, int64_t m, int64_t n, const void *x, int64_t ldx, const Packed &out,
                        hipStream_t stream);
// y = act(x), zeros in columns n .. fill - 1; low as Restore's, of an activation
hipError_t launch_unpack8(int dtype, int64_t m, int64_t n, const Packed &x, int act, void *y, int64_t ldy, int64_t fill,
                          hipStream_t stream, void *low = nullptr);
hipError_t launch_rms_norm(const dip_rms_norm_args &a, hipStream_t stream);
hipError_t launch_rms_norm_grad(const dip_rms_norm_grad_args &a, hipStream_t stream);
int64_t rms_norm_grad_workspace(const dip_rms_norm_grad_args &a);
hipError_t launch_rotary(const dip_rotary_args &a, hipStream_t stream);

hipError_t launch_group_norm(const dip_group_norm_args &a, hipStream_t stream);
hipError_t launch_group_norm_grad(const dip_group_norm_grad_args &a, hipStream_t stream);
int64_t group_norm_workspace(const dip_group_norm_args &a);
int64_t group_norm_grad_workspace(const dip_group_norm_grad_args &a);

inline bool aligned16(const void *p, int64_t ld, int elem) {
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld * elem % 16 == 0;
}
inline int64_t up16(int64_t bytes) { return (bytes + 15) / 16 * 16; }

}  // namespace dipops
