// kern_elementwise.hip -- dropout, the gradient before the matrix products, and
// sums over rows.
#include <algorithm>

#include "ops_internal.h"

namespace dipops {
namespace {

constexpr int kThreads = 256;

// Eight columns of a row a thread.
template <class T>
__global__ __launch_bounds__(kThreads) void dropout_add_kernel(int64_t m, int64_t n, const T *x,
                                                               int64_t ldx, const T *r,
                                                               int64_t ldr, Drop d, T *y,
                                                               int64_t ldy, bool vx, bool vr,
                                                               bool vy) {
  const int64_t per = (n + 7) / 8, all = m * per;
  for (int64_t i = int64_t(blockIdx.x) * kThreads + threadIdx.x; i < all;
       i += int64_t(gridDim.x) * kThreads) {
    const int64_t row = i / per, col = i % per * 8;
    const int left = int(min(int64_t(8), n - col));
    float v[8], q[8];
    load8(x + row * ldx + col, left, vx, v);
    if (d.drop_of) drop8(d, uint32_t(col / 8), uint32_t(row), v);
    if (r) {
      load8(r + row * ldr + col, left, vr, q);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] += q[j];
    }
    store8(y + row * ldy + col, left, vy, v);
  }
}

template <class T>
hipError_t dropout_add(int64_t m, int64_t n, const void *x, int64_t ldx, const void *r, int64_t ldr,
                       const Drop &d, void *y, int64_t ldy, hipStream_t stream) {
  const int64_t blocks = (m * ((n + 7) / 8) + kThreads - 1) / kThreads;
  dropout_add_kernel<T><<<dim3(uint32_t(std::min<int64_t>(blocks, 1 << 20))), dim3(kThreads), 0, stream>>>(
      m, n, static_cast<const T *>(x), ldx, static_cast<const T *>(r), ldr, d, static_cast<T *>(y),
      ldy, aligned16(x, ldx, sizeof(T)), aligned16(r, ldr, sizeof(T)), aligned16(y, ldy, sizeof(T)));
  return hipGetLastError();
}

// A block takes 256 columns (32 threads of eight) of one chunk of rows, eight
// rows at a time, and adds its eight row lanes at the end.
template <class T>
__global__ __launch_bounds__(kThreads) void grad_in_kernel(GradIn g) {
  __shared__ float s[8][256 + 8];
  const int tx = threadIdx.x % 32, ty = threadIdx.x / 32;
  const int64_t col = int64_t(blockIdx.x) * 256 + tx * 8;
  const int64_t per = (g.m + g.row_chunks - 1) / g.row_chunks;
  const int64_t r0 = per * blockIdx.y, r1 = min(r0 + per, g.m);
  const int left = int(max(int64_t(0), min(int64_t(8), g.n - col)));
  float sum[8] = {};
  if (left > 0) {
    for (int64_t row = r0 + ty; row < r1; row += 8) {
      float v[8], z[8];
      load8(static_cast<const T *>(g.dy) + row * g.ldy + col, left, g.vec_dy, v);
      if (g.drop.drop_of) drop8(g.drop, uint32_t(col / 8), uint32_t(row), v);
      if (g.pre) {
        load8(static_cast<const T *>(g.pre) + row * g.ldp + col, left, g.vec_pre, z);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] *= act_slope(z[j], g.act);
      }
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (j >= left) v[j] = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) sum[j] += v[j];
      if (g.out) store8(static_cast<T *>(g.out) + row * g.ldo + col, 8, true, v);
    }
  }
  if (!g.partial) return;
#pragma unroll
  for (int j = 0; j < 8; ++j) s[ty][tx * 8 + j] = sum[j];
  __syncthreads();
  const int c = threadIdx.x;
  const int64_t out = int64_t(blockIdx.x) * 256 + c;
  if (out < g.n) {
    float v = 0.f;
    for (int i = 0; i < 8; ++i) v += s[i][c];
    g.partial[int64_t(blockIdx.y) * g.n + out] = v;
  }
}

template <class O>
__global__ __launch_bounds__(kThreads) void sum_rows_kernel(const float *p, int64_t rows,
                                                            int64_t cols, O *out, int accumulate) {
  const int64_t c = int64_t(blockIdx.x) * kThreads + threadIdx.x;
  if (c >= cols) return;
  float v = 0.f;
  for (int64_t r = 0; r < rows; ++r) v += p[r * cols + c];
  if (accumulate) v += float(out[c]);
  out[c] = O(v);
}

}  // namespace

hipError_t launch_dropout_add(int dtype, int64_t m, int64_t n, const void *x, int64_t ldx,
                              const void *residual, int64_t ldr, const Drop &drop, void *y,
                              int64_t ldy, hipStream_t stream) {
  switch (dtype) {
    case DIP_F32: return dropout_add<float>(m, n, x, ldx, residual, ldr, drop, y, ldy, stream);
    case DIP_F16: return dropout_add<_Float16>(m, n, x, ldx, residual, ldr, drop, y, ldy, stream);
    default: return dropout_add<__bf16>(m, n, x, ldx, residual, ldr, drop, y, ldy, stream);
  }
}

int32_t grad_row_chunks(int64_t m, int64_t n) {
  const int64_t cols = (n + 255) / 256;
  return int32_t(std::max<int64_t>(1, std::min<int64_t>((m + 31) / 32, 2048 / cols)));
}

hipError_t launch_grad_in(int dtype, const GradIn &g, hipStream_t stream) {
  const dim3 grid(uint32_t((g.n + 255) / 256), uint32_t(g.row_chunks));
  if (dtype == DIP_BF16)
    grad_in_kernel<__bf16><<<grid, dim3(kThreads), 0, stream>>>(g);
  else
    grad_in_kernel<_Float16><<<grid, dim3(kThreads), 0, stream>>>(g);
  return hipGetLastError();
}

hipError_t launch_sum_rows(const float *partial, int64_t rows, int64_t cols, void *out,
                           int out_dtype, int accumulate, hipStream_t stream) {
  const dim3 grid(uint32_t((cols + kThreads - 1) / kThreads)), block(kThreads);
  switch (out_dtype) {
    case DIP_F32:
      sum_rows_kernel<<<grid, block, 0, stream>>>(partial, rows, cols, static_cast<float *>(out), accumulate);
      break;
    case DIP_F16:
      sum_rows_kernel<<<grid, block, 0, stream>>>(partial, rows, cols, static_cast<_Float16 *>(out), accumulate);
      break;
    default:
      sum_rows_kernel<<<grid, block, 0, stream>>>(partial, rows, cols, static_cast<__bf16 *>(out), accumulate);
  }
  return hipGetLastError();
}

}  // namespace dipops
