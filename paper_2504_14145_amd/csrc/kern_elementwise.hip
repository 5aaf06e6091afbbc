// kern_elementwise.hip -- dropout, the gradient before the matrix products, and
// sums over rows.
#include <algorithm>
#include <type_traits>

#include "ops_internal.h"

namespace dipops {
namespace {

constexpr int kThreads = 256;

// Bound by memory while a counter's 128 bits serve eight elements: its twenty
// 32 x 32 products take 320 cycles a wave, less than the wave's 24 bytes a lane
// take to come and go.  Eight columns of a row a thread.  65,536 x 3584 bf16 with a
// residual 240 us (5.9 TB/s), without 146 (6.4).
template <class T, bool RESIDUAL>
__global__ __launch_bounds__(kThreads) void dropout_add_kernel(uint32_t items, uint32_t row0, Divide per, int64_t n,
                                                               const T *x, int64_t ldx, const T *r, int64_t ldr,
                                                               Drop d, T *y, int64_t ldy) {
  const uint32_t i = blockIdx.x * kThreads + threadIdx.x;
  if (i >= items) return;
  const uint32_t in = per(i), row = row0 + in;
  const int64_t col = int64_t(i - in * per.by) * 8;
  const int left = int(min(int64_t(8), n - col));
  float v[8], q[8];
  load8(x + row * ldx + col, left, v);
  if constexpr (RESIDUAL) load8(r + row * ldr + col, left, q);
  if (d.drop_of) drop8(d, uint32_t(col / 8), row, v);
  if constexpr (RESIDUAL) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] += q[j];
  }
  store8(y + row * ldy + col, left, v);
}

template <class T>
hipError_t dropout_add(int64_t m, int64_t n, const void *x, int64_t ldx, const void *r, int64_t ldr,
                       const Drop &d, void *y, int64_t ldy, hipStream_t stream) {
  const int64_t per = (n + 7) / 8, most = ((int64_t(1) << 31) - 1) / per;   // rows a launch
  for (int64_t row0 = 0; row0 < m; row0 += most) {
    const uint32_t items = uint32_t(std::min(most, m - row0) * per);
    const dim3 grid((items + kThreads - 1) / kThreads);
    auto go = [&](auto kernel) {
      kernel<<<grid, dim3(kThreads), 0, stream>>>(items, uint32_t(row0), Divide(uint32_t(per)), n,
                                                  static_cast<const T *>(x), ldx, static_cast<const T *>(r), ldr, d,
                                                  static_cast<T *>(y), ldy);
    };
    if (r) go(dropout_add_kernel<T, true>);
    else go(dropout_add_kernel<T, false>);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// g = D(dy) act'(pre) and its column sums.  g is rounded to the type because the
// matrix instructions take it so; the factor of the kept elements is left to the
// float32 products (and the sums), so that without an activation, and with ReLU,
// whose slopes are 0 and 1, g is dy or 0 and that rounding changes nothing.  Slopes
// of SiLU and GELU leave dx and dw 0.0024 of their norm from the exact values in
// bf16, where the rounding of the result alone is 0.0017; a second product with
// what the rounding left off would take that back and double the products.
// Bound by memory, dy and pre read and g written once.  A block takes 256 columns (32 threads of eight) of one chunk of
// rows, sixteen rows at a time, and adds its eight row lanes at the end; the
// chunks' sums are added in their order by sum_rows_kernel.  65,536 x 2560 with
// GELU 217 us (4.6 TB/s; the slope's arithmetic is the rest).
typedef float GradSums[8][256 + 8];
template <class T, bool KEPT>
__device__ __forceinline__ void grad_in_block(const GradIn &g, uint32_t bx, uint32_t by, GradSums &s) {
  const int tx = threadIdx.x % 32, ty = threadIdx.x / 32;
  const int64_t col = int64_t(bx) * 256 + tx * 8;
  const int64_t per = (g.m + g.row_chunks - 1) / g.row_chunks;
  const int64_t r0 = per * by, r1 = min(r0 + per, g.m);
  const int left = int(max(int64_t(0), min(int64_t(8), g.n - col)));
  float sum[8] = {};
  if (left > 0) {
    const T *dy = static_cast<const T *>(g.dy) + col, *pre = static_cast<const T *>(g.pre) + col;
    // U rows at a time, their loads first
    auto rows = [&](int64_t row, auto u_) {
      constexpr int U = decltype(u_)::value;
      float v[U][8], z[U][8];
#pragma unroll
      for (int u = 0; u < U; ++u) load8(dy + (row + 8 * u) * g.ldy, left, v[u]);
      if constexpr (KEPT) {
        u32x2 bits[U];
        uint32_t scale[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          bits[u] = load8bits(g.kept.q + (row + 8 * u) * g.kept.ld, int(col), int(g.n));
          scale[u] = g.kept.s[(row + 8 * u) * g.kept.lds + col / 32];
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
          place8bits(int(col), int(g.n), bits[u]);
          from8bits(bits[u], scale_of(scale[u]), z[u]);
        }
      } else if (g.pre) {
#pragma unroll
        for (int u = 0; u < U; ++u) load8(pre + (row + 8 * u) * g.ldp, left, z[u]);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (g.act == DIP_ACT_GELU) {
#pragma unroll
          for (int j = 0; j < 8; ++j) v[u][j] *= act_slope(z[u][j], DIP_ACT_GELU);
        } else if (g.act == DIP_ACT_SILU) {
#pragma unroll
          for (int j = 0; j < 8; ++j) v[u][j] *= act_slope(z[u][j], DIP_ACT_SILU);
        } else if (g.act == DIP_ACT_RELU) {
#pragma unroll
          for (int j = 0; j < 8; ++j) v[u][j] *= act_slope(z[u][j], DIP_ACT_RELU);
        }
        // after the slope, which is NaN where pre is not finite: dropped ones are 0
        // whatever they held
        if (g.drop.drop_of) drop8(g.drop, uint32_t(col / 8), uint32_t(row + 8 * u), 1.f, v[u]);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          if (j >= left) v[u][j] = 0.f;
          sum[j] += v[u][j];
        }
        if (g.out) store8(static_cast<T *>(g.out) + (row + 8 * u) * g.ldo + col, 8, v[u]);
        if (g.again) store8(static_cast<T *>(g.again) + (row + 8 * u) * g.ldo + col, 8, v[u]);
      }
    };
    int64_t row = r0 + ty;
    for (; row + 8 < r1; row += 16) rows(row, std::integral_constant<int, 2>{});
    for (; row < r1; row += 8) rows(row, std::integral_constant<int, 1>{});
  }
  if (!g.partial) return;
#pragma unroll
  for (int j = 0; j < 8; ++j) s[ty][tx * 8 + j] = sum[j];
  __syncthreads();
  const int c = threadIdx.x;
  const int64_t out = int64_t(bx) * 256 + c;
  if (out < g.n) {
    float v = 0.f;
    for (int i = 0; i < 8; ++i) v += s[i][c];
    g.partial[int64_t(by) * g.n + out] = v * g.drop.scale;
  }
}
template <class T, bool KEPT>
__global__ __launch_bounds__(kThreads) void grad_in_kernel(GradIn g) {
  __shared__ GradSums s;
  grad_in_block<T, KEPT>(g, blockIdx.x, blockIdx.y, s);
}

// The same beside x restored from 8 bits and w copied where that is needed, in one
// launch: three passes that do not need each other, of which small ones leave most of the
// card idle.  Time of a whole backward pass with three launches and with one: 51.4 and
// 42.6 us at 1201 x 1795 x 1027 fp16, 413 and 409 at 8192 x 4096 x 3584 bf16.
struct Restoring {
  Restore x;
  Divide per;
  uint32_t items, x_blocks, g_cols, g_blocks;
};
template <class T, bool KEPT, bool ACT>
__global__ __launch_bounds__(kThreads) void grad_in_kept_kernel(GradIn g, Restoring r, PackJob w) {
  __shared__ GradSums s;
  uint32_t b = blockIdx.x;
  if (b < r.g_blocks) {
    const uint32_t by = b / r.g_cols;
    return grad_in_block<T, KEPT>(g, b - by * r.g_cols, by, s);
  }
  b -= r.g_blocks;
  if (b < r.x_blocks) {
    const uint32_t i = b * kThreads + threadIdx.x;
    if (i >= r.items) return;
    const uint32_t row = r.per(i);
    const int col = int(i - row * r.per.by) * 8;
    const int64_t at = int64_t(row) * r.x.ldo + col;
    return restore8<T, ACT>(r.x.x, row, col, r.x.n, r.x.act, static_cast<T *>(r.x.out) + at, 8,
                            r.x.low ? static_cast<T *>(r.x.low) + at : nullptr);
  }
  pack_item<T>(w, int64_t(b - r.x_blocks) * kThreads + threadIdx.x);
}

// 64 columns a workgroup, LANES threads a column.
template <class O, int LANES>
__global__ __launch_bounds__(64 * LANES) void sum_rows_kernel(SumRows a) {
  __shared__ float s[LANES][64];
  const int tx = threadIdx.x % 64, ty = threadIdx.x / 64;
  const int64_t col = int64_t(blockIdx.x) * 64 + tx, all = a.out1 ? 2 * a.c : a.c;
  float v = 0.f;
  if (col < all) {
    const float *p = a.partial + col;
    int64_t r = ty;
    for (; r + 3 * LANES < a.rows; r += 4 * LANES) {
      const float q0 = p[r * a.ld], q1 = p[(r + LANES) * a.ld], q2 = p[(r + 2 * LANES) * a.ld],
                  q3 = p[(r + 3 * LANES) * a.ld];
      v += (q0 + q1) + (q2 + q3);
    }
    for (; r < a.rows; r += LANES) v += p[r * a.ld];
  }
  s[ty][tx] = v;
  __syncthreads();
  if (ty != 0 || col >= all) return;
#pragma unroll
  for (int i = 1; i < LANES; ++i) v += s[i][tx];
  O *out = static_cast<O *>(col < a.c ? a.out0 : a.out1);
  if (!out) return;
  const int64_t at = col < a.c ? col : col - a.c;
  if (a.accumulate) v += float(out[at]);
  out[at] = O(v);
}

template <class O>
hipError_t sum_rows(const SumRows &a, hipStream_t stream) {
  if (!a.out0 && !a.out1) return hipSuccess;
  const dim3 grid(uint32_t(((a.out1 ? 2 * a.c : a.c) + 63) / 64));
  if (a.rows > 16)
    sum_rows_kernel<O, 16><<<grid, dim3(1024), 0, stream>>>(a);
  else
    sum_rows_kernel<O, 4><<<grid, dim3(256), 0, stream>>>(a);
  return hipGetLastError();
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
  return int32_t(std::max<int64_t>(1, std::min<int64_t>((m + 15) / 16, 2048 / cols)));
}

hipError_t launch_grad_in(int dtype, const GradIn &g, hipStream_t stream) {
  const dim3 grid(uint32_t((g.n + 255) / 256), uint32_t(g.row_chunks));
  auto go = [&](auto kernel) { kernel<<<grid, dim3(kThreads), 0, stream>>>(g); };
  if (dtype == DIP_BF16) g.kept.q ? go(grad_in_kernel<__bf16, true>) : go(grad_in_kernel<__bf16, false>);
  else g.kept.q ? go(grad_in_kernel<_Float16, true>) : go(grad_in_kernel<_Float16, false>);
  return hipGetLastError();
}

// Up to 2^22 vectors of x: larger passes fill the card by themselves, and x restored from
// a large array has too few waves in flight beside the gradient's registers and LDS (k
// 2560, n 256, gelu of x and of the product: 112.4 us apart and together at 16,384 rows,
// 244 apart and 262 together at 32,768; 784 and 812 at 131,072 without an activation of x).
bool grad_in_kept_fits(const GradIn &g, const Restore &x, const PackJob &w) {
  const int64_t items = x.m * (x.ldo / 8), pack = w.rows * (w.ldo / 8);
  const int64_t blocks = (items + pack) / kThreads + 2 + (g.n + 255) / 256 * g.row_chunks;
  return items <= (int64_t(1) << 22) && blocks < kMaxTiles;
}

hipError_t launch_grad_in_kept(int dtype, const GradIn &g, const Restore &x, const PackJob &w, hipStream_t stream) {
  const int64_t per = x.ldo / 8, items = x.m * per, pack = w.rows * (w.ldo / 8);
  Restoring r{x, Divide(uint32_t(per)), uint32_t(items), uint32_t((items + kThreads - 1) / kThreads),
              uint32_t((g.n + 255) / 256), 0};
  r.g_blocks = r.g_cols * uint32_t(g.row_chunks);
  const dim3 grid(r.g_blocks + r.x_blocks + uint32_t((pack + kThreads - 1) / kThreads));
  auto go = [&](auto kernel) { kernel<<<grid, dim3(kThreads), 0, stream>>>(g, r, w); };
  auto typed = [&](auto t) {
    typedef decltype(t) T;
    if (g.kept.q) x.act != DIP_ACT_NONE ? go(grad_in_kept_kernel<T, true, true>) : go(grad_in_kept_kernel<T, true, false>);
    else x.act != DIP_ACT_NONE ? go(grad_in_kept_kernel<T, false, true>) : go(grad_in_kept_kernel<T, false, false>);
  };
  if (dtype == DIP_BF16) typed(__bf16());
  else typed(_Float16());
  return hipGetLastError();
}

hipError_t launch_sum_rows(const SumRows &a, int out_dtype, hipStream_t stream) {
  return out_dtype == DIP_F32   ? sum_rows<float>(a, stream)
         : out_dtype == DIP_F16 ? sum_rows<_Float16>(a, stream)
                                : sum_rows<__bf16>(a, stream);
}

}  // namespace dipops
