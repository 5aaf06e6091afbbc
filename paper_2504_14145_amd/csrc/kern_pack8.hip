// kern_pack8.hip -- activations kept in 8 bits, and restored.
#include <algorithm>

#include "ops_internal.h"

namespace dipops {
namespace {

constexpr int kThreads = 256;

// Eight columns of a row a thread, four threads a scale; `per` is a multiple of four,
// so that those are of one wave and all there.
template <class T>
__global__ __launch_bounds__(kThreads) void pack8_kernel(uint32_t items, uint32_t row0, Divide per, int64_t n,
                                                         const T *x, int64_t ldx, Packed out) {
  const uint32_t i = blockIdx.x * kThreads + threadIdx.x;
  if (i >= items) return;
  const uint32_t in = per(i);
  const int64_t row = int64_t(row0) + in, col = int64_t(i - in * per.by) * 8;
  const int left = int(min(int64_t(8), n - col));
  float v[8];
  load8(x + row * ldx + col, left, v);
  pack8_quad(out, row, col, left, v);
}

template <class T>
__global__ __launch_bounds__(kThreads) void unpack8_kernel(uint32_t items, uint32_t row0, Divide per, int64_t n,
                                                           Packed x, int act, T *y, int64_t ldy, int64_t fill) {
  const uint32_t i = blockIdx.x * kThreads + threadIdx.x;
  if (i >= items) return;
  const uint32_t in = per(i);
  const int64_t row = int64_t(row0) + in, col = int64_t(i - in * per.by) * 8;
  const int left = int(min(int64_t(8), n - col));
  float v[8] = {};
  if (left > 0) {
    from8bits(load8bits(x.q + row * x.ld + col, left), scale_of(x.s[row * x.lds + col / 32]), v);
    if (act == DIP_ACT_SILU) {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = act_of(v[j], DIP_ACT_SILU);
    } else if (act == DIP_ACT_GELU) {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = act_of(v[j], DIP_ACT_GELU);
    } else if (act == DIP_ACT_RELU) {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = act_of(v[j], DIP_ACT_RELU);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = j < left ? within<T>(v[j]) : 0.f;
  }
  store8(y + row * ldy + col, int(min(int64_t(8), fill - col)), v);
}

// f(items, row0, Divide(per)) over launches of fewer than 2^31 items.
template <class F>
hipError_t pieces(int64_t m, int64_t per, F &&f) {
  const int64_t most = ((int64_t(1) << 31) - 1) / per;
  for (int64_t row0 = 0; row0 < m; row0 += most) {
    const uint32_t items = uint32_t(std::min(most, m - row0) * per);
    f(dim3((items + kThreads - 1) / kThreads), items, uint32_t(row0), Divide(uint32_t(per)));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <class T>
hipError_t pack(int64_t m, int64_t n, const void *x, int64_t ldx, const Packed &out, hipStream_t st) {
  return pieces(m, (n + 31) / 32 * 4, [&](dim3 grid, uint32_t items, uint32_t row0, const Divide &per) {
    pack8_kernel<T><<<grid, dim3(kThreads), 0, st>>>(items, row0, per, n, static_cast<const T *>(x), ldx, out);
  });
}
template <class T>
hipError_t unpack(int64_t m, int64_t n, const Packed &x, int act, void *y, int64_t ldy, int64_t fill, hipStream_t st) {
  return pieces(m, (fill + 7) / 8, [&](dim3 grid, uint32_t items, uint32_t row0, const Divide &per) {
    unpack8_kernel<T><<<grid, dim3(kThreads), 0, st>>>(items, row0, per, n, x, act, static_cast<T *>(y), ldy, fill);
  });
}

}  // namespace

hipError_t launch_pack8(int dtype, int64_t m, int64_t n, const void *x, int64_t ldx, const Packed &out,
                        hipStream_t stream) {
  switch (dtype) {
    case DIP_F32: return pack<float>(m, n, x, ldx, out, stream);
    case DIP_F16: return pack<_Float16>(m, n, x, ldx, out, stream);
    default: return pack<__bf16>(m, n, x, ldx, out, stream);
  }
}

hipError_t launch_unpack8(int dtype, int64_t m, int64_t n, const Packed &x, int act, void *y, int64_t ldy, int64_t fill,
                          hipStream_t stream) {
  switch (dtype) {
    case DIP_F32: return unpack<float>(m, n, x, act, y, ldy, fill, stream);
    case DIP_F16: return unpack<_Float16>(m, n, x, act, y, ldy, fill, stream);
    default: return unpack<__bf16>(m, n, x, act, y, ldy, fill, stream);
  }
}

}  // namespace dipops
