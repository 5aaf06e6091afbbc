// kern_thin.hip -- dip_linear for few rows of x: y = epilogue(x w^T).
//
// Bound by reading w once, and for small w by latency.  A workgroup takes 16 or 32
// rows of w and its eight waves an eighth of the contraction each; a lane reads its
// fragments of w and x straight into registers, eight of each at once, so that all
// of a wave's loads are on their way before the first product, and at any
// alignment.  The eight partial results meet in LDS: one launch, no workspace.
// bf16, one row: 4096 x 3584 7.7 us a call (3.8 TB/s of w), 4096 x 14336 27 us
// (4.4 TB/s); by tiles, split 16 ways and joined, the first took 14.
#include "ops_internal.h"

namespace dipops {
namespace {

constexpr int kWaves = 8;

// MF x 16 rows of x, NF x 16 rows of w a workgroup, U fragments at once.
template <class T, int MF, int NF, int U>
__global__ __launch_bounds__(64 * kWaves) void thin_kernel(int m, int64_t n, int64_t k, const T *x, int64_t ldx,
                                                           const T *w, int64_t ldw, Epilogue e) {
  typedef typename Vec8<T>::type V;
  typedef typename Any8<T>::type VA;
  __shared__ float s[kWaves][16 * MF][16 * NF + 1];
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, r = lane % 16, g = lane / 16;
  const int64_t n0 = int64_t(blockIdx.x) * (16 * NF);
  // rows beyond the arrays read the last one: their results are not written
  const T *wp[NF], *xp[MF];
#pragma unroll
  for (int f = 0; f < NF; ++f) wp[f] = w + min(n0 + 16 * f + r, n - 1) * ldw + 8 * g;
#pragma unroll
  for (int f = 0; f < MF; ++f) xp[f] = x + int64_t(min(16 * f + r, m - 1)) * ldx + 8 * g;
  const int64_t per = (k + 32 * kWaves - 1) / (32 * kWaves) * 32, k0 = per * wave, k1 = min(k0 + per, k);
  f32x4 acc[MF][NF];
#pragma unroll
  for (int i = 0; i < MF; ++i)
#pragma unroll
    for (int f = 0; f < NF; ++f) acc[i][f] = f32x4{0.f, 0.f, 0.f, 0.f};
  int64_t at = k0;
  for (; at + 32 * U <= k1; at += 32 * U) {
    V wv[U][NF], xv[U][MF];
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
      for (int f = 0; f < NF; ++f) wv[u][f] = *reinterpret_cast<const VA *>(wp[f] + at + 32 * u);
#pragma unroll
      for (int f = 0; f < MF; ++f) xv[u][f] = *reinterpret_cast<const VA *>(xp[f] + at + 32 * u);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < MF; ++i)
#pragma unroll
        for (int f = 0; f < NF; ++f) mfma16(wv[u][f], xv[u][i], acc[i][f]);
  }
  for (; at < k1; at += 32) {
    const int left = int(min(int64_t(8), k1 - at - 8 * g));
    V wv[NF], xv[MF];
    auto part = [&](const T *p) {
      float v[8];
      load8(p + at, left, v);
      return round8<T>(v);   // exact: the values are of the type
    };
#pragma unroll
    for (int f = 0; f < NF; ++f) wv[f] = part(wp[f]);
#pragma unroll
    for (int f = 0; f < MF; ++f) xv[f] = part(xp[f]);
#pragma unroll
    for (int i = 0; i < MF; ++i)
#pragma unroll
      for (int f = 0; f < NF; ++f) mfma16(wv[f], xv[i], acc[i][f]);
  }
#pragma unroll
  for (int i = 0; i < MF; ++i)
#pragma unroll
    for (int f = 0; f < NF; ++f) {
#pragma unroll
      for (int q = 0; q < 4; ++q) s[wave][16 * i + r][16 * f + 4 * g + q] = acc[i][f][q];
    }
  __syncthreads();
  constexpr int kParts = 2 * NF;   // of eight columns a row
  for (int j = threadIdx.x; j < 16 * MF * kParts; j += 64 * kWaves) {
    const int row = j / kParts, c = j % kParts * 8;
    if (row >= m || n0 + c >= n) continue;
    float v[8];
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      v[q] = s[0][row][c + q];
#pragma unroll
      for (int u = 1; u < kWaves; ++u) v[q] += s[u][row][c + q];
    }
    finish8<T>(e, row, n0 + c, int(min(int64_t(8), n - n0 - c)), v);
  }
}

template <class T>
hipError_t run(int m, int64_t n, int64_t k, const void *x, int64_t ldx, const void *w, int64_t ldw, const Epilogue &e,
               hipStream_t stream) {
  // 32 rows of w a workgroup where that still gives every CU one: x is read from
  // the caches half as often
  const bool two = n >= 32 * 256;
  const dim3 grid(uint32_t((n + (two ? 31 : 15)) / (two ? 32 : 16)));
  auto go = [&](auto kernel) {
    kernel<<<grid, dim3(64 * kWaves), 0, stream>>>(m, n, k, static_cast<const T *>(x), ldx, static_cast<const T *>(w),
                                                   ldw, e);
  };
  if (m <= 16) two ? go(thin_kernel<T, 1, 2, 8>) : go(thin_kernel<T, 1, 1, 8>);
  else two ? go(thin_kernel<T, 2, 2, 8>) : go(thin_kernel<T, 2, 1, 8>);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_thin(int dtype, int64_t m, int64_t n, int64_t k, const void *x, int64_t ldx, const void *w,
                       int64_t ldw, const Epilogue &e, hipStream_t stream) {
  return dtype == DIP_BF16 ? run<__bf16>(int(m), n, k, x, ldx, w, ldw, e, stream)
                           : run<_Float16>(int(m), n, k, x, ldx, w, ldw, e, stream);
}

}  // namespace dipops
