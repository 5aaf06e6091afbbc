// kern_linear.hip -- matrix products of the stage operators.
#include "ops_internal.h"

namespace dipops {
namespace {

constexpr int kTile = 64, kStep = 32, kPad = 40, kThreads = 256;

// out tile 64 x 64, four waves of 32 x 32; operands go to LDS element by element
// as [row][k], whatever their layout, zeros beyond their ends.  The product is
// taken transposed (the weight's rows as the matrix instruction's rows), and
// the tile goes through LDS so that a lane finishes eight columns of a row.
template <class T>
__global__ __launch_bounds__(kThreads) void gemm_kernel(int64_t m, int64_t n, int64_t k, Operand a,
                                                        Operand b, Epilogue e) {
  typedef typename Vec8<T>::type V;
  __shared__ __align__(16) T sa[kTile][kPad], sb[kTile][kPad];
  __shared__ float sc[kTile][kTile + 1];
  const int64_t tiles_n = (n + kTile - 1) / kTile;
  const int64_t m0 = int64_t(blockIdx.x) / tiles_n * kTile;
  const int64_t n0 = int64_t(blockIdx.x) % tiles_n * kTile;
  const int t = threadIdx.x, lane = t % 64, wave = t / 64;
  const int wm = wave / 2 * 32, wn = wave % 2 * 32;
  f32x4 acc[2][2] = {};
  auto stage = [&](T(&s)[kTile][kPad], const Operand &o, int64_t i0, int64_t rows, int64_t k0) {
    for (int j = t; j < kTile * kStep; j += kThreads) {
      const int r = o.k_rows ? j % kTile : j / kStep, c = o.k_rows ? j / kTile : j % kStep;
      const int64_t i = i0 + r, kk = k0 + c;
      T v = T(0.f);
      if (i < rows && kk < k) v = static_cast<const T *>(o.p)[o.k_rows ? kk * o.ld + i : i * o.ld + kk];
      s[r][c] = v;
    }
  };
  for (int64_t k0 = 0; k0 < k; k0 += kStep) {
    stage(sa, a, m0, m, k0);
    stage(sb, b, n0, n, k0);
    __syncthreads();
    for (int i = 0; i < 2; ++i)
      for (int j = 0; j < 2; ++j) {
        const V x = *reinterpret_cast<const V *>(&sa[wm + 16 * i + lane % 16][lane / 16 * 8]);
        const V w = *reinterpret_cast<const V *>(&sb[wn + 16 * j + lane % 16][lane / 16 * 8]);
        acc[i][j] = mfma16(w, x, acc[i][j]);
      }
    __syncthreads();
  }
  for (int i = 0; i < 2; ++i)
    for (int j = 0; j < 2; ++j)
      for (int q = 0; q < 4; ++q)
        sc[wm + 16 * i + lane % 16][wn + 16 * j + lane / 16 * 4 + q] = acc[i][j][q];
  __syncthreads();
  for (int j = t; j < kTile * kTile / 8; j += kThreads) {
    const int r = j / (kTile / 8), c = j % (kTile / 8) * 8;
    if (m0 + r >= m || n0 + c >= n) continue;
    float v[8];
    for (int q = 0; q < 8; ++q) v[q] = sc[r][c + q];
    finish8<T>(e, m0 + r, n0 + c, int(min(int64_t(8), n - n0 - c)), v);
  }
}

template <class T>
hipError_t run(int64_t m, int64_t n, int64_t k, const Operand &a, const Operand &b,
               const Epilogue &e, hipStream_t stream) {
  const int64_t tiles = ((m + kTile - 1) / kTile) * ((n + kTile - 1) / kTile);
  gemm_kernel<T><<<dim3(uint32_t(tiles)), dim3(kThreads), 0, stream>>>(m, n, k, a, b, e);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_gemm(int dtype, int64_t m, int64_t n, int64_t k, const Operand &a,
                       const Operand &b, const Epilogue &e, hipStream_t stream) {
  return dtype == DIP_BF16 ? run<__bf16>(m, n, k, a, b, e, stream)
                           : run<_Float16>(m, n, k, a, b, e, stream);
}

}  // namespace dipops
