// kern_thin.hip -- dip_linear for few rows of x: y = epilogue(x w^T).
//
// Bound by reading w once, and for small w by latency.  A workgroup takes 8 to 32
// rows of w and its eight waves an eighth of the contraction each; a lane reads its
// fragments of w and x straight into registers, eight of w at once, so that a wave's
// loads are on their way before the first product, at any alignment; what is left
// of the wave's part is one more batch.  The partial results meet in LDS: one
// launch, no workspace.
// bf16, w from memory: one row, 4096 x 3584 8.5 to 8.8 us alone (3.4 TB/s of w) and 9.6 a
// launch among others, 4096 x 14336 26 (4.5); 8 rows, 13696 x 1664 17.5 (28 with 16 rows
// of w a workgroup, on 104 CUs of 256), 7 rows, 5184 x 256 7.5 (12).
#include "ops_internal.h"

namespace dipops {
namespace {

// MF x R rows of x, NF x R rows of w a workgroup, U fragments at once, the
// contraction shared by kWaves waves.  A fragment's 16 rows are R rows of 16 / R
// pieces each, side by side along the contraction, of w as of x: the products of
// equal pieces stand in the result's diagonal blocks and are added, the others
// dropped.  A load then takes 64 * 16 / R bytes of a row.
template <class T, int MF, int NF, int U, int R, int kWaves>
__global__ __launch_bounds__(64 * kWaves) void thin_kernel(int m, int64_t n, int64_t k, const T *x, int64_t ldx,
                                                           const T *w, int64_t ldw, Epilogue e) {
  typedef typename Vec8<T>::type V;
  typedef typename Any8<T>::type VA;
  constexpr int kPieces = 16 / R, kAt = 32 * kPieces;   // contraction elements a fragment
  __shared__ float s[kWaves * kPieces][R * MF][R * NF + 1];
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, r = lane % R, piece = lane % 16 / R, g = lane / 16;
  const int mine = 32 * piece + 8 * g;   // a lane's eight elements of a fragment
  const int64_t n0 = int64_t(blockIdx.x) * (R * NF);
  // rows beyond the arrays read the last one: their results are not written
  const T *wp[NF], *xp[MF];
#pragma unroll
  for (int f = 0; f < NF; ++f) wp[f] = w + min(n0 + R * f + r, n - 1) * ldw + mine;
#pragma unroll
  for (int f = 0; f < MF; ++f) xp[f] = x + int64_t(min(R * f + r, m - 1)) * ldx + mine;
  const int64_t per = (k + kAt * kWaves - 1) / (kAt * kWaves) * kAt, k0 = per * wave, k1 = min(k0 + per, k);
  f32x4 acc[MF][NF];
#pragma unroll
  for (int i = 0; i < MF; ++i)
#pragma unroll
    for (int f = 0; f < NF; ++f) acc[i][f] = f32x4{0.f, 0.f, 0.f, 0.f};
  int64_t at = k0;
  for (; at + kAt * U <= k1; at += kAt * U) {
    V wv[U][NF], xv[U][MF];
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
      for (int f = 0; f < NF; ++f) wv[u][f] = *reinterpret_cast<const VA *>(wp[f] + at + kAt * u);
#pragma unroll
      for (int f = 0; f < MF; ++f) xv[u][f] = *reinterpret_cast<const VA *>(xp[f] + at + kAt * u);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < MF; ++i)
#pragma unroll
        for (int f = 0; f < NF; ++f) mfma16(wv[u][f], xv[u][i], acc[i][f]);
  }
  // what is left of the wave's part: whole vectors at once, zeros beyond them
  const int64_t whole = min(k1, k & ~int64_t(7));
  if (at < whole) {
    V wv[U][NF] = {}, xv[U][MF] = {};
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (at + kAt * u + mine >= whole) continue;
#pragma unroll
      for (int f = 0; f < NF; ++f) wv[u][f] = *reinterpret_cast<const VA *>(wp[f] + at + kAt * u);
#pragma unroll
      for (int f = 0; f < MF; ++f) xv[u][f] = *reinterpret_cast<const VA *>(xp[f] + at + kAt * u);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < MF; ++i)
#pragma unroll
        for (int f = 0; f < NF; ++f) mfma16(wv[u][f], xv[u][i], acc[i][f]);
  }
  // the last k % 8, by the wave whose part ends there
  if (k0 < k1 && whole < k1) {
    const int left = mine == 0 ? int(k1 - whole) : 0;
    V wv[NF], xv[MF];
    auto part = [&](const T *p) {
      float v[8];
      load8(p - mine + whole, left, v);
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
      if (4 * g / R != piece) continue;   // R >= 4: a lane's four are of one block
#pragma unroll
      for (int q = 0; q < 4; ++q) s[wave * kPieces + piece][R * i + r][R * f + 4 * g % R + q] = acc[i][f][q];
    }
  __syncthreads();
  for (int j = threadIdx.x; j < R * MF * R * NF; j += 64 * kWaves) {
    float *p = &s[0][j / (R * NF)][j % (R * NF)], v = p[0];
#pragma unroll
    for (int u = 1; u < kWaves * kPieces; ++u) v += p[u * (R * MF * (R * NF + 1))];
    p[0] = v;
  }
  __syncthreads();
  static_assert(R * NF % 8 == 0);
  constexpr int kParts = R * NF / 8;   // of eight columns a row
  for (int j = threadIdx.x; j < R * MF * kParts; j += 64 * kWaves) {
    const int row = j / kParts, c = j % kParts * 8;
    if (row >= m || n0 + c >= n) continue;
    float v[8];
#pragma unroll
    for (int q = 0; q < 8; ++q) v[q] = s[0][row][c + q];
    finish8<T>(e, row, n0 + c, int(min(int64_t(8), n - n0 - c)), v);
  }
}

template <class T>
hipError_t run(int m, int64_t n, int64_t k, const void *x, int64_t ldx, const void *w, int64_t ldw, const Epilogue &e,
               hipStream_t stream) {
  // 32 rows of w a workgroup where that still gives every CU one: x is read from
  // the caches half as often.  Below, 8 where x has no more (4096 x 3584, one row: 9.4
  // us, with 16 10.2), else 16.
  const bool two = n >= 32 * 256;
  auto go = [&](auto kernel, int rows, int waves) {
    kernel<<<dim3(uint32_t((n + rows - 1) / rows)), dim3(64 * waves), 0, stream>>>(
        m, n, k, static_cast<const T *>(x), ldx, static_cast<const T *>(w), ldw, e);
  };
  if (m <= 8) two ? go(thin_kernel<T, 1, 4, 2, 8, 8>, 32, 8) : go(thin_kernel<T, 1, 1, 8, 8, 8>, 8, 8);
  else if (m <= 16) two ? go(thin_kernel<T, 1, 2, 8, 16, 8>, 32, 8) : go(thin_kernel<T, 1, 1, 8, 16, 8>, 16, 8);
  else two ? go(thin_kernel<T, 2, 2, 8, 16, 8>, 32, 8) : go(thin_kernel<T, 2, 1, 8, 16, 8>, 16, 8);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_thin(int dtype, int64_t m, int64_t n, int64_t k, const void *x, int64_t ldx, const void *w,
                       int64_t ldw, const Epilogue &e, hipStream_t stream) {
  return dtype == DIP_BF16 ? run<__bf16>(int(m), n, k, x, ldx, w, ldw, e, stream)
                           : run<_Float16>(int(m), n, k, x, ldx, w, ldw, e, stream);
}

}  // namespace dipops
