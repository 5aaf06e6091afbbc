// kern_rmsnorm.hip -- root-mean-square norm with the residual's addition and an
// output in 8 bits, and its gradients.
//
// Bound by memory: x and the residual read, their sum and the norm written forward,
// dy, the sum and its gradient read and one array written backward, against some 15
// operations an element (36 instructions where it is packed too: 63 % of the issue).  A
// row of up to 16,384 columns is held in registers from its load to its stores; longer
// rows are read a second time, out of the caches.  The gradient's workgroups go over
// rows and keep the sums of dgamma on the way; of few rows dgamma is summed beside dx.
// bf16, 65,536 x 3584 with the residual: 372 us forward with the 8 bits (5.7 TB/s), 321
// without, 335 to 344 + 5 the gradient (5.5); 8192 x 4096 56 and 53; 149 x 4096 4.8 and 4.1
// a launch; 1201 x 1795 float32 7.7 and 7.9 + 5.  Rows
// beyond 16,384 columns: 4.2 TB/s, and 3 for the gradient, which reads dy and the sum
// in two launches.
#include <algorithm>
#include <type_traits>

#include "ops_internal.h"

namespace dipops {
namespace {

// Columns of a row held in registers; up to the second number the gradient's next row
// fits beside its own, and gamma (1024 threads have 128 registers each).
constexpr int kHeldMost = 16384, kAheadMost = 8192;

// The sum over LANES consecutive lanes of a wave, the same in all of them: neighbours,
// pairs, fours and eights within a row of sixteen, then rows and halves, without a way
// through the LDS.  What a step exchanges is already the same in the group that it
// comes from, so mirrored lanes serve.
template <class F>
__device__ __forceinline__ F exchanged(F v, int step) {
  constexpr int kWords = sizeof(F) / 4;
  struct Words {
    int w[kWords];
  };
  Words a = __builtin_bit_cast(Words, v);
#pragma unroll
  for (int i = 0; i < kWords; ++i) {
    if (step == 1) a.w[i] = __builtin_amdgcn_mov_dpp(a.w[i], 0xb1, 0xf, 0xf, true);         // lane ^ 1
    else if (step == 2) a.w[i] = __builtin_amdgcn_mov_dpp(a.w[i], 0x4e, 0xf, 0xf, true);    // lane ^ 2
    else if (step == 4) a.w[i] = __builtin_amdgcn_mov_dpp(a.w[i], 0x141, 0xf, 0xf, true);   // 7 - lane of eight
    else a.w[i] = __builtin_amdgcn_mov_dpp(a.w[i], 0x140, 0xf, 0xf, true);                  // 15 - lane of sixteen
  }
  return __builtin_bit_cast(F, a);
}
// The sum of a value and that 16 (HALVES: 32) lanes away.
template <bool HALVES, class F>
__device__ __forceinline__ F swapped_sum(F v) {
  constexpr int kWords = sizeof(F) / 4;
  struct Words {
    uint32_t w[kWords];
  };
  Words a = __builtin_bit_cast(Words, v), b = a;
#pragma unroll
  for (int i = 0; i < kWords; ++i) {
    if constexpr (HALVES) {
      const auto r = __builtin_amdgcn_permlane32_swap(a.w[i], b.w[i], false, false);
      a.w[i] = r[0], b.w[i] = r[1];
    } else {
      const auto r = __builtin_amdgcn_permlane16_swap(a.w[i], b.w[i], false, false);
      a.w[i] = r[0], b.w[i] = r[1];
    }
  }
  return __builtin_bit_cast(F, a) + __builtin_bit_cast(F, b);
}
template <int LANES, class F>
__device__ __forceinline__ F lanes_sum(F v) {
#pragma unroll
  for (int d = 1; d < (LANES < 16 ? LANES : 16); d *= 2) v += exchanged(v, d);
  if constexpr (LANES > 16) v = swapped_sum<false>(v);
  if constexpr (LANES > 32) v = swapped_sum<true>(v);
  return v;
}

// A row's threads: LANES of a wave, a power of two from four on, or, LANES 0, the whole
// workgroup, as many waves as the row fills.
template <int LANES>
struct Lanes {
  static constexpr bool kWide = LANES == 0;
  static constexpr int kMost = kWide ? 1024 : 256;           // threads a workgroup
  static constexpr int kRows = kWide ? 1 : 256 / LANES;      // rows a workgroup has at once
  static __device__ __forceinline__ int count() { return kWide ? int(blockDim.x) : LANES; }
  static __device__ __forceinline__ int mine() { return kWide ? int(threadIdx.x) : int(threadIdx.x) % LANES; }
  static __device__ __forceinline__ int row() { return kWide ? 0 : int(threadIdx.x) / LANES; }
  // Their sum; beyond a wave s holds two sets of the waves' values in turn, so that one
  // barrier a sum is enough.
  static constexpr int kSums = kWide ? 32 : 1;
  template <class F>
  static __device__ __forceinline__ F sum(F v, F *s, int &turn) {
    v = lanes_sum<(kWide ? 64 : LANES)>(v);
    if constexpr (kWide) {
      const int waves = int(blockDim.x) / 64;
      if (waves == 1) return v;
      F *q = s + turn * 16;
      turn ^= 1;
      if (threadIdx.x % 64 == 0) q[threadIdx.x / 64] = v;
      __syncthreads();
      v = lanes_sum<16>(int(threadIdx.x % 16) < waves ? q[threadIdx.x % 16] : F(0));
    }
    return v;
  }
};

template <class T>
__device__ __forceinline__ void gamma8(const void *gamma, int c, int n, float (&g)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) g[i] = 1.f;
  if (gamma) {
    Held<T> h;
    h.get(static_cast<const T *>(gamma), c, n);
    h.to(Held<T>::moved(c, n), g);
  }
}

// t = x + residual of eight columns, rounded to the type.
template <class T>
__device__ __forceinline__ void total8(const Held<T> &x, const Held<T> &r, bool residual, int by, float (&v)[8]) {
  x.to(by, v);
  if (residual) {
    float q[8];
    r.to(by, q);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = float(T(v[i] + q[i]));
  }
}

// 1 / sqrt(sum / n + eps) in float64, from the hardware's estimate and one step of third
// order, as a float32 and what its rounding left off.  Squares are exact in float64 and
// summed in it (two instructions an element, no time beside the memory's: 65,536 x 3584
// with the 8 bits 378 us as with float32 sums, 2^26 elements in rows of 515 to 2051
// within 1 %), so v + rest is off by 2^-47 at most, of the longest rows, 4096 squares a
// thread, by 2^-41, however alike the values, and rows whose squares no float32 holds
// have theirs too.
struct Rstd {
  float v, rest;
  __device__ __forceinline__ Rstd(double sum, double inv, float eps) {   // inv: 1 / n
    const double mean = fma(sum, inv, double(eps));
    double r = __builtin_amdgcn_rsq(mean);
    const double t = mean * r, below = fma(mean, r, -t);
    const double off = fma(-below, r, fma(-t, r, 1.0));                        // 1 - mean r^2
    r = fabs(off) < 1e-3 ? fma(r * off, fma(off, 0.375, 0.5), r) : r;          // not of an infinity or zero
    v = float(r);
    rest = v < INFINITY ? float(r - double(v)) : 0.f;
  }
};
__device__ __forceinline__ void add_squares(const float (&v)[8], double &sum) {
#pragma unroll
  for (int q = 0; q < 8; ++q) sum = fma(double(v[q]), double(v[q]), sum);
}

// t rstd as a float32 and what its rounding left off, together to 2^-45.  gamma comes
// after it: t rstd is at most sqrt(c), where gamma t may leave float32's range though y
// does not, and y is rounded once.
struct Normed {
  float s, e;
  __device__ __forceinline__ Normed(float t, const Rstd &rstd) {
    s = t * rstd.v;
    e = fmaf(t, rstd.rest, fmaf(t, rstd.v, -s));
  }
  __device__ __forceinline__ float times(float g) const { return fmaf(s, g, e * g); }
  // what is left of it beside y = times(g)
  __device__ __forceinline__ float beside(float g, float y) const { return fmaf(s, g, -y) + e * g; }
};

// y and its 8 bits from t; of the four lanes that share a scale all are here.
template <class T, bool PACK>
__device__ __forceinline__ void write8(const dip_rms_norm_args &a, const Packed &p, int64_t row, int c, const Rstd &rstd,
                                       const float (&v)[8]) {
  const int n = int(a.c), left = n - c;
  float g[8], y[8];
  gamma8<T>(a.gamma, c, n, g);
#pragma unroll
  for (int q = 0; q < 8; ++q) y[q] = Normed(v[q], rstd).times(g[q]);
  if (a.y && left > 0) put8(static_cast<T *>(a.y) + row * a.ldy + c, left, y);
  if constexpr (PACK) {
    // A float32 that ends in nineteen zeros may be the middle of two 8-bit values, on
    // which rounding has put what lies beside it: one in 2^19.  It goes to its side; what
    // is nearer than this arithmetic tells counts as the middle.
    constexpr uint32_t kLow = 0x7ffffu;
    uint32_t low = kLow;
    if (left >= 8) {
#pragma unroll
      for (int q = 0; q < 8; ++q) low = min(low, magnitude(y[q]) & kLow);
    } else if (left > 0) {   // not the zeros beyond the row
#pragma unroll
      for (int q = 0; q < 8; ++q) low = q < left ? min(low, magnitude(y[q]) & kLow) : low;
    }
    if (low == 0) {
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        const float beside = Normed(v[q], rstd).beside(g[q], y[q]);
        const uint32_t bits = magnitude(y[q]);
        if ((bits & kLow) == 0 && bits - 1 < kInfinity - 1 && fabsf(beside) > 0x1p-40f * fabsf(y[q])) {
          const bool out = (beside > 0.f) == (y[q] > 0.f);
          y[q] = copysignf(__builtin_bit_cast(float, bits + (out ? 1u : ~0u)), y[q]);
        }
      }
    }
    pack8_quad(p, row, c, left, y);   // zeros beyond the row, or NaN
  }
}

// NV vectors a thread.
template <class T, int LANES, int NV, bool PACK>
__global__ __launch_bounds__(Lanes<LANES>::kMost) void rms_rows_kernel(dip_rms_norm_args a, int64_t row0, double inv, Packed p) {
  typedef Lanes<LANES> L;
  __shared__ double s[L::kSums];
  int turn = 0;
  const int t = L::mine(), lanes = L::count(), n = int(a.c);
  const int64_t row = row0 + int64_t(blockIdx.x) * L::kRows + L::row();
  if (row >= a.m) return;   // all lanes of a row
  Held<T> x[NV], r[NV];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int c = (t + j * lanes) * 8;
    x[j].get(static_cast<const T *>(a.x) + row * a.ldx, c, n);
    if (a.residual) r[j].get(static_cast<const T *>(a.residual) + row * a.ldr, c, n);
  }
  float v[NV][8];
  double sum = 0.0;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    total8(x[j], r[j], a.residual != nullptr, Held<T>::moved((t + j * lanes) * 8, n), v[j]);
    add_squares(v[j], sum);
  }
  if (a.total) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (t + j * lanes) * 8;
      if (c < n) put8(static_cast<T *>(a.total) + row * a.ldt + c, n - c, v[j]);
    }
  }
  const Rstd rstd(L::sum(sum, s, turn), inv, a.eps);
  if (t == 0 && a.rstd) a.rstd[row] = rstd.v;
#pragma unroll
  for (int j = 0; j < NV; ++j) write8<T, PACK>(a, p, row, (t + j * lanes) * 8, rstd, v[j]);
}

// Rows of any length: a workgroup goes over its row twice.  Where the sum is stored a
// thread reads back what it wrote (the residual may be gone: they may be one array).
template <class T, bool PACK>
__global__ __launch_bounds__(1024) void rms_long_kernel(dip_rms_norm_args a, int64_t row0, double inv, Packed p) {
  __shared__ double s[Lanes<0>::kSums];
  int turn = 0;
  const int t = threadIdx.x, n = int(a.c);
  const int64_t row = row0 + blockIdx.x;
  const T *x = static_cast<const T *>(a.x) + row * a.ldx;
  const T *r = a.residual ? static_cast<const T *>(a.residual) + row * a.ldr : nullptr;
  T *total = a.total ? static_cast<T *>(a.total) + row * a.ldt : nullptr;
  auto first = [&](int c, float(&v)[8]) __attribute__((always_inline)) {
    const int left = n - c;
    load8(x + c, left, v);
    if (r) {
      float q[8];
      load8(r + c, left, q);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = float(T(v[i] + q[i]));
    }
  };
  double sum = 0.0;
  for (int c = t * 8; c < n; c += 1024 * 8) {
    float v[8];
    first(c, v);
    add_squares(v, sum);
    if (total) put8(total + c, n - c, v);
  }
  const Rstd rstd(Lanes<0>::sum(sum, s, turn), inv, a.eps);
  if (t == 0 && a.rstd) a.rstd[row] = rstd.v;
  for (int c = t * 8; c < (n + 31) / 32 * 32; c += 1024 * 8) {
    float v[8] = {};
    if (c < n) {
      if (total) load8(total + c, n - c, v);
      else first(c, v);
    }
    write8<T, PACK>(a, p, row, c, rstd, v);
  }
}

// ------------------------------------------------------------ gradients

// A workgroup goes over rows j, j + gridDim.x, .. (kRows at a time) and keeps the sums
// of dgamma of its columns on the way: partial[j][c].
template <class T, int LANES, int NV>
__global__ __launch_bounds__(Lanes<LANES>::kMost) void rms_grad_kernel(dip_rms_norm_grad_args a, float *partial) {
  typedef Lanes<LANES> L;
  constexpr int kRows = L::kRows;
  __shared__ float s[L::kSums];
  __shared__ float sums[kRows > 1 ? kRows * LANES * NV * 8 : 1];
  int turn = 0;
  const int t = L::mine(), lanes = L::count(), n = int(a.c);
  constexpr bool kAhead = LANES > 0 || NV == 1;
  float g[kAhead ? NV : 1][8], sg[NV][8] = {};
  if constexpr (kAhead) {
#pragma unroll
    for (int j = 0; j < NV; ++j) gamma8<T>(a.gamma, (t + j * lanes) * 8, n, g[j]);
  }
  // the next row is asked for before this one's sum is waited for
  Held<T> xn[NV], dn[NV], tn[NV];
  float rn = 0.f;
  auto fetch = [&](int64_t row) __attribute__((always_inline)) {
    rn = a.rstd[row];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (t + j * lanes) * 8;
      xn[j].get(static_cast<const T *>(a.total) + row * a.ldt, c, n);
      dn[j].get(static_cast<const T *>(a.dy) + row * a.ldy, c, n);
      if (a.dtotal && a.dx) tn[j].get(static_cast<const T *>(a.dtotal) + row * a.lddt, c, n);
    }
  };
  const int64_t step = int64_t(gridDim.x) * kRows;
  int64_t row = int64_t(blockIdx.x) * kRows + L::row();
  if (kAhead && row < a.m) fetch(row);
  for (; row < a.m; row += step) {   // all lanes of a row
    if (!kAhead) fetch(row);
    const float rstd = rn;
    float xh[NV][8], h[NV][8], dot = 0.f;
    Held<T> along[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (t + j * lanes) * 8, by = Held<T>::moved(c, n);
      xn[j].to(by, xh[j]);
      dn[j].to(by, h[j]);
      along[j] = tn[j];
      if constexpr (!kAhead) gamma8<T>(a.gamma, c, n, g[0]);
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        xh[j][q] *= rstd;
        sg[j][q] += h[j][q] * xh[j][q];
        h[j][q] *= g[kAhead ? j : 0][q];
        dot += h[j][q] * xh[j][q];
      }
    }
    if (kAhead && row + step < a.m) fetch(row + step);
    if (!a.dx) continue;
    dot = L::sum(dot, s, turn) / float(n);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (t + j * lanes) * 8;
      float v[8] = {};
      if (a.dtotal) along[j].to(Held<T>::moved(c, n), v);
#pragma unroll
      for (int q = 0; q < 8; ++q) v[q] += rstd * (h[j][q] - xh[j][q] * dot);
      if (c < n) put8(static_cast<T *>(a.dx) + row * a.lddx + c, n - c, v);
    }
  }
  if (!partial) return;
  if constexpr (kRows > 1) {   // its rows' sums, in their order
    float *mine = sums + L::row() * (LANES * NV * 8);
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int q = 0; q < 8; ++q) mine[(t + j * LANES) * 8 + q] = sg[j][q];
    __syncthreads();
    for (int c = threadIdx.x; c < n; c += 256) {
      float v = sums[c];
      for (int i = 1; i < kRows; ++i) v += sums[i * (LANES * NV * 8) + c];
      partial[int64_t(blockIdx.x) * n + c] = v;
    }
  } else {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (t + j * lanes) * 8;
      if (c < n) put8(partial + int64_t(blockIdx.x) * n + c, n - c, sg[j]);
    }
  }
}

// Few rows: dx by workgroups of kRows rows, and dgamma beside them by workgroups of 64
// columns that read the rows again, out of the caches: one launch, no workspace.
template <class T, class G, int LANES, int NV>
__global__ __launch_bounds__(Lanes<LANES>::kMost) void rms_few_grad_kernel(dip_rms_norm_grad_args a, int row_blocks) {
  typedef Lanes<LANES> L;
  __shared__ float s[L::kSums];
  __shared__ float sums[L::kMost / 8][64 + 2];
  const int n = int(a.c);
  if (int(blockIdx.x) < row_blocks) {
    int turn = 0;
    const int t = L::mine(), lanes = L::count();
    const int64_t row = int64_t(blockIdx.x) * L::kRows + L::row();
    if (row >= a.m) return;   // all lanes of a row
    const float rstd = a.rstd[row];
    Held<T> x[NV], d[NV], along[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (t + j * lanes) * 8;
      x[j].get(static_cast<const T *>(a.total) + row * a.ldt, c, n);
      d[j].get(static_cast<const T *>(a.dy) + row * a.ldy, c, n);
      if (a.dtotal) along[j].get(static_cast<const T *>(a.dtotal) + row * a.lddt, c, n);
    }
    float xh[NV][8], h[NV][8], dot = 0.f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      float g[8];
      gamma8<T>(a.gamma, (t + j * lanes) * 8, n, g);
      const int by = Held<T>::moved((t + j * lanes) * 8, n);
      x[j].to(by, xh[j]);
      d[j].to(by, h[j]);
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        xh[j][q] *= rstd;
        h[j][q] *= g[q];
        dot += h[j][q] * xh[j][q];
      }
    }
    dot = L::sum(dot, s, turn) / float(n);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (t + j * lanes) * 8;
      float v[8] = {};
      if (a.dtotal) along[j].to(Held<T>::moved(c, n), v);
#pragma unroll
      for (int q = 0; q < 8; ++q) v[q] += rstd * (h[j][q] - xh[j][q] * dot);
      if (c < n) put8(static_cast<T *>(a.dx) + row * a.lddx + c, n - c, v);
    }
    return;
  }
  const int c0 = (int(blockIdx.x) - row_blocks) * 64, c = c0 + int(threadIdx.x % 8) * 8, ty = threadIdx.x / 8;
  float sum[8] = {};
  if (c < n) {
    // rows ty, ty + step, ..: four at a time, their loads first
    const T *x = static_cast<const T *>(a.total), *dy = static_cast<const T *>(a.dy);
    const int step = int(blockDim.x) / 8;
    const int by = Held<T>::moved(c, n);
    for (int64_t row = ty; row < a.m; row += 4 * step) {
      Held<T> p[4], q[4];
      float r[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int64_t at = row + u * step;
        r[u] = 0.f;
        if (at < a.m) {
          r[u] = a.rstd[at];
          p[u].get(x + at * a.ldt, c, n);
          q[u].get(dy + at * a.ldy, c, n);
        } else {
          p[u].t = q[u].t = typename Held<T>::Words(0);
        }
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        float v[8], w[8];
        p[u].to(by, v);
        q[u].to(by, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[i] += w[i] * (v[i] * r[u]);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) sums[ty][threadIdx.x % 8 * 8 + i] = sum[i];
  __syncthreads();
  if (threadIdx.x < 64 && c0 + int(threadIdx.x) < n) {
    float v = 0.f;
#pragma unroll 8
    for (int i = 0; i < int(blockDim.x) / 8; ++i) v += sums[i][threadIdx.x];
    G *out = static_cast<G *>(a.dgamma) + c0 + threadIdx.x;
    if (a.accumulate) v += float(*out);
    *out = G(v);
  }
}

// Rows of any length: dx by a workgroup that goes over its row twice.
template <class T>
__global__ __launch_bounds__(1024) void rms_long_grad_kernel(dip_rms_norm_grad_args a, int64_t row0) {
  __shared__ float s[Lanes<0>::kSums];
  int turn = 0;
  const int t = threadIdx.x, n = int(a.c);
  const int64_t row = row0 + blockIdx.x;
  const T *x = static_cast<const T *>(a.total) + row * a.ldt, *dy = static_cast<const T *>(a.dy) + row * a.ldy;
  const float rstd = a.rstd[row];
  auto both = [&](int c, float(&xh)[8], float(&h)[8]) __attribute__((always_inline)) {
    float g[8];
    load8(x + c, n - c, xh);
    load8(dy + c, n - c, h);
    gamma8<T>(a.gamma, c, n, g);
#pragma unroll
    for (int q = 0; q < 8; ++q) xh[q] *= rstd, h[q] *= g[q];
  };
  float dot = 0.f;
  for (int c = t * 8; c < n; c += 1024 * 8) {
    float xh[8], h[8];
    both(c, xh, h);
#pragma unroll
    for (int q = 0; q < 8; ++q) dot += h[q] * xh[q];
  }
  dot = Lanes<0>::sum(dot, s, turn) / float(n);
  for (int c = t * 8; c < n; c += 1024 * 8) {
    float xh[8], h[8], along[8] = {};
    both(c, xh, h);
    if (a.dtotal) load8(static_cast<const T *>(a.dtotal) + row * a.lddt + c, n - c, along);
#pragma unroll
    for (int q = 0; q < 8; ++q) h[q] = along[q] + rstd * (h[q] - xh[q] * dot);
    put8(static_cast<T *>(a.dx) + row * a.lddx + c, n - c, h);
  }
}

// Their dgamma: 256 columns of a chunk of rows a workgroup.
template <class T>
__global__ __launch_bounds__(256) void rms_long_dgamma_kernel(dip_rms_norm_grad_args a, int64_t chunk, float *partial) {
  __shared__ float s[8][256 + 8];
  const int tx = threadIdx.x % 32, ty = threadIdx.x / 32, n = int(a.c);
  const int c = int(blockIdx.x) * 256 + tx * 8;
  const int64_t r1 = min(a.m, (int64_t(blockIdx.y) + 1) * chunk);
  float sum[8] = {};
  if (c < n) {
    for (int64_t row = int64_t(blockIdx.y) * chunk + ty; row < r1; row += 8) {
      float x[8], dy[8];
      load8(static_cast<const T *>(a.total) + row * a.ldt + c, n - c, x);
      load8(static_cast<const T *>(a.dy) + row * a.ldy + c, n - c, dy);
      const float rstd = a.rstd[row];
#pragma unroll
      for (int q = 0; q < 8; ++q) sum[q] += dy[q] * (x[q] * rstd);
    }
  }
#pragma unroll
  for (int q = 0; q < 8; ++q) s[ty][tx * 8 + q] = sum[q];
  __syncthreads();
  const int at = int(blockIdx.x) * 256 + threadIdx.x;
  if (at < n) {
    float v = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) v += s[i][threadIdx.x];
    partial[int64_t(blockIdx.y) * n + at] = v;
  }
}

__global__ __launch_bounds__(256) void rms_no_columns_kernel(int64_t n, float r, float *rstd) {
  for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < n; i += int64_t(gridDim.x) * 256) rstd[i] = r;
}

// How a row of c columns that registers hold is shared out: lanes of a wave (0: the
// workgroup), vectors a thread, threads a workgroup.
struct Shape {
  int lanes, vectors, threads;
  int rows() const { return lanes ? 256 / lanes : 1; }
};
// Up to 512 columns as many lanes as a row has vectors, to the next power of two.  Up to
// 1024 a wave with two vectors a lane (2^26 bf16 elements, us: 515 columns 125, by two
// waves 143; gradient of 768 103, 112), but for float32's gradient, whose registers
// leave two waves a SIMD (640 columns 374, by two waves 206).  Beyond that one vector a
// thread as far as a workgroup goes: two would take, bf16 4096 columns, 95 (93), float32
// 199 (186); gradient of 65,536 x 3584 325 (318).
Shape row_shape(int64_t c, bool heavy) {
  const int v = int((c + 7) / 8);
  int lanes = 4;
  while (lanes < v) lanes *= 2;
  if (lanes <= 64) return Shape{lanes, 1, 256};
  if (v <= 128 && !heavy) return Shape{64, 2, 256};
  const int vectors = c <= kAheadMost ? 1 : 2;
  return Shape{0, vectors, (v + 64 * vectors - 1) / (64 * vectors) * 64};
}
Shape forward_shape(const dip_rms_norm_args &a) { return row_shape(a.c, false); }
Shape grad_shape(const dip_rms_norm_grad_args &a) { return row_shape(a.c, a.dtype == DIP_F32); }
// f(LANES, NV)
template <class F>
void with(const Shape &s, F &&f) {
  using std::integral_constant;
  const integral_constant<int, 1> one;
  switch (s.lanes) {
    case 4: return f(integral_constant<int, 4>{}, one);
    case 8: return f(integral_constant<int, 8>{}, one);
    case 16: return f(integral_constant<int, 16>{}, one);
    case 32: return f(integral_constant<int, 32>{}, one);
    case 64:
      if (s.vectors == 1) return f(integral_constant<int, 64>{}, one);
      return f(integral_constant<int, 64>{}, integral_constant<int, 2>{});
    default:
      if (s.vectors == 1) f(integral_constant<int, 0>{}, one);
      else f(integral_constant<int, 0>{}, integral_constant<int, 2>{});
  }
}
// Bytes of a column up to which dgamma is summed beside dx in one launch: 768 rows of
// 2-byte types, 384 of float32.  In two launches a call takes 12 us and more, host
// included; in one 7, and at bf16 1024 rows of 512, 4096 and 8192 columns 7.8, 12.2 and
// 20.5 (two: 12.3, 12.6, 17.5), float32 600 of 1024 and 2048 13.7 and 18.8 (12.2, 13).
constexpr int64_t kFewBytes = 1536;
bool few_rows(const dip_rms_norm_grad_args &a) {
  return a.m * (a.dtype == DIP_F32 ? 4 : 2) <= kFewBytes && a.c <= kHeldMost && a.dgamma;
}

struct GradPlan {
  int64_t blocks = 1, chunk = 0;   // workgroups that each leave a row of partial sums; rows a chunk (long rows)
  int64_t bytes = 0;
};
GradPlan grad_plan(const dip_rms_norm_grad_args &a) {
  GradPlan p;
  if (a.c > kHeldMost) {
    const int64_t cols = (a.c + 255) / 256;
    p.blocks = std::max<int64_t>(1, std::min<int64_t>((a.m + 15) / 16, 2048 / cols));
    p.chunk = (a.m + p.blocks - 1) / p.blocks;
  } else {
    // As many workgroups as have about 30 KB a CU on their way, the next rows not counted:
    // more leave more sums and run into each other (2^26 elements bf16, us by KB a CU:
    // 264 columns 12.7 144, 25 118; 512 24.6 101, 49 109; 2051 12.3 160, 25 139, 37 131;
    // 65,536 x 3584 21.5 318, 43 332, 86 357).
    const Shape h = grad_shape(a);
    const int64_t bytes = h.rows() * a.c * (a.dtype == DIP_F32 ? 4 : 2) * (a.dtotal && a.dx ? 3 : 2);
    const int64_t a_cu = std::max<int64_t>(1, (30720 + bytes / 2) / bytes);
    p.blocks = std::max<int64_t>(1, std::min<int64_t>((a.m + h.rows() - 1) / h.rows(), std::min<int64_t>(a_cu, 2048 / h.threads) * 256));
  }
  p.bytes = a.dgamma && !few_rows(a) ? up16(p.blocks * a.c * 4) : 0;
  return p;
}

template <class T, bool PACK>
hipError_t forward(const dip_rms_norm_args &a, hipStream_t st) {
  const Packed p = make_packed(a.packed);
  // a launch has fewer than 2^32 threads
  const Shape h = forward_shape(a);
  const int64_t most = (int64_t(1) << 31) / (a.c > kHeldMost ? 1024 : h.threads / h.rows());
  for (int64_t row0 = 0; row0 < a.m; row0 += most) {
    dip_rms_norm_args b = a;
    b.m = std::min(a.m, row0 + most);
    const int64_t rows = b.m - row0;
    if (a.c > kHeldMost) {
      rms_long_kernel<T, PACK><<<dim3(uint32_t(rows)), dim3(1024), 0, st>>>(b, row0, 1.0 / double(a.c), p);
    } else {
      with(h, [&](auto l, auto v) {
        rms_rows_kernel<T, decltype(l)::value, decltype(v)::value, PACK>
            <<<dim3(uint32_t((rows + h.rows() - 1) / h.rows())), dim3(h.threads), 0, st>>>(b, row0, 1.0 / double(a.c), p);
      });
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <class T>
hipError_t backward(const dip_rms_norm_grad_args &a, hipStream_t st) {
  if (few_rows(a)) {
    const Shape h = grad_shape(a);
    with(h, [&](auto l, auto v) {
      constexpr int kLanes = decltype(l)::value, kNV = decltype(v)::value;
      if constexpr (!(sizeof(T) == 4 && kLanes == 64 && kNV == 2)) {   // not a shape of float32's
        const int rows = a.dx ? int((a.m + h.rows() - 1) / h.rows()) : 0;
        const dim3 grid(uint32_t(rows + (a.c + 63) / 64));
        if (a.accumulate) rms_few_grad_kernel<T, float, kLanes, kNV><<<grid, dim3(h.threads), 0, st>>>(a, rows);
        else rms_few_grad_kernel<T, T, kLanes, kNV><<<grid, dim3(h.threads), 0, st>>>(a, rows);
      }
    });
    return hipGetLastError();
  }
  const GradPlan p = grad_plan(a);
  float *partial = a.dgamma ? static_cast<float *>(a.workspace) : nullptr;
  if (a.c > kHeldMost) {
    const int64_t most = int64_t(1) << 21;
    for (int64_t row0 = 0; a.dx && row0 < a.m; row0 += most) {
      rms_long_grad_kernel<T><<<dim3(uint32_t(std::min(most, a.m - row0))), dim3(1024), 0, st>>>(a, row0);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
    if (partial)
      rms_long_dgamma_kernel<T>
          <<<dim3(uint32_t((a.c + 255) / 256), uint32_t(p.blocks)), dim3(256), 0, st>>>(a, p.chunk, partial);
  } else {
    const Shape h = grad_shape(a);
    with(h, [&](auto l, auto v) {
      constexpr int kLanes = decltype(l)::value, kNV = decltype(v)::value;
      if constexpr (!(sizeof(T) == 4 && kLanes == 64 && kNV == 2))   // not a shape of float32's
        rms_grad_kernel<T, kLanes, kNV><<<dim3(uint32_t(p.blocks)), dim3(h.threads), 0, st>>>(a, partial);
    });
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !partial) return e;
  return launch_sum_rows(SumRows{partial, p.blocks, a.c, a.c, a.dgamma, nullptr, a.accumulate},
                         a.accumulate ? DIP_F32 : a.dtype, st);
}

}  // namespace

int64_t rms_norm_grad_workspace(const dip_rms_norm_grad_args &a) {
  return a.m == 0 || a.c == 0 ? 0 : grad_plan(a).bytes;
}

hipError_t launch_rms_norm(const dip_rms_norm_args &a, hipStream_t stream) {
  if (a.m == 0) return hipSuccess;
  if (a.c == 0) {   // a mean over nothing is 0
    if (!a.rstd) return hipSuccess;
    rms_no_columns_kernel<<<dim3(uint32_t(std::min<int64_t>((a.m + 255) / 256, 4096))), dim3(256), 0, stream>>>(
        a.m, 1.f / sqrtf(a.eps), a.rstd);
    return hipGetLastError();
  }
  const bool pack = a.packed.values != nullptr;
  switch (a.dtype) {
    case DIP_F32: return pack ? forward<float, true>(a, stream) : forward<float, false>(a, stream);
    case DIP_F16: return pack ? forward<_Float16, true>(a, stream) : forward<_Float16, false>(a, stream);
    default: return pack ? forward<__bf16, true>(a, stream) : forward<__bf16, false>(a, stream);
  }
}

hipError_t launch_rms_norm_grad(const dip_rms_norm_grad_args &a, hipStream_t stream) {
  if (a.c == 0 || (!a.dx && !a.dgamma)) return hipSuccess;
  if (a.m == 0)   // sums over nothing
    return a.dgamma && !a.accumulate
               ? launch_sum_rows(SumRows{nullptr, 0, a.c, a.c, a.dgamma, nullptr, 0}, a.dtype, stream)
               : hipSuccess;
  switch (a.dtype) {
    case DIP_F32: return backward<float>(a, stream);
    case DIP_F16: return backward<_Float16>(a, stream);
    default: return backward<__bf16>(a, stream);
  }
}

}  // namespace dipops
