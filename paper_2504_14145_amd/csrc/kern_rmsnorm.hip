// kern_rmsnorm.hip -- root-mean-square norm with the residual's addition and an
// output in 8 bits, and its gradients.
//
// Bound by memory: x and the residual read, their sum and the norm written forward,
// dy, the sum and its gradient read and one array written backward, against some 15
// operations an element.  A row of up to 16,384 columns is held in registers from its
// load to its stores, by LANES threads of NV vectors of eight; longer rows are read a
// second time, out of the caches.
#include <algorithm>
#include <type_traits>

#include "ops_internal.h"

namespace dipops {
namespace {

// columns of a row held in registers: 1024 threads have 128 each, and the gradient's
// next row has to fit beside its own
constexpr int kHeldMost = 16384, kGradHeldMost = 8192;

// Over LANES consecutive threads, a power of two; beyond a wave s holds two sets of
// the waves' values in turn, so that one barrier a sum is enough.
template <int LANES>
__device__ __forceinline__ float lanes_sum(float v, float *s, int &turn) {
#pragma unroll
  for (int d = 1; d < (LANES < 64 ? LANES : 64); d *= 2) v += __shfl_xor(v, d);
  if constexpr (LANES > 64) {
    float *q = s + turn * (LANES / 64);
    turn ^= 1;
    if (threadIdx.x % 64 == 0) q[threadIdx.x / 64] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int i = 0; i < LANES / 64; ++i) v += q[i];
  }
  return v;
}

// Columns c .. c + 7 of a row of n, as they lie in memory; zeros beyond it.  Where the
// row ends inside them the eight that end with it are read and moved into place: all
// lanes read whole vectors, and element by element the last lane costs a chain of loads.
template <class T>
struct Held {
  static constexpr int kWords = sizeof(T) * 2;   // 32-bit words of eight
  typedef uint32_t Words __attribute__((ext_vector_type(kWords)));
  typedef Words WordsAny __attribute__((aligned(sizeof(T))));
  Words t;
  __device__ __forceinline__ void get(const T *row, int c, int n) {
    const int left = n - c;
    if (left >= 8) {
      t = *reinterpret_cast<const WordsAny *>(row + c);
    } else if (left <= 0) {
      t = Words(0);
    } else if (n >= 8) {
      t = *reinterpret_cast<const WordsAny *>(row + n - 8);
      const int by = 8 - left;   // elements to move down
      if constexpr (sizeof(T) == 2) {
        if (by & 1) {
#pragma unroll
          for (int i = 0; i < kWords; ++i) t[i] = t[i] >> 16 | (i + 1 < kWords ? t[i + 1] << 16 : 0u);
        }
      }
      constexpr int per = sizeof(T) == 2 ? 2 : 1;   // elements a word
#pragma unroll
      for (int d = 1; d < kWords; d *= 2) {
        if (by / per & d) {
#pragma unroll
          for (int i = 0; i < kWords; ++i) t[i] = i + d < kWords ? t[i + d] : 0u;
        }
      }
    } else {
      float v[8];
      load8(row + c, left, v);
      put(v);
    }
  }
  __device__ __forceinline__ void put(const float (&v)[8]) {
    T e[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) e[i] = T(v[i]);
    t = __builtin_bit_cast(Words, e);
  }
  __device__ __forceinline__ void to(float (&v)[8]) const {
    struct Elements {
      T e[8];
    };
    const Elements e = __builtin_bit_cast(Elements, t);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = float(e.e[i]);
  }
};

template <class T>
__device__ __forceinline__ void gamma8(const void *gamma, int c, int n, float (&g)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) g[i] = 1.f;
  if (gamma) {
    Held<T> h;
    h.get(static_cast<const T *>(gamma), c, n);
    h.to(g);
  }
}

// t = x + residual of eight columns, rounded to the type.
template <class T>
__device__ __forceinline__ void total8(const Held<T> &x, const Held<T> &r, bool residual, float (&v)[8]) {
  x.to(v);
  if (residual) {
    float q[8];
    r.to(q);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = float(T(v[i] + q[i]));
  }
}

// 1 / sqrt(sum / n + eps) and what its rounding left off, by one step of Newton's
// iteration on the residual: the norm and its 8 bits are then as good as a product of
// exact factors (the root's rounding would put a whole row off by it).
struct Rstd {
  float v, rest;
  __device__ __forceinline__ Rstd(float sum, int n, float eps) {
    const float m = sum / float(n) + eps;
    v = 1.f / sqrtf(m);
    const float t = m * v, below = fmaf(m, v, -t);
    const float off = fmaf(-below, v, fmaf(-t, v, 1.f));   // 1 - m v^2
    rest = fabsf(off) < 1e-3f ? 0.5f * v * off : 0.f;      // not of an infinity or zero
  }
};

// y and its 8 bits from t; of the four lanes that share a scale all are here.
template <class T, bool PACK>
__device__ __forceinline__ void write8(const dip_rms_norm_args &a, const Packed &p, int64_t row, int c, const Rstd &rstd,
                                       const float (&v)[8]) {
  const int n = int(a.c), left = n - c;
  float g[8], y[8];
  gamma8<T>(a.gamma, c, n, g);
#pragma unroll
  for (int q = 0; q < 8; ++q) {
    const float t = v[q] * g[q];   // exact of 2-byte types
    y[q] = fmaf(t, rstd.v, t * rstd.rest);
  }
  if (a.y && left > 0) store8(static_cast<T *>(a.y) + row * a.ldy + c, left, y);
  if constexpr (PACK) pack8_quad(p, row, c, left, y);   // zeros beyond the row, or NaN
}

// LANES threads a row, at least four, NV vectors a thread.
template <class T, int LANES, int NV, bool PACK>
__global__ __launch_bounds__(LANES < 256 ? 256 : LANES) void rms_rows_kernel(dip_rms_norm_args a, int64_t row0, Packed p) {
  constexpr int kThreads = LANES < 256 ? 256 : LANES, kRows = kThreads / LANES;
  __shared__ float s[2 * (LANES > 64 ? LANES / 64 : 1)];
  int turn = 0;
  const int t = threadIdx.x % LANES, n = int(a.c);
  const int64_t row = row0 + int64_t(blockIdx.x) * kRows + threadIdx.x / LANES;
  if (row >= a.m) return;   // all lanes of a row
  Held<T> x[NV], r[NV];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int c = (t + j * LANES) * 8;
    x[j].get(static_cast<const T *>(a.x) + row * a.ldx, c, n);
    if (a.residual) r[j].get(static_cast<const T *>(a.residual) + row * a.ldr, c, n);
  }
  float v[NV][8], sum = 0.f;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    total8(x[j], r[j], a.residual != nullptr, v[j]);
#pragma unroll
    for (int q = 0; q < 8; ++q) sum += v[j][q] * v[j][q];
  }
  if (a.total) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (t + j * LANES) * 8;
      if (c < n) store8(static_cast<T *>(a.total) + row * a.ldt + c, n - c, v[j]);
    }
  }
  const Rstd rstd(lanes_sum<LANES>(sum, s, turn), n, a.eps);
  if (t == 0 && a.rstd) a.rstd[row] = rstd.v;
#pragma unroll
  for (int j = 0; j < NV; ++j) write8<T, PACK>(a, p, row, (t + j * LANES) * 8, rstd, v[j]);
}

// Rows of any length: a workgroup goes over its row twice.  Where the sum is stored a
// thread reads back what it wrote (the residual may be gone: they may be one array).
template <class T, bool PACK>
__global__ __launch_bounds__(1024) void rms_long_kernel(dip_rms_norm_args a, int64_t row0, Packed p) {
  __shared__ float s[2 * 16];
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
  float sum = 0.f;
  for (int c = t * 8; c < n; c += 1024 * 8) {
    float v[8];
    first(c, v);
#pragma unroll
    for (int q = 0; q < 8; ++q) sum += v[q] * v[q];
    if (total) store8(total + c, n - c, v);
  }
  const Rstd rstd(lanes_sum<1024>(sum, s, turn), n, a.eps);
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
__global__ __launch_bounds__(LANES < 256 ? 256 : LANES) void rms_grad_kernel(dip_rms_norm_grad_args a, float *partial) {
  constexpr int kThreads = LANES < 256 ? 256 : LANES, kRows = kThreads / LANES;
  __shared__ float s[2 * (LANES > 64 ? LANES / 64 : 1)];
  __shared__ float sums[kRows > 1 ? kRows * LANES * NV * 8 : 1];
  int turn = 0;
  const int t = threadIdx.x % LANES, n = int(a.c);
  const float inv = 1.f / float(n);
  float g[NV][8], sg[NV][8] = {};
#pragma unroll
  for (int j = 0; j < NV; ++j) gamma8<T>(a.gamma, (t + j * LANES) * 8, n, g[j]);
  // the next row is asked for before this one's sum is waited for
  Held<T> xn[NV], dn[NV], tn[NV];
  float rn = 0.f;
  auto fetch = [&](int64_t row) __attribute__((always_inline)) {
    rn = a.rstd[row];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (t + j * LANES) * 8;
      xn[j].get(static_cast<const T *>(a.total) + row * a.ldt, c, n);
      dn[j].get(static_cast<const T *>(a.dy) + row * a.ldy, c, n);
      if (a.dtotal && a.dx) tn[j].get(static_cast<const T *>(a.dtotal) + row * a.lddt, c, n);
    }
  };
  const int64_t step = int64_t(gridDim.x) * kRows;
  int64_t row = int64_t(blockIdx.x) * kRows + threadIdx.x / LANES;
  if (row < a.m) fetch(row);
  for (; row < a.m; row += step) {   // all lanes of a row
    const float rstd = rn;
    float xh[NV][8], h[NV][8], along[NV][8], dot = 0.f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      xn[j].to(xh[j]);
      dn[j].to(h[j]);
      if (a.dtotal && a.dx) tn[j].to(along[j]);
      else {
#pragma unroll
        for (int q = 0; q < 8; ++q) along[j][q] = 0.f;
      }
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        xh[j][q] *= rstd;
        sg[j][q] += h[j][q] * xh[j][q];
        h[j][q] *= g[j][q];
        dot += h[j][q] * xh[j][q];
      }
    }
    if (row + step < a.m) fetch(row + step);
    if (!a.dx) continue;
    dot = lanes_sum<LANES>(dot, s, turn) * inv;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (t + j * LANES) * 8;
#pragma unroll
      for (int q = 0; q < 8; ++q) h[j][q] = along[j][q] + rstd * (h[j][q] - xh[j][q] * dot);
      if (c < n) store8(static_cast<T *>(a.dx) + row * a.lddx + c, n - c, h[j]);
    }
  }
  if (!partial) return;
  if constexpr (kRows > 1) {   // its rows' sums, in their order
    float *mine = sums + (threadIdx.x / LANES) * (LANES * NV * 8);
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int q = 0; q < 8; ++q) mine[(t + j * LANES) * 8 + q] = sg[j][q];
    __syncthreads();
    for (int c = threadIdx.x; c < n; c += kThreads) {
      float v = sums[c];
      for (int i = 1; i < kRows; ++i) v += sums[i * (LANES * NV * 8) + c];
      partial[int64_t(blockIdx.x) * n + c] = v;
    }
  } else {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (t + j * LANES) * 8;
      if (c < n) store8(partial + int64_t(blockIdx.x) * n + c, n - c, sg[j]);
    }
  }
}

// Few rows: dx by workgroups of kRows rows, and dgamma beside them by workgroups of 64
// columns that read the rows again, out of the caches: one launch, no workspace.
template <class T, class G, int LANES, int NV>
__global__ __launch_bounds__(LANES < 256 ? 256 : LANES) void rms_few_grad_kernel(dip_rms_norm_grad_args a, int row_blocks) {
  constexpr int kThreads = LANES < 256 ? 256 : LANES, kRows = kThreads / LANES;
  __shared__ float s[2 * (LANES > 64 ? LANES / 64 : 1)];
  __shared__ float sums[kThreads / 8][64 + 2];
  const int n = int(a.c);
  if (int(blockIdx.x) < row_blocks) {
    int turn = 0;
    const int t = threadIdx.x % LANES;
    const int64_t row = int64_t(blockIdx.x) * kRows + threadIdx.x / LANES;
    if (row >= a.m) return;   // all lanes of a row
    const float rstd = a.rstd[row];
    Held<T> x[NV], d[NV], along[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (t + j * LANES) * 8;
      x[j].get(static_cast<const T *>(a.total) + row * a.ldt, c, n);
      d[j].get(static_cast<const T *>(a.dy) + row * a.ldy, c, n);
      if (a.dtotal) along[j].get(static_cast<const T *>(a.dtotal) + row * a.lddt, c, n);
    }
    float xh[NV][8], h[NV][8], dot = 0.f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      float g[8];
      gamma8<T>(a.gamma, (t + j * LANES) * 8, n, g);
      x[j].to(xh[j]);
      d[j].to(h[j]);
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        xh[j][q] *= rstd;
        h[j][q] *= g[q];
        dot += h[j][q] * xh[j][q];
      }
    }
    dot = lanes_sum<LANES>(dot, s, turn) / float(n);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (t + j * LANES) * 8;
      float v[8] = {};
      if (a.dtotal) along[j].to(v);
#pragma unroll
      for (int q = 0; q < 8; ++q) v[q] += rstd * (h[j][q] - xh[j][q] * dot);
      if (c < n) store8(static_cast<T *>(a.dx) + row * a.lddx + c, n - c, v);
    }
    return;
  }
  const int c0 = (int(blockIdx.x) - row_blocks) * 64, c = c0 + int(threadIdx.x % 8) * 8, ty = threadIdx.x / 8;
  float sum[8] = {};
  if (c < n) {
    // rows ty, ty + kThreads / 8, ..: four at a time, their loads first
    const T *x = static_cast<const T *>(a.total), *dy = static_cast<const T *>(a.dy);
    constexpr int kStep = kThreads / 8;
    for (int64_t row = ty; row < a.m; row += 4 * kStep) {
      Held<T> p[4], q[4];
      float r[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int64_t at = row + u * kStep;
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
        p[u].to(v);
        q[u].to(w);
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
    for (int i = 0; i < kThreads / 8; ++i) v += sums[i][threadIdx.x];
    G *out = static_cast<G *>(a.dgamma) + c0 + threadIdx.x;
    if (a.accumulate) v += float(*out);
    *out = G(v);
  }
}

// Rows of any length: dx by a workgroup that goes over its row twice.
template <class T>
__global__ __launch_bounds__(1024) void rms_long_grad_kernel(dip_rms_norm_grad_args a, int64_t row0) {
  __shared__ float s[2 * 16];
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
  dot = lanes_sum<1024>(dot, s, turn) / float(n);
  for (int c = t * 8; c < n; c += 1024 * 8) {
    float xh[8], h[8], along[8] = {};
    both(c, xh, h);
    if (a.dtotal) load8(static_cast<const T *>(a.dtotal) + row * a.lddt + c, n - c, along);
#pragma unroll
    for (int q = 0; q < 8; ++q) h[q] = along[q] + rstd * (h[q] - xh[q] * dot);
    store8(static_cast<T *>(a.dx) + row * a.lddx + c, n - c, h);
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

// f(lanes, vectors) for a row of c columns that registers hold.  Up to 4096 columns the
// gradient, which has more to hold, takes 512 threads of one vector (65,536 x 3584 bf16
// 318 us, 256 threads of two 325).
template <bool GRAD, class F>
void shape(int64_t c, F &&f) {
  const auto i = [](auto v) { return v; };
  using std::integral_constant;
#define DIP_SHAPE(LANES, NV) \
  if (c <= LANES * NV * 8) return f(i(integral_constant<int, LANES>{}), i(integral_constant<int, NV>{}))
  DIP_SHAPE(4, 1);
  DIP_SHAPE(8, 1);
  DIP_SHAPE(16, 1);
  DIP_SHAPE(32, 1);
  DIP_SHAPE(64, 1);
  DIP_SHAPE(64, 2);
  DIP_SHAPE(256, 1);
  if constexpr (GRAD) {
    DIP_SHAPE(512, 1);
  } else {
    DIP_SHAPE(256, 2);
  }
  DIP_SHAPE(512, 2);
  DIP_SHAPE(1024, 2);
#undef DIP_SHAPE
}
template <bool GRAD>
int lanes_of(int64_t c) {
  int lanes = 1024;
  shape<GRAD>(c, [&](auto l, auto) { lanes = l; });
  return lanes;
}

// Rows up to which dgamma is summed beside dx
constexpr int64_t kFewRows = 256;
bool few_rows(const dip_rms_norm_grad_args &a) { return a.m <= kFewRows && a.c <= kGradHeldMost && a.dx && a.dgamma; }

struct GradPlan {
  int64_t blocks = 1, chunk = 0;   // workgroups that each leave a row of partial sums; rows a chunk (long rows)
  int64_t bytes = 0;
};
GradPlan grad_plan(const dip_rms_norm_grad_args &a) {
  GradPlan p;
  if (a.c > kGradHeldMost) {
    const int64_t cols = (a.c + 255) / 256;
    p.blocks = std::max<int64_t>(1, std::min<int64_t>((a.m + 15) / 16, 2048 / cols));
    p.chunk = (a.m + p.blocks - 1) / p.blocks;
  } else {
    const int lanes = lanes_of<true>(a.c), rows = lanes < 256 ? 256 / lanes : 1, threads = lanes < 256 ? 256 : lanes;
    // eight waves a CU: more keep no more loads on their way, leave more sums, and run
    // into each other (65,536 x 3584 bf16: 256 workgroups of 512 318 us, 512 332, 1024 357)
    p.blocks = std::max<int64_t>(1, std::min<int64_t>((a.m + rows - 1) / rows, std::max(1, 512 / threads) * 256));
  }
  p.bytes = a.dgamma && !few_rows(a) ? up16(p.blocks * a.c * 4) : 0;
  return p;
}

template <class T, bool PACK>
hipError_t forward(const dip_rms_norm_args &a, hipStream_t st) {
  const Packed p = make_packed(a.packed);
  // a launch has fewer than 2^32 threads
  const int64_t most = (int64_t(1) << 31) / (a.c > kHeldMost ? 1024 : lanes_of<false>(a.c));
  for (int64_t row0 = 0; row0 < a.m; row0 += most) {
    dip_rms_norm_args b = a;
    b.m = std::min(a.m, row0 + most);
    const int64_t rows = b.m - row0;
    if (a.c > kHeldMost) {
      rms_long_kernel<T, PACK><<<dim3(uint32_t(rows)), dim3(1024), 0, st>>>(b, row0, p);
    } else {
      shape<false>(a.c, [&](auto l, auto v) {
        constexpr int kLanes = decltype(l)::value, kThreads = kLanes < 256 ? 256 : kLanes, kRows = kThreads / kLanes;
        rms_rows_kernel<T, kLanes, decltype(v)::value, PACK>
            <<<dim3(uint32_t((rows + kRows - 1) / kRows)), dim3(kThreads), 0, st>>>(b, row0, p);
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
    shape<true>(a.c, [&](auto l, auto v) {
      constexpr int kLanes = decltype(l)::value, kNV = decltype(v)::value, kThreads = kLanes < 256 ? 256 : kLanes;
      if constexpr (kLanes * kNV * 8 <= kGradHeldMost) {
        const int rows = int((a.m + kThreads / kLanes - 1) / (kThreads / kLanes));
        const dim3 grid(uint32_t(rows + (a.c + 63) / 64));
        if (a.accumulate) rms_few_grad_kernel<T, float, kLanes, kNV><<<grid, dim3(kThreads), 0, st>>>(a, rows);
        else rms_few_grad_kernel<T, T, kLanes, kNV><<<grid, dim3(kThreads), 0, st>>>(a, rows);
      }
    });
    return hipGetLastError();
  }
  const GradPlan p = grad_plan(a);
  float *partial = a.dgamma ? static_cast<float *>(a.workspace) : nullptr;
  if (a.c > kGradHeldMost) {
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
    shape<true>(a.c, [&](auto l, auto v) {
      constexpr int kLanes = decltype(l)::value, kNV = decltype(v)::value, kThreads = kLanes < 256 ? 256 : kLanes;
      if constexpr (kLanes * kNV * 8 <= kGradHeldMost)
        rms_grad_kernel<T, kLanes, kNV><<<dim3(uint32_t(p.blocks)), dim3(kThreads), 0, st>>>(a, partial);
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
