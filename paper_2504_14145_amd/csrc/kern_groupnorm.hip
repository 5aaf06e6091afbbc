// kern_groupnorm.hip -- group norm with an activation over channels-last arrays,
// and its gradients.
//
// All of it is bound by memory: x read once and y written once forward, x and dy
// read and dx written backward, against some 30 operations an element.  Three
// ways, by the shape (plan below):
//  rows   one position a sample: a group is one contiguous row, held in registers
//         from the read to the write, one pass.  Up to 512 channels a wave or part
//         of one takes a row (narrow), beyond that a workgroup.
//  block  a workgroup takes a slab of whole groups of one sample, and holds the first
//         four rows of every thread from the sums to the write; what is beyond them
//         it reads a second time, out of the caches.
//  split  a sample's positions are cut into chunks: a pass for the sums of every
//         channel of a chunk, a small kernel that joins them, a pass that writes.
// Variances are sums of squares about the mean (rows), or about the mean of four
// rows at a time, joined by (count, mean, sum of squares about the mean) over a
// thread's rows, the threads and the channels (block, split): neither a mean far
// from zero nor a row unlike the others costs digits.  Sums are float32, in an
// order that depends on the shape alone.
// bf16: rows, 8192 x 4096, 28 us forward (4.9 TB/s), 37 + 5 for the gradient (5.8);
// 55,388 x 249 in fp16 with GELU, odd rows, 19 (2.8 TB/s) and 33 (2.5), where one wave
// a row and 512 at once, element by element at the row's end, took 360 together;
// split, four samples of 16,384 x 512 with SiLU, 15 + 6 + 25 us forward and 30 + 5
// + 36 + 4 for the gradient, whose passes over x and dy run at 4.5 and 5.6 TB/s;
// block, 64 x 320, 7.4 us, three samples of 577 x 120 in fp32 10.5 and 15.5: a chain
// of latencies (both passes from memory and every channel's sum over 256 rows by a
// tree took 8.5, 13.3 and 18.4).
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "ops_internal.h"

namespace dipops {
namespace {

// ------------------------------------------------------------ rows

// over the LANES lanes of a wave that share threadIdx.x / LANES
template <int LANES = 64>
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int d = 1; d < LANES; d *= 2) v += __shfl_xor(v, d);
  return v;
}
// over the waves of a workgroup; s holds two sets of values in turn, so that one
// barrier a sum is enough
template <int THREADS>
__device__ __forceinline__ float block_sum(float v, float *s, int &turn) {
  v = wave_sum<(THREADS < 64 ? THREADS : 64)>(v);
  if constexpr (THREADS > 64) {
    float *q = s + turn * (THREADS / 64);
    turn ^= 1;
    if (threadIdx.x % 64 == 0) q[threadIdx.x / 64] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int i = 0; i < THREADS / 64; ++i) v += q[i];
  }
  return v;
}

template <class T>
struct Affine {
  const T *gamma, *beta;
  // of columns c .. c + 7, ones and zeros where there are none
  __device__ __forceinline__ void get(int64_t c, int left, float (&g)[8], float (&b)[8]) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) g[i] = 1.f, b[i] = 0.f;
    if (gamma) load8(gamma + c, left, g);
    if (beta) load8(beta + c, left, b);
  }
};

// Eight elements as they lie in memory, held from their load to their use.
template <class T>
struct Held {
  typename Vec8<T>::type t;
  __device__ __forceinline__ void get(const T *p, int left) { t = take8(p, left); }
  __device__ __forceinline__ void to(float (&v)[8]) const {
#pragma unroll
    for (int q = 0; q < 8; ++q) v[q] = float(t[q]);
  }
};
template <>
struct Held<float> {
  float t[8];
  __device__ __forceinline__ void get(const float *p, int left) { load8(p, left, t); }
  __device__ __forceinline__ void to(float (&v)[8]) const {
#pragma unroll
    for (int q = 0; q < 8; ++q) v[q] = t[q];
  }
};
// Eight channels from c on of a run of n.  Where the run ends inside them the eight
// that end with it are taken, so that all lanes read whole vectors (element by
// element the odd lane costs a chain of loads); the first `skip` of those belong to
// the lane before.  A run below eight: its `left` channels.
struct Eight {
  int at, skip, left;
  __device__ __forceinline__ Eight(int c, int n)
      : at(max(0, min(c, n - 8))), skip(min(c - at, 8)), left(min(8, n - at)) {}
  __device__ __forceinline__ bool own(int q) const { return q >= skip && q < left; }
};

// Up to 512 channels: as many lanes as a row has vectors, to the next power of two.
template <class T, int LANES>
__global__ __launch_bounds__(256) void narrow_kernel(dip_group_norm_args a, int64_t rows) {
  const int64_t row = int64_t(blockIdx.x) * (256 / LANES) + threadIdx.x / LANES;
  if (row >= rows) return;   // all lanes of a row
  const uint32_t i = uint32_t(row) / uint32_t(a.groups), g = uint32_t(row) % uint32_t(a.groups);
  const int per = int(a.c) / a.groups, t = threadIdx.x % LANES;
  const Eight e(t * 8, per);
  const int64_t c = int64_t(g) * per + e.at;
  float v[8], ga[8], be[8];
  load8(static_cast<const T *>(a.x) + i * a.x_sb + c, e.left, v);
  Affine<T>{static_cast<const T *>(a.gamma), static_cast<const T *>(a.beta)}.get(c, e.left, ga, be);
  const float inv = 1.f / float(per);
  float sum = 0.f;
#pragma unroll
  for (int q = 0; q < 8; ++q) sum += e.own(q) ? v[q] : 0.f;
  const float mean = wave_sum<LANES>(sum) * inv;
  sum = 0.f;
#pragma unroll
  for (int q = 0; q < 8; ++q) {
    v[q] -= mean;
    sum += e.own(q) ? v[q] * v[q] : 0.f;
  }
  const float rstd = 1.f / sqrtf(wave_sum<LANES>(sum) * inv + a.eps);
  if (t == 0) {
    if (a.mean) a.mean[row] = mean;
    if (a.rstd) a.rstd[row] = rstd;
  }
  if (t * 8 >= per) return;
#pragma unroll
  for (int q = 0; q < 8; ++q) v[q] = act_of(v[q] * rstd * ga[q] + be[q], a.act);
  store8(static_cast<T *>(a.y) + i * a.y_sb + c, e.left, v);   // the skipped ones: what their own lane writes
}

// THREADS a row of `per` channels, NV vectors of eight a thread.
template <class T, int THREADS, int NV>
__global__ __launch_bounds__(256) void rows_kernel(dip_group_norm_args a, int64_t rows) {
  constexpr int kRows = 256 / THREADS;
  __shared__ float s[2 * 4];
  int turn = 0;
  const int t = threadIdx.x % THREADS;
  const int64_t row = int64_t(blockIdx.x) * kRows + threadIdx.x / THREADS;
  if (row >= rows) return;   // all threads of a row
  const uint32_t i = uint32_t(row) / uint32_t(a.groups), g = uint32_t(row) % uint32_t(a.groups);
  const int per = int(a.c) / a.groups;
  const int64_t c0 = int64_t(g) * per;
  const T *x = static_cast<const T *>(a.x) + i * a.x_sb + c0;
  T *y = static_cast<T *>(a.y) + i * a.y_sb + c0;
  float v[NV][8];
  float sum = 0.f;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    load8(x + (t + j * THREADS) * 8, per - (t + j * THREADS) * 8, v[j]);
#pragma unroll
    for (int q = 0; q < 8; ++q) sum += v[j][q];
  }
  const float inv = 1.f / float(per);
  const float mean = block_sum<THREADS>(sum, s, turn) * inv;
  sum = 0.f;
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      const float d = v[j][q] - mean;
      v[j][q] = d;
      sum += (t + j * THREADS) * 8 + q < per ? d * d : 0.f;
    }
  const float rstd = 1.f / sqrtf(block_sum<THREADS>(sum, s, turn) * inv + a.eps);
  if (t == 0) {
    if (a.mean) a.mean[row] = mean;
    if (a.rstd) a.rstd[row] = rstd;
  }
  const Affine<T> affine{static_cast<const T *>(a.gamma), static_cast<const T *>(a.beta)};
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int c = (t + j * THREADS) * 8;
    if (c >= per) continue;
    float ga[8], be[8];
    affine.get(c0 + c, per - c, ga, be);
#pragma unroll
    for (int q = 0; q < 8; ++q) v[j][q] = act_of(v[j][q] * rstd * ga[q] + be[q], a.act);
    store8(y + c, per - c, v[j]);
  }
}

// A workgroup goes over the samples j, j + gridDim.x, .. of one group, and keeps
// the sums of dgamma and dbeta of its channels on the way: partial[j][2][c].
template <class T, int THREADS, int NV>
__global__ __launch_bounds__(THREADS) void rows_grad_kernel(dip_group_norm_grad_args a, float *partial) {
  __shared__ float s[2 * 2 * THREADS / 64];
  int turn = 0, turn2 = 0;
  const int t = threadIdx.x, per = int(a.c) / a.groups;
  const uint32_t g = blockIdx.y;
  const int64_t c0 = int64_t(g) * per;
  const Affine<T> affine{static_cast<const T *>(a.gamma), static_cast<const T *>(a.beta)};
  float sg[NV][8] = {}, sb[NV][8] = {}, ga[NV][8], be[NV][8];
#pragma unroll
  for (int j = 0; j < NV; ++j) affine.get(c0 + (t + j * THREADS) * 8, per - (t + j * THREADS) * 8, ga[j], be[j]);
  const float inv = 1.f / float(per);
  // the next sample's row is asked for before this one's sums are waited for
  Held<T> xn[NV], dn[NV];
  auto fetch = [&](int64_t i) __attribute__((always_inline)) {
    const T *x = static_cast<const T *>(a.x) + i * a.x_sb + c0;
    const T *dy = static_cast<const T *>(a.dy) + i * a.dy_sb + c0;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (t + j * THREADS) * 8;
      xn[j].get(x + c, per - c);
      dn[j].get(dy + c, per - c);   // zeros beyond the row
    }
  };
  if (int64_t(blockIdx.x) < a.b) fetch(blockIdx.x);
  for (int64_t i = blockIdx.x; i < a.b; i += gridDim.x) {
    const float mean = a.mean[i * a.groups + g], rstd = a.rstd[i * a.groups + g];
    float xh[NV][8], h[NV][8];
    float m1 = 0.f, m2 = 0.f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      xn[j].to(xh[j]);
      dn[j].to(h[j]);
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        xh[j][q] = (xh[j][q] - mean) * rstd;
        const float v = a.act == DIP_ACT_NONE ? h[j][q] : h[j][q] * act_slope(xh[j][q] * ga[j][q] + be[j][q], a.act);
        sg[j][q] += v * xh[j][q];
        sb[j][q] += v;
        h[j][q] = v * ga[j][q];
        m1 += h[j][q];
        m2 += h[j][q] * xh[j][q];
      }
    }
    if (i + gridDim.x < a.b) fetch(i + gridDim.x);
    if (!a.dx) continue;
    m1 = block_sum<THREADS>(m1, s, turn) * inv;
    m2 = block_sum<THREADS>(m2, s + 2 * THREADS / 64, turn2) * inv;
    T *dx = static_cast<T *>(a.dx) + i * a.dx_sb + c0;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (t + j * THREADS) * 8;
#pragma unroll
      for (int q = 0; q < 8; ++q) h[j][q] = rstd * (h[j][q] - m1 - xh[j][q] * m2);
      store8(dx + c, per - c, h[j]);
    }
  }
  if (!partial) return;
  float *p = partial + int64_t(blockIdx.x) * 2 * a.c + c0;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int c = (t + j * THREADS) * 8;
    store8(p + c, per - c, sg[j]);
    store8(p + a.c + c, per - c, sb[j]);
  }
}

// ------------------------------------------------------------ block and split

// How a workgroup's threads lie over a slab: vector vx of eight channels, rows
// ty, ty + TY, .., TY a power of two.
struct Lanes {
  int vx, ty, TY;
  bool on;
  __device__ Lanes(int vectors, int lanes_y) {
    TY = lanes_y;
    vx = int(threadIdx.x) % vectors;
    ty = int(threadIdx.x) / vectors;
    on = ty < TY;
  }
};

// Adds two values a channel over the workgroup's TY rows of `width` channels; every
// thread then finds the sums of channel c at s[c] and s[half + c], half = width TY.
// s is not in use before.  A thread adds up to sixteen rows, as many threads as
// that takes side by side, and a second step their sums.
__device__ __forceinline__ void channel_sums(int width, int ty, int TY, bool on, int at, int skip, const float (&a)[8],
                                             const float (&b)[8], float *s) {
  const int half = width * TY;
  if (on) {
    float *p = s + ty * width + at;
    if (skip == 0) {
#pragma unroll
      for (int q = 0; q < 8; ++q) p[q] = a[q], p[half + q] = b[q];
    } else {
#pragma unroll
      for (int q = 0; q < 8; ++q)
        if (q >= skip) p[q] = a[q], p[half + q] = b[q];
    }
  }
  __syncthreads();
  for (int rows = TY; rows > 1;) {
    const int parts = rows / min(rows, 16), step = parts * width;
    for (int j = threadIdx.x; j < 2 * step; j += blockDim.x) {
      float *p = s + (j >= step ? half + j - step : j), v = p[0];
#pragma unroll 8
      for (int r = step; r < rows * width; r += step) v += p[r];
      p[0] = v;   // row j / width of the half: no other thread of the step reads it
    }
    __syncthreads();
    rows = parts;
  }
}

// A sum of squares less what its mean was off, which rounding may take below zero.
// One beyond float32 stays infinite, NaN stays NaN.
__device__ __forceinline__ float less(float v, float off) { return v < INFINITY ? fmaxf(v - off, 0.f) : v; }

// Joins the threads' moments of `n` rows, of which thread row ty has ty, ty + TY, ..;
// every thread then finds channel c's mean at s[c] and the squares about it at
// s[half + c], half = width TY.  s is not in use before.  As above a thread joins up
// to sixteen rows; the mean is taken twice, the second time about the first, so that
// it and the squares lose nothing to a row unlike the others.
__device__ __forceinline__ void channel_moments(int width, int ty, int TY, bool on, int at, int skip, const float (&mean)[8],
                                                const float (&m2)[8], int64_t n, float *s) {
  const int half = width * TY;
  if (on) {
    float *p = s + ty * width + at;
#pragma unroll
    for (int q = 0; q < 8; ++q)
      if (q >= skip) p[q] = mean[q], p[half + q] = m2[q];
  }
  __syncthreads();
  for (int rows = TY; rows > 1;) {
    const int parts = rows / min(rows, 16), step = parts * width;
    // rows seen by the r-th of them: n / rows, and one more of the first n % rows
    const int shift = __ffs(rows) - 1, more = int(n & (rows - 1));
    const float few = float(n >> shift);
    auto join = [&](auto count_) __attribute__((always_inline)) {
      constexpr int kCount = decltype(count_)::value;
      for (int j = threadIdx.x; j < step; j += blockDim.x) {
        float *p = s + j, v[kCount], w[kCount], sum = 0.f, total = 0.f, a = 0.f, b = 0.f, c = 0.f;
        const int first = j / width;
#pragma unroll
        for (int r = 0; r < kCount; ++r) {
          v[r] = p[r * step];
          c += p[half + r * step];
        }
#pragma unroll
        for (int r = 0; r < kCount; ++r) {
          w[r] = few + (first + r * parts < more ? 1.f : 0.f);
          sum += w[r] * v[r];
          total += w[r];
        }
        const float inv = total > 0.f ? __builtin_amdgcn_rcpf(total) : 0.f, about = sum * inv;
#pragma unroll
        for (int r = 0; r < kCount; ++r) {
          const float d = v[r] - about, wd = w[r] * d;
          a += wd;
          b += wd * d;
        }
        // row j / width of either half: no other thread of the step reads them
        p[0] = about + a * inv;
        p[half] = c + less(b, a * (a * inv));
      }
    };
    if (rows >= 16) join(std::integral_constant<int, 16>{});
    else if (rows == 8) join(std::integral_constant<int, 8>{});
    else if (rows == 4) join(std::integral_constant<int, 4>{});
    else join(std::integral_constant<int, 2>{});
    __syncthreads();
    rows = parts;
  }
}

// Mean and sum of squares about it of eight channels over the rows a thread has
// seen.  The mean is held as hi + lo, so that adding to it rounds away nothing that
// counts.  Four rows are summed about hi and then about their own mean, and joined:
// no sum is larger than what the rows are apart.
struct Moments {
  float n = 0.f, hi[8] = {}, lo[8] = {}, m2[8] = {};
  // the first `count` of four rows; count at least 1
  template <bool FOUR>
  __device__ __forceinline__ void add(float (&v)[4][8], int count) {
    if (n == 0.f) {
#pragma unroll
      for (int q = 0; q < 8; ++q) hi[q] = v[0][q];
    }
    // reciprocals to a rounding or two: of what the rows are apart
    const float c = FOUR ? 4.f : float(count), inv = FOUR ? 0.25f : __builtin_amdgcn_rcpf(c), total = n + c,
                part = n == 0.f ? 1.f : c * __builtin_amdgcn_rcpf(total), both = n * part;
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      float sum = 0.f;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        v[u][q] = FOUR || u < count ? v[u][q] - hi[q] : 0.f;
        sum += v[u][q];
      }
      const float mean = sum * inv;
      float sq = 0.f;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const float d = FOUR || u < count ? v[u][q] - mean : 0.f;
        sq += d * d;
      }
      const float apart = mean - lo[q], low = lo[q] + apart * part, high = hi[q] + low;
      m2[q] += sq + apart * (apart * both);   // 0 of the first rows, however far apart
      lo[q] = low - (high - hi[q]);
      hi[q] = high;
    }
    n = total;
  }
};

// The moments of rows r, r + TY, .. below r1.
template <class T>
__device__ __forceinline__ void moments(const T *x, int64_t ss, int left, const Lanes &l, int64_t r, int64_t r1,
                                        Moments &m) {
  float v[4][8];
  for (; r + 3 * l.TY < r1; r += 4 * l.TY) {
#pragma unroll
    for (int u = 0; u < 4; ++u) load8(x + (r + u * l.TY) * ss, left, v[u]);
    m.add<true>(v, 4);
  }
  if (r >= r1) return;
  const int count = int((r1 - r + l.TY - 1) / l.TY);
#pragma unroll
  for (int u = 0; u < 4; ++u) load8(x + min(r + u * l.TY, r1 - 1) * ss, left, v[u]);
  m.add<false>(v, count);
}

// Eight channels' part in the forward's second pass and in both of the
// gradient's: z = x scale + shift, xh = (x - mean) rstd.
struct Channels {
  float mean[8], rstd[8], gamma[8], beta[8];
};

template <class T>
__device__ __forceinline__ void write_row(T *y, int left, const Channels &c, int act, float (&v)[8]) {
#pragma unroll
  for (int q = 0; q < 8; ++q) v[q] = (v[q] - c.mean[q]) * (c.rstd[q] * c.gamma[q]) + c.beta[q];
  if (act == DIP_ACT_SILU) {
#pragma unroll
    for (int q = 0; q < 8; ++q) v[q] = act_of(v[q], DIP_ACT_SILU);
  } else if (act != DIP_ACT_NONE) {
#pragma unroll
    for (int q = 0; q < 8; ++q) v[q] = act_of(v[q], act);
  }
  store8(y, left, v);
}

template <class T>
__device__ __forceinline__ void write_rows(const T *x, int64_t x_ss, T *y, int64_t y_ss, int left, const Lanes &l,
                                           int64_t r, int64_t r1, const Channels &c, int act) {
  if (!l.on) return;
  auto one = [&](int64_t r, float(&v)[8]) { write_row(y + r * y_ss, left, c, act, v); };
  for (; r + l.TY < r1; r += 2 * l.TY) {
    float v[2][8];
    load8(x + r * x_ss, left, v[0]);
    load8(x + (r + l.TY) * x_ss, left, v[1]);
    one(r, v[0]);
    one(r + l.TY, v[1]);
  }
  if (r < r1) {
    float v[8];
    load8(x + r * x_ss, left, v);
    one(r, v);
  }
}

// v = dy act'(z) and xh of eight channels of one row
__device__ __forceinline__ void grad_terms(const Channels &c, int act, float (&xv)[8], float (&dv)[8]) {
#pragma unroll
  for (int q = 0; q < 8; ++q) xv[q] = (xv[q] - c.mean[q]) * c.rstd[q];
  if (act == DIP_ACT_SILU) {
#pragma unroll
    for (int q = 0; q < 8; ++q) dv[q] *= act_slope(xv[q] * c.gamma[q] + c.beta[q], DIP_ACT_SILU);
  } else if (act != DIP_ACT_NONE) {
#pragma unroll
    for (int q = 0; q < 8; ++q) dv[q] *= act_slope(xv[q] * c.gamma[q] + c.beta[q], act);
  }
}

// a += v xh, b += v
__device__ __forceinline__ void add_grad(const Channels &c, int act, float (&xv)[8], float (&dv)[8], float (&a)[8],
                                         float (&b)[8]) {
  grad_terms(c, act, xv, dv);
#pragma unroll
  for (int q = 0; q < 8; ++q) {
    a[q] += dv[q] * xv[q];
    b[q] += dv[q];
  }
}
// the same over rows r, r + TY, .. below r1
template <class T>
__device__ __forceinline__ void grad_sums(const T *x, int64_t x_ss, const T *dy, int64_t dy_ss, int left,
                                          const Lanes &l, int64_t r, int64_t r1, const Channels &c, int act,
                                          float (&a)[8], float (&b)[8]) {
  if (!l.on) return;
  auto add = [&](float(&xv)[8], float(&dv)[8]) { add_grad(c, act, xv, dv, a, b); };
  for (; r + l.TY < r1; r += 2 * l.TY) {
    float xv[2][8], dv[2][8];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      load8(x + (r + u * l.TY) * x_ss, left, xv[u]);
      load8(dy + (r + u * l.TY) * dy_ss, left, dv[u]);
    }
    add(xv[0], dv[0]);
    add(xv[1], dv[1]);
  }
  if (r < r1) {
    float xv[8], dv[8];
    load8(x + r * x_ss, left, xv);
    load8(dy + r * dy_ss, left, dv);
    add(xv, dv);
  }
}

// dx = rstd (h - m1 - xh m2), h = v gamma
template <class T>
__device__ __forceinline__ void write_grad_row(T *dx, int left, const Channels &c, const float (&m1)[8],
                                               const float (&m2)[8], int act, float (&xv)[8], float (&dv)[8]) {
  grad_terms(c, act, xv, dv);
#pragma unroll
  for (int q = 0; q < 8; ++q) dv[q] = c.rstd[q] * (dv[q] * c.gamma[q] - m1[q] - xv[q] * m2[q]);
  store8(dx, left, dv);
}
template <class T>
__device__ __forceinline__ void write_grad(const T *x, int64_t x_ss, const T *dy, int64_t dy_ss, T *dx, int64_t dx_ss,
                                           int left, const Lanes &l, int64_t r, int64_t r1, const Channels &c,
                                           const float (&m1)[8], const float (&m2)[8], int act) {
  if (!l.on) return;
  auto one = [&](int64_t r, float(&xv)[8], float(&dv)[8]) {
    write_grad_row(dx + r * dx_ss, left, c, m1, m2, act, xv, dv);
  };
  for (; r + l.TY < r1; r += 2 * l.TY) {
    float xv[2][8], dv[2][8];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      load8(x + (r + u * l.TY) * x_ss, left, xv[u]);
      load8(dy + (r + u * l.TY) * dy_ss, left, dv[u]);
    }
    one(r, xv[0], dv[0]);
    one(r + l.TY, xv[1], dv[1]);
  }
  if (r < r1) {
    float xv[8], dv[8];
    load8(x + r * x_ss, left, xv);
    load8(dy + r * dy_ss, left, dv);
    one(r, xv, dv);
  }
}

// two values a group (statistics or means), for the groups of eight channels from
// c on; those beyond `left` (at least one) get the last one's
__device__ __forceinline__ void of_groups(const float *p, const float *r, int64_t c, int per, int left, float (&u)[8],
                                          float (&v)[8]) {
  uint32_t g = uint32_t(c) / uint32_t(per), rest = uint32_t(c) - g * per;   // c < 2^22
#pragma unroll
  for (int q = 0; q < 8; ++q) {
    u[q] = p[g];
    v[q] = r[g];
    if (q + 1 < left && ++rest == uint32_t(per)) rest = 0, ++g;
  }
}

constexpr int kHeld = 4;   // a thread's rows that a slab reads once, as many as Moments takes

// Lanes for the channels of one group, a power of two, so that each adds up about
// four of them.
__device__ __forceinline__ int group_lanes(int per) {
  int n = 1;
  while (n < 64 && n * 4 < per) n *= 2;
  return n;
}
__device__ __forceinline__ float lanes_sum(float v, int lanes) {
  for (int d = 1; d < lanes; d *= 2) v += __shfl_xor(v, d);
  return v;
}

// One workgroup: a slab of `groups` whole groups of one sample.
template <class T>
__global__ __launch_bounds__(512) void block_kernel(dip_group_norm_args a, int groups, int vectors, int lanes_y) {
  extern __shared__ float s[];
  Lanes l(vectors, lanes_y);
  const int tiles = (a.groups + groups - 1) / groups;
  const int per = int(a.c) / a.groups, g0 = int(blockIdx.x % tiles) * groups, count = min(groups, a.groups - g0);
  const int slab = count * per;
  const int64_t i = blockIdx.x / tiles;
  const Eight e(l.vx * 8, slab);
  const int64_t c = int64_t(g0) * per + e.at;
  l.on = l.on && l.vx * 8 < slab;
  const T *x = static_cast<const T *>(a.x) + i * a.x_sb + c;
  Channels ch;
  Moments mo;
  Held<T> held[kHeld];
  if (l.on) {
#pragma unroll
    for (int j = 0; j < kHeld; ++j) held[j].get(x + min(int64_t(l.ty) + j * l.TY, a.s - 1) * a.x_ss, e.left);
    Affine<T>{static_cast<const T *>(a.gamma), static_cast<const T *>(a.beta)}.get(c, e.left, ch.gamma, ch.beta);
    float w[kHeld][8];
#pragma unroll
    for (int j = 0; j < kHeld; ++j) held[j].to(w[j]);
    const int64_t count = (a.s - l.ty + l.TY - 1) / l.TY;
    if (count >= kHeld) mo.add<true>(w, kHeld);
    else mo.add<false>(w, int(count));
    moments(x, a.x_ss, e.left, l, l.ty + int64_t(kHeld) * l.TY, a.s, mo);
  }
  const int width = vectors * 8, half = width * l.TY;
  channel_moments(width, l.ty, l.TY, l.on, e.at, e.skip, mo.hi, mo.m2, a.s, s);
  const float n = float(a.s);
  float *stat = s + 2 * half;   // [2][groups]
  const int lanes = group_lanes(per), t = threadIdx.x % lanes, at_once = blockDim.x / lanes;
  for (int b = 0; b < count; b += at_once) {
    const int g = b + threadIdx.x / lanes;
    const float *m = s + min(g, count - 1) * per;
    float mean = 0.f, m2 = 0.f;
#pragma unroll 4
    for (int j = t; j < per; j += lanes) mean += m[j];
    mean = lanes_sum(mean, lanes) / float(per);
#pragma unroll 4
    for (int j = t; j < per; j += lanes) {
      const float d = m[j] - mean;
      m2 += m[half + j] + n * d * d;
    }
    const float rstd = 1.f / sqrtf(lanes_sum(m2, lanes) / (n * float(per)) + a.eps);
    if (t == 0 && g < count) {
      stat[g] = mean;
      stat[groups + g] = rstd;
      if (a.mean) a.mean[i * a.groups + g0 + g] = mean;
      if (a.rstd) a.rstd[i * a.groups + g0 + g] = rstd;
    }
  }
  __syncthreads();
  if (!l.on) return;
  of_groups(stat, stat + groups, e.at, per, e.left, ch.mean, ch.rstd);
  T *y = static_cast<T *>(a.y) + i * a.y_sb + c;
#pragma unroll
  for (int j = 0; j < kHeld; ++j) {
    const int64_t r = l.ty + j * l.TY;
    float w[8];
    held[j].to(w);
    if (r < a.s) write_row(y + r * a.y_ss, e.left, ch, a.act, w);
  }
  write_rows(x, a.x_ss, y, a.y_ss, e.left, l, l.ty + int64_t(kHeld) * l.TY, a.s, ch, a.act);
}

// Sums of dgamma and dbeta of a workgroup's channels: to partial[at][2][c], or, of
// the only workgroup that has these channels, to the gradients themselves.
template <class T>
__device__ __forceinline__ void put_sums(const dip_group_norm_grad_args &a, float *partial, int64_t at, int64_t c0,
                                         int n, const float *s, int half) {
  T *dgamma = static_cast<T *>(a.dgamma), *dbeta = static_cast<T *>(a.dbeta);
  float *p = partial + at * 2 * a.c + c0;
  for (int j = threadIdx.x; j < n; j += blockDim.x) {
    if (partial) {
      p[j] = s[j], p[a.c + j] = s[half + j];
    } else if (a.accumulate) {
      if (dgamma) static_cast<float *>(a.dgamma)[c0 + j] += s[j];
      if (dbeta) static_cast<float *>(a.dbeta)[c0 + j] += s[half + j];
    } else {
      if (dgamma) dgamma[c0 + j] = T(s[j]);
      if (dbeta) dbeta[c0 + j] = T(s[half + j]);
    }
  }
}

template <class T>
__global__ __launch_bounds__(512) void block_grad_kernel(dip_group_norm_grad_args a, int groups, int vectors,
                                                          int lanes_y, float *partial) {
  extern __shared__ float s[];
  Lanes l(vectors, lanes_y);
  const int tiles = (a.groups + groups - 1) / groups;
  const int per = int(a.c) / a.groups, g0 = int(blockIdx.x % tiles) * groups, count = min(groups, a.groups - g0);
  const int slab = count * per;
  const int64_t i = blockIdx.x / tiles, c0 = int64_t(g0) * per;
  const Eight e(l.vx * 8, slab);
  const int64_t c = c0 + e.at;
  l.on = l.on && l.vx * 8 < slab;
  const T *x = static_cast<const T *>(a.x) + i * a.x_sb + c, *dy = static_cast<const T *>(a.dy) + i * a.dy_sb + c;
  Channels ch;
  float u[8] = {}, v[8] = {};
  Held<T> hx[kHeld], hd[kHeld];
  if (l.on) {
#pragma unroll
    for (int j = 0; j < kHeld; ++j) {
      const int64_t r = min(int64_t(l.ty) + j * l.TY, a.s - 1);
      hx[j].get(x + r * a.x_ss, e.left);
      hd[j].get(dy + r * a.dy_ss, e.left);
    }
    of_groups(a.mean + i * a.groups, a.rstd + i * a.groups, c, per, e.left, ch.mean, ch.rstd);
    Affine<T>{static_cast<const T *>(a.gamma), static_cast<const T *>(a.beta)}.get(c, e.left, ch.gamma, ch.beta);
#pragma unroll
    for (int j = 0; j < kHeld; ++j) {
      float xv[8], dv[8];
      hx[j].to(xv);
      hd[j].to(dv);
      if (l.ty + j * l.TY < a.s) add_grad(ch, a.act, xv, dv, u, v);
    }
  }
  grad_sums(x, a.x_ss, dy, a.dy_ss, e.left, l, l.ty + int64_t(kHeld) * l.TY, a.s, ch, a.act, u, v);
  const int width = vectors * 8, half = width * l.TY;
  channel_sums(width, l.ty, l.TY, l.on, e.at, e.skip, u, v, s);
  if (partial || a.b == 1) put_sums<T>(a, partial, i, c0, slab, s, half);
  if (!a.dx) return;
  const T *gamma = static_cast<const T *>(a.gamma);
  float *mean = s + 2 * half;   // [2][groups]
  const int lanes = group_lanes(per), t = threadIdx.x % lanes, at_once = blockDim.x / lanes;
  for (int b = 0; b < count; b += at_once) {
    const int g = b + threadIdx.x / lanes, first = min(g, count - 1) * per;
    float m1 = 0.f, m2 = 0.f;
#pragma unroll 4
    for (int j = t; j < per; j += lanes) {
      const float w = gamma ? float(gamma[c0 + first + j]) : 1.f;
      m2 += w * s[first + j];
      m1 += w * s[half + first + j];
    }
    const float inv = 1.f / (float(a.s) * float(per));
    m1 = lanes_sum(m1, lanes) * inv;
    m2 = lanes_sum(m2, lanes) * inv;
    if (t == 0 && g < count) mean[g] = m1, mean[groups + g] = m2;
  }
  __syncthreads();
  if (!l.on) return;
  float m1[8], m2[8];
  of_groups(mean, mean + groups, e.at, per, e.left, m1, m2);
  T *dx = static_cast<T *>(a.dx) + i * a.dx_sb + c;
#pragma unroll
  for (int j = 0; j < kHeld; ++j) {
    const int64_t r = l.ty + j * l.TY;
    float xv[8], dv[8];
    hx[j].to(xv);
    hd[j].to(dv);
    if (r < a.s) write_grad_row(dx + r * a.dx_ss, e.left, ch, m1, m2, a.act, xv, dv);
  }
  write_grad(x, a.x_ss, dy, a.dy_ss, dx, a.dx_ss, e.left, l, l.ty + int64_t(kHeld) * l.TY, a.s, ch, m1, m2, a.act);
}

// The gradient of rows of up to 512 channels (one position a sample), LANES lanes a
// row and 256 / LANES rows at once; dgamma and dbeta as in rows_grad_kernel.
template <class T, int LANES>
__global__ __launch_bounds__(256) void narrow_grad_kernel(dip_group_norm_grad_args a, float *partial) {
  constexpr int kRows = 256 / LANES;
  __shared__ float s[2 * 256 * 8];
  const int t = threadIdx.x % LANES, ty = threadIdx.x / LANES, per = int(a.c) / a.groups;
  const uint32_t g = blockIdx.y;
  const int64_t c0 = int64_t(g) * per;
  const Eight e(t * 8, per);
  const bool on = t * 8 < per;
  const T *x = static_cast<const T *>(a.x) + c0 + e.at, *dy = static_cast<const T *>(a.dy) + c0 + e.at;
  const int64_t first = int64_t(blockIdx.x) * kRows + ty, step = int64_t(gridDim.x) * kRows;
  Held<T> xn, dn;
  float mean = 0.f, rstd = 0.f;
  // the next row is asked for before this one's sums are waited for
  auto fetch = [&](int64_t i) __attribute__((always_inline)) {
    xn.get(x + i * a.x_sb, e.left);
    dn.get(dy + i * a.dy_sb, e.left);
    mean = a.mean[i * a.groups + g];
    rstd = a.rstd[i * a.groups + g];
  };
  if (first < a.b) fetch(first);
  float ga[8], be[8], sg[8] = {}, sb[8] = {};
  Affine<T>{static_cast<const T *>(a.gamma), static_cast<const T *>(a.beta)}.get(c0 + e.at, e.left, ga, be);
  const float inv = 1.f / float(per);
  for (int64_t i = first; i < a.b; i += step) {   // all lanes of a row
    float xh[8], h[8], m1 = 0.f, m2 = 0.f;
    const float r = rstd;
    xn.to(xh);
    dn.to(h);
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      xh[q] = (xh[q] - mean) * r;
      if (a.act != DIP_ACT_NONE) h[q] *= act_slope(xh[q] * ga[q] + be[q], a.act);
      sg[q] += h[q] * xh[q];
      sb[q] += h[q];
      h[q] *= ga[q];
      m1 += e.own(q) ? h[q] : 0.f;
      m2 += e.own(q) ? h[q] * xh[q] : 0.f;
    }
    if (i + step < a.b) fetch(i + step);
    if (!a.dx) continue;
    m1 = wave_sum<LANES>(m1) * inv;
    m2 = wave_sum<LANES>(m2) * inv;
#pragma unroll
    for (int q = 0; q < 8; ++q) h[q] = r * (h[q] - m1 - xh[q] * m2);
    if (on) store8(static_cast<T *>(a.dx) + i * a.dx_sb + c0 + e.at, e.left, h);   // skipped ones: the same values
  }
  if (!a.dgamma && !a.dbeta) return;
  channel_sums(LANES * 8, ty, kRows, on, e.at, e.skip, sg, sb, s);
  put_sums<T>(a, partial, blockIdx.x, c0, per, s, LANES * 8 * kRows);
}

// Split: a workgroup a column tile, chunk and sample, 256 threads.
struct Part {
  int64_t i, c, left, r0, r1, at;   // sample, channel, rows, index among all chunks
  __device__ Part(const Lanes &l, int vectors, int tiles, int chunks, int64_t chunk, int64_t all_c, int64_t all_s,
                  bool backwards) {
    const uint32_t tile = blockIdx.x % tiles, rest = blockIdx.x / tiles;
    uint32_t q = rest % chunks;
    if (backwards) q = chunks - 1 - q;
    i = rest / chunks;
    at = i * chunks + q;
    c = (int64_t(tile) * vectors + l.vx) * 8;
    left = min(all_c - c, int64_t(8));
    r0 = chunk * q;
    r1 = min(r0 + chunk, all_s);
  }
};

// A chunk's channels: partial[sample][chunk][2][c], mean and squares about it.
template <class T>
__global__ __launch_bounds__(256) void split_sums_kernel(dip_group_norm_args a, int vectors, int lanes_y, int tiles,
                                                         int chunks, int64_t chunk, float *partial) {
  extern __shared__ float s[];
  const Lanes l(vectors, lanes_y);
  const Part w(l, vectors, tiles, chunks, chunk, a.c, a.s, false);
  const int left = int(w.left);
  Moments mo;
  if (l.on && left > 0)
    moments(static_cast<const T *>(a.x) + w.i * a.x_sb + w.c, a.x_ss, left, l, w.r0 + l.ty, w.r1, mo);
  channel_moments(vectors * 8, l.ty, l.TY, l.on, l.vx * 8, 0, mo.hi, mo.m2, max(w.r1 - w.r0, int64_t(0)), s);
  const int half = vectors * 8 * l.TY;
  if (!l.on || l.ty != 0) return;
  float *p = partial + w.at * 2 * a.c + w.c, u[8], v[8];
#pragma unroll
  for (int q = 0; q < 8; ++q) u[q] = s[l.vx * 8 + q], v[q] = s[half + l.vx * 8 + q];
  store8(p, left, u);
  store8(p + a.c, left, v);
}

// A workgroup's threads over [chunks][per] values of one sample and group, whole
// runs of channels side by side: f(chunk, channel), eight of a thread's at once.
template <class F>
__device__ __forceinline__ void over_chunks(int chunks, int per, F &&f) {
  const int side = min(per, 256), rows = 256 / side;
  const int tx = threadIdx.x % side, ty = threadIdx.x / side;
  if (ty >= rows) return;
  for (int j = tx; j < per; j += side) {
#pragma unroll 8
    for (int q = ty; q < chunks; q += rows) f(q, j);
  }
}

// One workgroup a sample and group joins its chunks' channels.
__global__ __launch_bounds__(256) void split_join_kernel(const float *partial, int64_t s_all, int64_t chunk,
                                                         int chunks, int64_t c, int per, float eps, float *mean,
                                                         float *rstd, float *stat) {
  __shared__ float s[2 * 4], s2[2 * 4];
  int turn = 0, turn2 = 0;
  const uint32_t groups = uint32_t(c / per), i = blockIdx.x / groups, g = blockIdx.x % groups;
  const float *p = partial + int64_t(i) * chunks * 2 * c + int64_t(g) * per;
  const float total = float(s_all) * float(per), full = float(chunk);
  const float rest = float(s_all - chunk * (chunks - 1));   // rows of the last chunk
  // every value times its count, about the first chunk's first channel
  const float k = p[0];
  float u = 0.f;
  over_chunks(chunks, per, [&](int q, int j) {
    u += (p[int64_t(q) * 2 * c + j] - k) * (q + 1 < chunks ? full : rest);
  });
  float m = k + block_sum<256>(u, s, turn) / total;
  // squares about that, and what it is off where k is unlike the other values
  float off = 0.f;
  u = 0.f;
  over_chunks(chunks, per, [&](int q, int j) {
    const float *v = p + int64_t(q) * 2 * c + j;
    const float d = v[0] - m, w = d * (q + 1 < chunks ? full : rest);
    off += w;
    u += v[c] + d * w;
  });
  off = block_sum<256>(off, s2, turn2) / total;
  m += off;
  const float r = 1.f / sqrtf(less(block_sum<256>(u, s, turn) / total, off * off) + eps);
  if (threadIdx.x == 0) {
    stat[blockIdx.x] = m;
    stat[gridDim.x + blockIdx.x] = r;
    if (mean) mean[blockIdx.x] = m;
    if (rstd) rstd[blockIdx.x] = r;
  }
}

template <class T>
__global__ __launch_bounds__(256) void split_write_kernel(dip_group_norm_args a, int vectors, int lanes_y, int tiles,
                                                          int chunks, int64_t chunk, const float *stat) {
  const Lanes l(vectors, lanes_y);
  // the chunks read last come first: they may still be in the caches
  const Part w(l, vectors, tiles, chunks, chunk, a.c, a.s, true);
  const int left = int(w.left), per = int(a.c) / a.groups;
  const int64_t i = w.i, c = w.c;
  if (left <= 0) return;
  Channels ch;
  of_groups(stat + i * a.groups, stat + (a.b + i) * a.groups, c, per, left, ch.mean, ch.rstd);
  Affine<T>{static_cast<const T *>(a.gamma), static_cast<const T *>(a.beta)}.get(c, left, ch.gamma, ch.beta);
  write_rows(static_cast<const T *>(a.x) + i * a.x_sb + c, a.x_ss, static_cast<T *>(a.y) + i * a.y_sb + c, a.y_ss, left,
             l, w.r0 + l.ty, w.r1, ch, a.act);
}

template <class T>
__global__ __launch_bounds__(256) void split_grad_sums_kernel(dip_group_norm_grad_args a, int vectors, int lanes_y, int tiles,
                                                              int chunks, int64_t chunk, float *partial) {
  extern __shared__ float s[];
  const Lanes l(vectors, lanes_y);
  const Part w(l, vectors, tiles, chunks, chunk, a.c, a.s, false);
  const int left = int(w.left), per = int(a.c) / a.groups;
  const int64_t i = w.i, c = w.c;
  Channels ch;
  float u[8] = {}, v[8] = {};
  if (left > 0) {
    of_groups(a.mean + i * a.groups, a.rstd + i * a.groups, c, per, left, ch.mean, ch.rstd);
    Affine<T>{static_cast<const T *>(a.gamma), static_cast<const T *>(a.beta)}.get(c, left, ch.gamma, ch.beta);
    grad_sums(static_cast<const T *>(a.x) + i * a.x_sb + c, a.x_ss, static_cast<const T *>(a.dy) + i * a.dy_sb + c,
              a.dy_ss, left, l, w.r0 + l.ty, w.r1, ch, a.act, u, v);
  }
  channel_sums(vectors * 8, l.ty, l.TY, l.on, l.vx * 8, 0, u, v, s);
  const int half = vectors * 8 * l.TY;
  if (!l.on || l.ty != 0) return;
#pragma unroll
  for (int q = 0; q < 8; ++q) u[q] = s[l.vx * 8 + q], v[q] = s[half + l.vx * 8 + q];
  float *p = partial + w.at * 2 * a.c + c;
  store8(p, left, u);
  store8(p + a.c, left, v);
}

// One workgroup a sample and group: its channels' sums over the chunks to
// sums[sample][2][c], and the group's means of h and h xh to mean[2][b][groups].
template <class T>
__global__ __launch_bounds__(256) void split_grad_join_kernel(const float *partial, int64_t s_all, int chunks,
                                                              int64_t c, int per, const T *gamma, float *sums,
                                                              float *mean) {
  __shared__ float s[2][256];
  __shared__ float sw[2 * 2 * 4];
  int turn = 0, turn2 = 0;
  const uint32_t groups = uint32_t(c / per), i = blockIdx.x / groups, g = blockIdx.x % groups;
  const int64_t c0 = int64_t(g) * per;
  const float *p = partial + int64_t(i) * chunks * 2 * c + c0;
  const int side = min(per, 256), rows = 256 / side;
  const int tx = threadIdx.x % side, ty = threadIdx.x / side;
  float m1 = 0.f, m2 = 0.f;
  for (int j0 = 0; j0 < per; j0 += side) {
    const int j = j0 + tx;
    float u = 0.f, v = 0.f;
    if (ty < rows && j < per) {
#pragma unroll 8
      for (int q = ty; q < chunks; q += rows) {
        u += p[int64_t(q) * 2 * c + j];
        v += p[int64_t(q) * 2 * c + c + j];
      }
    }
    __syncthreads();
    s[0][threadIdx.x] = u;
    s[1][threadIdx.x] = v;
    __syncthreads();
    if (ty == 0 && j < per) {
      for (int r = 1; r < rows; ++r) {
        u += s[0][r * side + tx];
        v += s[1][r * side + tx];
      }
      if (sums) {
        sums[int64_t(i) * 2 * c + c0 + j] = u;
        sums[int64_t(i) * 2 * c + c + c0 + j] = v;
      }
      const float w = gamma ? float(gamma[c0 + j]) : 1.f;
      m2 += w * u;
      m1 += w * v;
    }
  }
  const float inv = 1.f / (float(s_all) * float(per));
  m1 = block_sum<256>(m1, sw, turn) * inv;
  m2 = block_sum<256>(m2, sw + 2 * 4, turn2) * inv;
  if (threadIdx.x == 0) {
    mean[blockIdx.x] = m1;
    mean[gridDim.x + blockIdx.x] = m2;
  }
}

template <class T>
__global__ __launch_bounds__(256) void split_grad_write_kernel(dip_group_norm_grad_args a, int vectors, int lanes_y, int tiles,
                                                               int chunks, int64_t chunk, const float *mean) {
  const Lanes l(vectors, lanes_y);
  const Part w(l, vectors, tiles, chunks, chunk, a.c, a.s, true);
  const int left = int(w.left), per = int(a.c) / a.groups;
  const int64_t i = w.i, c = w.c;
  if (left <= 0) return;
  Channels ch;
  of_groups(a.mean + i * a.groups, a.rstd + i * a.groups, c, per, left, ch.mean, ch.rstd);
  Affine<T>{static_cast<const T *>(a.gamma), static_cast<const T *>(a.beta)}.get(c, left, ch.gamma, ch.beta);
  float m1[8], m2[8];
  of_groups(mean + i * a.groups, mean + (a.b + i) * a.groups, c, per, left, m1, m2);
  write_grad(static_cast<const T *>(a.x) + i * a.x_sb + c, a.x_ss, static_cast<const T *>(a.dy) + i * a.dy_sb + c,
             a.dy_ss, static_cast<T *>(a.dx) + i * a.dx_sb + c, a.dx_ss, left, l, w.r0 + l.ty, w.r1, ch, m1, m2, a.act);
}

// The statistics of groups of nothing: mean 0, variance 0.
__global__ __launch_bounds__(256) void no_values_kernel(int64_t n, float r, float *mean, float *rstd) {
  for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < n; i += int64_t(gridDim.x) * 256) {
    if (mean) mean[i] = 0.f;
    if (rstd) rstd[i] = r;
  }
}

// ------------------------------------------------------------ plans

enum Way { kRows, kBlock, kSplit };
struct Plan {
  Way way = kRows;
  int groups = 1, vectors = 1, lanes_y = 1, threads = 256, tiles = 1;   // block: groups a slab
  int64_t chunk = 0, chunks = 1;                                       // split
  int64_t row_blocks = 1;                                              // rows' gradient
  int lanes = 8;                                                       // narrow rows
  size_t lds = 0;
  int64_t partial = 0, stat = 0, sums = 0;   // floats
  int64_t stat_at() const { return up16(partial * 4); }
  int64_t sums_at() const { return stat_at() + up16(stat * 4); }
  int64_t bytes() const { return sums_at() + up16(sums * 4); }
};

int pow2_at_most(int64_t n) {
  int p = 1;
  while (2 * p <= n) p *= 2;
  return p;
}

constexpr int kRowMost = 16384;      // channels a row held in registers
constexpr int kSlabMost = 4096;      // channels a slab, eight a thread

// of at least one sample, position and channel
Plan plan(int64_t b, int64_t s, int64_t c, int groups, int elem, bool grad) {
  Plan p;
  const int64_t per = c / groups;
  if (s == 1 && per <= kRowMost && groups < 65536) {
    p.way = kRows;
    if (per <= 512) {   // narrow rows: four workgroups a CU
      while (p.lanes < 64 && p.lanes * 8 < per) p.lanes *= 2;
      const int64_t at_once = 256 / p.lanes;
      p.row_blocks = std::max<int64_t>(1, std::min<int64_t>((b + at_once - 1) / at_once, std::max(1, 1024 / groups)));
    } else {
      p.row_blocks = std::max<int64_t>(1, std::min<int64_t>(b, std::max(1, 512 / groups)));
    }
    // one workgroup a group of narrow rows writes the parameters' gradients itself
    p.partial = grad && !(per <= 512 && p.row_blocks == 1) ? p.row_blocks * 2 * c : 0;
    return p;
  }
  // a slab of at least 128 bytes of a row, and beyond that as many groups as still
  // leave workgroups for the whole card; where that would leave most of it idle,
  // of eight channels (the lines that slabs share come out of the caches)
  const int64_t least = b * c * elem >= 128 * 256 ? 128 / elem : 8;
  int64_t slab = std::max<int64_t>(1, std::min<int64_t>(groups, (least + per - 1) / per));
  while (slab * 2 <= groups && slab * 2 * per <= 512 && b * ((groups + slab * 2 - 1) / (slab * 2)) >= 1024) slab *= 2;
  const int64_t blocks = b * ((groups + slab - 1) / slab);
  if (slab * per <= kSlabMost && (s * slab * per <= 32768 || blocks >= 512)) {
    p.way = kBlock;
    p.groups = int(slab);
    p.vectors = int((slab * per + 7) / 8);
    p.threads = s * p.vectors > 256 ? 512 : 256;
    p.lanes_y = pow2_at_most(std::min<int64_t>(s, p.threads / p.vectors));
    p.tiles = int((groups + slab - 1) / slab);
    p.lds = size_t(2) * p.vectors * 8 * p.lanes_y * 4 + size_t(2) * slab * 4;
    p.partial = grad && b > 1 ? b * 2 * c : 0;
    return p;
  }
  p.way = kSplit;
  const int64_t cv = (c + 7) / 8;
  p.tiles = int((cv + 255) / 256);
  p.vectors = int((cv + p.tiles - 1) / p.tiles);
  p.lanes_y = pow2_at_most(256 / p.vectors);
  // chunks for about four workgroups a CU, of at least two rows a thread
  const int64_t most = std::max<int64_t>(1, s / (int64_t(p.lanes_y) * 2));
  p.chunks = std::max<int64_t>(1, std::min<int64_t>(most, 1024 / std::max<int64_t>(1, b * p.tiles)));
  p.chunk = (s + p.chunks - 1) / p.chunks;
  p.chunks = (s + p.chunk - 1) / p.chunk;
  p.lds = size_t(2) * p.vectors * 8 * p.lanes_y * 4;
  p.partial = b * p.chunks * 2 * c;
  p.stat = 2 * b * groups;
  p.sums = grad ? b * 2 * c : 0;
  return p;
}

// Samples that one launch of each of a plan's kernels takes: a launch has fewer than
// 2^32 threads, and one sample has at most 2^31.
int64_t samples_a_launch(const Plan &p, int64_t per, int64_t groups) {
  const int64_t a_row = per <= 512 ? p.lanes : per <= 1024 ? 64 : 256;
  const int64_t threads = p.way == kRows    ? groups * a_row
                          : p.way == kBlock ? int64_t(p.tiles) * p.threads
                                            : std::max(p.tiles * p.chunks, groups) * 256;
  return std::max<int64_t>(1, (int64_t(1) << 31) / threads);
}

template <class T>
hipError_t forward_piece(const dip_group_norm_args &a, const Plan &p, float *partial, float *stat, hipStream_t st) {
  const int64_t per = a.c / a.groups, rows = a.b * a.groups;
  if (p.way == kRows) {
    const dim3 narrow(uint32_t((rows + 256 / p.lanes - 1) / (256 / p.lanes)));
    if (per <= 64)
      narrow_kernel<T, 8><<<narrow, dim3(256), 0, st>>>(a, rows);
    else if (per <= 128)
      narrow_kernel<T, 16><<<narrow, dim3(256), 0, st>>>(a, rows);
    else if (per <= 256)
      narrow_kernel<T, 32><<<narrow, dim3(256), 0, st>>>(a, rows);
    else if (per <= 512)
      narrow_kernel<T, 64><<<narrow, dim3(256), 0, st>>>(a, rows);
    else if (per <= 1024)
      rows_kernel<T, 64, 2><<<dim3(uint32_t((rows + 3) / 4)), dim3(256), 0, st>>>(a, rows);
    else if (per <= 2048)
      rows_kernel<T, 256, 1><<<dim3(uint32_t(rows)), dim3(256), 0, st>>>(a, rows);
    else if (per <= 4096)
      rows_kernel<T, 256, 2><<<dim3(uint32_t(rows)), dim3(256), 0, st>>>(a, rows);
    else
      rows_kernel<T, 256, 8><<<dim3(uint32_t(rows)), dim3(256), 0, st>>>(a, rows);
    return hipGetLastError();
  }
  if (p.way == kBlock) {
    block_kernel<T><<<dim3(uint32_t(p.tiles * a.b)), dim3(p.threads), p.lds, st>>>(a, p.groups, p.vectors,
                                                                                      p.lanes_y);
    return hipGetLastError();
  }
  const dim3 grid(uint32_t(p.tiles * p.chunks * a.b));
  split_sums_kernel<T><<<grid, dim3(256), p.lds, st>>>(a, p.vectors, p.lanes_y, p.tiles, int(p.chunks), p.chunk, partial);
  split_join_kernel<<<dim3(uint32_t(rows)), dim3(256), 0, st>>>(partial, a.s, p.chunk, int(p.chunks), a.c, int(per),
                                                               a.eps, a.mean, a.rstd, stat);
  split_write_kernel<T><<<grid, dim3(256), 0, st>>>(a, p.vectors, p.lanes_y, p.tiles, int(p.chunks), p.chunk, stat);
  return hipGetLastError();
}

// f(first sample, samples) over pieces of b samples until one fails.
template <class F>
hipError_t pieces(int64_t b, int64_t at_once, F &&f) {
  for (int64_t i = 0; i < b; i += at_once) {
    const hipError_t e = f(i, std::min(at_once, b - i));
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <class T>
hipError_t forward(const dip_group_norm_args &a, hipStream_t st) {
  const Plan p = plan(a.b, a.s, a.c, a.groups, a.dtype == DIP_F32 ? 4 : 2, false);
  float *partial = static_cast<float *>(a.workspace);
  float *stat = reinterpret_cast<float *>(static_cast<char *>(a.workspace) + p.stat_at());
  return pieces(a.b, samples_a_launch(p, a.c / a.groups, a.groups), [&](int64_t i, int64_t n) {
    dip_group_norm_args q = a;
    q.b = n;
    q.x = static_cast<const T *>(a.x) + i * a.x_sb;
    q.y = static_cast<T *>(a.y) + i * a.y_sb;
    if (a.mean) q.mean += i * a.groups;
    if (a.rstd) q.rstd += i * a.groups;
    return forward_piece<T>(q, p, partial + i * p.chunks * 2 * a.c, stat + i * 2 * a.groups, st);
  });
}

// of dgamma and dbeta
int param_type(const dip_group_norm_grad_args &a) { return a.accumulate ? DIP_F32 : a.dtype; }

template <class T>
hipError_t backward(const dip_group_norm_grad_args &a, hipStream_t st) {
  const Plan p = plan(a.b, a.s, a.c, a.groups, a.dtype == DIP_F32 ? 4 : 2, true);
  const int64_t per = a.c / a.groups, at_once = samples_a_launch(p, per, a.groups);
  float *partial = static_cast<float *>(a.workspace);
  float *sums = p.partial > 0 && (a.dgamma || a.dbeta) ? partial : nullptr;
  auto piece = [&](int64_t i, int64_t n) {
    dip_group_norm_grad_args q = a;
    q.b = n;
    q.dy = static_cast<const T *>(a.dy) + i * a.dy_sb;
    q.x = static_cast<const T *>(a.x) + i * a.x_sb;
    q.mean += i * a.groups;
    q.rstd += i * a.groups;
    if (a.dx) q.dx = static_cast<T *>(a.dx) + i * a.dx_sb;
    return q;
  };
  if (p.way == kSplit) {
    float *means = reinterpret_cast<float *>(static_cast<char *>(a.workspace) + p.stat_at());
    if (sums) sums = reinterpret_cast<float *>(static_cast<char *>(a.workspace) + p.sums_at());
    const hipError_t e = pieces(a.b, at_once, [&](int64_t i, int64_t n) {
      const dip_group_norm_grad_args q = piece(i, n);
      float *part = partial + i * p.chunks * 2 * a.c, *mean = means + i * 2 * a.groups;
      const dim3 grid(uint32_t(p.tiles * p.chunks * n));
      split_grad_sums_kernel<T><<<grid, dim3(256), p.lds, st>>>(q, p.vectors, p.lanes_y, p.tiles, int(p.chunks), p.chunk, part);
      split_grad_join_kernel<T><<<dim3(uint32_t(n * a.groups)), dim3(256), 0, st>>>(
          part, a.s, int(p.chunks), a.c, int(per), static_cast<const T *>(a.gamma), sums ? sums + i * 2 * a.c : nullptr,
          mean);
      if (a.dx) split_grad_write_kernel<T><<<grid, dim3(256), 0, st>>>(q, p.vectors, p.lanes_y, p.tiles, int(p.chunks), p.chunk, mean);
      return hipGetLastError();
    });
    if (e != hipSuccess || !sums) return e;
    return launch_sum_rows(SumRows{sums, a.b, 2 * a.c, a.c, a.dgamma, a.dbeta, a.accumulate}, param_type(a), st);
  }
  int64_t rows = a.b;
  if (p.way == kRows) {
    rows = p.row_blocks;
    const dim3 grid(uint32_t(p.row_blocks), uint32_t(a.groups));
    if (per <= 64)
      narrow_grad_kernel<T, 8><<<grid, dim3(256), 0, st>>>(a, sums);
    else if (per <= 128)
      narrow_grad_kernel<T, 16><<<grid, dim3(256), 0, st>>>(a, sums);
    else if (per <= 256)
      narrow_grad_kernel<T, 32><<<grid, dim3(256), 0, st>>>(a, sums);
    else if (per <= 512)
      narrow_grad_kernel<T, 64><<<grid, dim3(256), 0, st>>>(a, sums);
    else if (per <= 2048)
      rows_grad_kernel<T, 256, 1><<<grid, dim3(256), 0, st>>>(a, sums);
    else if (per <= 4096)
      rows_grad_kernel<T, 512, 1><<<grid, dim3(512), 0, st>>>(a, sums);
    else if (per <= 8192)
      rows_grad_kernel<T, 512, 2><<<grid, dim3(512), 0, st>>>(a, sums);
    else
      rows_grad_kernel<T, 512, 4><<<grid, dim3(512), 0, st>>>(a, sums);
  } else {
    const hipError_t e = pieces(a.b, at_once, [&](int64_t i, int64_t n) {
      block_grad_kernel<T><<<dim3(uint32_t(p.tiles * n)), dim3(p.threads), p.lds, st>>>(
          piece(i, n), p.groups, p.vectors, p.lanes_y, sums ? sums + i * 2 * a.c : nullptr);
      return hipGetLastError();
    });
    if (e != hipSuccess) return e;
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !sums) return e;
  return launch_sum_rows(SumRows{partial, rows, 2 * a.c, a.c, a.dgamma, a.dbeta, a.accumulate}, param_type(a), st);
}

}  // namespace

int64_t group_norm_workspace(const dip_group_norm_args &a) {
  return a.b > 0 && a.c > 0 && a.s > 0 ? plan(a.b, a.s, a.c, a.groups, a.dtype == DIP_F32 ? 4 : 2, false).bytes() : 0;
}
int64_t group_norm_grad_workspace(const dip_group_norm_grad_args &a) {
  return a.b > 0 && a.c > 0 && a.s > 0 ? plan(a.b, a.s, a.c, a.groups, a.dtype == DIP_F32 ? 4 : 2, true).bytes() : 0;
}

hipError_t launch_group_norm(const dip_group_norm_args &a, hipStream_t st) {
  if (a.s == 0 || a.c == 0) {
    const int64_t n = a.b * a.groups;
    if (n == 0 || (!a.mean && !a.rstd)) return hipSuccess;
    no_values_kernel<<<dim3(uint32_t(std::min<int64_t>((n + 255) / 256, 4096))), dim3(256), 0, st>>>(
        n, 1.f / std::sqrt(a.eps), a.mean, a.rstd);
    return hipGetLastError();
  }
  return a.dtype == DIP_F32   ? forward<float>(a, st)
         : a.dtype == DIP_F16 ? forward<_Float16>(a, st)
                              : forward<__bf16>(a, st);
}

hipError_t launch_group_norm_grad(const dip_group_norm_grad_args &a, hipStream_t st) {
  if (a.b == 0 || a.s == 0)   // sums over nothing
    return launch_sum_rows(SumRows{nullptr, 0, 0, a.c, a.dgamma, a.dbeta, a.accumulate}, param_type(a), st);
  return a.dtype == DIP_F32   ? backward<float>(a, st)
         : a.dtype == DIP_F16 ? backward<_Float16>(a, st)
                              : backward<__bf16>(a, st);
}

}  // namespace dipops
