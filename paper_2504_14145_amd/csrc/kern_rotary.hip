// kern_rotary.hip -- rotary positions with several axes: the pairs of every head of a
// token turned by the angles of its positions.
//
// Bound by memory, every head read and written once; a token's sines and cosines are
// as many as one head has pairs and serve all heads.  A workgroup takes a token or a
// few, or a share of one token's heads: it asks for all its pairs, a vector a thread,
// puts the sines and cosines into LDS meanwhile (in float64 up to their rounding: far
// positions lose nothing), and turns and stores.
// bf16, 65,536 tokens of 56 heads of 128: 319 to 323 us, 5.9 TB/s; 28 heads of q alone
// 160, 5.9.  2^26 elements of 16 + 16 heads, us: 128 elements a head 47, 112 50, 72 51,
// 20 (4 + 4 heads) 57; one head of q and k each 69, sines and cosines then being as many
// as pairs.
#include <algorithm>
#include <type_traits>

#include "ops_internal.h"

namespace dipops {
namespace {

constexpr int kThreads = 512;   // at most

__device__ __forceinline__ double position(const dip_rotary_args &a, int64_t at) {
  if (a.pos_type == DIP_POS_I64) return double(static_cast<const int64_t *>(a.pos)[at]);
  const int32_t v = static_cast<const int32_t *>(a.pos)[at];
  return a.pos_type == DIP_POS_I32 ? double(v) : double(__builtin_bit_cast(float, v));
}

template <class T, int V>
struct Vector {
  typedef T type __attribute__((ext_vector_type(V)));
  typedef type any __attribute__((aligned(sizeof(T))));
};
template <class T>
struct Vector<T, 1> {
  typedef T type, any;
};
template <class T, int V>
__device__ __forceinline__ typename Vector<T, V>::type load(const T *p) {
  return *reinterpret_cast<const typename Vector<T, V>::any *>(p);
}
template <class T, int V>
__device__ __forceinline__ void floats(const typename Vector<T, V>::type &t, float (&v)[V]) {
  if constexpr (V == 1) v[0] = float(t);
  else {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = float(t[i]);
  }
}
template <class T, int V>
__device__ __forceinline__ void store(T *p, const float (&v)[V]) {
  typename Vector<T, V>::type t;
  if constexpr (V == 1) t = T(v[0]);
  else {
#pragma unroll
    for (int i = 0; i < V; ++i) t[i] = T(v[i]);
  }
  *reinterpret_cast<typename Vector<T, V>::any *>(p) = t;
}

// Tokens and heads a workgroup takes; dividers of an item's index.
struct Shares {
  int32_t tokens, heads;
  Divide vectors, in_head;   // vectors a head; heads a token
};

// Where an item's pairs lie and go.
template <class T>
struct Item {
  const T *p;
  T *o;
  uint32_t first, n;   // first pair, token of the workgroup
  __device__ __forceinline__ Item(const dip_rotary_args &a, const Shares &sh, int V, uint32_t i, int64_t i0, int h0,
                                  int heads) {
    const uint32_t x = sh.vectors(i);
    first = min((i - x * sh.vectors.by) * V, uint32_t(a.pairs - V));
    n = heads == sh.heads ? sh.in_head(x) : x / uint32_t(heads);
    const int h = int(x - n * uint32_t(heads)) + h0;
    const int64_t token = i0 + n;
    const bool of_q = h < a.heads;
    const int64_t hk = of_q ? h : h - a.heads;
    p = of_q ? static_cast<const T *>(a.q) + token * a.q_st + hk * a.q_sh
             : static_cast<const T *>(a.k) + token * a.k_st + hk * a.k_sh;
    o = of_q ? static_cast<T *>(a.q_out) + token * a.qo_st + hk * a.qo_sh
             : static_cast<T *>(a.k_out) + token * a.ko_st + hk * a.ko_sh;
  }
};

// (cosine, sine) of an angle in turns: less its whole turns and its nearest quarter by the
// Taylor series about that, in float64 to 2^-36 of themselves, and rounded once.  (The
// hardware's way, sincospif of a float32 argument, leaves 2^-23 beside that rounding.)
__device__ __forceinline__ float2 turned_by(double turns) {
  turns -= rint(turns);
  const double quarter = rint(4.0 * turns), a = fma(quarter, -0.25, turns) * 6.283185307179586477, z = a * a;
  double s = fma(z, -1.0 / 39916800, 1.0 / 362880), c = fma(z, 1.0 / 479001600, -1.0 / 3628800);
  s = fma(z, s, -1.0 / 5040);
  c = fma(z, c, 1.0 / 40320);
  s = fma(z, s, 1.0 / 120);
  c = fma(z, c, -1.0 / 720);
  s = fma(z, s, -1.0 / 6);
  c = fma(z, c, 1.0 / 24);
  s = fma(a * z, s, a);
  c = fma(z, c, -0.5);
  c = fma(z, c, 1.0);
  const int q = int(quarter);   // -2 .. 2: to (-s, c), (-c, -s) and (s, -c)
  const float u = float(q & 1 ? s : c), v = float(q & 1 ? c : s);
  return float2{(q + 1) & 2 ? -u : u, q & 2 ? -v : v};
}

// V pairs a thread; a head's last vector ends with its pairs and has some of the one
// before, which come out the same.  All loads are before the barrier and all stores
// behind it, and a head is one workgroup's: outputs may be the inputs.  What is loaded
// stays as it is up to there, so that nothing waits for it before.
template <class T, int V, bool INTERLEAVED>
__global__ __launch_bounds__(kThreads) void rotary_kernel(dip_rotary_args a, int64_t token0, Shares sh) {
  extern __shared__ float2 table[];   // [tokens][pairs]: cosine, sine
  const int64_t i0 = token0 + int64_t(blockIdx.x) * sh.tokens;
  const int tokens = int(min(int64_t(sh.tokens), a.t - i0)), all = a.heads + a.keys;
  const int h0 = int(blockIdx.y) * sh.heads, heads = min(sh.heads, all - h0);
  const bool on = threadIdx.x < uint32_t(tokens) * uint32_t(heads) * sh.vectors.by;
  const Item<T> it(a, sh, V, on ? threadIdx.x : 0, i0, h0, heads);
  const int at = int(it.first) * (INTERLEAVED ? 2 : 1), step = INTERLEAVED ? V : a.pairs;
  const int angles = tokens * a.pairs;
  auto turns = [&](int j) __attribute__((always_inline)) {   // of the pair's angle; 0 without an axis
    const int n = j / a.pairs, pair = j - n * a.pairs, axis = a.axis[pair];
    const double f = a.freq[pair] * 0.15915494309189533577;   // asked for with the axis, not behind the position
    const bool has = uint32_t(axis) < uint32_t(a.axes);
    const double p = has ? position(a, (i0 + n) * a.p_st + axis * a.p_sa) : 0.0;
    return has ? p * f : 0.0;
  };
  auto put = [&](int j, double turns) __attribute__((always_inline)) {
    float2 cs = turned_by(turns);
    if (a.inverse) cs.y = -cs.y;
    table[j] = cs;
  };
  typename Vector<T, V>::type ru, rw;
  if (on) {   // on their way while the table is made
    ru = load<T, V>(it.p + at);
    rw = load<T, V>(it.p + at + step);
  }
  for (int j = threadIdx.x; j < angles; j += blockDim.x) put(j, turns(j));
  // what overlaps at a head's end another wave may write in its input's place
  if (a.pairs % V) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (!on) return;
  float u[V], w[V];
  floats<T, V>(ru, u);
  floats<T, V>(rw, w);
  const float2 *cs = table + it.n * a.pairs + it.first;
  float ou[V], ow[V];
  if constexpr (INTERLEAVED && V > 1) {
#pragma unroll
    for (int j = 0; j < V / 2; ++j) {
      const float2 c = cs[j], d = cs[V / 2 + j];
      ou[2 * j] = u[2 * j] * c.x - u[2 * j + 1] * c.y;
      ou[2 * j + 1] = u[2 * j] * c.y + u[2 * j + 1] * c.x;
      ow[2 * j] = w[2 * j] * d.x - w[2 * j + 1] * d.y;
      ow[2 * j + 1] = w[2 * j] * d.y + w[2 * j + 1] * d.x;
    }
  } else {
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const float2 c = cs[j];
      ou[j] = u[j] * c.x - w[j] * c.y;
      ow[j] = u[j] * c.y + w[j] * c.x;
    }
  }
  store<T, V>(it.o + at, ou);
  store<T, V>(it.o + at + step, ow);
}

// Elements 2 pairs .. dim - 1 of every head, where the output is not the input.
template <class T>
__global__ __launch_bounds__(kThreads) void rotary_rest_kernel(dip_rotary_args a, int64_t items) {
  const int rest = a.dim - 2 * a.pairs, all = a.heads + a.keys;
  for (int64_t i = int64_t(blockIdx.x) * kThreads + threadIdx.x; i < items; i += int64_t(gridDim.x) * kThreads) {
    const int64_t x = i / rest, token = x / all;
    const int e = 2 * a.pairs + int(i - x * rest), h = int(x - token * all);
    if (h < a.heads)
      static_cast<T *>(a.q_out)[token * a.qo_st + h * a.qo_sh + e] = static_cast<const T *>(a.q)[token * a.q_st + h * a.q_sh + e];
    else
      static_cast<T *>(a.k_out)[token * a.ko_st + (h - a.heads) * a.ko_sh + e] =
          static_cast<const T *>(a.k)[token * a.k_st + (h - a.heads) * a.k_sh + e];
  }
}

template <class T>
hipError_t rotary(const dip_rotary_args &a, hipStream_t st) {
  const int all = a.heads + a.keys;
  if (a.pairs > 0) {
    const int V = a.pairs >= 8 ? 8 : a.pairs >= 4 ? 4 : a.pairs >= 2 ? 2 : 1;
    const int vectors = (a.pairs + V - 1) / V;   // at most 128
    // One item a thread: as many tokens as 256 threads take, with tables of up to 2048
    // pairs; or one token by a workgroup of its items, in even shares where they are many
    // (65,536 x 28 heads of 128, bf16: one token 153 us, 6.1 TB/s, two 166, four 171,
    // sixteen 186: a workgroup that loops waits for each round's loads).
    Shares sh{1, all, Divide(uint32_t(vectors)), Divide(1)};
    const int64_t an = int64_t(all) * vectors;
    if (an <= 256) {
      sh.tokens = int32_t(std::max<int64_t>(1, std::min<int64_t>(256 / an, 2048 / a.pairs)));
    } else {
      const int64_t parts = std::min<int64_t>((an + kThreads - 1) / kThreads, 65535);
      sh.heads = int32_t(std::min<int64_t>((all + parts - 1) / parts, kThreads / vectors));
    }
    sh.in_head = Divide(uint32_t(sh.heads));
    const uint32_t parts = uint32_t((all + sh.heads - 1) / sh.heads);
    const int threads = (sh.tokens * sh.heads * vectors + 63) / 64 * 64;
    // a launch has fewer than 2^32 threads
    const int64_t blocks = std::max<int64_t>(1, ((int64_t(1) << 31) / threads) / parts), most = blocks * sh.tokens;
    for (int64_t token0 = 0; token0 < a.t; token0 += most) {
      dip_rotary_args b = a;
      b.t = std::min(a.t, token0 + most);
      const dim3 grid(uint32_t((b.t - token0 + sh.tokens - 1) / sh.tokens), parts);
      const size_t lds = size_t(sh.tokens) * a.pairs * sizeof(float2);
      auto go = [&](auto v) {
        constexpr int kV = decltype(v)::value;
        if (a.interleaved) rotary_kernel<T, kV, true><<<grid, dim3(threads), lds, st>>>(b, token0, sh);
        else rotary_kernel<T, kV, false><<<grid, dim3(threads), lds, st>>>(b, token0, sh);
      };
      if (V == 8) go(std::integral_constant<int, 8>{});
      else if (V == 4) go(std::integral_constant<int, 4>{});
      else if (V == 2) go(std::integral_constant<int, 2>{});
      else go(std::integral_constant<int, 1>{});
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
  }
  const bool moved = (a.heads > 0 && a.q != a.q_out) || (a.keys > 0 && a.k != a.k_out);
  if (a.dim > 2 * a.pairs && moved) {
    const int64_t items = a.t * all * (a.dim - 2 * a.pairs);
    rotary_rest_kernel<T><<<dim3(uint32_t(std::min<int64_t>((items + kThreads - 1) / kThreads, 1 << 16))), dim3(kThreads), 0, st>>>(a, items);
    return hipGetLastError();
  }
  return hipSuccess;
}

}  // namespace

hipError_t launch_rotary(const dip_rotary_args &a, hipStream_t stream) {
  switch (a.dtype) {
    case DIP_F32: return rotary<float>(a, stream);
    case DIP_F16: return rotary<_Float16>(a, stream);
    default: return rotary<__bf16>(a, stream);
  }
}

}  // namespace dipops
