// ops_device.h -- what the stage operators' kernels share: element types, vector
// accesses, activations, dropout draws and the epilogue of the matrix products.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "dip_ops.h"

namespace dipops {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

template <class T>
struct Vec8;
template <>
struct Vec8<__bf16> {
  typedef bf16x8 type;
};
template <>
struct Vec8<_Float16> {
  typedef f16x8 type;
};

// c[i][j] += sum_k a[i][k] b[j][k], 16 x 16 x 32: lane l holds row l % 16 and
// k = 8 (l / 16) .. + 7 of either operand, and c's column l % 16, rows
// 4 (l / 16) .. + 3.
__device__ __forceinline__ void mfma16(bf16x8 a, bf16x8 b, f32x4 &c) {
  c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ void mfma16(f16x8 a, f16x8 b, f32x4 &c) {
  c = __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}
// A product's result may be read some cycles after its issue at the earliest; this
// waits longer than the slowest takes, for reads that the compiler does not place.
__device__ __forceinline__ void products_wait() { asm volatile("s_nop 15\n\ts_nop 15" ::: "memory"); }
__device__ __forceinline__ float from_accumulator(float a) {
  float v;
  asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(v) : "a"(a));
  return v;
}
// Keeps a result in accumulation registers up to here: with 256 of them a lane
// the compiler otherwise moves them back and forth.
__device__ __forceinline__ void in_accumulators(f32x4 &a, f32x4 &b) { asm volatile("" : "+a"(a), "+a"(b)); }

// Eight consecutive elements from any address aligned to its element (the
// hardware takes vector accesses at such addresses, and a row of odd length
// costs an extra cache line, not eight loads); `left` of them exist, the others
// read as zero and are not written.
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
template <class T>
struct Any8 {
  typedef typename Vec8<T>::type type __attribute__((aligned(2)));
};
template <class T>
__device__ __forceinline__ void load8(const T *p, int left, float (&v)[8]) {
  if (left >= 8) {
    if constexpr (sizeof(T) == 2) {
      const typename Vec8<T>::type t = *reinterpret_cast<const typename Any8<T>::type *>(p);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = float(t[i]);
    } else {
      const f32x4 a = reinterpret_cast<const f32x4_any *>(p)[0], b = reinterpret_cast<const f32x4_any *>(p)[1];
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = a[i], v[4 + i] = b[i];
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < left ? float(p[i]) : 0.f;
  }
}
// The same as one vector of 2-byte elements.
template <class T>
__device__ __forceinline__ typename Vec8<T>::type take8(const T *p, int left) {
  if (left >= 8) return *reinterpret_cast<const typename Any8<T>::type *>(p);
  typename Vec8<T>::type t;
#pragma unroll
  for (int i = 0; i < 8; ++i) t[i] = i < left ? p[i] : T(0.f);
  return t;
}
template <class T>
__device__ __forceinline__ typename Vec8<T>::type round8(const float (&v)[8]) {
  typename Vec8<T>::type t;
#pragma unroll
  for (int i = 0; i < 8; ++i) t[i] = T(v[i]);
  return t;
}
template <class T>
__device__ __forceinline__ void store8(T *p, int left, const float (&v)[8]) {
  if (left >= 8) {
    if constexpr (sizeof(T) == 2) {
      *reinterpret_cast<typename Any8<T>::type *>(p) = round8<T>(v);
    } else {
      f32x4 a, b;
#pragma unroll
      for (int i = 0; i < 4; ++i) a[i] = v[i], b[i] = v[4 + i];
      reinterpret_cast<f32x4_any *>(p)[0] = a;
      reinterpret_cast<f32x4_any *>(p)[1] = b;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < left) p[i] = T(v[i]);
  }
}

// ------------------------------------------------------------ ends of rows

// Columns c .. c + 7 of a row of n, zeros beyond it.  Where the row ends inside them the
// eight that end with it are read, and moved into place when they are used: all lanes
// read whole vectors (element by element the last lane costs a chain of loads), and no
// lane waits for its loads before it has asked for all of them.
template <class T>
struct Held {
  static constexpr int kWords = sizeof(T) * 2;   // 32-bit words of eight
  typedef uint32_t Words __attribute__((ext_vector_type(kWords)));
  typedef Words WordsAny __attribute__((aligned(sizeof(T))));
  Words t;
  __device__ __forceinline__ void get(const T *row, int c, int n) {
    if (n >= 8) {
      t = *reinterpret_cast<const WordsAny *>(row + min(c, n - 8));
    } else {
      float v[8];
      load8(row, n, v);
      T e[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) e[i] = T(v[i]);   // exact
      t = __builtin_bit_cast(Words, e);
    }
  }
  // by: elements to move down, 8 and more for a vector beyond the row
  static __device__ __forceinline__ int moved(int c, int n) { return n >= 8 ? max(c - (n - 8), 0) : c; }
  __device__ __forceinline__ Words words(int by) const {
    Words w = t;
    if (by) {
      if constexpr (sizeof(T) == 2) {
        if (by & 1) {
#pragma unroll
          for (int i = 0; i < kWords; ++i) w[i] = w[i] >> 16 | (i + 1 < kWords ? w[i + 1] << 16 : 0u);
        }
      }
      constexpr int per = sizeof(T) == 2 ? 2 : 1;   // elements a word
#pragma unroll
      for (int d = 1; d < kWords; d *= 2) {
        if (by / per & d) {
#pragma unroll
          for (int i = 0; i < kWords; ++i) w[i] = i + d < kWords ? w[i + d] : 0u;
        }
      }
      if (by >= 8) w = Words(0);
    }
    return w;
  }
  __device__ __forceinline__ void to(int by, float (&v)[8]) const {
    struct Elements {
      T e[8];
    };
    const Elements e = __builtin_bit_cast(Elements, words(by));
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = float(e.e[i]);
  }
};

// Stores `left` of eight columns, at a row's end four, two and one at once.
template <class T>
__device__ __forceinline__ void put8(T *p, int left, const float (&v)[8]) {
  if (left >= 8) return store8(p, 8, v);
  float w[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) w[i] = v[i];
  if (left & 4) {
    typedef T T4 __attribute__((ext_vector_type(4)));
    typedef T4 T4Any __attribute__((aligned(sizeof(T))));
    *reinterpret_cast<T4Any *>(p) = T4{T(w[0]), T(w[1]), T(w[2]), T(w[3])};
    p += 4;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = w[i + 4];
  }
  if (left & 2) {
    p[0] = T(w[0]);
    p[1] = T(w[1]);
    p += 2;
    w[0] = w[2];
  }
  if (left & 1) p[0] = T(w[0]);
}

// ------------------------------------------------------------ activations

// 1 / (1 + 2^t) with the hardware's exponential and reciprocal: within 1e-6 of
// the value for the t at which an output of it is not rounded to 0 or 1.
__device__ __forceinline__ float logistic2(float t) {
  return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(t));
}

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kGeluA = 0.7978845608028654f;   // sqrt(2 / pi)
constexpr float kGeluC = 0.044715f;

// the logistic function's argument of each, times -log2 e: z, and 2 u of GELU
__device__ __forceinline__ float silu_arg(float z) { return -kLog2e * z; }
__device__ __forceinline__ float gelu_arg(float z) {
  return z * (z * z * (-2.f * kLog2e * kGeluA * kGeluC) - 2.f * kLog2e * kGeluA);
}

__device__ __forceinline__ float act_of(float z, int act) {
  switch (act) {
    case DIP_ACT_RELU: return z > 0.f ? z : (z != z ? z : 0.f);
    case DIP_ACT_SILU: return z * logistic2(silu_arg(z));
    case DIP_ACT_GELU: return z * logistic2(gelu_arg(z));
    default: return z;
  }
}
__device__ __forceinline__ float act_slope(float z, int act) {
  switch (act) {
    case DIP_ACT_RELU: return z > 0.f ? 1.f : (z != z ? z : 0.f);
    case DIP_ACT_SILU: {
      // e is 0 or 1 beyond 120, and z may be infinite: a pre beyond float16's range is
      // stored so.  NaN comes through e.
      const float e = logistic2(silu_arg(z));
      return e * (1.f + __builtin_amdgcn_fmed3f(z, -120.f, 120.f) * (1.f - e));
    }
    case DIP_ACT_GELU: {
      if (fabsf(z) > 12.f) return z > 0.f ? 1.f : 0.f;   // e is 0 or 1 there, z^2 may overflow
      const float e = logistic2(gelu_arg(z));
      return e * (1.f + z * (1.f - e) * (2.f * kGeluA + 6.f * kGeluA * kGeluC * z * z));
    }
    default: return 1.f;
  }
}

// ------------------------------------------------------------ values in 8 bits

struct Packed {
  uint8_t *q;
  int64_t ld;
  uint8_t *s;
  int64_t lds;
};
inline Packed make_packed(const dip_packed8 &p) {
  return Packed{static_cast<uint8_t *>(p.values), p.ld, static_cast<uint8_t *>(p.scales), p.lds};
}

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef u32x2 u32x2_any __attribute__((aligned(1)));

// Magnitudes are compared as integers: infinity and NaN are above all others.
constexpr uint32_t kInfinity = 0x7f800000u;
__device__ __forceinline__ uint32_t magnitude(float v) { return __builtin_bit_cast(uint32_t, v) & 0x7fffffffu; }
// By the three-operand maximum, which passes over NaN: those are NaN in 8 bits anyway.
__device__ __forceinline__ uint32_t most_of(const float (&v)[8]) {
  float most = fmaxf(fabsf(v[0]), fabsf(v[1]));
#pragma unroll
  for (int i = 2; i < 8; i += 2) most = fmaxf(fmaxf(most, fabsf(v[i])), fabsf(v[i + 1]));
  return magnitude(most);
}
// Makes what is not finite NaN, and the largest magnitude of the others.
__device__ __forceinline__ uint32_t finite_most(float (&v)[8]) {
  uint32_t most = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t a = magnitude(v[i]);
    if (a >= kInfinity) v[i] = NAN;
    else most = max(most, a);
  }
  return most;
}
// The largest over the four lanes 4 j .. 4 j + 3, which are all on.
__device__ __forceinline__ uint32_t quad_most(uint32_t a) {
  a = max(a, uint32_t(__builtin_amdgcn_mov_dpp(int(a), 0xb1, 0xf, 0xf, true)));      // lane ^ 1
  return max(a, uint32_t(__builtin_amdgcn_mov_dpp(int(a), 0x4e, 0xf, 0xf, true)));   // lane ^ 2
}
// The byte e + 127 of the smallest 2^e, e >= -126, with most / 2^e <= 448 = 1.75 2^8,
// by the bits of most.
__device__ __forceinline__ uint32_t scale_byte(uint32_t most) {
  return uint32_t(max(int(most >> 23) - 8 + ((most & 0x7fffffu) > 0x600000u ? 1 : 0), 1));
}
__device__ __forceinline__ float scale_of(uint32_t byte) {
  const uint32_t b = byte ? byte << 23 : 0x400000u;
  return __builtin_bit_cast(float, byte == 255 ? 0x7fc00000u : b);
}
// Eight values over 2^e in 8 bits: at most 448 each, or NaN.  The conversions divide by
// the scale and round to nearest even: as the arithmetic does for every 16-bit value under
// every scale that it can have, and for float32 on and beside every border.
typedef short s16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ u32x2 round8bits(uint32_t byte, const float (&v)[8]) {
  const float scale = __builtin_bit_cast(float, byte << 23);   // byte 1 .. 247
  u32x2 r;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    s16x2 w = {0, 0};
    w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, v[4 * i], v[4 * i + 1], scale, false);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, v[4 * i + 2], v[4 * i + 3], scale, true);
    r[i] = __builtin_bit_cast(uint32_t, w);
  }
  return r;
}
__device__ __forceinline__ void store8bits(uint8_t *p, int left, u32x2 r) {
  if (left >= 8) {
    *reinterpret_cast<u32x2_any *>(p) = r;
    return;
  }
  uint32_t w = r[0];
  if (left & 4) {
    typedef uint32_t u32_any __attribute__((aligned(1)));
    *reinterpret_cast<u32_any *>(p) = w;
    p += 4;
    w = r[1];
  }
  if (left & 2) {
    p[0] = uint8_t(w);
    p[1] = uint8_t(w >> 8);
    p += 2;
    w >>= 16;
  }
  if (left & 1) p[0] = uint8_t(w);
}
// Columns c .. c + 7, c < n, of a row of n; as Held: moved into place behind the loads.
__device__ __forceinline__ u32x2 load8bits(const uint8_t *row, int c, int n) {
  if (n >= 8) return *reinterpret_cast<const u32x2_any *>(row + min(c, n - 8));
  uint64_t r = 0;
  for (int i = 0; i < n; ++i) r |= uint64_t(row[i]) << (8 * i);   // c is 0
  return __builtin_bit_cast(u32x2, r);
}
__device__ __forceinline__ void place8bits(int c, int n, u32x2 &r) {
  if (n >= 8 && c > n - 8) r = __builtin_bit_cast(u32x2, __builtin_bit_cast(uint64_t, r) >> (8 * (c - (n - 8))));
}
// Exact for every value and scale.
__device__ __forceinline__ void from8bits(u32x2 r, float scale, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const auto lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(r[i], scale, false),
               hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(r[i], scale, true);
    v[4 * i] = lo[0];
    v[4 * i + 1] = lo[1];
    v[4 * i + 2] = hi[0];
    v[4 * i + 3] = hi[1];
  }
}
// The same in 16 bits, for scales from 2^-15 to 2^7 in float16, whose values that holds,
// and from 2^-124 to 2^119 in bfloat16 (float32: up to 2^119).
__device__ __forceinline__ bool held_by(float, uint32_t byte) { return byte <= 246u; }
__device__ __forceinline__ bool held_by(_Float16, uint32_t byte) { return byte - 112u <= 22u; }
__device__ __forceinline__ bool held_by(__bf16, uint32_t byte) { return byte - 3u <= 243u; }
template <class T>
__device__ __forceinline__ typename Vec8<T>::type from8bits_to(u32x2 r, float scale) {
  typedef T T2 __attribute__((ext_vector_type(2)));
  T2 q[4];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if constexpr (__is_same(T, _Float16)) {
      q[2 * i] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(r[i], scale, false);
      q[2 * i + 1] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(r[i], scale, true);
    } else {
      q[2 * i] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(r[i], scale, false);
      q[2 * i + 1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(r[i], scale, true);
    }
  }
  return typename Vec8<T>::type{q[0][0], q[0][1], q[1][0], q[1][1], q[2][0], q[2][1], q[3][0], q[3][1]};
}
// What rounded up beyond the largest value of T in 8 bits is that value; NaN stays.
template <class T>
__device__ __forceinline__ float within(float v) {
  constexpr float kMost = sizeof(T) == 4 ? 3.402823466e38f
                          : __is_same(T, _Float16) ? 65504.f : 3.389531389e38f;   // (2 - 2^-7) 2^127
  return v > kMost ? kMost : v < -kMost ? -kMost : v;
}
// Columns col .. col + 7 of act of a row in 8 bits, of which n exist, to `left` columns
// from out on: zeros beyond n.  Behind an activation rounded once to T, which as a
// product's operand is all that the matrix instructions take (0.0017 of the norm of a bf16
// gradient, beside as much of its own rounding); without one exact.  What the rounding
// left off goes to `low`, if given.
template <class T, bool ACT>
__device__ __forceinline__ void restore8(const Packed &x, int64_t row, int col, int n, int act, T *out, int left,
                                         T *low = nullptr) {
  u32x2 bits = {0, 0};
  uint32_t byte = 127;
  if (col < n) {
    bits = load8bits(x.q + row * x.ld, col, n);
    byte = x.s[row * x.lds + (col >> 5)];
    place8bits(col, n, bits);
  }
  if constexpr (!ACT && sizeof(T) == 2) {
    if (held_by(T(), byte) && left >= 8) {
      *reinterpret_cast<typename Any8<T>::type *>(out) = from8bits_to<T>(bits, scale_of(byte));
      return;
    }
  }
  float v[8];
  from8bits(bits, scale_of(byte), v);
  if constexpr (ACT) {
    if (!held_by(0.f, byte)) {   // before the activation, which of an infinity may be NaN
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = within<float>(v[j]);
    }
    if (act == DIP_ACT_SILU) {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = act_of(v[j], DIP_ACT_SILU);
    } else if (act == DIP_ACT_GELU) {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = act_of(v[j], DIP_ACT_GELU);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = act_of(v[j], DIP_ACT_RELU);
    }
  }
  if (!held_by(T(), byte)) {   // an activation makes nothing larger
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = within<T>(v[j]);
  }
  put8(out, left, v);   // beyond n act(0) = 0
  if constexpr (ACT) {
    if (low) {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] -= float(T(v[j]));   // exact
      put8(low, left, v);
    }
  }
}
// Packs a quad's 32 columns from `col` % 32 == 8 (lane % 4) on, of which the lane has
// `left`, zeros beyond them; all four lanes are on, one without columns writes nothing.
__device__ __forceinline__ void pack8_quad(const Packed &p, int64_t row, int col, int left, float (&v)[8]) {
  uint32_t most = quad_most(most_of(v));
  if (most >= kInfinity) most = quad_most(finite_most(v));   // the four lanes agree
  if (left <= 0) return;
  const uint32_t byte = scale_byte(most);
  store8bits(p.q + row * p.ld + col, left, round8bits(byte, v));
  if ((col & 31) == 0) p.s[row * p.lds + (col >> 5)] = uint8_t(byte);
}

// ------------------------------------------------------------ dropout

struct Drop {
  uint32_t k0, k1, c2, c3, row0, drop_of;
  float scale;
};

inline Drop make_drop(const dip_dropout &d) {
  return Drop{uint32_t(d.seed), uint32_t(d.seed >> 32), uint32_t(d.offset),
              uint32_t(d.offset >> 32), d.row0, d.drop_of,
              65536.f / float(65536u - d.drop_of)};
}

// The 128 bits of one counter: 16 bits for each of eight consecutive columns.
__device__ __forceinline__ uint4 draws(const Drop &d, uint32_t block, uint32_t row) {
  uint32_t c0 = block, c1 = d.row0 + row, c2 = d.c2, c3 = d.c3, k0 = d.k0, k1 = d.k1;
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t p0 = uint64_t(0xD2511F53u) * c0, p1 = uint64_t(0xCD9E8D57u) * c2;
    c0 = uint32_t(p1 >> 32) ^ c1 ^ k0;
    c1 = uint32_t(p1);
    c2 = uint32_t(p0 >> 32) ^ c3 ^ k1;
    c3 = uint32_t(p0);
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return make_uint4(c0, c1, c2, c3);
}

// Drops columns 8 block .. + 7 of a row and multiplies the kept ones by `scale`.
// Dropped values are set to zero, not multiplied by it, so an infinity or NaN
// under the mask is gone.
__device__ __forceinline__ void drop8(const Drop &d, uint32_t block, uint32_t row, float scale, float (&v)[8]) {
  const uint4 r = draws(d, block, row);
  const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t u = (i & 1) ? w[i / 2] >> 16 : w[i / 2] & 0xffffu;
    v[i] = u >= d.drop_of ? v[i] * scale : 0.f;
  }
}
__device__ __forceinline__ void drop8(const Drop &d, uint32_t block, uint32_t row, float (&v)[8]) {
  drop8(d, block, row, d.scale, v);
}

// ------------------------------------------------------------ epilogues

// What follows a matrix product: out = residual + D(act(acc + bias)), or of a
// gradient, with no bias, activation or mask, scale acc of either type, added to
// or not.
struct Epilogue {
  const void *bias, *residual;
  void *out, *pre;
  int64_t ldr, ldo, ldp;
  Drop drop;
  float scale;   // 1 forward
  int32_t act;
  uint8_t out_f32, accumulate;
};

// Eight consecutive columns of one row; `left`: columns up to the matrix's end.
template <class T>
__device__ __forceinline__ void finish8(const Epilogue &e, int64_t row, int64_t col, int left,
                                        float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] *= e.scale;
  if (e.bias) {
    float b[8];
    load8(static_cast<const T *>(e.bias) + col, left, b);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] += b[i];
  }
  if (e.pre) store8(static_cast<T *>(e.pre) + row * e.ldp + col, left, v);
  if (e.act != DIP_ACT_NONE) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = act_of(v[i], e.act);
  }
  if (e.drop.drop_of) drop8(e.drop, uint32_t(col >> 3), uint32_t(row), v);
  if (e.residual) {
    float r[8];
    load8(static_cast<const T *>(e.residual) + row * e.ldr + col, left, r);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] += r[i];
  }
  if (e.out_f32) {
    float *o = static_cast<float *>(e.out) + row * e.ldo + col;
    if (e.accumulate) {
      float r[8];
      load8(o, left, r);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] += r[i];
    }
    store8(o, left, v);
  } else {
    T *o = static_cast<T *>(e.out) + row * e.ldo + col;
    if (e.accumulate) {
      float r[8];
      load8(o, left, r);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] += r[i];
    }
    store8(o, left, v);
  }
}

}  // namespace dipops
