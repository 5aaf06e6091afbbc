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
