// kern_pack8.hip -- activations kept in 8 bits, and restored.
//
// A value is q 2^e with q of four significant bits and one e for 32 columns: the
// conversion instructions take such a scale, a kept value is exact in bfloat16, and a
// group's largest value costs the others bits only where they are below a 2^-14th of it
// (it divides to between 224 and 448, and steps stop shrinking at 2^-6: from 2^-13.8 to
// 2^-14.8 of it).  Bound by memory: read once, written once.  A thread has one vector of
// eight columns, and nothing waits but for its own load: two a thread, sixteen columns
// a thread and non-temporal accesses were 2 to 5 % slower (235 million bf16: 116 us,
// 6.1 TB/s, either way; 119, 121 with two and four vectors, 123 with sixteen columns).
// That leaves some 60 instructions a vector before they are what bounds it: hence
// magnitudes compared as integers two at a time, and whole vectors at the ends of rows
// (65,536 x 2560 fp16 packed 87 to 99 us, restored 83 to 86, through GELU 99; float32 144,
// 145 and 158, 5.8 TB/s without an activation;
// 2^26 bf16 in rows of 100 44 and 44, where elements one by one at the end took 61 and 75).
#include <algorithm>

#include "ops_internal.h"

namespace dipops {
namespace {

constexpr int kThreads = 256;

// Eight columns of a row a thread, four threads a scale; `per` is a multiple of four,
// so that those are of one wave and all there.
template <class T>
__global__ __launch_bounds__(kThreads) void pack8_kernel(uint32_t items, uint32_t row0, Divide per, int n,
                                                         const T *x, int64_t ldx, Packed out) {
  const uint32_t i = blockIdx.x * kThreads + threadIdx.x;
  if (i >= items) return;
  const uint32_t in = per(i);
  const int64_t row = int64_t(row0) + in;
  const int col = int(i - in * per.by) * 8, left = min(8, n - col), by = Held<T>::moved(col, n);
  Held<T> h;
  h.get(x + row * ldx, col, n);
  if constexpr (sizeof(T) == 2) {
    // magnitudes compared and rounded two at a time, as they lie in memory
    typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    typedef T T2 __attribute__((ext_vector_type(2)));
    const u32x4 words = h.words(by), w = words & 0x7fff7fffu;
    const auto t = __builtin_bit_cast(typename Vec8<T>::type, words);
    auto two = [&](int j) { return __builtin_bit_cast(u16x2, uint32_t(w[j])); };
    const u16x2 m = __builtin_elementwise_max(__builtin_elementwise_max(two(0), two(1)),
                                              __builtin_elementwise_max(two(2), two(3)));
    const uint32_t most = quad_most(max(uint32_t(m[0]), uint32_t(m[1])));
    if (most < (__is_same(T, _Float16) ? 0x7c00u : 0x7f80u)) {   // the four lanes agree
      if (left <= 0) return;
      const uint32_t byte = scale_byte(magnitude(float(__builtin_bit_cast(T, uint16_t(most)))));
      const float scale = scale_of(byte);
      u32x2 r;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const T2 a = {t[4 * j], t[4 * j + 1]}, b = {t[4 * j + 2], t[4 * j + 3]};
        s16x2 q = {0, 0};
        if constexpr (__is_same(T, _Float16)) {
          q = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(q, a, scale, false);
          q = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(q, b, scale, true);
        } else {
          q = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(q, a, scale, false);
          q = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(q, b, scale, true);
        }
        r[j] = __builtin_bit_cast(uint32_t, q);
      }
      store8bits(out.q + row * out.ld + col, left, r);
      if ((col & 31) == 0) out.s[row * out.lds + (col >> 5)] = uint8_t(byte);
      return;
    }
  }
  float v[8];
  h.to(by, v);
  pack8_quad(out, row, col, left, v);
}

template <class T, bool ACT>
__global__ __launch_bounds__(kThreads) void unpack8_kernel(uint32_t items, uint32_t row0, Divide per, int n,
                                                           Packed x, int act, T *y, int64_t ldy, int fill, T *low) {
  const uint32_t i = blockIdx.x * kThreads + threadIdx.x;
  if (i >= items) return;
  const uint32_t in = per(i);
  const int64_t row = int64_t(row0) + in;
  const int col = int(i - in * per.by) * 8;
  const int64_t at = row * ldy + col;
  restore8<T, ACT>(x, row, col, n, act, y + at, min(8, fill - col), low ? low + at : nullptr);
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
    pack8_kernel<T><<<grid, dim3(kThreads), 0, st>>>(items, row0, per, int(n), static_cast<const T *>(x), ldx, out);
  });
}
template <class T>
hipError_t unpack(int64_t m, int64_t n, const Packed &x, int act, void *y, int64_t ldy, int64_t fill, hipStream_t st, void *low) {
  return pieces(m, (fill + 7) / 8, [&](dim3 grid, uint32_t items, uint32_t row0, const Divide &per) {
    auto go = [&](auto kernel) {
      kernel<<<grid, dim3(kThreads), 0, st>>>(items, row0, per, int(n), x, act, static_cast<T *>(y), ldy, int(fill),
                                              static_cast<T *>(low));
    };
    act != DIP_ACT_NONE ? go(unpack8_kernel<T, true>) : go(unpack8_kernel<T, false>);
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
                          hipStream_t stream, void *low) {
  switch (dtype) {
    case DIP_F32: return unpack<float>(m, n, x, act, y, ldy, fill, stream, low);
    case DIP_F16: return unpack<_Float16>(m, n, x, act, y, ldy, fill, stream, low);
    default: return unpack<__bf16>(m, n, x, act, y, ldy, fill, stream, low);
  }
}

}  // namespace dipops
