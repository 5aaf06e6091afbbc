// kern_groupnorm.hip -- group norm with an activation over channels-last arrays.
#include "ops_internal.h"

namespace dipops {
namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ float block_sum(float v, float *s) {
  for (int d = 1; d < 64; d *= 2) v += __shfl_xor(v, d);
  __syncthreads();
  if (threadIdx.x % 64 == 0) s[threadIdx.x / 64] = v;
  __syncthreads();
  return (s[0] + s[1]) + (s[2] + s[3]);
}

// One block a sample and group; statistics in two passes over the data.
template <class T>
__global__ __launch_bounds__(kThreads) void norm_kernel(dip_group_norm_args a) {
  __shared__ float s[4];
  const int64_t i = blockIdx.x / a.groups;
  const int g = int(blockIdx.x % a.groups), per = int(a.c / a.groups);
  const int64_t count = a.s * per;
  const T *x = static_cast<const T *>(a.x) + i * a.x_sb + int64_t(g) * per;
  T *y = static_cast<T *>(a.y) + i * a.y_sb + int64_t(g) * per;
  const T *gamma = static_cast<const T *>(a.gamma), *beta = static_cast<const T *>(a.beta);
  float v = 0.f;
  for (int64_t j = threadIdx.x; j < count; j += kThreads) v += float(x[j / per * a.x_ss + j % per]);
  const float mean = block_sum(v, s) / float(max(count, int64_t(1)));
  v = 0.f;
  for (int64_t j = threadIdx.x; j < count; j += kThreads) {
    const float d = float(x[j / per * a.x_ss + j % per]) - mean;
    v += d * d;
  }
  const float rstd = 1.f / sqrtf(block_sum(v, s) / float(max(count, int64_t(1))) + a.eps);
  if (threadIdx.x == 0) {
    if (a.mean) a.mean[blockIdx.x] = mean;
    if (a.rstd) a.rstd[blockIdx.x] = rstd;
  }
  for (int64_t j = threadIdx.x; j < count; j += kThreads) {
    const int c = int(j % per);
    float z = (float(x[j / per * a.x_ss + c]) - mean) * rstd;
    z = z * (gamma ? float(gamma[g * per + c]) : 1.f) + (beta ? float(beta[g * per + c]) : 0.f);
    y[j / per * a.y_ss + c] = T(act_of(z, a.act));
  }
}

// One block a sample and group; its channels' sums over positions go to
// partial[2][b][c] (dgamma's first).
template <class T>
__global__ __launch_bounds__(kThreads) void norm_grad_kernel(dip_group_norm_grad_args a) {
  __shared__ float s[4];
  const int64_t i = blockIdx.x / a.groups;
  const int g = int(blockIdx.x % a.groups), per = int(a.c / a.groups);
  const int64_t count = a.s * per;
  const T *x = static_cast<const T *>(a.x) + i * a.x_sb + int64_t(g) * per;
  const T *dy = static_cast<const T *>(a.dy) + i * a.dy_sb + int64_t(g) * per;
  const T *gamma = static_cast<const T *>(a.gamma), *beta = static_cast<const T *>(a.beta);
  const float mean = a.mean[blockIdx.x], rstd = a.rstd[blockIdx.x];
  float *pg = static_cast<float *>(a.workspace) + i * a.c + int64_t(g) * per;
  float *pb = pg + a.b * a.c;
  auto grad = [&](int64_t p, int c, float &xh) {
    xh = (float(x[p * a.x_ss + c]) - mean) * rstd;
    const float z = xh * (gamma ? float(gamma[g * per + c]) : 1.f) + (beta ? float(beta[g * per + c]) : 0.f);
    return float(dy[p * a.dy_ss + c]) * act_slope(z, a.act);
  };
  float h_sum = 0.f, hx_sum = 0.f;
  for (int c = 0; c < per; ++c) {
    float sg = 0.f, sb = 0.f;
    for (int64_t p = threadIdx.x; p < a.s; p += kThreads) {
      float xh;
      const float v = grad(p, c, xh);
      sg += v * xh;
      sb += v;
    }
    sg = block_sum(sg, s);
    sb = block_sum(sb, s);
    if (threadIdx.x == 0) {
      pg[c] = sg;
      pb[c] = sb;
    }
    const float w = gamma ? float(gamma[g * per + c]) : 1.f;
    h_sum += sb * w;
    hx_sum += sg * w;
  }
  if (!a.dx) return;
  const float h_mean = h_sum / float(count), hx_mean = hx_sum / float(count);
  T *dx = static_cast<T *>(a.dx) + i * a.dx_sb + int64_t(g) * per;
  for (int64_t j = threadIdx.x; j < count; j += kThreads) {
    const int c = int(j % per);
    float xh;
    const float h = grad(j / per, c, xh) * (gamma ? float(gamma[g * per + c]) : 1.f);
    dx[j / per * a.dx_ss + c] = T(rstd * (h - h_mean - xh * hx_mean));
  }
}

template <class T>
hipError_t norm(const dip_group_norm_args &a, hipStream_t st) {
  norm_kernel<T><<<dim3(uint32_t(a.b * a.groups)), dim3(kThreads), 0, st>>>(a);
  return hipGetLastError();
}
template <class T>
hipError_t norm_grad(const dip_group_norm_grad_args &a, hipStream_t st) {
  norm_grad_kernel<T><<<dim3(uint32_t(a.b * a.groups)), dim3(kThreads), 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace

int64_t group_norm_workspace(const dip_group_norm_args &) { return 0; }
int64_t group_norm_grad_workspace(const dip_group_norm_grad_args &a) { return up16(2 * a.b * a.c * 4); }

hipError_t launch_group_norm(const dip_group_norm_args &a, hipStream_t st) {
  return a.dtype == DIP_F32 ? norm<float>(a, st) : a.dtype == DIP_F16 ? norm<_Float16>(a, st) : norm<__bf16>(a, st);
}

hipError_t launch_group_norm_grad(const dip_group_norm_grad_args &a, hipStream_t st) {
  if (a.b > 0 && a.s > 0) {
    const hipError_t e = a.dtype == DIP_F32   ? norm_grad<float>(a, st)
                         : a.dtype == DIP_F16 ? norm_grad<_Float16>(a, st)
                                              : norm_grad<__bf16>(a, st);
    if (e != hipSuccess) return e;
  }
  const float *p = static_cast<const float *>(a.workspace);
  const int64_t rows = a.s > 0 ? a.b : 0;
  for (int j = 0; j < 2; ++j) {
    void *out = j ? a.dbeta : a.dgamma;
    if (!out) continue;
    const hipError_t e = launch_sum_rows(p + j * a.b * a.c, rows, a.c, out, a.dtype, 0, st);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace dipops
