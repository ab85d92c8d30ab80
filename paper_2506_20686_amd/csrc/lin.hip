// Linear projection with bias, activation and residual, and its backward.
#include "kernels.h"
#include "timing.h"
#include "triattn.h"

namespace triattn {
namespace {

__device__ inline float act_value(float z, int act) {
  if (act == TRIATTN_ACT_RELU) return z > 0.f ? z : 0.f;
  if (act == TRIATTN_ACT_GELU) return 0.5f * z * (1.f + erff(z * 0.70710678118654752f));
  if (act == TRIATTN_ACT_SILU) return z / (1.f + expf(-z));
  return z;
}

__device__ inline float act_grad(float z, int act) {
  if (act == TRIATTN_ACT_RELU) return z > 0.f ? 1.f : 0.f;
  if (act == TRIATTN_ACT_GELU)
    return 0.5f * (1.f + erff(z * 0.70710678118654752f)) +
           z * 0.39894228040143268f * expf(-0.5f * z * z);
  if (act == TRIATTN_ACT_SILU) {
    const float s = 1.f / (1.f + expf(-z));
    return s * (1.f + z * (1.f - s));
  }
  return 1.f;
}

// A 16 x 16 output tile per workgroup: C[i][j] = sum over t of A(i, t) B(t, j), the
// operands staged through LDS in fp32.
template <typename FA, typename FB>
__device__ inline float tile_product(int64_t t0, int64_t t1, FA fa, FB fb) {
  __shared__ float sa[16][17], sb[16][17];
  const int ti = threadIdx.x >> 4, tj = threadIdx.x & 15;
  float acc = 0.f;
  for (int64_t t = t0; t < t1; t += 16) {
    sa[ti][tj] = t + tj < t1 ? fa(ti, t + tj) : 0.f;
    sb[ti][tj] = t + ti < t1 ? fb(t + ti, tj) : 0.f;
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 16; ++e) acc += sa[ti][e] * sb[e][tj];
    __syncthreads();
  }
  return acc;
}

template <typename T>
__global__ __launch_bounds__(256) void lin_fwd_kernel(LinArgs a) {
  const int64_t i0 = (int64_t)blockIdx.x * 16;
  const int j0 = blockIdx.y * 16;
  const T *x = (const T*)a.x, *w = (const T*)a.w;
  float z = tile_product(
      0, a.k, [&](int i, int64_t t) { return i0 + i < a.m ? (float)x[(i0 + i) * a.k + t] : 0.f; },
      [&](int64_t t, int j) { return j0 + j < a.n ? (float)w[t * a.n + j0 + j] : 0.f; });
  const int64_t i = i0 + (threadIdx.x >> 4);
  const int j = j0 + (threadIdx.x & 15);
  if (i >= a.m || j >= a.n) return;
  if (a.bias) z += (float)((const T*)a.bias)[j];
  float o = act_value(z, a.act);
  if (a.residual) o += (float)((const T*)a.residual)[i * a.n + j];
  ((T*)a.out)[i * a.n + j] = (T)o;
  if (a.z) ((T*)a.z)[i * a.n + j] = (T)z;
}

template <typename T>
__device__ inline float dz_at(const LinBwdArgs& a, int64_t i, int j) {
  const float dy = (float)((const T*)a.dout)[i * a.n + j];
  return a.act == TRIATTN_ACT_NONE ? dy
                                   : dy * act_grad((float)((const T*)a.z)[i * a.n + j], a.act);
}

template <typename T>
__global__ __launch_bounds__(256) void lin_bwd_dx_kernel(LinBwdArgs a) {
  const int64_t i0 = (int64_t)blockIdx.x * 16;
  const int j0 = blockIdx.y * 16;
  const T* w = (const T*)a.w;
  const float d = tile_product(
      0, a.n, [&](int i, int64_t t) { return i0 + i < a.m ? dz_at<T>(a, i0 + i, (int)t) : 0.f; },
      [&](int64_t t, int j) { return j0 + j < a.k ? (float)w[(int64_t)(j0 + j) * a.n + t] : 0.f; });
  const int64_t i = i0 + (threadIdx.x >> 4);
  const int j = j0 + (threadIdx.x & 15);
  if (i < a.m && j < a.k) ((T*)a.dx)[i * a.k + j] = (T)d;
}

// Workgroup (i tile, j tile, split): one split's rows of dw and, in the i tile past the
// last one, of dbias (x taken as ones).
template <typename T>
__global__ __launch_bounds__(256) void lin_bwd_w_kernel(LinBwdArgs a) {
  const int64_t per = (a.m + a.splits - 1) / a.splits;
  const int64_t r0 = blockIdx.z * per, r1 = min(a.m, r0 + per);
  const int i0 = blockIdx.x * 16, j0 = blockIdx.y * 16;
  const bool ones = i0 >= a.k;
  const T* x = (const T*)a.x;
  const float d = tile_product(
      r0, r1,
      [&](int i, int64_t t) {
        return ones ? 1.f : (i0 + i < a.k ? (float)x[t * a.k + i0 + i] : 0.f);
      },
      [&](int64_t t, int j) { return j0 + j < a.n ? dz_at<T>(a, t, j0 + j) : 0.f; });
  const int i = i0 + (threadIdx.x >> 4);
  const int j = j0 + (threadIdx.x & 15);
  float* part = a.part + (int64_t)blockIdx.z * ((int64_t)a.k * a.n + a.n);
  if (j >= a.n) return;
  if (ones) {
    if ((threadIdx.x >> 4) == 0) part[(int64_t)a.k * a.n + j] = d;
  } else if (i < a.k) {
    part[(int64_t)i * a.n + j] = d;
  }
}

__global__ __launch_bounds__(256) void lin_reduce_kernel(LinBwdArgs a) {
  const int64_t kn = (int64_t)a.k * a.n, i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= kn + a.n) return;
  float s = 0.f;
  for (int w = 0; w < a.splits; ++w) s += a.part[w * (kn + a.n) + i];
  if (i < kn) {
    if (a.dw) a.dw[i] = s;
  } else if (a.dbias) {
    a.dbias[i - kn] = s;
  }
}

template <typename T>
hipError_t fwd(const LinArgs& a, hipStream_t s) {
  KernelTimer t(K_LIN_FWD, s);
  hipLaunchKernelGGL(lin_fwd_kernel<T>, dim3((unsigned)((a.m + 15) / 16), (a.n + 15) / 16),
                     dim3(256), 0, s, a);
  return hipGetLastError();
}

template <typename T>
hipError_t bwd(const LinBwdArgs& a, hipStream_t s) {
  if (a.dx) {
    KernelTimer t(K_LIN_BWD_DX, s);
    hipLaunchKernelGGL(lin_bwd_dx_kernel<T>, dim3((unsigned)((a.m + 15) / 16), (a.k + 15) / 16),
                       dim3(256), 0, s, a);
  }
  if (a.dw || a.dbias) {
    {
      KernelTimer t(K_LIN_BWD_W, s);
      hipLaunchKernelGGL(lin_bwd_w_kernel<T>,
                         dim3((a.k + 15) / 16 + 1, (a.n + 15) / 16, a.splits), dim3(256), 0, s, a);
    }
    KernelTimer t(K_LIN_REDUCE, s);
    hipLaunchKernelGGL(lin_reduce_kernel,
                       dim3((unsigned)(((int64_t)a.k * a.n + a.n + 255) / 256)), dim3(256), 0, s,
                       a);
  }
  return hipGetLastError();
}

}  // namespace

int lin_bwd_splits(int, int64_t m, int, int) { return (int)((m + 511) / 512 < 128 ? (m + 511) / 512 : 128); }

hipError_t launch_lin_fwd(int dtype, const LinArgs& a, hipStream_t s) {
  return dtype == TRIATTN_BF16 ? fwd<bf16>(a, s) : fwd<float>(a, s);
}
hipError_t launch_lin_bwd(int dtype, const LinBwdArgs& a, hipStream_t s) {
  return dtype == TRIATTN_BF16 ? bwd<bf16>(a, s) : bwd<float>(a, s);
}

}  // namespace triattn
