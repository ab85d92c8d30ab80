// Layer norm over rows of any width, forward and backward.
#include "kernels.h"
#include "timing.h"
#include "triattn.h"

namespace triattn {
namespace {

__device__ inline float wave_sum(float v) {
#pragma unroll
  for (int i = 32; i > 0; i >>= 1) v += __shfl_xor(v, i);
  return v;
}

// One wave per row: mean, then the mean square about it, then the row.
template <typename T>
__global__ __launch_bounds__(256) void ln_fwd_kernel(LnArgs a) {
  const int lane = threadIdx.x & 63;
  const T *gamma = (const T*)a.gamma, *beta = (const T*)a.beta;
  for (int64_t r = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); r < a.m;
       r += (int64_t)gridDim.x * 4) {
    const T* x = (const T*)a.x + r * a.c;
    T* out = (T*)a.out + r * a.c;
    float s = 0.f, q = 0.f;
    for (int i = lane; i < a.c; i += 64) s += (float)x[i];
    const float mean = wave_sum(s) / (float)a.c;
    for (int i = lane; i < a.c; i += 64) {
      const float d = (float)x[i] - mean;
      q += d * d;
    }
    const float rstd = 1.f / sqrtf(wave_sum(q) / (float)a.c + a.eps);
    for (int i = lane; i < a.c; i += 64) {
      float o = ((float)x[i] - mean) * rstd;
      if (gamma) o *= (float)gamma[i];
      if (beta) o += (float)beta[i];
      out[i] = (T)o;
    }
    if (lane == 0) {
      a.mean[r] = mean;
      a.rstd[r] = rstd;
    }
  }
}

template <typename T>
__global__ __launch_bounds__(256) void ln_bwd_dx_kernel(LnBwdArgs a) {
  const int lane = threadIdx.x & 63;
  const T* gamma = (const T*)a.gamma;
  for (int64_t r = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); r < a.m;
       r += (int64_t)gridDim.x * 4) {
    const T* x = (const T*)a.x + r * a.c;
    const T* dy = (const T*)a.dout + r * a.c;
    T* dx = (T*)a.dx + r * a.c;
    const float mean = a.mean[r], rstd = a.rstd[r];
    float s1 = 0.f, s2 = 0.f;
    for (int i = lane; i < a.c; i += 64) {
      const float w = gamma ? (float)dy[i] * (float)gamma[i] : (float)dy[i];
      s1 += w * (((float)x[i] - mean) * rstd);
      s2 += w;
    }
    const float c1 = wave_sum(s1) / (float)a.c, c2 = wave_sum(s2) / (float)a.c;
    for (int i = lane; i < a.c; i += 64) {
      const float w = gamma ? (float)dy[i] * (float)gamma[i] : (float)dy[i];
      dx[i] = (T)(rstd * (w - c1 * (((float)x[i] - mean) * rstd) - c2));
    }
  }
}

// One thread per column and workgroup's stretch of rows.
template <typename T>
__global__ __launch_bounds__(256) void ln_bwd_part_kernel(LnBwdArgs a) {
  const int64_t per = (a.m + a.nwg - 1) / a.nwg;
  const int64_t r0 = blockIdx.x * per, r1 = min(a.m, r0 + per);
  float* part = a.part + (int64_t)blockIdx.x * 2 * a.c;
  for (int i = threadIdx.x; i < a.c; i += 256) {
    float g = 0.f, b = 0.f;
    for (int64_t r = r0; r < r1; ++r) {
      const float dy = (float)((const T*)a.dout)[r * a.c + i];
      g += dy * (((float)((const T*)a.x)[r * a.c + i] - a.mean[r]) * a.rstd[r]);
      b += dy;
    }
    part[i] = g;
    part[a.c + i] = b;
  }
}

__global__ __launch_bounds__(256) void ln_reduce_kernel(const float* part, int nwg, int c,
                                                        float* dgamma, float* dbeta) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i >= 2 * c) return;
  float s = 0.f;
  for (int w = 0; w < nwg; ++w) s += part[(int64_t)w * 2 * c + i];
  float* out = i < c ? dgamma : dbeta;
  if (out) out[i < c ? i : i - c] = s;
}

unsigned grid_rows(int64_t m) { return (unsigned)(m + 3 < 4 * 8192 ? (m + 3) / 4 : 8192); }

template <typename T>
hipError_t fwd(const LnArgs& a, hipStream_t s) {
  KernelTimer t(K_LN_FWD, s);
  hipLaunchKernelGGL(ln_fwd_kernel<T>, dim3(grid_rows(a.m)), dim3(256), 0, s, a);
  return hipGetLastError();
}

template <typename T>
hipError_t bwd(const LnBwdArgs& a, hipStream_t s) {
  if (a.dgamma || a.dbeta) {
    KernelTimer t(K_LN_BWD, s);
    hipLaunchKernelGGL(ln_bwd_part_kernel<T>, dim3(a.nwg), dim3(256), 0, s, a);
  }
  {
    KernelTimer t(K_LN_BWD, s);
    hipLaunchKernelGGL(ln_bwd_dx_kernel<T>, dim3(grid_rows(a.m)), dim3(256), 0, s, a);
  }
  if (a.dgamma || a.dbeta) {
    KernelTimer t(K_LN_REDUCE, s);
    hipLaunchKernelGGL(ln_reduce_kernel, dim3((2 * a.c + 255) / 256), dim3(256), 0, s, a.part,
                       a.nwg, a.c, a.dgamma, a.dbeta);
  }
  return hipGetLastError();
}

}  // namespace

int ln_bwd_parts(int, int64_t m, int) { return (int)(m < 512 ? m : 512); }

hipError_t launch_ln_fwd(int dtype, const LnArgs& a, hipStream_t s) {
  return dtype == TRIATTN_BF16 ? fwd<bf16>(a, s) : fwd<float>(a, s);
}
hipError_t launch_ln_bwd(int dtype, const LnBwdArgs& a, hipStream_t s) {
  return dtype == TRIATTN_BF16 ? bwd<bf16>(a, s) : bwd<float>(a, s);
}

}  // namespace triattn
