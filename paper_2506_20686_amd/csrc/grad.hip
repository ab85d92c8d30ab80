// Norm of many gradients together, and their scaling.  Bound by memory: each is read once for
// the norm; read again (from the last-level cache, as far as it holds them) and written once.
//
// Squares are summed in 64 bits: an fp32 square has 48, so a term is exact, no sum of them
// overflows, and what is lost are terms below 2^-53 of it.  The workgroups' sums are added in a
// fixed order.
// 150,000,001 bf16 elements: 55 us, 5.5 TB/s.  60 tensors, 64,000,000 elements in both types (162
// MB): 31 us for the sum, 53 to scale them.
#include "common.h"
#include "ops.h"
#include "timing.h"
#include "triattn.h"

namespace triattn {
namespace {

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

// Which tensor workgroup wg belongs to.
__device__ inline int tensor_of(const GradArgs& a, int wg) {
  int lo = 0, hi = a.count;
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (a.first[mid] <= wg) lo = mid;
    else hi = mid;
  }
  return lo;
}

__device__ inline void add_square(double& s, float x) {
  const double d = (double)x;
  s = fma(d, d, s);
}

template <typename T>
__device__ inline double squares(const T* p, int64_t n) {
  constexpr int W = 16 / (int)sizeof(T);
  struct E {
    T x[W];
  };
  const int64_t words = n / W;
  double s[4] = {};
  int64_t i = threadIdx.x;
  for (; i + 3 * 256 < words; i += 4 * 256) {
    u32x4 v[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) v[u] = ((const u32x4*)p)[i + 256 * u];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const E e = __builtin_bit_cast(E, v[u]);
#pragma unroll
      for (int k = 0; k < W; ++k) add_square(s[u], (float)e.x[k]);
    }
  }
  for (; i < words; i += 256) {
    const E e = __builtin_bit_cast(E, ((const u32x4*)p)[i]);
#pragma unroll
    for (int k = 0; k < W; ++k) add_square(s[0], (float)e.x[k]);
  }
  if (words * W + threadIdx.x < n) add_square(s[1], (float)p[words * W + threadIdx.x]);
  return (s[0] + s[1]) + (s[2] + s[3]);
}

// Sum over the workgroup, in thread 0.
__device__ inline double group_sum(double s) {
  __shared__ double part[256];
  part[threadIdx.x] = s;
  for (int half = 128; half > 0; half >>= 1) {
    __syncthreads();
    if ((int)threadIdx.x < half) part[threadIdx.x] += part[threadIdx.x + half];
  }
  return part[0];
}

__global__ __launch_bounds__(256) void grad_squares_kernel(GradArgs a) {
  const int wg = blockIdx.x, t = tensor_of(a, wg);
  const int64_t at = (int64_t)(wg - a.first[t]) * a.span;
  const int64_t n = a.size[t] - at < a.span ? a.size[t] - at : a.span;
  double s = a.dtype[t] == TRIATTN_BF16 ? squares((const bf16*)a.src[t] + at, n)
                                        : squares((const float*)a.src[t] + at, n);
  s = group_sum(s);
  if (threadIdx.x == 0) a.part[a.wg0 + wg] = s;
}

__global__ __launch_bounds__(256) void grad_root_kernel(const double* part, int64_t count,
                                                        float* norm) {
  double s = 0.;
#pragma unroll 8
  for (int64_t i = threadIdx.x; i < count; i += 256) s += part[i];
  s = group_sum(s);
  if (threadIdx.x == 0) *norm = (float)sqrt(s);
}

template <typename T, typename F>
__device__ inline u32x4 scaled(u32x4 v, F f) {
  constexpr int W = 16 / (int)sizeof(T);
  struct E {
    T x[W];
  };
  E e = __builtin_bit_cast(E, v);
#pragma unroll
  for (int k = 0; k < W; ++k) e.x[k] = (T)(float)((F)(float)e.x[k] * f);
  return __builtin_bit_cast(u32x4, e);
}
template <typename T, typename F>
__device__ inline void scale(const T* p, T* o, int64_t n, F f) {
  constexpr int W = 16 / (int)sizeof(T);
  const int64_t words = n / W;
  int64_t i = threadIdx.x;
  for (; i + 3 * 256 < words; i += 4 * 256) {
    u32x4 v[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) v[u] = ((const u32x4*)p)[i + 256 * u];
#pragma unroll
    for (int u = 0; u < 4; ++u)
      __builtin_nontemporal_store(scaled<T>(v[u], f), (u32x4*)o + i + 256 * u);
  }
  for (; i < words; i += 256) ((u32x4*)o)[i] = scaled<T>(((const u32x4*)p)[i], f);
  i = words * W + threadIdx.x;
  if (i < n) o[i] = (T)(float)((F)(float)p[i] * f);
}
template <typename F>
__device__ inline void scale_tensor(const GradArgs& a, int t, int64_t at, F f) {
  const int64_t n = a.size[t] - at < a.span ? a.size[t] - at : a.span;
  if (a.dtype[t] == TRIATTN_BF16) scale((const bf16*)a.src[t] + at, (bf16*)a.dst[t] + at, n, f);
  else scale((const float*)a.src[t] + at, (float*)a.dst[t] + at, n, f);
}

__global__ __launch_bounds__(256) void grad_scale_kernel(GradArgs a) {
  const int wg = blockIdx.x, t = tensor_of(a, wg);
  const float norm = *a.norm;
  // a norm that is not finite scales nothing: the caller sees it and drops the step
  const bool finite = (__float_as_uint(norm) & 0x7f800000u) != 0x7f800000u;
  const float f = finite && norm > a.limit ? a.limit / norm : 1.f;
  if (f == 1.f && a.src[t] == a.dst[t]) return;
  const int64_t at = (int64_t)(wg - a.first[t]) * a.span;
  // a factor below fp32's normal numbers has lost bits, though its products need not be small
  if (f >= 0x1p-126f) scale_tensor(a, t, at, f);
  else scale_tensor(a, t, at, (double)a.limit / (double)norm);
}

}  // namespace

hipError_t launch_grad_squares(const GradArgs& a, hipStream_t s) {
  KernelTimer t(K_GRAD_NORM, s);
  hipLaunchKernelGGL(grad_squares_kernel, dim3((unsigned)a.first[a.count]), dim3(256), 0, s, a);
  return hipGetLastError();
}
hipError_t launch_grad_root(const double* part, int64_t count, float* norm, hipStream_t s) {
  KernelTimer t(K_GRAD_NORM, s);
  hipLaunchKernelGGL(grad_root_kernel, dim3(1), dim3(256), 0, s, part, count, norm);
  return hipGetLastError();
}
hipError_t launch_grad_scale(const GradArgs& a, hipStream_t s) {
  KernelTimer t(K_GRAD_CLIP, s);
  hipLaunchKernelGGL(grad_scale_kernel, dim3((unsigned)a.first[a.count]), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace triattn
