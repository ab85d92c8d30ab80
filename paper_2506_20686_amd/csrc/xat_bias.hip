// Cross attention: the pair bias [query][key][head] as planes, one row of keys a (head, query),
// and the planes of its gradient back again.  Bound by memory: both are read and written once.
#include "timing.h"
#include "triattn.h"
#include "xat.h"

namespace triattn {
namespace {

// Keys of a workgroup: 4096 elements of all heads.
__host__ __device__ inline int plane_keys(int h) { return h <= 16 ? 256 : h <= 64 ? 64 : 16; }

template <typename T>
__global__ __launch_bounds__(256) void xat_planes_kernel(XatArgs a, int chunks) {
  __shared__ T x[4096 + 256];
  const int kc = plane_keys(a.h), k0 = (int)(blockIdx.x % chunks) * kc;
  const int64_t row = blockIdx.x / chunks;  // sample, query
  const int64_t b = row / a.nq;
  const int qi = (int)(row % a.nq), keys = a.nk - k0 < kc ? a.nk - k0 : kc, rows = a.nq * a.group;
  const T* src = (const T*)a.bias + (row * a.nk + k0) * a.h;
  // a line of keys of each head, one element apart from the banks of the next
  const int line = kc + 1;
  for (int i = threadIdx.x; i < keys * a.h; i += 256) x[i % a.h * line + i / a.h] = src[i];
  __syncthreads();
  const int width = a.nkp - k0 < kc ? a.nkp - k0 : kc;
  for (int i = threadIdx.x; i < width * a.h; i += 256) {
    const int head = i / width, key = i % width, kh = head / a.group;
    T* dst = (T*)a.planes +
             ((b * a.hk + kh) * rows + (int64_t)qi * a.group + head - kh * a.group) * a.nkp + k0;
    dst[key] = key < keys ? x[head * line + key] : (T)0.f;
  }
}

template <typename T>
__global__ __launch_bounds__(256) void xat_dbias_kernel(XatArgs a, int chunks) {
  __shared__ float x[4096 + 256];
  const int kc = plane_keys(a.h), k0 = (int)(blockIdx.x % chunks) * kc;
  const int64_t row = blockIdx.x / chunks;
  const int64_t b = row / a.nq;
  const int qi = (int)(row % a.nq), keys = a.nk - k0 < kc ? a.nk - k0 : kc, rows = a.nq * a.group;
  const int line = kc + 1, samples = a.bias_batch == 1 ? (int)a.batch : 1;
  for (int i = threadIdx.x; i < keys * a.h; i += 256) {
    const int head = i / keys, key = i % keys, kh = head / a.group;
    const float* src = a.dplanes +
        ((b * a.hk + kh) * rows + (int64_t)qi * a.group + head - kh * a.group) * a.nkp + k0 + key;
    float s = 0.f;
    for (int n = 0; n < samples; ++n) s += src[(int64_t)n * a.hk * rows * a.nkp];
    x[head * line + key] = s;
  }
  __syncthreads();
  T* dst = (T*)a.dbias + (row * a.nk + k0) * a.h;
  for (int i = threadIdx.x; i < keys * a.h; i += 256) dst[i] = (T)x[i % a.h * line + i / a.h];
}

// Sum over the samples of maps of dbias's layout, 4 elements a thread (their number is a
// multiple of 4).
template <typename T>
__global__ __launch_bounds__(256) void xat_dbias_sum_kernel(XatArgs a) {
  const int64_t all = (int64_t)a.nq * a.nk * a.h;
  const int64_t i = 4 * ((int64_t)blockIdx.x * 256 + threadIdx.x);
  if (i >= all) return;
  f32x4 s{};
#pragma unroll 4
  for (int64_t b = 0; b < a.batch; ++b) s += *(const f32x4*)(a.dplanes + b * all + i);
  store4((T*)a.dbias + i, s);
}

int64_t groups(const XatArgs& a, int& chunks) {
  const int kc = plane_keys(a.h);
  chunks = (a.nkp + kc - 1) / kc;
  return a.bias_batch * a.nq * chunks;
}

}  // namespace

hipError_t launch_xat_planes(int dtype, const XatArgs& a, hipStream_t s) {
  KernelTimer t(K_XAT_PLANES, s);
  int chunks;
  const dim3 grid((unsigned)groups(a, chunks)), wg(256);
  if (dtype == TRIATTN_BF16) hipLaunchKernelGGL(xat_planes_kernel<bf16>, grid, wg, 0, s, a, chunks);
  else hipLaunchKernelGGL(xat_planes_kernel<float>, grid, wg, 0, s, a, chunks);
  return hipGetLastError();
}

hipError_t launch_xat_dbias(int dtype, const XatArgs& a, bool heads, hipStream_t s) {
  KernelTimer t(K_XAT_DBIAS, s);
  if (heads) {
    const dim3 grid((unsigned)(((int64_t)a.nq * a.nk * a.h / 4 + 255) / 256)), wg(256);
    if (dtype == TRIATTN_BF16) hipLaunchKernelGGL(xat_dbias_sum_kernel<bf16>, grid, wg, 0, s, a);
    else hipLaunchKernelGGL(xat_dbias_sum_kernel<float>, grid, wg, 0, s, a);
    return hipGetLastError();
  }
  int chunks;
  const dim3 grid((unsigned)groups(a, chunks)), wg(256);
  if (dtype == TRIATTN_BF16) hipLaunchKernelGGL(xat_dbias_kernel<bf16>, grid, wg, 0, s, a, chunks);
  else hipLaunchKernelGGL(xat_dbias_kernel<float>, grid, wg, 0, s, a, chunks);
  return hipGetLastError();
}

}  // namespace triattn
