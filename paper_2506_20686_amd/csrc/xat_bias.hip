// Cross attention: the pair bias [query][key][head] as planes, one row of keys a (head, query),
// and the planes of its gradient back again.  Bound by memory: both are read and written once.
#include "slabs.h"
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
  const int line = kc + 1;
  for (int i = threadIdx.x; i < keys * a.h; i += 256) {
    const int head = i / keys, key = i % keys, kh = head / a.group;
    const float* src = a.dplanes +
        ((b * a.hk + kh) * rows + (int64_t)qi * a.group + head - kh * a.group) * a.nkp + k0 + key;
    x[head * line + key] = *src;
  }
  __syncthreads();
  T* dst = (T*)a.dbias + (row * a.nk + k0) * a.h;
  for (int i = threadIdx.x; i < keys * a.h; i += 256) dst[i] = (T)x[i % a.h * line + i / a.h];
}

// Sums over the samples of their maps ([batch][stride]): 4 columns a thread, or, of many samples
// and few columns, 16 columns and 64 slices of the samples a workgroup.  To dbias itself, or
// (PLANES) to the first sample's map, each column by the one workgroup that reads it.
template <typename T, bool PLANES>
__global__ __launch_bounds__(256) void xat_sum_kernel(XatArgs a, int64_t cols) {
  const int64_t i = 4 * ((int64_t)blockIdx.x * 256 + threadIdx.x);
  if (i >= cols) return;
  f32x4 s{};
#pragma unroll 4
  for (int64_t b = 0; b < a.batch; ++b) s += *(const f32x4*)(a.dplanes + b * cols + i);
  if (PLANES) *(f32x4*)(a.dplanes + i) = s;
  else store4((T*)a.dbias + i, s);
}
template <typename T, bool PLANES>
__global__ __launch_bounds__(SLAB_WG) void xat_slab_sum_kernel(XatArgs a, int64_t cols) {
  const float s = slab_column_sum(a.dplanes, (int)a.batch, cols, cols);
  const int64_t i = (int64_t)blockIdx.x * SLAB_COLS + threadIdx.x;
  if (threadIdx.x >= SLAB_COLS || i >= cols) return;
  if (PLANES) a.dplanes[i] = s;
  else ((T*)a.dbias)[i] = (T)s;
}
template <typename T, bool PLANES>
void sum_launch(const XatArgs& a, int64_t cols, hipStream_t s) {
  // (the columns, a multiple of 4, make fewer than 2^24 workgroups either way)
  if (a.batch >= 16 && cols < (int64_t)1 << 20)
    hipLaunchKernelGGL((xat_slab_sum_kernel<T, PLANES>), dim3(slab_grid(cols)), dim3(SLAB_WG), 0, s,
                       a, cols);
  else
    hipLaunchKernelGGL((xat_sum_kernel<T, PLANES>), dim3((unsigned)((cols / 4 + 255) / 256)),
                       dim3(256), 0, s, a, cols);
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
    const int64_t cols = (int64_t)a.nq * a.nk * a.h;
    if (dtype == TRIATTN_BF16) sum_launch<bf16, false>(a, cols, s);
    else sum_launch<float, false>(a, cols, s);
    return hipGetLastError();
  }
  if (a.bias_batch < a.batch) sum_launch<float, true>(a, (int64_t)a.h * a.nq * a.nkp, s);
  int chunks;
  const dim3 grid((unsigned)groups(a, chunks)), wg(256);
  if (dtype == TRIATTN_BF16) hipLaunchKernelGGL(xat_dbias_kernel<bf16>, grid, wg, 0, s, a, chunks);
  else hipLaunchKernelGGL(xat_dbias_kernel<float>, grid, wg, 0, s, a, chunks);
  return hipGetLastError();
}

}  // namespace triattn
