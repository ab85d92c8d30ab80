// Learned relative position bias by buckets, and the gradient of its table.
#include "kernels.h"
#include "timing.h"
#include "triattn.h"

namespace triattn {
namespace {

// Number of edges at or below d (edges ascending, in LDS).
__device__ inline int bucket_of(const int32_t* edges, int ne, int64_t d) {
  int lo = 0, hi = ne;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (edges[mid] <= d) lo = mid + 1;
    else hi = mid;
  }
  return lo;
}

__device__ inline int pair_bucket(const RelArgs& a, const int32_t* edges, int64_t q, int64_t k) {
  if (a.chain && a.chain[q] != a.chain[k]) return a.ne + 1;
  return bucket_of(edges, a.ne, (int64_t)a.pos[q] - (int64_t)a.pos[k]);
}

template <typename T>
__global__ __launch_bounds__(256) void rel_fwd_kernel(RelArgs a) {
  __shared__ int32_t edges[REL_MAX_EDGES + 1];
  if ((int)threadIdx.x < a.ne) edges[threadIdx.x] = a.edges[threadIdx.x];
  __syncthreads();
  const int64_t total = a.batch * a.n * a.n * a.h;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total;
       i += (int64_t)gridDim.x * 256) {
    const int64_t pair = i / a.h, row = pair / a.n, b = row / a.n;
    const int c = (int)(i - pair * a.h);
    const int r = pair_bucket(a, edges, row, b * a.n + (pair - row * a.n));
    float o = (float)((const T*)a.table)[r * a.h + c];
    if (a.base) o += (float)((const T*)a.base)[i];
    ((T*)a.out)[i] = (T)o;
  }
}

// Workgroup (stretch of query rows, 64 channels): one thread per channel adds its pairs
// into its own column of the LDS sums.
template <typename T>
__global__ __launch_bounds__(64) void rel_bwd_kernel(RelArgs a) {
  __shared__ int32_t edges[REL_MAX_EDGES + 1];
  __shared__ float sum[REL_MAX_EDGES + 2][64];
  for (int i = threadIdx.x; i < a.ne; i += 64) edges[i] = a.edges[i];
  for (int r = 0; r < a.rows; ++r) sum[r][threadIdx.x] = 0.f;
  __syncthreads();
  const int c = blockIdx.y * 64 + threadIdx.x;
  if (c >= a.h) return;
  const int64_t nrow = a.batch * a.n, per = (nrow + a.nwg - 1) / a.nwg;
  const int64_t r0 = blockIdx.x * per, r1 = min(nrow, r0 + per);
  for (int64_t row = r0; row < r1; ++row) {
    const int64_t b = row / a.n;
    for (int k = 0; k < a.n; ++k)
      sum[pair_bucket(a, edges, row, b * a.n + k)][threadIdx.x] +=
          (float)((const T*)a.dout)[(row * a.n + k) * a.h + c];
  }
  for (int r = 0; r < a.rows; ++r)
    a.part[((int64_t)blockIdx.x * a.rows + r) * a.h + c] = sum[r][threadIdx.x];
}

__global__ __launch_bounds__(256) void rel_reduce_kernel(const float* part, int nwg, int total,
                                                         float* dtable) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i >= total) return;
  float s = 0.f;
  for (int w = 0; w < nwg; ++w) s += part[(int64_t)w * total + i];
  dtable[i] = s;
}

}  // namespace

int rel_bwd_parts(int, int64_t batch, int64_t n, int) {
  return (int)(batch * n < 512 ? batch * n : 512);
}

hipError_t launch_rel_fwd(int dtype, const RelArgs& a, hipStream_t s) {
  KernelTimer t(K_REL_FWD, s);
  const int64_t wgs = (a.batch * a.n * a.n * a.h + 255) / 256;
  const dim3 grid((unsigned)(wgs < 16384 ? wgs : 16384));
  if (dtype == TRIATTN_BF16)
    hipLaunchKernelGGL(rel_fwd_kernel<bf16>, grid, dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL(rel_fwd_kernel<float>, grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_rel_bwd(int dtype, const RelArgs& a, hipStream_t s) {
  {
    KernelTimer t(K_REL_BWD, s);
    const dim3 grid(a.nwg, (a.h + 63) / 64);
    if (dtype == TRIATTN_BF16)
      hipLaunchKernelGGL(rel_bwd_kernel<bf16>, grid, dim3(64), 0, s, a);
    else
      hipLaunchKernelGGL(rel_bwd_kernel<float>, grid, dim3(64), 0, s, a);
  }
  KernelTimer t(K_REL_REDUCE, s);
  const int total = a.rows * a.h;
  hipLaunchKernelGGL(rel_reduce_kernel, dim3((total + 255) / 256), dim3(256), 0, s, a.part, a.nwg,
                     total, a.dtable);
  return hipGetLastError();
}

}  // namespace triattn
