// Fixed-order sums of partial results: slabs [count][stride] added up column by column.
#pragma once

#include "common.h"

namespace triattn {

constexpr int SLAB_COLS = 16;  // columns of a workgroup (64-byte pieces of a slab)
constexpr int SLAB_WG = 1024;

// Sum over the slabs of column blockIdx.x * SLAB_COLS + threadIdx.x % SLAB_COLS, valid in
// the first SLAB_COLS threads: 64 threads to a column, each every 64th slab with its
// loads in flight together, then their sums through LDS.
__device__ inline float slab_column_sum(const float* part, int count, int64_t stride, int64_t cols) {
  __shared__ float sum[64][SLAB_COLS + 1];
  const int col = threadIdx.x % SLAB_COLS, k = threadIdx.x / SLAB_COLS;
  const int64_t i = (int64_t)blockIdx.x * SLAB_COLS + col;
  float s = 0.f;
  if (i < cols) {
#pragma unroll 8
    for (int w = k; w < count; w += 64) s += part[w * stride + i];
  }
  sum[k][col] = s;
  for (int half = 32; half > 0; half >>= 1) {
    __syncthreads();
    if (k < half) sum[k][col] += sum[k + half][col];
  }
  return sum[0][col];  // of the thread that summed it last: k = 0
}

inline unsigned slab_grid(int64_t cols) { return (unsigned)((cols + SLAB_COLS - 1) / SLAB_COLS); }

}  // namespace triattn
