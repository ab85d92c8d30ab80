// Layer norm over rows of any width, forward and backward.
//
// Both passes are bound by memory: 2 (forward) and 3 (backward) values moved per element
// for some ten operations on it.  So every value is read once and kept in registers: a
// row belongs to L lanes of V chunks of 16 bytes each (chunk v of lane l is the row's
// chunk v L + l), and the row sums meet over those lanes only.  L = 1, 4, 16 or 64 lanes
// of one wave, or a workgroup of 256 (see dispatch()), so that narrow rows leave few
// lanes idle and wide ones fit the registers.
//
// Rows of a width that is no whole number of chunks start at any element; a 16-byte
// access may start at any byte on this machine, so only the row's last, partial chunk
// goes element by element.
//
// The variance is the mean square of the deviations from the mean (the row is at hand),
// not a difference of squares, which would lose what a row far from zero has of it.
#include "ops.h"
#include "slabs.h"
#include "timing.h"
#include "triattn.h"

namespace triattn {
namespace {

constexpr int LN_WG = 256;

template <typename T>
struct Chunk {
  static constexpr int N = 16 / (int)sizeof(T);
  T x[N];
};
struct __attribute__((packed)) Raw16 {
  unsigned v[4];
};

// Chunk `at` of a row of c elements: all of it, its first elements with zeros after them,
// or zeros where it lies past the row.
template <typename T>
__device__ inline Chunk<T> load_chunk(const T* row, int at, int c) {
  constexpr int N = Chunk<T>::N;
  Chunk<T> r;
  const int e0 = at * N;
  if (e0 + N <= c) {
    r = __builtin_bit_cast(Chunk<T>, *(const Raw16*)(row + e0));
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e) r.x[e] = e0 + e < c ? row[e0 + e] : (T)0.f;
  }
  return r;
}
template <typename T>
__device__ inline void store_chunk(T* row, int at, int c, const Chunk<T>& r) {
  constexpr int N = Chunk<T>::N;
  const int e0 = at * N;
  if (e0 + N <= c) {
    *(Raw16*)(row + e0) = __builtin_bit_cast(Raw16, r);
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (e0 + e < c) row[e0 + e] = r.x[e];
  }
}

template <int CTRL>
__device__ inline float dpp_add(float v) {
  const int o = __builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true);
  return v + __int_as_float(o);
}
// Adds the lanes l ^ 16.
__device__ inline float xor16_sum(float v) {
  const auto r =
      __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Sum over each aligned group of L lanes, the same bits in all of them: pairs, quads,
// then halves of eight and sixteen mirrored onto each other (whose lanes already agree).
template <int L>
__device__ inline float group_sum(float v) {
  if (L >= 4) {
    v = dpp_add<0xB1>(v);   // quad_perm 1 0 3 2
    v = dpp_add<0x4E>(v);   // quad_perm 2 3 0 1
  }
  if (L >= 16) {
    v = dpp_add<0x141>(v);  // row_half_mirror
    v = dpp_add<0x140>(v);  // row_mirror
  }
  if (L >= 64) {
    v = xor16_sum(v);
    v = wave_xor32_sum(v);
  }
  return v;
}

// The row's sum for a workgroup that shares it: the waves' sums through LDS.  `turn`
// alternates between two slots, so one barrier per sum is enough: a wave writes a slot
// again only after the barrier of the other one, which every wave reaches after reading.
__device__ inline float wg_sum(float v, float (*slot)[4], int& turn) {
  v = group_sum<64>(v);
  if ((threadIdx.x & 63) == 0) slot[turn][threadIdx.x >> 6] = v;
  __syncthreads();
  const float s = (slot[turn][0] + slot[turn][1]) + (slot[turn][2] + slot[turn][3]);
  turn ^= 1;
  return s;
}
template <int L>
__device__ inline float row_sum(float v, float (*slot)[4], int& turn) {
  return L == LN_WG ? wg_sum(v, slot, turn) : group_sum<L>(v);
}

// Forward.  589,824 x 128 bf16: 55 us, 5.5 TB/s of x and out (a large copy reaches 5.1); 65,536 x
// 1024: 46, 5.9 TB/s; 9001 x 833 bf16, rows at any element: 14 us.  A chunk's load lies in the
// branch of whole chunks, behind which the compiler waits for it, so with few rows a wave the
// chunks' latencies (of gamma, beta and x) add up.
template <typename T, int L, int V>
__global__ __launch_bounds__(LN_WG) void ln_fwd_kernel(LnArgs a) {
  constexpr int N = Chunk<T>::N, G = LN_WG / L;
  __shared__ float slot[2][4];
  int turn = 0;
  const int lane = threadIdx.x % L, group = threadIdx.x / L;
  const float inv = 1.f / (float)a.c;
  Chunk<T> gamma[V], beta[V];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    if (a.gamma) gamma[v] = load_chunk((const T*)a.gamma, v * L + lane, a.c);
    if (a.beta) beta[v] = load_chunk((const T*)a.beta, v * L + lane, a.c);
  }
  for (int64_t r = (int64_t)blockIdx.x * G + group; r < a.m; r += (int64_t)gridDim.x * G) {
    const T* row = (const T*)a.x + r * a.c;
    Chunk<T> x[V];
#pragma unroll
    for (int v = 0; v < V; ++v) x[v] = load_chunk(row, v * L + lane, a.c);
    float s = 0.f;
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int e = 0; e < N; ++e) s += (float)x[v].x[e];
    const float mean = row_sum<L>(s, slot, turn) * inv;
    float q = 0.f;
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const float d = (float)x[v].x[e] - mean;
        // elements past the row are zeros, not deviations
        q += (v * L + lane) * N + e < a.c ? d * d : 0.f;
      }
    const float rstd = 1.f / sqrtf(row_sum<L>(q, slot, turn) * inv + a.eps);
    T* out = (T*)a.out + r * a.c;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      Chunk<T> o;
#pragma unroll
      for (int e = 0; e < N; ++e) {
        float y = ((float)x[v].x[e] - mean) * rstd;
        if (a.gamma) y *= (float)gamma[v].x[e];
        if (a.beta) y += (float)beta[v].x[e];
        o.x[e] = (T)y;
      }
      store_chunk(out, v * L + lane, a.c, o);
    }
    if (lane == 0) {
      a.mean[r] = mean;
      a.rstd[r] = rstd;
    }
  }
}

// Backward: dx as in the forward, and each lane's terms of dgamma and dbeta kept in its
// registers over all of its rows; the workgroup's totals go to its slab of the workspace
// (fixed order: lanes, then waves), which ln_reduce_kernel adds up.  589,824 x 128 bf16: 99 us,
// 4.6 TB/s of x, dout and dx, with 1024 slabs of 1 KB; 100,000 x 384: 60, 3.9 TB/s; 9001 x 833
// bf16: 17 to 19 us (a chunk's loads wait for each other as in the forward).
template <typename T, int L, int V, bool WG>
__global__ __launch_bounds__(LN_WG) void ln_bwd_kernel(LnBwdArgs a) {
  constexpr int N = Chunk<T>::N, G = LN_WG / L, ROW = (L < 64 ? L : 64) * V * N;
  __shared__ float slot[2][4];
  int turn = 0;
  const int lane = threadIdx.x % L, group = threadIdx.x / L;
  const float inv = 1.f / (float)a.c;
  Chunk<T> gamma[V];
  if (a.gamma)
#pragma unroll
    for (int v = 0; v < V; ++v) gamma[v] = load_chunk((const T*)a.gamma, v * L + lane, a.c);
  float dg[V][N], db[V][N];
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int e = 0; e < N; ++e) dg[v][e] = db[v][e] = 0.f;
  for (int64_t r = (int64_t)blockIdx.x * G + group; r < a.m; r += (int64_t)gridDim.x * G) {
    Chunk<T> x[V], dy[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      x[v] = load_chunk((const T*)a.x + r * a.c, v * L + lane, a.c);
      dy[v] = load_chunk((const T*)a.dout + r * a.c, v * L + lane, a.c);
    }
    const float mean = a.mean[r], rstd = a.rstd[r];
    float s1 = 0.f, s2 = 0.f;  // dout is zero past the row, so both sums are the row's
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const float d = (float)dy[v].x[e], xhat = ((float)x[v].x[e] - mean) * rstd;
        const float w = a.gamma ? d * (float)gamma[v].x[e] : d;
        s1 += w * xhat;
        s2 += w;
        if (WG) {
          dg[v][e] += d * xhat;
          db[v][e] += d;
        }
      }
    const float c1 = row_sum<L>(s1, slot, turn) * inv, c2 = row_sum<L>(s2, slot, turn) * inv;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      Chunk<T> o;
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const float d = (float)dy[v].x[e], xhat = ((float)x[v].x[e] - mean) * rstd;
        const float w = a.gamma ? d * (float)gamma[v].x[e] : d;
        o.x[e] = (T)(rstd * (w - c1 * xhat - c2));
      }
      store_chunk((T*)a.dx + r * a.c, v * L + lane, a.c, o);
    }
  }
  if (!WG) return;
  // the totals themselves where there is one workgroup
  float* part_g = gridDim.x > 1 ? a.part + (int64_t)blockIdx.x * 2 * a.c : a.dgamma;
  float* part_b = gridDim.x > 1 ? part_g + a.c : a.dbeta;
  if (L < 64) {  // the wave's groups
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int e = 0; e < N; ++e)
#pragma unroll
        for (int o = L; o < 64; o <<= 1) {
          dg[v][e] += __shfl_xor(dg[v][e], o);
          db[v][e] += __shfl_xor(db[v][e], o);
        }
  }
  if (L < LN_WG) {  // the waves: 2 and 3 onto 0 and 1, then 1 onto 0
    __shared__ float sum[2][2][ROW];
    const int wave = threadIdx.x >> 6, at = threadIdx.x & 63;
    for (int half = 2; half > 0; half >>= 1) {
      __syncthreads();
      if (wave >= half && wave < 2 * half && at < L)
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
          for (int e = 0; e < N; ++e) {
            sum[wave - half][0][(v * N + e) * (L < 64 ? L : 64) + at] = dg[v][e];
            sum[wave - half][1][(v * N + e) * (L < 64 ? L : 64) + at] = db[v][e];
          }
      __syncthreads();
      if (wave < half && at < L)
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
          for (int e = 0; e < N; ++e) {
            dg[v][e] += sum[wave][0][(v * N + e) * (L < 64 ? L : 64) + at];
            db[v][e] += sum[wave][1][(v * N + e) * (L < 64 ? L : 64) + at];
          }
    }
    if (threadIdx.x >= L) return;
  }
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const int i = (v * L + lane) * N + e;
      if (i < a.c) {
        if (part_g) part_g[i] = dg[v][e];
        if (part_b) part_b[i] = db[v][e];
      }
    }
}

// The slabs' sums, a column of [2][c] at a time: 4 to 5 us, two rounds of loads and a launch.
__global__ __launch_bounds__(SLAB_WG) void ln_reduce_kernel(const float* part, int nwg, int c,
                                                            float* dgamma, float* dbeta) {
  const float s = slab_column_sum(part, nwg, 2 * c, 2 * c);
  const int i = blockIdx.x * SLAB_COLS + threadIdx.x;
  if (threadIdx.x >= SLAB_COLS || i >= 2 * c) return;
  float* out = i < c ? dgamma : dbeta;
  if (out) out[i < c ? i : i - c] = s;
}

// Lanes a row of `chunks` 16-byte chunks takes: the fewest chunks a lane with no more
// than half of the lanes idle, few variants, and at most four chunks a lane (eight for
// the widest fp32 rows) so that a row's values and its weights' sums stay in registers.
int lanes_for(int chunks) {
  return chunks <= 4 ? 1 : chunks <= 8 ? 4 : chunks <= 64 ? 16 : chunks <= 256 ? 64 : LN_WG;
}

template <int L, int V>
struct Shape {
  static constexpr int lanes = L, chunks = V;
};

// Calls f with the shape of rows of c elements of T.
template <typename T, typename F>
void dispatch(int c, F f) {
  const int chunks = (c + Chunk<T>::N - 1) / Chunk<T>::N, L = lanes_for(chunks);
  const int v = (chunks + L - 1) / L;
  if (L == 1) {
    if (v == 1) f(Shape<1, 1>());
    else if (v == 2) f(Shape<1, 2>());
    else if (v == 3) f(Shape<1, 3>());
    else f(Shape<1, 4>());
  } else if (L == 4) {
    f(Shape<4, 2>());
  } else if (L == 16) {
    if (v == 1) f(Shape<16, 1>());
    else if (v == 2) f(Shape<16, 2>());
    else if (v == 3) f(Shape<16, 3>());
    else f(Shape<16, 4>());
  } else if (L == 64) {
    if (v == 2) f(Shape<64, 2>());
    else if (v == 3) f(Shape<64, 3>());
    else f(Shape<64, 4>());
  } else {
    if (v == 2) f(Shape<LN_WG, 2>());
    else if (v == 3) f(Shape<LN_WG, 3>());
    else if (v == 4) f(Shape<LN_WG, 4>());
    else if constexpr (sizeof(T) == 4) f(Shape<LN_WG, 8>());
  }
}

int64_t row_groups(int chunks, int64_t m) {
  const int64_t g = LN_WG / lanes_for(chunks);
  return (m + g - 1) / g;
}

template <typename T>
hipError_t fwd(const LnArgs& a, hipStream_t s) {
  KernelTimer t(K_LN_FWD, s);
  // eight workgroups fill a CU; with many rounds each keeps its weights over its own, with
  // few the dispatcher evens them out
  const int64_t g = row_groups((a.c + Chunk<T>::N - 1) / Chunk<T>::N, a.m);
  const dim3 grid((unsigned)(g < 256 * 32 ? g : 256 * 8));
  dispatch<T>(a.c, [&](auto shape) {
    hipLaunchKernelGGL((ln_fwd_kernel<T, shape.lanes, shape.chunks>), grid, dim3(LN_WG), 0, s, a);
  });
  return hipGetLastError();
}

template <typename T>
hipError_t bwd(const LnBwdArgs& a, hipStream_t s) {
  const bool weights = a.dgamma || a.dbeta;
  {
    KernelTimer t(K_LN_BWD, s);
    dispatch<T>(a.c, [&](auto shape) {
      constexpr int L = shape.lanes, V = shape.chunks;
      if (weights)
        hipLaunchKernelGGL((ln_bwd_kernel<T, L, V, true>), dim3(a.nwg), dim3(LN_WG), 0, s, a);
      else
        hipLaunchKernelGGL((ln_bwd_kernel<T, L, V, false>), dim3(a.nwg), dim3(LN_WG), 0, s, a);
    });
  }
  if (weights && a.nwg > 1) {
    KernelTimer t(K_LN_REDUCE, s);
    hipLaunchKernelGGL(ln_reduce_kernel, dim3(slab_grid(2 * a.c)), dim3(SLAB_WG), 0, s, a.part,
                       a.nwg, a.c, a.dgamma, a.dbeta);
  }
  return hipGetLastError();
}

}  // namespace

// Workgroups (and slabs) of the backward: up to four a CU, fewer where their slabs,
// written and read once, would pass a third of the rows' traffic (3 values an element),
// and one alone, which needs no further sum, for up to 4 rounds.
int ln_bwd_parts(int dtype, int64_t m, int c) {
  const int e = dtype == TRIATTN_BF16 ? 2 : 4;
  const int64_t groups = row_groups((c * e + 15) / 16, m);
  int64_t most = m * e / 16;
  most = groups <= 4 ? 1 : most < 256 ? 256 : most > 1024 ? 1024 : most;
  const int64_t rounds = (groups + most - 1) / most;  // as many for every workgroup
  return (int)((groups + rounds - 1) / rounds);
}

hipError_t launch_ln_fwd(int dtype, const LnArgs& a, hipStream_t s) {
  return dtype == TRIATTN_BF16 ? fwd<bf16>(a, s) : fwd<float>(a, s);
}
hipError_t launch_ln_bwd(int dtype, const LnBwdArgs& a, hipStream_t s) {
  return dtype == TRIATTN_BF16 ? bwd<bf16>(a, s) : bwd<float>(a, s);
}

}  // namespace triattn
