// Learned relative position bias by buckets, and the gradient of its table.
//
// A pair's bucket is the number of edges at or below the difference of its positions.
// Where the edges span fewer than REL_SPAN differences (a clipped difference and buckets
// that widen up to four thousand tokens do), the bucket is one read of a table by difference
// in LDS; edges further apart are searched, eight dependent LDS reads a pair (940 tokens x 16
// heads with 209 edges, forward and backward: 328 us by search, 87 by table).  The host makes
// tables of up to REL_LUT bytes, which travel in the kernel's arguments in the place of the
// edges; longer ones every workgroup makes of the edges.
#include <limits.h>

#include "dma.h"
#include "ops.h"
#include "slabs.h"
#include "timing.h"
#include "triattn.h"

namespace triattn {
namespace {

constexpr int REL_LDS_BUCKETS = REL_SPAN + REL_MAX_EDGES * 4 + 4;

struct Buckets {
  const uint8_t* lut;    // LDS: bucket of difference low + i
  const int32_t* edges;  // LDS
};

__device__ inline int search(const int32_t* edges, int ne, int64_t d) {
  int lo = 0, hi = ne;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (edges[mid] <= d) lo = mid + 1;
    else hi = mid;
  }
  return lo;
}

// Brings the table or the edges from the arguments to LDS (REL_LDS_BUCKETS bytes).  A table
// too long for the arguments is made here: a thread searches its first difference and walks
// on from there.  The caller's barrier follows.
template <bool LUT>
__device__ inline Buckets load_buckets(const RelArgs& a, char* lds) {
  int32_t* edges = (int32_t*)(lds + REL_SPAN);
  uint8_t* lut = (uint8_t*)lds;
  if (LUT && a.span < REL_LUT) {
    for (int i = threadIdx.x; i <= a.span / 4; i += blockDim.x)
      ((uint32_t*)lds)[i] = ((const uint32_t*)a.lut)[i];
    return Buckets{lut, edges};
  }
  for (int i = threadIdx.x; i < a.ne; i += blockDim.x) edges[i] = a.edges[i];
  if constexpr (LUT) {
    __syncthreads();
    const int per = (a.span / (int)blockDim.x + 4) / 4 * 4, i0 = threadIdx.x * per;
    if (i0 <= a.span) {
      int r = search(edges, a.ne, (int64_t)a.low + i0);
      for (int i = i0; i < i0 + per && i <= a.span; ++i) {
        while (r < a.ne && edges[r] <= a.low + i) ++r;
        lut[i] = (uint8_t)r;
      }
    }
  }
  return Buckets{lut, edges};
}

// Bucket of position pq less pk.  The difference may need 33 bits: LUT saturates it,
// which keeps its order against any edge above -2^31 (the host sees to that); the search
// takes it in 64.
template <bool LUT>
__device__ inline int bucket_of(const RelArgs& a, const Buckets& b, int32_t pq, int32_t pk) {
  if constexpr (LUT) {
    const int32_t d = __builtin_elementwise_sub_sat(
        __builtin_elementwise_sub_sat(pq, pk), a.low);
    int32_t i;  // d clipped to [0, span]
    asm("v_med3_i32 %0, %1, 0, %2" : "=v"(i) : "v"(d), "s"(a.span));
    return b.lut[i];
  } else {
    return search(b.edges, a.ne, (int64_t)pq - (int64_t)pk);
  }
}

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
struct __attribute__((packed)) Any16 {
  u32x4 v;
};

// Forward.  Bound by the write of the result (and the read of base).  A wave takes 64 U
// consecutive 16-byte chunks of one query's row; P elements of a chunk (P divides the
// chunk and h) belong to one pair and take one bucket and one read of the table, which
// lies in LDS if it has room.  Rows need not start at 16 bytes; a row's last, partial
// chunk goes element by element.  2 x 333 tokens x 128 channels bf16 (57 MB): 14 us, where a
// plain fill takes 10; 768 tokens x 4 heads with base (9 MB): 5.5 us, mostly the launch.
template <typename T, int P>
constexpr int task_chunks() {  // a lane's: more where a chunk is one piece
  return P == 16 / (int)sizeof(T) ? 4 : 2;
}
template <typename T, int P, bool LUT, bool LDS_TABLE>
__global__ __launch_bounds__(256) void rel_fwd_kernel(RelArgs a) {
  constexpr int N = 16 / (int)sizeof(T), U = task_chunks<T, P>();
  struct Piece {
    T x[P];
  };
  struct Elems {
    T x[N];
  };
  __shared__ __attribute__((aligned(16))) char bucket_lds[REL_LDS_BUCKETS];
  extern __shared__ __attribute__((aligned(16))) char table_lds[];
  const Buckets buckets = load_buckets<LUT>(a, bucket_lds);
  const T* table = (const T*)a.table;
  if (LDS_TABLE) {
    // in 16-byte words (the table starts at one), then what is left of it
    T* t = (T*)table_lds;
    const int all = a.rows * a.h, words = all / N;
    for (int i = threadIdx.x; i < words; i += 256) ((u32x4*)t)[i] = ((const u32x4*)table)[i];
    for (int i = words * N + threadIdx.x; i < all; i += 256) t[i] = table[i];
    table = t;
  }
  __syncthreads();
  const int len = a.n * a.h, chunks = (len + N - 1) / N;
  const int segs = (chunks + 64 * U - 1) / (64 * U), lane = threadIdx.x & 63;
  // below 2^31 for fewer than 2^39 elements; divided in 32 bits, as in 64 the two divisions
  // took longer than the rest of a task
  const uint32_t tasks = (uint32_t)(a.batch * a.n * segs);
  for (uint32_t task = blockIdx.x * 4 + (threadIdx.x >> 6); task < tasks; task += gridDim.x * 4) {
    const uint32_t r32 = task / (uint32_t)segs;  // row b n + q
    const int seg = (int)(task - r32 * (uint32_t)segs);
    const int64_t row = r32, b0 = (int64_t)(r32 / (uint32_t)a.n) * a.n;  // its sample's first
    const int32_t pq = a.pos[row], cq = a.chain ? a.chain[row] : 0;
    const T* base = a.base ? (const T*)a.base + row * len : nullptr;
    T* out = (T*)a.out + row * len;
    // all of the task's loads first; a piece past the row (never stored) takes the last one's
    Elems add[U];
    int32_t pk[U][N / P], ck[U][N / P];
    int column[U][N / P];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int e0 = ((seg * U + u) * 64 + lane) * N;
      if (base) {
        if (e0 + N <= len) {
          add[u] = __builtin_bit_cast(Elems, *(const Any16*)(base + e0));
        } else {
#pragma unroll
          for (int e = 0; e < N; ++e) add[u].x[e] = base[min(e0 + e, len - 1)];
        }
      }
#pragma unroll
      for (int i = 0; i < N / P; ++i) {
        const unsigned at = min(e0 + i * P, len - P);
        const int k = a.inv_h ? (int)__umulhi(at, a.inv_h) : (int)at;
        column[u][i] = (int)at - k * a.h;
        pk[u][i] = a.pos[b0 + k];
        ck[u][i] = a.chain ? a.chain[b0 + k] : 0;
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int e0 = ((seg * U + u) * 64 + lane) * N;
      Elems o;
#pragma unroll
      for (int i = 0; i < N / P; ++i) {
        int r = bucket_of<LUT>(a, buckets, pq, pk[u][i]);
        if (ck[u][i] != cq) r = a.ne + 1;
        const Piece t = *(const Piece*)(table + r * a.h + column[u][i]);
#pragma unroll
        for (int e = 0; e < P; ++e)
          o.x[i * P + e] = base ? (T)((float)t.x[e] + (float)add[u].x[i * P + e]) : t.x[e];
      }
      if (e0 + N <= len) {
        *(Any16*)(out + e0) = __builtin_bit_cast(Any16, o);
      } else {
#pragma unroll
        for (int e = 0; e < N; ++e)
          if (e0 + e < len) out[e0 + e] = o.x[e];
      }
    }
  }
}

// Backward: sums over the pairs of a bucket, for any positions in any order.
//
// A lane belongs to one channel (lane = pair offset * h + channel for h <= 64; 64 channels of
// one pair at a time above) and adds its values into its own column of the wave's LDS sums
// [rows][64]: no two lanes share a sum, so nothing depends on the order lanes run in, no
// atomics are needed, and a wave's lanes never meet in an LDS bank.  A read, an add and a
// write take 14 cycles a wave and CU with the lookup before them (8 waves in turn); the LDS's
// own fp32 add, although nothing waits for it, takes 200.  A wave keeps its keys (positions in
// registers) and walks over query rows.  At the end the workgroup adds its lanes' and waves'
// columns in a fixed order into its slab, and rel_reduce_kernel the slabs.
//
// 1536 tokens x 16 heads bf16 (75 MB): 25 us, 3.0 TB/s; 2 x 333 tokens x 128 channels: 24 us;
// 768 x 4: 11 us.  Bound by the chain of LDS accesses at the eight waves that the sums (17 KB
// a wave for 66 rows) leave on a CU.
constexpr int REL_K = 4;  // key groups of a wave
constexpr int REL_Q = 4;  // query rows whose loads are in flight together

// Geometry of the backward, from the sizes alone.
struct RelPlan {
  int hc;      // channels of a wave: min(h, 64)
  int groups;  // channel groups of 64
  int pl;      // pairs of a wave's load
  int waves;   // waves of a workgroup: what leaves their sums 64 KB of LDS, or half of it
  int kblocks; // workgroups along the keys
  int units;   // row chunks of a sample
  int qlen;    // rows of a chunk
  int w;       // workgroups that share a key block's units
  __host__ __device__ int slabs() const { return w * kblocks; }
};

__host__ __device__ inline RelPlan rel_plan(int64_t batch, int n, int h, int rows) {
  RelPlan p;
  p.hc = h < 64 ? h : 64;
  p.groups = (h + 63) / 64;
  p.pl = 64 / p.hc;
  p.waves = rows <= 64 + 8 ? 4 : rows <= 128 + 8 ? 2 : 1;
  const int keys = p.pl * REL_K * p.waves;
  p.kblocks = (n + keys - 1) / keys;
  // about as many workgroups as the CUs' LDS holds at once, each of at least 4 rows; one
  // alone, which needs no further sum, for up to 32 rows
  const int lds = p.waves * rows * 256 + REL_LDS_BUCKETS, fit = 160 * 1024 / lds;
  int64_t want = 256 * fit / (p.groups * p.kblocks);
  if (want < 1 || (p.groups * p.kblocks == 1 && batch * n <= 32)) want = 1;
  // a workgroup has one chunk of a sample's rows, or, where there are more samples than
  // that, whole samples in turn
  int64_t units = want / batch, most = (n + REL_Q - 1) / REL_Q;
  if (units > most) units = most;
  if (units < 1) units = 1;
  p.qlen = (int)((n + units - 1) / units);
  p.units = (n + p.qlen - 1) / p.qlen;
  p.w = (int)(batch * p.units < want ? batch * p.units : want);
  return p;
}

// One element by a buffer load (zero past the resource).
__device__ inline float load_one(rsrc_t r, uint32_t off, bf16) {
  return __uint_as_float((uint32_t)__builtin_amdgcn_raw_buffer_load_b16(r, (int)off, 0, 0) << 16);
}
__device__ inline float load_one(rsrc_t r, uint32_t off, float) {
  return __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(r, (int)off, 0, 0));
}

// Value V of a group of SPREAD lanes, in all of them.
template <int SPREAD, int V>
__device__ inline int spread(int x) {
  if constexpr (SPREAD == 4)
    return __builtin_amdgcn_update_dpp(0, x, 0x55 * V, 0xf, 0xf, true);  // quad_perm V V V V
  else
    return __builtin_amdgcn_update_dpp(0, x, 0x150 + V, 0xf, 0xf, true);  // row_newbcast V
}

// SPREAD: the lanes of a pair (h = 4, 16, or 64 and up) look up one row of their key each,
// SPREAD rows at a time, and hand the buckets round; 0: every lane looks up every row of
// its key itself.
template <typename T, bool LUT, int SPREAD>
__global__ __launch_bounds__(256) void rel_bwd_kernel(RelArgs a, RelPlan p) {
  constexpr int BLOCK = SPREAD ? SPREAD : 64;  // rows whose positions (or buckets) lanes hold
  const bool chains = a.chain != nullptr;
  __shared__ __attribute__((aligned(16))) char bucket_lds[REL_LDS_BUCKETS];
  extern __shared__ __attribute__((aligned(16))) float sums[];  // [waves][rows][64]
  const Buckets buckets = load_buckets<LUT>(a, bucket_lds);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  float* mine = sums + wave * a.rows * 64;
  for (int i = 4 * lane; i < a.rows * 64; i += 256) *(f32x4*)(mine + i) = f32x4{};
  __syncthreads();
  const int kb = blockIdx.x % p.kblocks, w = blockIdx.x / p.kblocks, c0 = blockIdx.y * 64;
  const int off = lane / p.hc, c = c0 + lane % p.hc;
  const int k0 = (kb * p.waves + wave) * p.pl * REL_K + off;
  const uint32_t row_bytes = (uint32_t)(a.n * a.h) * sizeof(T);  // at most 8 MB
  // lanes without a channel and keys past the last read zeros (and add them to a sum of
  // their own column)
  int key[REL_K];
  uint32_t at[REL_K];
#pragma unroll
  for (int u = 0; u < REL_K; ++u) {
    const int k = k0 + u * p.pl;
    const bool in = off < p.pl && c < a.h && k < a.n;
    key[u] = k < a.n ? k : 0;  // the same for all lanes of a pair, with or without a channel
    at[u] = in ? (uint32_t)(k * a.h + c) * sizeof(T) : 0x80000000u;
  }
  float* column = mine + lane;
  for (int64_t unit = w; unit < a.batch * p.units; unit += p.w) {
    const int64_t b0 = unit / p.units * a.n;  // the sample's first row
    const int q0 = (int)(unit % p.units) * p.qlen, q1 = min(q0 + p.qlen, a.n);
    int32_t pk[REL_K], ck[REL_K];
#pragma unroll
    for (int u = 0; u < REL_K; ++u) {
      pk[u] = a.pos[b0 + key[u]];
      ck[u] = chains ? a.chain[b0 + key[u]] : 0;
    }
    float x[REL_Q][REL_K];
    auto load = [&](int q) {  // rows past the chunk give zeros
#pragma unroll
      for (int v = 0; v < REL_Q; ++v) {
        const rsrc_t row = buf_rsrc_n((const char*)a.dout + (b0 + q + v) * row_bytes,
                                      q + v < q1 ? row_bytes : 0u);
#pragma unroll
        for (int u = 0; u < REL_K; ++u) x[v][u] = load_one(row, at[u], T());
      }
    };
    load(q0);
    // position and chain of one row of the current block and of the next one
    const int mine_of = lane % BLOCK;
    auto row_of = [&](int q) { return b0 + min(q + mine_of, q1 - 1); };
    int32_t next_pos = a.pos[row_of(q0)], next_chain = chains ? a.chain[row_of(q0)] : 0;
    int32_t prow = 0, crow = 0;
    int bucket[REL_K];  // SPREAD: of this lane's row and key u
    for (int q = q0; q < q1; q += REL_Q) {
      const int at_row = (q - q0) % BLOCK;
      float f[REL_Q][REL_K];
#pragma unroll
      for (int v = 0; v < REL_Q; ++v)
#pragma unroll
        for (int u = 0; u < REL_K; ++u) f[v][u] = x[v][u];
      if (at_row == 0) {
        prow = next_pos;
        crow = next_chain;
        next_pos = a.pos[row_of(q + BLOCK)];
        if (chains) next_chain = a.chain[row_of(q + BLOCK)];
        if constexpr (SPREAD != 0) {
#pragma unroll
          for (int u = 0; u < REL_K; ++u) {
            bucket[u] = bucket_of<LUT>(a, buckets, prow, pk[u]);
            if (chains && ck[u] != crow) bucket[u] = a.ne + 1;
          }
        }
      }
      // the next rows' loads leave now, not where the scheduler finds registers for them
      __builtin_amdgcn_sched_barrier(0);
      load(q + REL_Q);
      __builtin_amdgcn_sched_barrier(0);
      int r[REL_Q][REL_K];
      if constexpr (SPREAD == 0) {
#pragma unroll
        for (int v = 0; v < REL_Q; ++v) {
          const int32_t pq = __builtin_amdgcn_readlane(prow, at_row + v);
          const int32_t cq = __builtin_amdgcn_readlane(crow, at_row + v);
#pragma unroll
          for (int u = 0; u < REL_K; ++u) {
            r[v][u] = bucket_of<LUT>(a, buckets, pq, pk[u]);
            if (chains && ck[u] != cq) r[v][u] = a.ne + 1;
          }
        }
      } else if constexpr (SPREAD == 64) {
#pragma unroll
        for (int v = 0; v < REL_Q; ++v)
#pragma unroll
          for (int u = 0; u < REL_K; ++u) r[v][u] = __builtin_amdgcn_readlane(bucket[u], at_row + v);
      } else {
        static_assert(REL_Q == 4, "spread's constants");
#pragma unroll
        for (int u = 0; u < REL_K; ++u) {
          r[0][u] = spread<SPREAD, 0>(bucket[u]);
          r[1][u] = spread<SPREAD, 1>(bucket[u]);
          r[2][u] = spread<SPREAD, 2>(bucket[u]);
          r[3][u] = spread<SPREAD, 3>(bucket[u]);
          // the next four rows' buckets to the front (row_ror 12)
          if (SPREAD == 16) bucket[u] = __builtin_amdgcn_update_dpp(0, bucket[u], 0x12c, 0xf, 0xf, true);
        }
      }
      // two at a time, which halves the chain of dependent LDS accesses: if both fall into
      // one bucket, the second goes on from the first one's new value and its write stays
#pragma unroll
      for (int v = 0; v < REL_Q; ++v)
#pragma unroll
        for (int u = 0; u < REL_K; u += 2) {
          const int r0 = r[v][u], r1 = r[v][u + 1];
          const float x0 = column[r0 * 64], x1 = column[r1 * 64], y0 = x0 + f[v][u];
          column[r0 * 64] = y0;
          column[r1 * 64] = (r1 == r0 ? y0 : x1) + f[v][u + 1];
        }
    }
  }
  __syncthreads();
  // the waves' sums onto the first wave's, row by row
  for (int i = threadIdx.x; i < a.rows * 64; i += blockDim.x) {
    float s = sums[i];
    for (int v = 1; v < p.waves; ++v) s += sums[v * a.rows * 64 + i];
    sums[i] = s;
  }
  __syncthreads();
  // channel c of row r: the lanes off * hc + c, beginning at another one in every row so that
  // the rows' reads fall into different banks
  float* slab = p.slabs() > 1 ? a.part + (int64_t)blockIdx.x * a.rows * a.h : a.dtable;
  for (int i = threadIdx.x; i < a.rows * p.hc; i += blockDim.x) {
    const int r = i / p.hc, ch = i - r * p.hc;
    if (c0 + ch >= a.h) continue;
    const float* row = sums + r * 64 + ch;
    float s = 0.f;
    int at = r % p.pl;
#pragma unroll 4
    for (int t = 0; t < p.pl; ++t) {
      s += row[at * p.hc];
      at = at + 1 == p.pl ? 0 : at + 1;
    }
    slab[r * a.h + c0 + ch] = s;
  }
}

// The slabs' sums (462 of 1 KB: 4 us; 252 of 34 KB: 6 us).
__global__ __launch_bounds__(SLAB_WG) void rel_reduce_kernel(const float* part, int count,
                                                             int total, float* dtable) {
  const float s = slab_column_sum(part, count, total, total);
  const int i = blockIdx.x * SLAB_COLS + threadIdx.x;
  if (threadIdx.x < SLAB_COLS && i < total) dtable[i] = s;
}

// Fills in the table's range.  False: the edges are searched.
bool use_lut(RelArgs& a) {
  const int64_t span = (int64_t)a.edges[a.ne - 1] - a.edges[0] + 1;
  if (a.edges[0] == INT_MIN || span >= REL_SPAN) return false;
  a.low = a.edges[0] - 1;
  a.span = (int32_t)span;  // difference low + span is the last edge
  if (span < REL_LUT) {
    int32_t edges[REL_MAX_EDGES];
    for (int i = 0; i < a.ne; ++i) edges[i] = a.edges[i];  // the table takes their place
    a.lut[0] = 0;
    for (int i = 0; i < a.ne; ++i) {
      const int from = edges[i] - a.low, to = i + 1 < a.ne ? edges[i + 1] - a.low : a.span + 1;
      for (int d = from; d < to; ++d) a.lut[d] = (uint8_t)(i + 1);
    }
  }
  return true;
}

constexpr size_t REL_LDS_TABLE = 32 << 10;

template <typename T, int P>
void fwd_piece(const RelArgs& a, bool lut, hipStream_t s) {
  constexpr int SEG = 64 * task_chunks<T, P>();
  const size_t table = (size_t)a.rows * a.h * sizeof(T);
  const int64_t chunks = ((int64_t)a.n * a.h * sizeof(T) + 15) / 16;
  const int64_t wgs = (a.batch * a.n * ((chunks + SEG - 1) / SEG) + 3) / 4;
  const dim3 g((unsigned)(wgs < 256 * 8 ? wgs : 256 * 8)), wg(256);
  if (table <= REL_LDS_TABLE) {
    if (lut) hipLaunchKernelGGL((rel_fwd_kernel<T, P, true, true>), g, wg, table, s, a);
    else hipLaunchKernelGGL((rel_fwd_kernel<T, P, false, true>), g, wg, table, s, a);
  } else {
    if (lut) hipLaunchKernelGGL((rel_fwd_kernel<T, P, true, false>), g, wg, 0, s, a);
    else hipLaunchKernelGGL((rel_fwd_kernel<T, P, false, false>), g, wg, 0, s, a);
  }
}

template <typename T>
hipError_t fwd(RelArgs a, hipStream_t s) {
  KernelTimer t(K_REL_FWD, s);
  const bool lut = use_lut(a);
  a.inv_h = a.h == 1 ? 0u : (uint32_t)((((uint64_t)1 << 32) + a.h - 1) / a.h);
  constexpr int N = 16 / (int)sizeof(T);
  if (a.h % N == 0) fwd_piece<T, N>(a, lut, s);
  else if (N > 4 && a.h % 4 == 0) fwd_piece<T, 4>(a, lut, s);
  else if (a.h % 2 == 0) fwd_piece<T, 2>(a, lut, s);
  else fwd_piece<T, 1>(a, lut, s);
  return hipGetLastError();
}

template <typename T>
hipError_t bwd(RelArgs a, hipStream_t s) {
  const RelPlan p = rel_plan(a.batch, a.n, a.h, a.rows);
  const bool lut = use_lut(a);
  {
    KernelTimer t(K_REL_BWD, s);
    const dim3 grid((unsigned)p.slabs(), (unsigned)p.groups), wg(64 * p.waves);
    const size_t lds = (size_t)p.waves * a.rows * 64 * sizeof(float);
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, wg, lds, s, a, p); };
    if (p.hc == 64) go(lut ? rel_bwd_kernel<T, true, 64> : rel_bwd_kernel<T, false, 64>);
    else if (p.hc == 16) go(lut ? rel_bwd_kernel<T, true, 16> : rel_bwd_kernel<T, false, 16>);
    else if (p.hc == 4) go(lut ? rel_bwd_kernel<T, true, 4> : rel_bwd_kernel<T, false, 4>);
    else go(lut ? rel_bwd_kernel<T, true, 0> : rel_bwd_kernel<T, false, 0>);
  }
  if (p.slabs() == 1) return hipGetLastError();
  KernelTimer t(K_REL_REDUCE, s);
  const int total = a.rows * a.h;
  hipLaunchKernelGGL(rel_reduce_kernel, dim3(slab_grid(total)), dim3(SLAB_WG), 0, s, a.part,
                     p.slabs(), total, a.dtable);
  return hipGetLastError();
}

}  // namespace

size_t rel_bwd_ws(int64_t batch, int n, int h, int rows) {
  return (size_t)rel_plan(batch, n, h, rows).slabs() * (size_t)rows * h * sizeof(float);
}

hipError_t launch_rel_fwd(int dtype, const RelArgs& a, hipStream_t s) {
  return dtype == TRIATTN_BF16 ? fwd<bf16>(a, s) : fwd<float>(a, s);
}
hipError_t launch_rel_bwd(int dtype, const RelArgs& a, hipStream_t s) {
  return dtype == TRIATTN_BF16 ? bwd<bf16>(a, s) : bwd<float>(a, s);
}

}  // namespace triattn
