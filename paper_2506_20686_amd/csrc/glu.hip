// Gated linear projection: [a | b] = x W + bias, out = act(a) b, W [k][2 f].
//
// Both projections are one product (lin_tile.h): a tile of W holds the same columns of both
// halves, 8 and 8 in turn, so that a thread ends with a and b of the same outputs and neither is
// written.  The backward forms them again, with
//   da = dout b act'(a),  db = dout act(a)
// in the product's epilogue, as dz = [da | db] in 24 bits: three planes of bf16 where rows are whole
// words (6 bytes an element moved, but a tile that reads dz need not split it: 6001 x 512 x 2048,
// products 240 us from fp32, 221 from planes), else fp32.  dx = dz W^T, dW = x^T dz and the sums
// of dz are the linear projection's products.
#include "lin_tile.h"
#include "timing.h"

namespace triattn {
namespace {

// sigmoid(z) and sigmoid(-z), neither taken from 1: z is a sum in fp32, never rounded to the
// tensors' 8 bits, and far out the sigmoid's derivative is the small side's.  The hardware's
// exponential serves for bf16 tensors: it is off by twice |z| half steps, as z's own half step is
// by |z|.  (silu's derivative is p + z p q, where a q taken from 1 is off by |z| half steps of
// 1: the narrow backward of it took 343 us so, and 363 with both sides.)
template <bool FULL>
__device__ inline void both_sides(float z, float& s, float& other) {
  if constexpr (FULL) return sigmoid<true>(z, s, other);
  const float e = __expf(-fabsf(z)), big = fast_rcp(1.f + e), small = e * big;
  s = z < 0.f ? small : big;
  other = z < 0.f ? big : small;
}

// The activation of tensors of T and its derivative.
template <typename T>
__device__ inline void act_both(float z, int act, float& value, float& slope) {
  float p, q;
  if (act == TRIATTN_ACT_GELU) {
    normal_cdf<sizeof(T) == 4>(z, p, q);
    value = z * p;
    slope = p + z * 0.39894228040143268f * q;
  } else if (act == TRIATTN_ACT_RELU) {
    value = z > 0.f ? z : 0.f;
    slope = z > 0.f ? 1.f : 0.f;
  } else if (act == TRIATTN_ACT_NONE) {
    value = z;
    slope = 1.f;
  } else if (act == TRIATTN_ACT_SILU) {
    sigmoid<sizeof(T) == 4>(z, p, q);
    value = z * p;
    slope = p * (1.f + z * q);
  } else {
    both_sides<sizeof(T) == 4>(z, p, q);
    value = p;
    slope = p * q;
  }
}
template <typename T>
__device__ inline float gate_value(float z, int act) {
  if (act != TRIATTN_ACT_SIGMOID) return act_value<T>(z, act);
  float p, q;
  sigmoid<sizeof(T) == 4>(z, p, q);
  return p;
}

// Four packed bf16 of an accumulator quad.
__device__ inline u32x2 pack4(float a, float b, float c, float d) {
  return __builtin_bit_cast(u32x2, bf16x4{(bf16)a, (bf16)b, (bf16)c, (bf16)d});
}
// The four values' next plane of bf16, taken off them.
__device__ inline u32x2 take_plane(float& a, float& b, float& c, float& d) {
  const u32x2 w = pack4(a, b, c, d);
  a -= __uint_as_float(w[0] << 16);
  b -= __uint_as_float(w[0] & 0xffff0000u);
  c -= __uint_as_float(w[1] << 16);
  d -= __uint_as_float(w[1] & 0xffff0000u);
  return w;
}

// The first `have` (whole words) of 8 values as three planes of bf16, `plane` elements apart.
__device__ inline void put_planes(bf16* p, int64_t plane, int have, float (&f)[8]) {
#pragma unroll
  for (int u = 0; u < 3; ++u) {
    const u32x2 lo = take_plane(f[0], f[1], f[2], f[3]), hi = take_plane(f[4], f[5], f[6], f[7]);
    const u32x4 w{lo[0], lo[1], hi[0], hi[1]};
    // (fp32's whole words are 4 elements: half a word here, and the second half may start there)
    if (have >= 8) ((Any16*)(p + u * plane))->v = w;
    else if (have > 0) *(u32x2*)(p + u * plane) = lo;
  }
}

// 6001 x 512 x 2048 bf16: 45 us (560 TFLOP/s), with dz as its result 65 (50 and 73 in the first
// passes); as the linear projection's forward, LDS reads and staging beside the products.
template <typename T, int R, bool ALIGNED, bool DZ>
__global__ __launch_bounds__(256, sizeof(T) == 2 ? 2 : 1) void glu_kernel(GluArgs a) {
  using G = Product<T, T, R, step_k(R, 2 * planes<T>()), true, false, planes<T>(), planes<T>(),
                    DZ_X, DZ_X, ALIGNED, false, true>;
  __shared__ __attribute__((aligned(16))) char lds[G::LDS];
  const int nj = (a.f + R / 2 - 1) / (R / 2), wg = xcd_swizzle(blockIdx.x, gridDim.x);
  const int64_t i0 = (int64_t)(wg / nj) * R;
  const int j0 = (wg % nj) * (R / 2), j = j0 + G::pair_col(), have = a.f - j;
  // what the epilogue reads is on its way before the product
  Raw8<T> dy[ALIGNED && DZ ? G::PAIRS : 1];
  float ba[8] = {}, bb[8] = {};
  if (ALIGNED && DZ) {
#pragma unroll
    for (int t = 0; t < G::PAIRS; ++t) {
      const int64_t i = i0 + G::pair_row(t);
      if (i < a.m && have > 0) dy[t] = get8<T, ALIGNED>((const T*)a.dout + i * a.f + j, have);
    }
  }
  if (a.bias && have > 0) {
    unpack(get8<T, ALIGNED>((const T*)a.bias + j, have), ba);
    unpack(get8<T, ALIGNED>((const T*)a.bias + a.f + j, have), bb);
  }
  f32x16 acc[G::NT][G::NT];
  float none[8];
  G::run(lds, Mat<T>{(const T*)a.x, a.m, a.k}, nullptr, Mat<T>{(const T*)a.w, a.k, 2 * a.f},
         nullptr, 0, i0, j0, 0, a.k, false, none, acc);
  G::pairs(lds, acc, [&](int t, float (&za)[8], float (&zb)[8]) {
    const int64_t i = i0 + G::pair_row(t);
    if (i >= a.m || have <= 0) return;
#pragma unroll
    for (int e = 0; e < 8; ++e) za[e] += ba[e], zb[e] += bb[e];
    if constexpr (DZ) {
      float d[8];
      if constexpr (ALIGNED) unpack(dy[t], d);
      else unpack(get8<T, false>((const T*)a.dout + i * a.f + j, have), d);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float value, slope;
        act_both<T>(za[e], a.act, value, slope);
        za[e] = d[e] * zb[e] * slope;
        zb[e] = d[e] * value;
      }
      const int64_t at = i * 2 * a.f + j;
      if constexpr (ALIGNED) {
        bf16* dz = (bf16*)a.dz + at;
        put_planes(dz, a.m * 2 * a.f, have, za);
        put_planes(dz + a.f, a.m * 2 * a.f, have, zb);
      } else {
        put8<float, false>(a.dz + at, have, za);
        put8<float, false>(a.dz + at + a.f, have, zb);
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) za[e] = gate_value<T>(za[e], a.act) * zb[e];
      put8<T, ALIGNED>((T*)a.out + i * a.f + j, have, za);
    }
  });
}

// ---- narrow bf16 projections (k, f <= 128): the pair channels -----------------------------
//
// Rows of 128 + 128 channels move as many bytes as 4 f k operations take to multiply in a
// fraction of the time, so a workgroup keeps W in registers, from the start to its last row,
// and walks over blocks of 32 rows; nothing but x, dout, out and dx crosses memory.
constexpr int GLU_ROWS = 32;

// W to LDS as two squares (lines k, columns of a half each), zeros past the ends.
template <int THREADS>
__device__ inline void stage_w(const GluArgs& a, char* t) {
  const Mat<bf16> w{(const bf16*)a.w, a.k, 2 * a.f};
#pragma unroll
  for (int u = 0; u < 2 * 128 * 16 / THREADS; ++u) {
    const int id = (int)threadIdx.x + THREADS * u, half = id / 2048, line = id / 16 % 128;
    const int c = id % 16;
    const rsrc_t rs = buf_rsrc_n(w.p, (uint32_t)(a.k * 2 * a.f) * 2u);
    const uint32_t off = line < a.k && 8 * c < a.f
                             ? (uint32_t)((line * 2 + half) * a.f + 8 * c) * 2u
                             : 0x80000000u;
    *(u32x4*)(t + half * 128 * 256 + Square::chunk_at(line, c)) = __builtin_bit_cast(
        u32x4, __builtin_amdgcn_raw_buffer_load_b128(rs, (int)off, 0, 0));
  }
}

// Quads i (columns 8 i + 4 g ..) of a row's 32 results -> this lane's columns 16 g .. + 7 and
// 16 g + 8 .. + 15, by exchanges between the two halves of the wave.
__device__ inline void row_words(const u32x2 (&q)[4], u32x4 (&w)[2]) {
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const auto x = __builtin_amdgcn_permlane32_swap(q[u][0], q[u + 2][0], false, false);
    const auto y = __builtin_amdgcn_permlane32_swap(q[u][1], q[u + 2][1], false, false);
    w[u] = u32x4{x[0], y[0], x[1], y[1]};
  }
}

// Forward: a wave has 32 columns of both halves; blocks of 64 rows through LDS, the next one's on
// their way meanwhile.  Bound by memory: 589,824 x 128 x 128 in 70 us, 4.3 TB/s (x straight into
// operand registers, a lane a row: 128 us, each line of it fetched four times).
template <int ACT>
__global__ __launch_bounds__(256, 2) void glu_narrow_fwd_kernel(GluArgs a) {
  __shared__ __attribute__((aligned(16))) char lds[2 * 128 * 256];
  stage_w<256>(a, lds);
  __syncthreads();
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 5;
  const int c0 = 32 * wave;
  bf16x8 wa[8], wb[8];
#pragma unroll
  for (int t = 0; t < 8; ++t) {
    wa[t] = Square::across(lds, c0, 16 * t, lane);
    wb[t] = Square::across(lds + 128 * 256, c0, 16 * t, lane);
  }
  f32x16 ba{}, bb{};
  if (a.bias) {
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      const int c = c0 + acc_row(v, g);
      if (c < a.f) {
        ba[v] = (float)((const bf16*)a.bias)[c];
        bb[v] = (float)((const bf16*)a.bias)[a.f + c];
      }
    }
  }
  // chunks of 64 rows, a row's 16 by 16 consecutive threads
  constexpr int M = 2 * GLU_ROWS, N = M * 16 / 256;
  const int chunk = threadIdx.x % 16;
  u32x4 x[N];
  auto load = [&](int64_t r0) {
    const int64_t left = a.m - r0;
    const int rows = left < 0 ? 0 : left < M ? (int)left : M;
    const rsrc_t rs = buf_rsrc_n((const bf16*)a.x + r0 * a.k, (uint32_t)(rows * a.k) * 2u);
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const int line = threadIdx.x / 16 + 16 * u;
      const uint32_t off = 8 * chunk < a.k ? (uint32_t)(line * a.k + 8 * chunk) * 2u : 0x80000000u;
      x[u] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rs, (int)off, 0, 0));
    }
  };
  const int64_t step = (int64_t)gridDim.x * M;
  int64_t r0 = (int64_t)blockIdx.x * M;
  load(r0);
  __syncthreads();  // W has been read
  int buf = 0;
  for (; r0 < a.m; r0 += step, buf ^= 1) {
    char* tx = lds + buf * M * 256;
#pragma unroll
    for (int u = 0; u < N; ++u)
      *(u32x4*)(tx + Square::chunk_at(threadIdx.x / 16 + 16 * u, chunk)) = x[u];
    load(r0 + step);
    // this buffer was last read two blocks ago, before the barrier of the last block
    __syncthreads();
    if (c0 >= a.f) continue;
#pragma unroll
    for (int j = 0; j < M; j += 32) {
      f32x16 za = ba, zb = bb;
#pragma unroll
      for (int t = 0; t < 8; ++t) {
        const bf16x8 fx = Square::along(tx, j, 16 * t, lane);
        za = Mma<bf16>::mma(wa[t], fx, za);
        zb = Mma<bf16>::mma(wb[t], fx, zb);
      }
      u32x2 q[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float o[4];
#pragma unroll
        for (int e = 0; e < 4; ++e)
          o[e] = gate_value<bf16>(za[4 * i + e], ACT) * zb[4 * i + e];
        q[i] = pack4(o[0], o[1], o[2], o[3]);
      }
      u32x4 w[2];
      row_words(q, w);
      const int64_t r = r0 + j + (lane & 31);
      bf16* out = (bf16*)a.out + r * a.f + c0 + 16 * g;
#pragma unroll
      for (int u = 0; u < 2; ++u)
        if (r < a.m && c0 + 16 * g + 8 * u < a.f) *(u32x4*)(out + 8 * u) = w[u];
    }
  }
}

// Backward: eight waves on a block of 32 rows.
//   z    a wave has 16 columns of either half (one tile: rows 0 .. 15 a, 16 .. 31 b, so that a
//        lane has a and b of the same output); dz goes to LDS in three planes;
//   dW   32 columns of dz a wave, all of k, in registers to the end;
//   dx   a tile of 32 of k and one half of dz's columns a wave; the halves meet in LDS.
// 48 of a wave's 56 matrix instructions a block are the three planes' (24 bits of dz).  589,824 x
// 128 x 128: 312 us, 350 in the first passes; 270 GFLOP of matrix instructions; the matrix cores
// are busy 44% of the time, the vector units 34%, LDS 31%, in phases that follow each other.
// (First passes too: the general kernels 598 us; the next block's z and dz beside this one's dW,
// with a barrier less, 380.)  All 256 registers are taken, and with an activation 2 to 6 spilled.
constexpr int GLU_BWD_WG = 512;
template <int ACT>
__global__ __launch_bounds__(GLU_BWD_WG) void glu_narrow_bwd_kernel(GluArgs a, LinBwdArgs o) {
  constexpr int LINES = GLU_ROWS * 256;  // bytes of 32 lines of 128 bf16
  // W first; then x (two buffers), dz (three planes of two halves), the halves of dx
  constexpr int X = 0, Z = 2 * LINES, P = Z + 6 * LINES;
  __shared__ __attribute__((aligned(16))) char lds[P + 4 * 64 * 16 * 4];
  static_assert(sizeof(lds) >= 2 * 128 * 256, "room for W");
  stage_w<GLU_BWD_WG>(a, lds);
  __syncthreads();
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 5;
  const int kt = 32 * (wave & 3), half = wave >> 2;  // of dx
  bf16x8 wz[8], wx[8];
  {
    const char* mine = lds + (lane & 16 ? 128 * 256 : 0);
    const int i = lane & 15, col = 16 * wave + 4 * (i & 3);
    typedef TRIATTN_LDS s16x4* lds4;
#pragma unroll
    for (int t = 0; t < 8; ++t) {
      const int line = 16 * t + 8 * g + (i >> 2);
      const char* p = mine + Square::chunk_at(line, col >> 3) + (col & 4) * 2;
      const char* q = mine + Square::chunk_at(line + 4, col >> 3) + (col & 4) * 2;
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(uintptr_t)lds_addr(p));
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(uintptr_t)lds_addr(q));
      wz[t] = __builtin_bit_cast(bf16x8,
                                 __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
      wx[t] = Square::along(lds + half * 128 * 256, kt, 16 * t, lane);
    }
  }
  f32x16 bias{};
  if (a.bias) {
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      const int c = 16 * wave + acc_row(v & 7, g);
      if (c < a.f) bias[v] = (float)((const bf16*)a.bias)[(v >> 3) * a.f + c];
    }
  }
  // this thread's chunk of x, and its row's dout (columns of its part of dz)
  const int line = threadIdx.x / 16, chunk = threadIdx.x % 16;
  u32x4 x;
  u32x2 dy[2];
  auto load = [&](int64_t r0) {
    const int64_t left = a.m - r0;
    const int rows = left < 0 ? 0 : left < GLU_ROWS ? (int)left : GLU_ROWS;
    const rsrc_t rx = buf_rsrc_n((const bf16*)a.x + r0 * a.k, (uint32_t)(rows * a.k) * 2u);
    const uint32_t off = 8 * chunk < a.k ? (uint32_t)(line * a.k + 8 * chunk) * 2u : 0x80000000u;
    x = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rx, (int)off, 0, 0));
    const rsrc_t rd = buf_rsrc_n((const bf16*)a.dout + r0 * a.f, (uint32_t)(rows * a.f) * 2u);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int c = 16 * wave + 8 * i + 4 * g;
      const uint32_t at = c < a.f ? (uint32_t)((lane & 31) * a.f + c) * 2u : 0x80000000u;
      dy[i] = __builtin_bit_cast(u32x2,
                                 __builtin_amdgcn_raw_buffer_load_b64(rd, (int)at, 0, 0));
    }
  };
  f32x16 gw[4] = {};
  f32x16 col{};  // this lane's rows' sums of dz
  const int64_t step = (int64_t)gridDim.x * GLU_ROWS;
  int64_t r0 = (int64_t)blockIdx.x * GLU_ROWS;
  load(r0);
  __syncthreads();  // W has been read
  int buf = 0;
  for (; r0 < a.m; r0 += step, buf ^= 1) {
    char* tx = lds + X + buf * LINES;
    *(u32x4*)(tx + Square::chunk_at(line, chunk)) = x;
    float d[8];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const bf16x4 y = __builtin_bit_cast(bf16x4, dy[i]);
#pragma unroll
      for (int e = 0; e < 4; ++e) d[4 * i + e] = (float)y[e];
    }
    __syncthreads();
    load(r0 + step);
    f32x16 z = bias;
#pragma unroll
    for (int t = 0; t < 8; ++t) z = Mma<bf16>::mma(wz[t], Square::along(tx, 0, 16 * t, lane), z);
#pragma unroll
    for (int v = 0; v < 8; ++v) {
      float value, slope;
      act_both<bf16>(z[v], ACT, value, slope);
      z[v] = d[v] * z[v + 8] * slope;
      z[v + 8] = d[v] * value;
    }
    col += z;
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        float f[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) f[e] = z[8 * h + 4 * i + e];
        char* to = lds + Z + h * LINES + Square::chunk_at(lane & 31, 2 * wave + i) + 8 * g;
#pragma unroll
        for (int p = 0; p < 3; ++p)
          *(u32x2*)(to + 2 * p * LINES) = take_plane(f[0], f[1], f[2], f[3]);
      }
    __syncthreads();
    if (o.dw) {
      // columns 32 (wave % 4) of half wave / 4
#pragma unroll
      for (int kk = 0; kk < GLU_ROWS; kk += 16) {
        bf16x8 fx[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) fx[u] = Square::across(tx, 32 * u, kk, lane);
#pragma unroll
        for (int p = 2; p >= 0; --p) {
          const bf16x8 fz = Square::across(lds + Z + (2 * p + half) * LINES, kt, kk, lane);
#pragma unroll
          for (int u = 0; u < 4; ++u) gw[u] = Mma<bf16>::mma(fz, fx[u], gw[u]);
        }
      }
    }
    if (o.dx) {
      f32x16 gx{};
#pragma unroll
      for (int p = 2; p >= 0; --p)
#pragma unroll
        for (int t = 0; t < 8; ++t)
          gx = Mma<bf16>::mma(
              wx[t], Square::along(lds + Z + (2 * p + half) * LINES, 0, 16 * t, lane), gx);
      f32x4* part = (f32x4*)(lds + P) + (wave & 3) * 256 + lane;
      if (half) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          part[64 * i] = f32x4{gx[4 * i], gx[4 * i + 1], gx[4 * i + 2], gx[4 * i + 3]};
      }
      __syncthreads();
      if (!half) {
        u32x2 q[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const f32x4 y = part[64 * i];
          q[i] = pack4(gx[4 * i] + y[0], gx[4 * i + 1] + y[1], gx[4 * i + 2] + y[2],
                       gx[4 * i + 3] + y[3]);
        }
        u32x4 w[2];
        row_words(q, w);
        const int64_t r = r0 + (lane & 31);
        bf16* dx = (bf16*)o.dx + r * a.k + kt + 16 * g;
#pragma unroll
        for (int u = 0; u < 2; ++u)
          if (r < a.m && kt + 16 * g + 8 * u < a.k) *(u32x4*)(dx + 8 * u) = w[u];
      }
    }
  }
  const int n = 2 * a.f;
  float* dw = o.splits > 1 ? o.part + blockIdx.x * slab_floats(a.k, n) : o.dw;
  float* db = o.splits > 1 ? dw + (int64_t)a.k * n : o.dbias;
  if (o.dw) {
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int i = 32 * u + (lane & 31);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int j = kt + 8 * q + 4 * g;
        if (i < a.k && j < a.f)
          *(f32x4*)(dw + (int64_t)i * n + half * a.f + j) =
              f32x4{gw[u][4 * q], gw[u][4 * q + 1], gw[u][4 * q + 2], gw[u][4 * q + 3]};
      }
    }
  }
  if (o.dbias) {  // the 32 lanes of a half hold rows of the same columns
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      float s = col[v];
      for (int i = 1; i < 32; i *= 2) s += __shfl_xor(s, i);
      const int c = 16 * wave + acc_row(v & 7, g);
      if ((lane & 31) == 0 && c < a.f) db[(v >> 3) * a.f + c] = s;
    }
  }
}

// f(constant) for the activation: one inside a row's loop would branch for every value.
template <typename F>
void with_act(int act, F f) {
  switch (act) {
    case TRIATTN_ACT_NONE: f(std::integral_constant<int, TRIATTN_ACT_NONE>()); break;
    case TRIATTN_ACT_RELU: f(std::integral_constant<int, TRIATTN_ACT_RELU>()); break;
    case TRIATTN_ACT_GELU: f(std::integral_constant<int, TRIATTN_ACT_GELU>()); break;
    case TRIATTN_ACT_SILU: f(std::integral_constant<int, TRIATTN_ACT_SILU>()); break;
    default: f(std::integral_constant<int, TRIATTN_ACT_SIGMOID>());
  }
}

bool narrow(int dtype, int k, int f) {
  return dtype == TRIATTN_BF16 && k <= 128 && f <= 128 && k % 8 == 0 && f % 8 == 0;
}
// Workgroups of the narrow kernels: one a CU backward, two forward, with blocks for all.
int narrow_wgs(int64_t m, int most) {
  const int64_t blocks = (m + GLU_ROWS - 1) / GLU_ROWS;
  return (int)(blocks < most ? blocks : most);
}

// Rows of every tensor, and the halves of W's, are whole 16-byte words.
bool whole(int dtype, int k, int f) {
  const int word = dtype == TRIATTN_BF16 ? WORD<bf16> : WORD<float>;
  return k % word == 0 && f % word == 0;
}

template <typename T, bool DZ>
hipError_t launch(const GluArgs& a, hipStream_t s) {
  KernelTimer t(DZ ? K_GLU_DZ : K_GLU_FWD, s);
  const bool al = whole(sizeof(T) == 2 ? TRIATTN_BF16 : TRIATTN_F32, a.k, a.f);
  // 128-wide tiles where there are enough of them for the 256 CUs, as in the linear projection
  const bool big = (al || sizeof(T) == 2) && a.f > 32 &&
                   (a.m + 127) / 128 * ((a.f + 63) / 64) >= 256 && (sizeof(T) == 2 || a.k >= 256);
  const int64_t rows = big ? 128 : 64, cols = rows / 2;
  const dim3 grid((unsigned)((a.m + rows - 1) / rows * ((a.f + cols - 1) / cols))), wg(256);
  if (big && al) hipLaunchKernelGGL((glu_kernel<T, 128, true, DZ>), grid, wg, 0, s, a);
  else if (big) hipLaunchKernelGGL((glu_kernel<bf16, 128, false, DZ>), grid, wg, 0, s, a);
  else if (al) hipLaunchKernelGGL((glu_kernel<T, 64, true, DZ>), grid, wg, 0, s, a);
  else hipLaunchKernelGGL((glu_kernel<T, 64, false, DZ>), grid, wg, 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_glu_fwd(int dtype, const GluArgs& a, hipStream_t s) {
  if (narrow(dtype, a.k, a.f)) {
    KernelTimer t(K_GLU_FWD, s);
    const dim3 grid(narrow_wgs((a.m + 1) / 2, 512)), wg(256);
    with_act(a.act, [&](auto act) {
      hipLaunchKernelGGL((glu_narrow_fwd_kernel<decltype(act)::value>), grid, wg, 0, s, a);
    });
    return hipGetLastError();
  }
  return dtype == TRIATTN_BF16 ? launch<bf16, false>(a, s) : launch<float, false>(a, s);
}

LinBwdPlan glu_bwd_plan(int dtype, int64_t m, int k, int f) {
  if (!narrow(dtype, k, f)) return lin_made_plan(dtype, m, k, 2 * f, whole(dtype, k, f));
  LinBwdPlan p{};
  p.splits = narrow_wgs(m, 256);
  if (p.splits > 1) p.part = lin_slab_bytes(k, 2 * f, p.splits);
  return p;
}
hipError_t launch_glu_bwd(int dtype, const GluArgs& a, const LinBwdArgs& b, hipStream_t s) {
  if (narrow(dtype, a.k, a.f)) {
    {
      KernelTimer t(K_GLU_DZ, s);
      const dim3 grid(b.splits), wg(GLU_BWD_WG);
      with_act(a.act, [&](auto act) {
        hipLaunchKernelGGL((glu_narrow_bwd_kernel<decltype(act)::value>), grid, wg, 0, s, a, b);
      });
    }
    return (b.dw || b.dbias) && b.splits > 1 ? launch_lin_reduce(b, s) : hipGetLastError();
  }
  const hipError_t e = dtype == TRIATTN_BF16 ? launch<bf16, true>(a, s) : launch<float, true>(a, s);
  return e != hipSuccess ? e : launch_lin_made(dtype, b, whole(dtype, a.k, a.f), s);
}

}  // namespace triattn
