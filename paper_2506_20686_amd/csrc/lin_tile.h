// Tiles, staging and products of the linear projections (lin.hip, glu.hip).
#pragma once

#include "dma.h"
#include "ops.h"
#include "triattn.h"

namespace triattn {
namespace {

// Activations of fp32 tensors keep fp32's bits in the tails too: value and derivative are
// good to 14 half steps of themselves (the derivative, of its two terms).  With bf16
// tensors the linear projection's z is known to 8 bits, so the hardware's exponential and
// reciprocal serve as they are: near 0 both are as good, and far out an exponential of a is off
// by |a| half steps.
// (In full they cost a bf16 forward of 589,824 x 128 x 128 15%: 100 -> 115 us with gelu.)

// exp(a), and exp(a + b) with |b| below a's last place, for -2^20 < a <= 0: the hardware's
// power of two of the rounded a log2(e), then what the rounding left of a, to first order.
__device__ inline float exp_part(float a, float& rest) {
  constexpr float LN2_LO = -1.90465430e-9f;  // ln(2) less LN2
  const float p = a * LOG2E;
  rest = fmaf(-p, LN2_LO, fmaf(-p, LN2, a));
  return __builtin_amdgcn_exp2f(p);
}
__device__ inline float exp_full(float a) {
  float rest;
  const float r = exp_part(a, rest);
  return fmaf(r, rest, r);
}
__device__ inline float exp_full(float a, float b) {
  float rest;
  const float r = exp_part(a, rest);
  return fmaf(r, rest + b, r);
}

// Phi(z) and exp(-z^2 / 2).  Phi(-a) = exp(-a^2 / 2) t R(t) with t = 1 / (1 + 0.26 a)
// (Hastings' form, Abramowitz and Stegun 7.1.23 to 7.1.28, whose own coefficients are good
// to 1.5e-7 of 1, not of Phi).  R is a polynomial in t - 1/2, which keeps its terms small
// beside the sum, of the degree that leaves a third of a half step: fitted for 0 <= a <=
// 13.5 by weighted least squares, largest relative error 2.2e-8.
template <bool FULL>
__device__ inline void normal_cdf(float z, float& cdf, float& e) {
  const float a = FULL ? fminf(fabsf(z), 20.f) : fabsf(z);  // exp(-200) is 0
  const float h = -0.5f * a, sq = h * a;
  e = FULL ? exp_full(sq, fmaf(h, a, -sq)) : __expf(sq);
  const float d = fmaf(a, 0.26f, 1.f), q = fast_rcp(d);
  // in full, one Newton step: t enters three times
  const float t = FULL ? fmaf(fmaf(-d, q, 1.f), q, q) : q, v = t - 0.5f;
  float r = 0.0307835574f;
  r = fmaf(v, r, -0.0310549279f);
  r = fmaf(v, r, -0.0698595991f);
  r = fmaf(v, r, 0.0147384053f);
  r = fmaf(v, r, 0.191496291f);
  r = fmaf(v, r, 0.343348547f);
  r = fmaf(v, r, 0.38113254f);
  r = fmaf(v, r, 0.309965674f);
  r = fmaf(v, r, 0.19560028f);
  const float tail = e * t * r;
  cdf = z < 0.f ? tail : 1.f - tail;
}
// sigmoid(z) and sigmoid(-z); in full neither is taken from 1, so both keep their bits.
template <bool FULL>
__device__ inline void sigmoid(float z, float& s, float& other) {
  if (FULL) {
    const float e = exp_full(-fminf(fabsf(z), 128.f));  // exp(-128) is 0
    const float big = fast_rcp(1.f + e), small = e * big;
    s = z < 0.f ? small : big;
    other = z < 0.f ? big : small;
  } else {
    s = fast_rcp(1.f + __expf(-z));
    other = 1.f - s;
  }
}

// The activation of tensors of T, and its derivative.
template <typename T>
__device__ inline float act_value(float z, int act) {
  if (act == TRIATTN_ACT_RELU) return z > 0.f ? z : 0.f;
  float p, q;
  if (act == TRIATTN_ACT_GELU) {
    normal_cdf<sizeof(T) == 4>(z, p, q);
    return z * p;
  }
  if (act == TRIATTN_ACT_SILU) {
    sigmoid<sizeof(T) == 4>(z, p, q);
    return z * p;
  }
  return z;
}

template <typename T>
__device__ inline float act_grad(float z, int act) {
  if (act == TRIATTN_ACT_RELU) return z > 0.f ? 1.f : 0.f;
  float p, q;
  if (act == TRIATTN_ACT_GELU) {
    normal_cdf<sizeof(T) == 4>(z, p, q);
    return p + z * 0.39894228040143268f * q;
  }
  if (act == TRIATTN_ACT_SILU) {
    sigmoid<sizeof(T) == 4>(z, p, q);
    return p * (1.f + z * q);
  }
  return 1.f;
}

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

// Eight consecutive elements as they lie in memory.
template <typename T>
struct Raw8 {
  static constexpr int N = (int)sizeof(T) / 2;  // 16-byte words
  u32x4 v[N];
};
template <typename T>
constexpr int WORD = 16 / (int)sizeof(T);  // elements of a 16-byte word
template <typename T>
__device__ inline void unpack(const Raw8<T>& r, float (&f)[8]) {
  struct E {
    T x[8];
  };
  const E e = __builtin_bit_cast(E, r);
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = (float)e.x[i];
}

struct __attribute__((packed)) Any16 {
  u32x4 v;
};

// The first `have` of 8 values (zeros after them); ALIGNED: whole words of them.  A
// partial chunk is 8 loads at once, those past its end of its last element.
template <typename T, bool ALIGNED>
__device__ inline Raw8<T> get8(const T* p, int have) {
  Raw8<T> r{};
  if (ALIGNED) {
#pragma unroll
    for (int i = 0; i < Raw8<T>::N; ++i)
      if (i * WORD<T> < have) r.v[i] = ((const u32x4*)p)[i];
  } else if (have >= 8) {
#pragma unroll
    for (int i = 0; i < Raw8<T>::N; ++i) r.v[i] = ((const Any16*)p)[i].v;
  } else {
    struct E {
      T e[8];
    } y;
#pragma unroll
    for (int i = 0; i < 8; ++i) y.e[i] = p[min(i, have - 1)];
#pragma unroll
    for (int i = 1; i < 8; ++i)
      if (i >= have) y.e[i] = (T)0.f;
    r = __builtin_bit_cast(Raw8<T>, y);
  }
  return r;
}

// A row-major matrix [rows][cols] seen from a tile's corner.
template <typename T>
struct Mat {
  const T* p;
  int64_t rows;
  int cols;
};

// Chunk (r, c .. c + 7) of the window at (r0, c0) of a matrix whose rows are whole 16-byte
// words, `lim` rows high: zeros outside.  A word is all in or all out, and the buffer
// resource's range check gives the zeros.
template <typename T>
__device__ inline Raw8<T> fetch(const Mat<T>& m, int64_t r0, int c0, int lim, int r, int c) {
  Raw8<T> x;
  // rows of the window inside the matrix; the step after the last one may lie past the end,
  // and `lim` be negative there
  const int64_t left = c0 < m.cols ? m.rows - r0 : 0, high = left < lim ? left : lim;
  const int rows = high > 0 ? (int)high : 0;
  const T* base = m.p + r0 * m.cols + c0;
  // the last row's end past the corner; a row is at most 32 KB, a window 4 MB
  const rsrc_t rs = buf_rsrc_n(base, rows ? (uint32_t)(rows * m.cols - c0) * sizeof(T) : 0u);
#pragma unroll
  for (int i = 0; i < Raw8<T>::N; ++i) {
    const int ci = c + i * WORD<T>;
    const uint32_t off = c0 + ci < m.cols ? (uint32_t)(r * m.cols + ci) * sizeof(T) : 0x80000000u;
    x.v[i] = __builtin_bit_cast(u32x4,
                                __builtin_amdgcn_raw_buffer_load_b128(rs, (int)off, 0, 0));
  }
  return x;
}

// The same of any width: rows start at any element (16-byte loads may), a row's last chunk
// runs on into the next row, and what would pass the matrix's end is read from its last 8
// elements.  `info` says what to make of it once it is needed (in repair): the valid
// elements in bits 0..3, how far they lie behind in bits 4..6.  So nothing waits for a load
// before its values are stored.  Matrices of fewer than 8 elements go element by
// element.
template <typename T>
__device__ inline Raw8<T> fetch_any(const Mat<T>& m, int64_t r0, int c0, int lim, int r, int c,
                                    int& info, int half = 0) {
  // this matrix's rows (and their halves) are whole words after all
  if (m.cols % WORD<T> == 0 && half % WORD<T> == 0) {
    info = 8;
    return fetch<T>(m, r0, c0, lim, r, c);
  }
  const int64_t total = m.rows * m.cols, corner = r0 * m.cols + c0;
  const int have = r < lim && r0 + r < m.rows ? min(max(m.cols - (c0 + c), 0), 8) : 0;
  if (total < 8) {  // element by element, zeros past the end
    const rsrc_t rs = buf_rsrc_n(m.p, (uint32_t)total * sizeof(T));
    const uint32_t off = have > 0 ? (uint32_t)(corner + r * m.cols + c) * sizeof(T) : 0x80000000u;
    struct E {
      T e[8];
    } y;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if constexpr (sizeof(T) == 4)
        y.e[i] = __builtin_bit_cast(
            T, __builtin_amdgcn_raw_buffer_load_b32(rs, (int)(off + 4 * i), 0, 0));
      else
        y.e[i] = __builtin_bit_cast(
            T, __builtin_amdgcn_raw_buffer_load_b16(rs, (int)(off + 2 * i), 0, 0));
    }
    info = have;
    return __builtin_bit_cast(Raw8<T>, y);
  }
  // 32-bit offsets from the corner, or from the last 8 elements if it lies past those
  const int64_t last = total - 8, from = corner < last ? corner : last;
  const int room = last - from < 0x7fffffff ? (int)(last - from) : 0x7fffffff;
  const int at = r * m.cols + c + (int)(corner - from), in = min(at, room);
  info = have | (have > 0 ? (at - in) << 4 : 0);
  Raw8<T> x;
  if (have > 0) {
#pragma unroll
    for (int i = 0; i < Raw8<T>::N; ++i) x.v[i] = ((const Any16*)(m.p + from + in))[i].v;
  }
  return x;
}
template <typename T>
__device__ inline Raw8<T> repair(const Raw8<T>& x, int info) {
  if (info == 8) return x;
  struct E {
    T e[8];
  } y = __builtin_bit_cast(E, x);
#pragma unroll
  for (int bit = 1; bit < 8; bit *= 2)
    if (info & (bit << 4))
#pragma unroll
      for (int i = 0; i + bit < 8; ++i) y.e[i] = y.e[i + bit];
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (i >= (info & 15)) y.e[i] = (T)0.f;
  return __builtin_bit_cast(Raw8<T>, y);
}

// One operand's tile of R rows x BK contraction indices in LDS, as P planes of bf16.
// Reads of a fragment (32 rows x 16 indices: lane l holds row l % 32, indices
// 8 (l / 32) .. + 7) and the stores of staged chunks are free of bank conflicts whether
// the LDS serves 128 or 256 bytes a cycle: the 16-byte chunks of a K major row are
// permuted by XOR with a value that differs between any 8 (and, with the row's parity or
// row % 4, any 16) consecutive rows; the 64-byte pieces of a transposed tile's line by
// one that differs between the four lines of a transposing read.
template <int R, int BK, bool KM, int P>
struct Tile {
  static constexpr int PLANE = R * BK * 2;
  static constexpr int BYTES = P * PLANE;
  static constexpr int LINE = KM ? BK / 8 : R / 8;  // chunks of a line
  __device__ static inline int chunk_at(int line, int c) {
    if constexpr (KM) {
      static_assert(BK == 64 || BK == 32, "chunks of a line");
      const int s = BK == 64 ? (line & 7) ^ ((line >> 3) & 1) : swz(line);
      return (line * LINE + (c ^ s)) * 16;
    } else {
      static_assert(R == 128 || R == 64, "chunks of a line");
      const int s = R == 128 ? (line & 3) << 2 : ((line >> 1) & 1) << 2;
      return (line * LINE + (c ^ s)) * 16;
    }
  }
  // Fragment of rows r0 .. r0 + 31, indices k0 .. k0 + 15.
  __device__ static inline bf16x8 frag(const char* plane, int r0, int k0, int lane) {
    if constexpr (KM) {
      return *(const bf16x8*)(plane + chunk_at(r0 + (lane & 31), (k0 >> 3) + (lane >> 5)));
    } else {
      // lane 4 e + j of a group of 16 gives 8 bytes (rows r0 + 16 G + 4 j .. + 3) of index
      // k0 + 8 g + e (+ 4) and receives its own row's four indices
      const int i = lane & 15, row = r0 + (lane & 16) + 4 * (i & 3);
      const int k = k0 + 8 * (lane >> 5) + (i >> 2);
      typedef TRIATTN_LDS s16x4* lds4;
      const char* a = plane + chunk_at(k, row >> 3) + (row & 4) * 2;
      const char* b = plane + chunk_at(k + 4, row >> 3) + (row & 4) * 2;
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(uintptr_t)lds_addr(a));
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(uintptr_t)lds_addr(b));
      return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
  }
};

// What dz is made of in the staging: the tensor itself; dout where z > 0; dout act'(z); (not in
// the staging) dz made beforehand; or made and split beforehand, its planes of bf16 one after
// the other.
enum Dz { DZ_X, DZ_RELU, DZ_ACT, DZ_MADE, DZ_PLANES };

// Staging of one operand: this thread's chunks of a tile, from memory to LDS.  GATED: the
// matrix is two side by side (cols / 2 columns each), and a tile holds R / 2 columns of both, 8
// of the first, the same 8 of the second, and so on.
template <typename T, int R, int BK, bool KM, int P, int DZ, bool ALIGNED, bool GATED = false>
struct Stage {
  using L = Tile<R, BK, KM, P>;
  static constexpr int N = R * BK / 8 / 256;  // chunks a thread
  static constexpr bool SPLIT = DZ == DZ_PLANES, WITH_Z = DZ == DZ_RELU || DZ == DZ_ACT;
  static_assert(!SPLIT || ALIGNED, "planes of whole words");
  Raw8<T> x[SPLIT ? P * N : N], z[WITH_Z ? N : 1];
  int info[ALIGNED ? 1 : N];

  // Tile at rows i0, indices k0 (of k1): lines are rows (K major) or indices.
  __device__ inline void load(const Mat<T>& m, const T* zp, int64_t i0, int64_t k0, int64_t k1) {
    Mat<T> w = m;
    if (!KM && ALIGNED) w.rows = k1;
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const int id = (int)threadIdx.x + 256 * u, line = id / L::LINE, ch = id % L::LINE;
      const int half = GATED ? m.cols / 2 : 0;
      const int c = GATED ? 8 * (ch >> 1) + (ch & 1) * half : 8 * ch;
      const int64_t r0 = KM ? i0 : k0;
      const int c0 = (int)(KM ? k0 : i0);
      if constexpr (SPLIT) {
#pragma unroll
        for (int p = 0; p < P; ++p)
          x[P * u + p] = fetch<T>(Mat<T>{m.p + p * m.rows * m.cols, w.rows, w.cols}, r0, c0,
                                  KM ? R : BK, line, c);
      } else if constexpr (ALIGNED) {
        x[u] = fetch<T>(w, r0, c0, KM ? R : BK, line, c);
        if constexpr (WITH_Z)
          z[u] = fetch<T>(Mat<T>{zp, w.rows, w.cols}, r0, c0, KM ? R : BK, line, c);
      } else {
        const int lim = KM ? R : (int)(k1 - k0 < BK ? k1 - k0 : BK);
        x[u] = fetch_any<T>(w, r0, c0, lim, line, c, info[u], half);
        if constexpr (WITH_Z) {
          int same;
          z[u] = fetch_any<T>(Mat<T>{zp, w.rows, w.cols}, r0, c0, lim, line, c, same);
        }
      }
    }
  }
  __device__ inline Raw8<T> raw(const Raw8<T>& r, int u) const {
    if constexpr (ALIGNED) return r;
    else return repair(r, info[u]);
  }
  // The values of chunk u.
  __device__ inline void values(int u, int act, float (&f)[8]) const {
    unpack(raw(x[SPLIT ? P * u : u], u), f);
    if constexpr (SPLIT) {  // the smaller planes together first
      float g[8], h[8];
      static_assert(P == 3, "planes");
      unpack(x[P * u + 1], g);
      unpack(x[P * u + 2], h);
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] += g[e] + h[e];
    }
    if constexpr (WITH_Z) {
      float g[8];
      unpack(raw(z[u], u), g);
#pragma unroll
      for (int e = 0; e < 8; ++e)
        f[e] = DZ == DZ_RELU ? (g[e] > 0.f ? f[e] : 0.f) : f[e] * act_grad<T>(g[e], act);
    }
  }
  // Stores the planes; with SUM, adds the values to the thread's column sums (its chunks
  // lie in the same columns of every line).
  template <bool SUM>
  __device__ inline void store(char* tile, int act, bool sum, float (&col)[8]) const {
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const int id = (int)threadIdx.x + 256 * u;
      char* d = tile + L::chunk_at(id / L::LINE, id % L::LINE);
      float f[8];
      if ((!SPLIT && (P > 1 || WITH_Z)) || SUM) values(u, act, f);
      if (SUM && sum) {
#pragma unroll
        for (int e = 0; e < 8; ++e) col[e] += f[e];
      }
      if constexpr (SPLIT) {
#pragma unroll
        for (int p = 0; p < P; ++p) *(u32x4*)(d + p * L::PLANE) = x[P * u + p].v[0];
      } else if constexpr (P == 1 && DZ == DZ_X) {
        *(u32x4*)d = raw(x[u], u).v[0];
      } else {
#pragma unroll
        for (int p = 0; p < P; ++p) {
          bf16x8 b;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            b[e] = (bf16)f[e];
            if (p + 1 < P) f[e] -= (float)b[e];
          }
          *(bf16x8*)(d + p * L::PLANE) = b;
        }
      }
    }
  }
};

// C tile (rows i0 .. i0 + R - 1, columns j0 .. j0 + R - 1) = sum over indices [k0, k1) of
// A(i, k) B(k, j), in registers: acc[u][v] of wave (wi, wj) holds rows wi R/2 + 32 u + l % 32
// and columns wj R/2 + 32 v + accumulator rows (acc_row).
template <typename TA, typename TB, int R, int BK, bool AKM, bool BKM, int PA, int PB, int DZA,
          int DZB, bool ALIGNED, bool SUM, bool GATED = false>
struct Product {
  static constexpr int NT = R / 64;  // 32-wide tiles of a wave, each way
  using SA = Stage<TA, R, BK, AKM, PA, DZA, ALIGNED>;
  using SB = Stage<TB, R, BK, BKM, PB, DZB, ALIGNED, GATED>;
  using LA = typename SA::L;
  using LB = typename SB::L;
  static constexpr int BUF = LA::BYTES + LB::BYTES;
  // steps whose loads are in flight: two where the registers allow three workgroups on a CU,
  // one where rows are ragged
  static constexpr int D = R == 64 && ALIGNED ? 2 : 1;
  static constexpr int EPI = 4 * 32 * (R / 2 + 4) * 4;  // the result's staging
  static constexpr int LDS = 2 * BUF > EPI ? 2 * BUF : EPI;

  __device__ static inline void run(char* lds, const Mat<TA>& a, const TA* az, const Mat<TB>& b,
                                    const TB* bz, int act, int64_t i0, int j0, int64_t k0,
                                    int64_t k1, bool sum, float (&col)[8],
                                    f32x16 (&acc)[NT][NT]) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int ri = (wave >> 1) * (R / 2), rj = (wave & 1) * (R / 2);
#pragma unroll
    for (int u = 0; u < NT; ++u)
#pragma unroll
      for (int v = 0; v < NT; ++v) acc[u][v] = f32x16{};
    // Loads run D steps ahead and without a condition (past the end they give zeros and
    // touch no memory), so that a step waits for its own loads only.
    const int steps = (int)((k1 - k0 + BK - 1) / BK);
    SA sa[D];
    SB sb[D];
    auto load = [&](int d, int it) {
      sa[d].load(a, az, i0, k0 + (int64_t)it * BK, k1);
      sb[d].load(b, bz, j0, k0 + (int64_t)it * BK, k1);
    };
    auto step = [&](int d, char* buf, int it) {
      const int next = it + D;
      const int64_t left = k1 - k0 - (int64_t)it * BK;  // indices of this step and on
      float none[8];
      sa[d].template store<false>(buf, act, false, none);
      sb[d].template store<SUM>(buf + LA::BYTES, act, sum, col);
      load(d, next);
      // this buffer was last read two steps ago, before the barrier of the last step
      __syncthreads();
      multiply(buf, ri, rj, lane, left, acc);
    };
#pragma unroll
    for (int d = 0; d < D; ++d) load(d, d);
    // Ragged fp32 operands have the longest code by far (repair and split of both), so where
    // few steps run it, one copy of a step and its loads instead of two.  One copy against two:
    // gradients at 2777 x 449 x 131 (5 and 6 steps) 20.6 and 24.6 us; at 25,152 x 453 x 1179
    // (37 and 132) 886 and 840, at 40 x 1001 x 1001 (32 and 2) 52 and 47.
    constexpr bool LONG = !ALIGNED && sizeof(TA) == 4 && sizeof(TB) == 4;
    if (!LONG || steps >= 16) {
      int it = 0;
      for (; it + 2 <= steps; it += 2) {
        step(0, lds, it);
        step(D - 1, lds + BUF, it + 1);
      }
      if (it < steps) step(0, lds, it);
    } else {
      for (int it = 0; it < steps; ++it) step(0, lds + (it & 1) * BUF, it);
    }
  }

  __device__ static inline void multiply(const char* buf, int ri, int rj, int lane, int64_t left,
                                         f32x16 (&acc)[NT][NT]) {
#pragma unroll
    for (int kk = 0; kk < BK; kk += 16) {
      if (kk > 0 && kk >= left) break;
      bf16x8 fa[PA][NT], fb[PB][NT];
#pragma unroll
      for (int p = 0; p < PA; ++p)
#pragma unroll
        for (int u = 0; u < NT; ++u)
          fa[p][u] = LA::frag(buf + p * LA::PLANE, ri + 32 * u, kk, lane);
#pragma unroll
      for (int p = 0; p < PB; ++p)
#pragma unroll
        for (int v = 0; v < NT; ++v)
          fb[p][v] = LB::frag(buf + LA::BYTES + p * LB::PLANE, rj + 32 * v, kk, lane);
      // plane products down to 2^-24 of the whole, the smallest first
      constexpr int MOST = (PA > PB ? PA : PB) - 1;
#pragma unroll
      for (int order = MOST; order >= 0; --order)
#pragma unroll
        for (int p = 0; p < PA; ++p) {
          const int q = order - p;
          if (q < 0 || q >= PB) continue;
#pragma unroll
          for (int u = 0; u < NT; ++u)
#pragma unroll
            for (int v = 0; v < NT; ++v)
              acc[u][v] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fb[q][v], fa[p][u], acc[u][v], 0,
                                                                  0, 0);
        }
    }
  }

  // The result is handed out 8 consecutive columns at a time: piece t of PIECES of this
  // thread lies at row piece_row(t), column piece_col() of the tile.
  static constexpr int W = R / 2, PER = 64 / (W / 8), PIECES = NT * 32 / PER;
  __device__ static inline int piece_row(int t) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    return (wave >> 1) * W + PER * t + lane / (W / 8);
  }
  __device__ static inline int piece_col() {
    return ((threadIdx.x >> 6) & 1) * W + 8 * ((threadIdx.x & 63) % (W / 8));
  }
  // f(t, values) for every piece: through LDS, 32 rows a wave at a time, so that the
  // accesses f makes are whole rows' pieces.
  template <typename F>
  __device__ static inline void result(char* lds, const f32x16 (&acc)[NT][NT], F f) {
    constexpr int ROW = W + 4;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    float* mine = (float*)lds + wave * 32 * ROW;
    const int j = 8 * (lane % (W / 8));
#pragma unroll
    for (int u = 0; u < NT; ++u) {
      __syncthreads();
#pragma unroll
      for (int v = 0; v < NT; ++v)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const f32x16& c = acc[u][v];
          *(f32x4*)(mine + (lane & 31) * ROW + 32 * v + 8 * q + 4 * (lane >> 5)) =
              f32x4{c[4 * q], c[4 * q + 1], c[4 * q + 2], c[4 * q + 3]};
        }
      __syncthreads();
#pragma unroll
      for (int s = 0; s < 32; s += PER) {
        const int i = s + lane / (W / 8);
        float o[8];
#pragma unroll
        for (int e = 0; e < 8; e += 4) {
          const f32x4 x = *(const f32x4*)(mine + i * ROW + j + e);
          o[e] = x[0], o[e + 1] = x[1], o[e + 2] = x[2], o[e + 3] = x[3];
        }
        f((32 * u + s) / PER, o);
      }
    }
  }

  // The same of a gated product: f(t, a, b) with 8 columns of the first half and the same 8 of
  // the second; piece t of PAIRS at row pair_row(t), column pair_col() of either.
  static constexpr int PER2 = 64 / (W / 16), PAIRS = NT * 32 / PER2;
  __device__ static inline int pair_row(int t) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    return (wave >> 1) * W + PER2 * t + lane / (W / 16);
  }
  __device__ static inline int pair_col() {
    return ((threadIdx.x >> 6) & 1) * (W / 2) + 8 * ((threadIdx.x & 63) % (W / 16));
  }
  template <typename F>
  __device__ static inline void pairs(char* lds, const f32x16 (&acc)[NT][NT], F f) {
    constexpr int ROW = W + 4;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    float* mine = (float*)lds + wave * 32 * ROW;
    const int j = 16 * (lane % (W / 16));
#pragma unroll
    for (int u = 0; u < NT; ++u) {
      __syncthreads();
#pragma unroll
      for (int v = 0; v < NT; ++v)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const f32x16& c = acc[u][v];
          *(f32x4*)(mine + (lane & 31) * ROW + 32 * v + 8 * q + 4 * (lane >> 5)) =
              f32x4{c[4 * q], c[4 * q + 1], c[4 * q + 2], c[4 * q + 3]};
        }
      __syncthreads();
#pragma unroll
      for (int s = 0; s < 32; s += PER2) {
        const int i = s + lane / (W / 16);
        float o[16];
#pragma unroll
        for (int e = 0; e < 16; e += 4) {
          const f32x4 x = *(const f32x4*)(mine + i * ROW + j + e);
          o[e] = x[0], o[e + 1] = x[1], o[e + 2] = x[2], o[e + 3] = x[3];
        }
        float a[8], b[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) a[e] = o[e], b[e] = o[8 + e];
        f((32 * u + s) / PER2, a, b);
      }
    }
  }
};

// Writes the first `have` of 8 values to p; ALIGNED: whole words of them.
template <typename T, bool ALIGNED>
__device__ inline void put_raw(T* p, int have, const Raw8<T>& r) {
  if (ALIGNED) {
#pragma unroll
    for (int i = 0; i < Raw8<T>::N; ++i)
      if (i * WORD<T> < have) ((u32x4*)p)[i] = r.v[i];
  } else if (have >= 8) {
#pragma unroll
    for (int i = 0; i < Raw8<T>::N; ++i) ((Any16*)p)[i].v = r.v[i];
  } else {
    struct E {
      T e[8];
    } y = __builtin_bit_cast(E, r);
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < have) p[i] = y.e[i];
  }
}
template <typename T, bool ALIGNED>
__device__ inline void put8(T* p, int have, const float (&f)[8]) {
  struct E {
    T e[8];
  } y;
#pragma unroll
  for (int i = 0; i < 8; ++i) y.e[i] = (T)f[i];
  put_raw<T, ALIGNED>(p, have, __builtin_bit_cast(Raw8<T>, y));
}

// Contraction indices a step: 64 while the two buffers leave room for two workgroups on a
// CU, else 32 (three planes of each operand, or of one and 128 rows).
constexpr int step_k(int r, int planes) { return r * planes <= 256 ? 64 : 32; }
template <typename T>
constexpr int planes() {
  return sizeof(T) == 2 ? 1 : 3;
}

// Floats of one split's partial sums: dw, then dbias.
__host__ __device__ inline int64_t slab_floats(int k, int n) {
  return ((int64_t)k * n + n + 3) / 4 * 4;
}

struct Square {  // lines of 128 bf16, read along and across
  // Both reads are free of bank conflicts: s differs between any 16 consecutive lines
  // (its low three bits between 8) for 16-byte reads down the lines, and its bits 3, 2 as
  // well as its bits 2, 1 between the four lines of a transposing read.
  __device__ static inline int chunk_at(int line, int c) {
    const int e = line & 3, s = ((e ^ (e << 1)) << 1) ^ ((line >> 2) & 3);
    return (line * 16 + (c ^ s)) * 16;
  }
  // lines r0 .. + 31 as rows, columns k0 .. + 15 as indices
  __device__ static inline bf16x8 along(const char* t, int r0, int k0, int lane) {
    return *(const bf16x8*)(t + chunk_at(r0 + (lane & 31), (k0 >> 3) + (lane >> 5)));
  }
  // columns r0 .. + 31 as rows, lines k0 .. + 15 as indices
  __device__ static inline bf16x8 across(const char* t, int r0, int k0, int lane) {
    const int i = lane & 15, col = r0 + (lane & 16) + 4 * (i & 3);
    const int line = k0 + 8 * (lane >> 5) + (i >> 2);
    typedef TRIATTN_LDS s16x4* lds4;
    const char* a = t + chunk_at(line, col >> 3) + (col & 4) * 2;
    const char* b = t + chunk_at(line + 4, col >> 3) + (col & 4) * 2;
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(uintptr_t)lds_addr(a));
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(uintptr_t)lds_addr(b));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  }
};

}  // namespace
}  // namespace triattn
