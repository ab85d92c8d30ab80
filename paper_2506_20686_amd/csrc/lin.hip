// Linear projection with bias, activation and residual, and its backward:
//   forward  z = x W + bias, out = act(z) + residual      contraction over k
//   dx = dz W^T, dz = dout act'(z)                        contraction over n
//   dW = x^T dz, dbias = column sums of dz                contraction over the m rows
//
// All three products run through one kernel body: a workgroup of 4 waves (2 x 2) makes an
// R x R tile of the result, R = 128 or 64, staging tiles of both operands through
// registers into two LDS buffers in turn, and multiplies them on the matrix cores (bf16
// 32 x 32 x 16, fp32 sums).  The loads of the next tile, or two, are in flight while one
// is multiplied; one barrier a step.
//
// Operands: a tile is stored as it lies in memory, either [row][contraction] ("K major":
// fragments are 16-byte reads) or [contraction][row] (fragments are the LDS's transposing
// reads), so neither W, W^T nor x^T is ever copied.
//
// Precision: an fp32 value is the sum of three bf16 (8 bits each, rounded to nearest), so fp32
// operands are staged as three planes and a product is the six plane products above 2^-24 of it;
// sums are fp32 throughout.  (The matrix cores take subnormal bf16 as they are, so the third plane
// ends at 2^-133: values below 2^-110 keep fewer bits.)  Six bf16 instructions for what would be 8
// fp32 ones of four times the length each.  With bf16 tensors, dz of a smooth activation is not a
// bf16 value: it enters dx and dW as three planes.  (dx is rounded to bf16 itself, but where its
// sum cancels, the cut of a dz to two planes, 16 bits, would show.)
//
// Every sum over rows is split over workgroups; their partial sums, in the workspace, are
// added in a fixed order.
#include "dma.h"
#include "ops.h"
#include "timing.h"
#include "triattn.h"

namespace triattn {
namespace {

// Activations of fp32 tensors keep fp32's bits in the tails too: value and derivative are
// good to 14 half steps of themselves (the derivative, of its two terms).  With bf16
// tensors z is known to 8 bits, so the hardware's exponential and reciprocal serve as they
// are: near 0 both are as good, and far out an exponential of a is off by |a| half steps.
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
                                    int& info) {
  if (m.cols % WORD<T> == 0) {  // this matrix's rows are whole words after all
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

// What dz is made of in the staging: the tensor itself; dout where z > 0; dout act'(z); and
// (not in the staging) dz made beforehand.
enum Dz { DZ_X, DZ_RELU, DZ_ACT, DZ_MADE };

// Staging of one operand: this thread's chunks of a tile, from memory to LDS.
template <typename T, int R, int BK, bool KM, int P, int DZ, bool ALIGNED>
struct Stage {
  using L = Tile<R, BK, KM, P>;
  static constexpr int N = R * BK / 8 / 256;  // chunks a thread
  Raw8<T> x[N], z[DZ == DZ_X ? 1 : N];
  int info[ALIGNED ? 1 : N];

  // Tile at rows i0, indices k0 (of k1): lines are rows (K major) or indices.
  __device__ inline void load(const Mat<T>& m, const T* zp, int64_t i0, int64_t k0, int64_t k1) {
    Mat<T> w = m;
    if (!KM && ALIGNED) w.rows = k1;
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const int id = (int)threadIdx.x + 256 * u, line = id / L::LINE, c = 8 * (id % L::LINE);
      const int64_t r0 = KM ? i0 : k0;
      const int c0 = (int)(KM ? k0 : i0);
      if constexpr (ALIGNED) {
        x[u] = fetch<T>(w, r0, c0, KM ? R : BK, line, c);
        if constexpr (DZ != DZ_X)
          z[u] = fetch<T>(Mat<T>{zp, w.rows, w.cols}, r0, c0, KM ? R : BK, line, c);
      } else {
        const int lim = KM ? R : (int)(k1 - k0 < BK ? k1 - k0 : BK);
        x[u] = fetch_any<T>(w, r0, c0, lim, line, c, info[u]);
        if constexpr (DZ != DZ_X) {
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
    unpack(raw(x[u], u), f);
    if constexpr (DZ != DZ_X) {
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
      if (P > 1 || DZ != DZ_X || SUM) values(u, act, f);
      if (SUM && sum) {
#pragma unroll
        for (int e = 0; e < 8; ++e) col[e] += f[e];
      }
      if constexpr (P == 1 && DZ == DZ_X) {
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
          int DZB, bool ALIGNED, bool SUM>
struct Product {
  static constexpr int NT = R / 64;  // 32-wide tiles of a wave, each way
  using SA = Stage<TA, R, BK, AKM, PA, DZA, ALIGNED>;
  using SB = Stage<TB, R, BK, BKM, PB, DZB, ALIGNED>;
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

// Forward.  589,824 x 128 x 128 bf16 with residual: 87 us, 5.2 TB/s; 32,768 x 1024 x 512: 45 to 54
// us on different cards, 640 to 750 TFLOP/s, LDS reads and staging beside the products; 16,384 x
// 1024 x 1024 fp32: 150 TFLOP/s.  Two workgroups on a CU (bf16) hide one's loads and epilogue
// behind the other's products.
template <typename T, int R, bool ALIGNED>
__global__ __launch_bounds__(256, sizeof(T) == 2 ? 2 : 1) void lin_fwd_kernel(LinArgs a) {
  using G = Product<T, T, R, step_k(R, 2 * planes<T>()), true, false, planes<T>(), planes<T>(), DZ_X,
                    DZ_X, ALIGNED, false>;
  __shared__ __attribute__((aligned(16))) char lds[G::LDS];
  const int nj = (a.n + R - 1) / R, wg = xcd_swizzle(blockIdx.x, gridDim.x);
  const int64_t i0 = (int64_t)(wg / nj) * R;
  const int j0 = (wg % nj) * R;
  // what the epilogue reads is on its way before the product: the product of a narrow
  // projection is shorter than a memory access
  const int j = j0 + G::piece_col(), have = a.n - j;
  // (ragged rows have no registers to spare for the residual)
  Raw8<T> res[ALIGNED ? G::PIECES : 1];
  float bias[8] = {};
  if (ALIGNED && a.residual) {
#pragma unroll
    for (int t = 0; t < G::PIECES; ++t) {
      const int64_t i = i0 + G::piece_row(t);
      if (i < a.m && have > 0) res[t] = get8<T, ALIGNED>((const T*)a.residual + i * a.n + j, have);
    }
  }
  if (a.bias && have > 0) unpack(get8<T, ALIGNED>((const T*)a.bias + j, have), bias);
  f32x16 acc[G::NT][G::NT];
  float none[8];
  G::run(lds, Mat<T>{(const T*)a.x, a.m, a.k}, nullptr, Mat<T>{(const T*)a.w, a.k, a.n}, nullptr,
         0, i0, j0, 0, a.k, false, none, acc);
  G::result(lds, acc, [&](int t, float (&o)[8]) {
    const int64_t i = i0 + G::piece_row(t), at = i * a.n + j;
    if (i >= a.m || have <= 0) return;
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] += bias[e];
    if (a.z) put8<T, ALIGNED>((T*)a.z + at, have, o);
    if (a.act != TRIATTN_ACT_NONE) {
#pragma unroll
      for (int e = 0; e < 8; ++e) o[e] = act_value<T>(o[e], a.act);
    }
    if (a.residual) {
      float r[8];
      if constexpr (ALIGNED) unpack(res[t], r);
      else unpack(get8<T, false>((const T*)a.residual + at, have), r);
#pragma unroll
      for (int e = 0; e < 8; ++e) o[e] += r[e];
    }
    put8<T, ALIGNED>((T*)a.out + at, have, o);
  });
}

// What dz is read from, and as what: the call's dout (and z) in its own type, or the fp32
// dz that lin_dz_kernel made of them.  P: planes of dz.
template <typename T, int DZ>
struct DzSource {
  using E = T;
  static constexpr int STAGE = DZ, P = sizeof(T) == 4 || DZ == DZ_ACT ? 3 : 1;
};
template <typename T>
struct DzSource<T, DZ_MADE> {
  using E = float;
  static constexpr int STAGE = DZ_X, P = 3;
};

// dz = dout act'(z) in fp32, where several column tiles of dx and dW would each form it again from
// the two tensors (an exponential an element).  Bound by memory and a launch: 1500 x 1536 in 8.5
// us; 1500 x 384 x 1536 backward with it 41 us, without 71; 16,384 x 512 x 2048 with it 271,
// without 412.
template <typename T>
__global__ __launch_bounds__(256) void lin_dz_kernel(LinBwdArgs a) {
  const int64_t all = a.m * a.n;
  for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8; i < all;
       i += (int64_t)gridDim.x * 2048) {
    const int have = all - i < 8 ? (int)(all - i) : 8;
    float d[8], z[8];
    unpack(get8<T, false>((const T*)a.dout + i, have), d);
    unpack(get8<T, false>((const T*)a.z + i, have), z);
#pragma unroll
    for (int e = 0; e < 8; ++e) d[e] *= act_grad<T>(z[e], a.act);
    put8<float, false>(a.dz + i, have, d);
  }
}

// dx = dz W^T: W's rows are the columns of dx, its columns the contraction.  Bound by memory
// for few columns (294,912 x 256 x 128 bf16 in 128-wide tiles: 45 us, 5.0 TB/s), by LDS reads
// and, with planes, by the matrix cores for many (16,384 x 512 x 2048 with GELU: 106 us, and dW
// 106, three plane products each, 970 TFLOP/s of matrix instructions).
template <typename T, int R, int DZ, bool ALIGNED>
using DxProduct = Product<typename DzSource<T, DZ>::E, T, R,
                          step_k(R, DzSource<T, DZ>::P + planes<T>()), true, true,
                          DzSource<T, DZ>::P, planes<T>(), DzSource<T, DZ>::STAGE, DZ_X, ALIGNED,
                          false>;
template <typename T, int R, int DZ, bool ALIGNED>
__device__ inline void dx_tile(const LinBwdArgs& a, char* lds, int wg) {
  using E = typename DzSource<T, DZ>::E;
  using G = DxProduct<T, R, DZ, ALIGNED>;
  const int nj = (a.k + R - 1) / R;
  const int64_t i0 = (int64_t)(wg / nj) * R;
  const int j0 = (wg % nj) * R;
  const E* src = DZ == DZ_MADE ? (const E*)a.dz : (const E*)a.dout;
  f32x16 acc[G::NT][G::NT];
  float none[8];
  G::run(lds, Mat<E>{src, a.m, a.n}, (const E*)a.z, Mat<T>{(const T*)a.w, a.k, a.n}, nullptr,
         a.act, i0, j0, 0, a.n, false, none, acc);
  const int j = j0 + G::piece_col(), have = a.k - j;
  G::result(lds, acc, [&](int t, float (&o)[8]) {
    const int64_t i = i0 + G::piece_row(t);
    if (i < a.m && have > 0) put8<T, ALIGNED>((T*)a.dx + i * a.k + j, have, o);
  });
}

// Rows of a split, a multiple of the largest step.
__host__ __device__ inline int64_t split_rows(int64_t m, int splits) {
  const int64_t per = (m + splits - 1) / splits;
  return (per + 63) / 64 * 64;
}
// Floats of one split's partial sums: dw, then dbias.
__host__ __device__ inline int64_t slab_floats(int k, int n) {
  return ((int64_t)k * n + n + 3) / 4 * 4;
}

// One split's dW tile and, in the first row of tiles, its dbias.  Without splits the
// results themselves.  The rows are split so that the GPU is full although dW has few tiles.
template <typename T, int R, int DZ, bool ALIGNED>
using DwProduct = Product<T, typename DzSource<T, DZ>::E, R,
                          step_k(R, planes<T>() + DzSource<T, DZ>::P), false, false, planes<T>(),
                          DzSource<T, DZ>::P, DZ_X, DzSource<T, DZ>::STAGE, ALIGNED, true>;
template <typename T, int R, int DZ, bool ALIGNED>
__device__ inline void dw_tile(const LinBwdArgs& a, char* lds, int wg) {
  using E = typename DzSource<T, DZ>::E;
  using G = DwProduct<T, R, DZ, ALIGNED>;
  const int ni = (a.k + R - 1) / R, nj = (a.n + R - 1) / R;
  const int split = wg / (ni * nj);
  const int i0 = wg % (ni * nj) / nj * R, j0 = wg % nj * R;
  const int64_t per = split_rows(a.m, a.splits), k0 = split * per;
  const int64_t k1 = k0 + per < a.m ? k0 + per : a.m;
  const bool sum = i0 == 0 && a.dbias != nullptr;
  float* dw = a.splits > 1 ? a.part + split * slab_floats(a.k, a.n) : a.dw;
  float* db = a.splits > 1 ? dw + (int64_t)a.k * a.n : a.dbias;
  f32x16 acc[G::NT][G::NT];
  float col[8] = {};
  const E* src = DZ == DZ_MADE ? (const E*)a.dz : (const E*)a.dout;
  G::run(lds, Mat<T>{(const T*)a.x, a.m, a.k}, nullptr, Mat<E>{src, a.m, a.n}, (const E*)a.z,
         a.act, i0, j0, k0, k1, sum, col, acc);
  const int j = j0 + G::piece_col(), have = a.n - j;
  if (a.dw)
    G::result(lds, acc, [&](int t, float (&o)[8]) {
      const int i = i0 + G::piece_row(t);
      if (i < a.k && have > 0) put8<float, ALIGNED>(dw + (int64_t)i * a.n + j, have, o);
    });
  if (sum) {  // the threads of a column chunk, in order
    constexpr int C = R / 8;
    __syncthreads();
    float* part = (float*)lds;
#pragma unroll
    for (int e = 0; e < 8; ++e) part[threadIdx.x / C * R + threadIdx.x % C * 8 + e] = col[e];
    __syncthreads();
    if ((int)threadIdx.x < R && j0 + (int)threadIdx.x < a.n) {
      float s = 0.f;
      for (int t = 0; t < 256 / C; ++t) s += part[t * R + threadIdx.x];
      db[j0 + threadIdx.x] = s;
    }
  }
}

template <typename T, int R, int DZ, bool ALIGNED>
__global__ __launch_bounds__(256) void lin_bwd_dx_kernel(LinBwdArgs a) {
  __shared__ __attribute__((aligned(16))) char lds[DxProduct<T, R, DZ, ALIGNED>::LDS];
  dx_tile<T, R, DZ, ALIGNED>(a, lds, xcd_swizzle(blockIdx.x, gridDim.x));
}
template <typename T, int R, int DZ, bool ALIGNED>
__global__ __launch_bounds__(256) void lin_bwd_w_kernel(LinBwdArgs a) {
  __shared__ __attribute__((aligned(16))) char lds[DwProduct<T, R, DZ, ALIGNED>::LDS];
  dw_tile<T, R, DZ, ALIGNED>(a, lds, xcd_swizzle(blockIdx.x, gridDim.x));
}
// Both in one launch, where dx does not fill the GPU: the first ndx workgroups make dx, the others
// dW (in tiles of RW).  1500 x 384 x 1536 with GELU: 28 us, where the two take 27 and 20.
template <typename T, int RW, int DZ, bool ALIGNED>
__global__ __launch_bounds__(256) void lin_bwd_both_kernel(LinBwdArgs a, int ndx) {
  constexpr int LX = DxProduct<T, 64, DZ, ALIGNED>::LDS, LW = DwProduct<T, RW, DZ, ALIGNED>::LDS;
  __shared__ __attribute__((aligned(16))) char lds[LX > LW ? LX : LW];
  const int wg = blockIdx.x, ndw = (int)gridDim.x - ndx;
  if (wg < ndx)
    dx_tile<T, 64, DZ, ALIGNED>(a, lds, xcd_swizzle(wg, ndx));
  else
    dw_tile<T, RW, DZ, ALIGNED>(a, lds, xcd_swizzle(wg - ndx, ndw));
}

// ---- the whole backward of a narrow bf16 projection (k, n <= 128) -------------------------
//
// Bound by memory: for rows of 128 + 128 channels it multiplies 128 times per value moved,
// a tenth of what the matrix cores do meanwhile.  So dx, dW and dbias come from one copy
// of x and dout (the two kernels above read dout twice): a workgroup of 8 waves walks over
// blocks of M rows, stages x and dz in LDS, and uses the dz tile both ways, its rows for
// dx = dz W^T (W stays in LDS) and its columns for dW += x^T dz (in registers until the
// end).  The next block's loads are in flight meanwhile.  dx goes through x's place in LDS,
// each wave's part by itself, to be stored in whole rows' pieces.
//
// M = 128, or 64 where dz takes three planes (96 KB of LDS either way) or where the repair
// of ragged rows would not fit the registers beside two times 128 rows.
// 589,824 x 128 x 128: 85 us (5.3 TB/s of x, dout and dx) and 6 for the sums of 256 slabs, where
// the two kernels above and their sums take 143.
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

constexpr int NARROW_WG = 512;
constexpr int narrow_rows(int dz, bool aligned) {
  return dz == DZ_ACT || !aligned ? 64 : 128;
}

template <int DZ, bool ALIGNED>
__global__ __launch_bounds__(NARROW_WG) void lin_narrow_kernel(LinBwdArgs a) {
  using S = DzSource<bf16, DZ>;
  constexpr int M = narrow_rows(DZ, ALIGNED), N = M / 32;       // chunks a thread stages of a tile
  constexpr int JT = M / 64, JW = 32 * JT;             // dx tiles, columns of a wave
  constexpr int TILE_BYTES = M * 256, W_BYTES = 128 * 256;
  __shared__ __attribute__((aligned(16))) char lds[W_BYTES + (1 + S::P) * TILE_BYTES];
  char *tw = lds, *tx = lds + W_BYTES, *tz = tx + TILE_BYTES;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const bool weights = a.dw || a.dbias;
  const Mat<bf16> mx{(const bf16*)a.x, a.m, a.k}, md{(const bf16*)a.dout, a.m, a.n},
      mz{(const bf16*)a.z, a.m, a.n}, mw{(const bf16*)a.w, a.k, a.n};
  const int line0 = threadIdx.x / 16, chunk = threadIdx.x % 16;
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const int line = line0 + 32 * u;
    int info = 8;
    Raw8<bf16> w;
    if constexpr (ALIGNED) w = fetch<bf16>(mw, 0, 0, 128, line, 8 * chunk);
    else w = fetch_any<bf16>(mw, 0, 0, 128, line, 8 * chunk, info);
    *(u32x4*)(tw + Square::chunk_at(line, chunk)) = repair(w, info).v[0];
  }
  Raw8<bf16> x[N], d[N], z[DZ == DZ_X ? 1 : N];
  int xi[N], ni[N];
  auto load = [&](int64_t r0) {
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const int line = line0 + 32 * u;
      xi[u] = ni[u] = 8;
      if constexpr (ALIGNED) {
        x[u] = fetch<bf16>(mx, r0, 0, M, line, 8 * chunk);
        d[u] = fetch<bf16>(md, r0, 0, M, line, 8 * chunk);
        if constexpr (DZ != DZ_X) z[u] = fetch<bf16>(mz, r0, 0, M, line, 8 * chunk);
      } else {
        x[u] = fetch_any<bf16>(mx, r0, 0, M, line, 8 * chunk, xi[u]);
        d[u] = fetch_any<bf16>(md, r0, 0, M, line, 8 * chunk, ni[u]);
        if constexpr (DZ != DZ_X) z[u] = fetch_any<bf16>(mz, r0, 0, M, line, 8 * chunk, ni[u]);
      }
    }
  };
  // this wave's tiles: dx rows di .. + 31, columns dj .. + JW - 1; dW rows (of k) wi .. + 31,
  // columns wj .. + 63
  const int di = M == 128 ? wave / 2 * 32 : wave / 4 * 32;
  const int dj = M == 128 ? wave % 2 * 64 : wave % 4 * 32;
  const int wi = wave / 2 * 32, wj = wave % 2 * 64;
  f32x16 gw[2] = {};
  float col[8] = {};
  load((int64_t)blockIdx.x * M);
  for (int64_t r0 = (int64_t)blockIdx.x * M; r0 < a.m; r0 += (int64_t)gridDim.x * M) {
    __syncthreads();  // dx of the last block has left x's place
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const int at = Square::chunk_at(line0 + 32 * u, chunk);
      *(u32x4*)(tx + at) = repair(x[u], xi[u]).v[0];
      float f[8];
      unpack(repair(d[u], ni[u]), f);
      if constexpr (DZ != DZ_X) {
        float g[8];
        unpack(repair(z[u], ni[u]), g);
#pragma unroll
        for (int e = 0; e < 8; ++e)
          f[e] = DZ == DZ_RELU ? (g[e] > 0.f ? f[e] : 0.f) : f[e] * act_grad<bf16>(g[e], a.act);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) col[e] += f[e];
#pragma unroll
      for (int p = 0; p < S::P; ++p) {
        bf16x8 b;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          b[e] = (bf16)f[e];
          if (p + 1 < S::P) f[e] -= (float)b[e];
        }
        *(bf16x8*)(tz + p * TILE_BYTES + at) = b;
      }
    }
    __syncthreads();
    load(r0 + (int64_t)gridDim.x * M);
    if (a.dw && wi < a.k && wj < a.n) {
#pragma unroll
      for (int kk = 0; kk < M; kk += 16) {
        const bf16x8 fx = Square::across(tx, wi, kk, lane);
#pragma unroll
        for (int p = S::P - 1; p >= 0; --p)
#pragma unroll
          for (int v = 0; v < 2; ++v)
            gw[v] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                Square::across(tz + p * TILE_BYTES, wj + 32 * v, kk, lane), fx, gw[v], 0, 0, 0);
      }
    }
    f32x16 gx[JT] = {};
    if (a.dx && dj < a.k) {
#pragma unroll
      for (int kk = 0; kk < 128; kk += 16) {
        if (kk >= a.n) break;
#pragma unroll
        for (int p = S::P - 1; p >= 0; --p) {
          const bf16x8 fz = Square::along(tz + p * TILE_BYTES, di, kk, lane);
#pragma unroll
          for (int v = 0; v < JT; ++v)
            gx[v] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                Square::along(tw, dj + 32 * v, kk, lane), fz, gx[v], 0, 0, 0);
        }
      }
    }
    __syncthreads();
    if (a.dx && dj < a.k) {
      // the wave's 32 rows x JW columns in its own part of x's place, 16-byte chunks
      // permuted by the row
      constexpr int CH = JW / 8;
      char* mine = tx + wave * 32 * JW * 2;
      auto at = [&](int i, int c) {
        return mine + (i * CH + (c ^ (CH == 8 ? i & 7 : (i >> 1) & 3))) * 16;
      };
#pragma unroll
      for (int v = 0; v < JT; ++v)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          *(bf16x4*)(at(lane & 31, 4 * v + q) + 8 * (lane >> 5)) =
              bf16x4{(bf16)gx[v][4 * q], (bf16)gx[v][4 * q + 1], (bf16)gx[v][4 * q + 2],
                     (bf16)gx[v][4 * q + 3]};
      // only this wave's lanes read it back, after their writes (LDS serves a wave in order)
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      const int j = dj + 8 * (lane % CH);
#pragma unroll
      for (int s = 0; s < 32; s += 64 / CH) {
        const int i = s + lane / CH;
        const Raw8<bf16> o = *(const Raw8<bf16>*)at(i, lane % CH);
        if (r0 + di + i < a.m && j < a.k)
          put_raw<bf16, ALIGNED>((bf16*)a.dx + (r0 + di + i) * a.k + j, a.k - j, o);
      }
    }
  }
  if (!weights) return;
  float* dw = a.splits > 1 ? a.part + blockIdx.x * slab_floats(a.k, a.n) : a.dw;
  float* db = a.splits > 1 ? dw + (int64_t)a.k * a.n : a.dbias;
  const int i = wi + (lane & 31);
  if (a.dw && i < a.k)
#pragma unroll
    for (int v = 0; v < 2; ++v)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int j = wj + 32 * v + 8 * q + 4 * (lane >> 5);
        if (ALIGNED) {
          if (j < a.n)
            *(f32x4*)(dw + i * a.n + j) =
                f32x4{gw[v][4 * q], gw[v][4 * q + 1], gw[v][4 * q + 2], gw[v][4 * q + 3]};
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (j + e < a.n) dw[i * a.n + j + e] = gw[v][4 * q + e];
        }
      }
  if (a.dbias) {  // the threads of a column, in order
    __syncthreads();
    float* part = (float*)lds;
#pragma unroll
    for (int e = 0; e < 8; ++e) part[line0 * 128 + 8 * chunk + e] = col[e];
    __syncthreads();
    if ((int)threadIdx.x < a.n) {
      float s = 0.f;
      for (int t = 0; t < 32; ++t) s += part[t * 128 + threadIdx.x];
      db[threadIdx.x] = s;
    }
  }
}

// Sums of the splits' slabs (256 of 66 KB: 6 us): `slices` threads (a power of two) to 4
// consecutive sums, each every slices-th slab, then their sums through LDS, in a fixed order.
__global__ __launch_bounds__(256) void lin_reduce_kernel(LinBwdArgs a, int slices) {
  __shared__ f32x4 sum[256];
  const int cols = 256 / slices, slice = threadIdx.x / cols;
  const int64_t kn = (int64_t)a.k * a.n, all = kn + a.n, slab = slab_floats(a.k, a.n);
  const int64_t i = ((int64_t)blockIdx.x * cols + threadIdx.x % cols) * 4;
  f32x4 s{};
  if (i < all) {
#pragma unroll 4
    for (int w = slice; w < a.splits; w += slices) s += *(const f32x4*)(a.part + w * slab + i);
  }
  sum[threadIdx.x] = s;
  for (int half = slices / 2; half > 0; half >>= 1) {
    __syncthreads();
    if (slice < half) sum[threadIdx.x] += sum[threadIdx.x + half * cols];
  }
  if (slice > 0) return;
  s = sum[threadIdx.x];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if (i + e < kn) {
      if (a.dw) a.dw[i + e] = s[e];
    } else if (i + e < all && a.dbias) {
      a.dbias[i + e - kn] = s[e];
    }
  }
}

// Rows of x, dx and of W, z, dout, out are whole 16-byte words.
template <typename T>
bool whole_words(int k, int n) {
  return k % WORD<T> == 0 && n % WORD<T> == 0;
}
int64_t tiles_of(int64_t m, int64_t n, int r) { return (m + r - 1) / r * ((n + r - 1) / r); }

// 128-wide tiles of an [m][width] result where there are enough of them for the 256 CUs and
// a second half of a tile to fill, else 64-wide ones (four times as many, at half the reuse
// of an operand).  fp32 tiles of 128 leave one workgroup on a CU (96 KB of planes), which
// pays where the products and not the memory take the time, from 256 terms a sum on
// (291,975 x 32 x 72 fp32 forward: 73 us in tiles of 128, 45 in tiles of 64).
template <typename T>
bool wide(int64_t m, int width, int terms) {
  return width > 64 && tiles_of(m, width, 128) >= 256 && (sizeof(T) == 2 || terms >= 256);
}

template <typename T>
hipError_t fwd(const LinArgs& a, hipStream_t s) {
  KernelTimer t(K_LIN_FWD, s);
  const bool al = whole_words<T>(a.k, a.n);
  // ragged fp32 rows in tiles of 64 only: 25,152 x 453 x 1179 in 253 against 301 us
  const bool big = (al || sizeof(T) == 2) && wide<T>(a.m, a.n, a.k);
  const dim3 grid((unsigned)tiles_of(a.m, a.n, big ? 128 : 64)), wg(256);
  if (big && al) hipLaunchKernelGGL((lin_fwd_kernel<T, 128, true>), grid, wg, 0, s, a);
  else if (big) hipLaunchKernelGGL((lin_fwd_kernel<bf16, 128, false>), grid, wg, 0, s, a);
  else if (al) hipLaunchKernelGGL((lin_fwd_kernel<T, 64, true>), grid, wg, 0, s, a);
  else hipLaunchKernelGGL((lin_fwd_kernel<T, 64, false>), grid, wg, 0, s, a);
  return hipGetLastError();
}

// Tiles of dW: 128 wide if that leaves 256 workgroups of at least 512 rows, else 64 wide
// (fewer splits for as many workgroups, and so fewer partial sums) or if k or n fills no
// more than half of one.
bool wide_w(int64_t m, int k, int n) {
  return k > 64 && n > 64 && tiles_of(k, n, 128) * ((m + 511) / 512) >= 256;
}

template <typename T, int DZ, bool AL>
void bwd_launch(const LinBwdArgs& a, hipStream_t s) {
  const bool weights = a.dw || a.dbias, ww = wide_w(a.m, a.k, a.n);
  const bool wx = wide<T>(a.m, a.k, a.n);
  const unsigned ndx = (unsigned)tiles_of(a.m, a.k, wx ? 128 : 64);
  const unsigned ndw = (unsigned)(tiles_of(a.k, a.n, ww ? 128 : 64) * a.splits);
  const dim3 wg(256), both(ndx + ndw);
  // (and a launch holds fewer than 2^32 threads)
  if (a.dx && weights && !wx && ndx < (1u << 20)) {
    KernelTimer t(K_LIN_BWD_BOTH, s);
    if (ww) hipLaunchKernelGGL((lin_bwd_both_kernel<T, 128, DZ, AL>), both, wg, 0, s, a, (int)ndx);
    else hipLaunchKernelGGL((lin_bwd_both_kernel<T, 64, DZ, AL>), both, wg, 0, s, a, (int)ndx);
    return;
  }
  if (a.dx) {
    KernelTimer t(K_LIN_BWD_DX, s);
    if (wx) hipLaunchKernelGGL((lin_bwd_dx_kernel<T, 128, DZ, AL>), dim3(ndx), wg, 0, s, a);
    else hipLaunchKernelGGL((lin_bwd_dx_kernel<T, 64, DZ, AL>), dim3(ndx), wg, 0, s, a);
  }
  if (weights) {
    KernelTimer t(K_LIN_BWD_W, s);
    if (ww) hipLaunchKernelGGL((lin_bwd_w_kernel<T, 128, DZ, AL>), dim3(ndw), wg, 0, s, a);
    else hipLaunchKernelGGL((lin_bwd_w_kernel<T, 64, DZ, AL>), dim3(ndw), wg, 0, s, a);
  }
}
template <typename T, int DZ>
void bwd_align(const LinBwdArgs& a, hipStream_t s) {
  if (whole_words<T>(a.k, a.n)) bwd_launch<T, DZ, true>(a, s);
  else bwd_launch<T, DZ, false>(a, s);
}
template <typename T>
void bwd_products(const LinBwdArgs& a, hipStream_t s) {
  if (a.act == TRIATTN_ACT_NONE) bwd_align<T, DZ_X>(a, s);
  else if (a.act == TRIATTN_ACT_RELU) bwd_align<T, DZ_RELU>(a, s);
  else if (a.dz) bwd_align<T, DZ_MADE>(a, s);
  else bwd_align<T, DZ_ACT>(a, s);
}

// A smooth activation's dz is made beforehand (fp32, in the workspace) where dx has several
// column tiles, and dW as many: for one, forming it twice moves half the bytes.  (relu's
// costs one comparison wherever it is formed.)
bool make_dz(int act, int k) { return act > TRIATTN_ACT_RELU && k > 128; }

hipError_t reduce(const LinBwdArgs& a, hipStream_t s) {
  KernelTimer t(K_LIN_REDUCE, s);
  int slices = 1;
  while (slices < 32 && slices * 4 < a.splits) slices *= 2;
  const int64_t quads = ((int64_t)a.k * a.n + a.n + 3) / 4, cols = 256 / slices;
  hipLaunchKernelGGL(lin_reduce_kernel, dim3((unsigned)((quads + cols - 1) / cols)), dim3(256), 0, s,
                     a, slices);
  return hipGetLastError();
}

bool narrow(int dtype, int k, int n) {
  return dtype == TRIATTN_BF16 && k <= 128 && n <= 128;
}
int narrow_parts(int64_t m, int k, int n, int act) {
  const int dz = act == TRIATTN_ACT_NONE ? DZ_X : act == TRIATTN_ACT_RELU ? DZ_RELU : DZ_ACT;
  const int rows = narrow_rows(dz, whole_words<bf16>(k, n));
  const int64_t blocks = (m + rows - 1) / rows;
  return (int)(blocks < 256 ? blocks : 256);  // one workgroup a CU
}
hipError_t bwd_narrow(const LinBwdArgs& a, hipStream_t s) {
  {
    KernelTimer t(K_LIN_NARROW, s);
    const dim3 grid(narrow_parts(a.m, a.k, a.n, a.act)), wg(NARROW_WG);
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, wg, 0, s, a); };
    const bool al = whole_words<bf16>(a.k, a.n);
    if (a.act == TRIATTN_ACT_NONE)
      go(al ? lin_narrow_kernel<DZ_X, true> : lin_narrow_kernel<DZ_X, false>);
    else if (a.act == TRIATTN_ACT_RELU)
      go(al ? lin_narrow_kernel<DZ_RELU, true> : lin_narrow_kernel<DZ_RELU, false>);
    else
      go(al ? lin_narrow_kernel<DZ_ACT, true> : lin_narrow_kernel<DZ_ACT, false>);
  }
  return (a.dw || a.dbias) && a.splits > 1 ? reduce(a, s) : hipGetLastError();
}

template <typename T>
hipError_t bwd(const LinBwdArgs& a, hipStream_t s) {
  if (sizeof(T) == 2 && narrow(TRIATTN_BF16, a.k, a.n)) return bwd_narrow(a, s);
  if (a.dz) {
    KernelTimer t(K_LIN_DZ, s);
    const int64_t wgs = (a.m * a.n + 2047) / 2048;
    hipLaunchKernelGGL(lin_dz_kernel<T>, dim3((unsigned)(wgs < 4096 ? wgs : 4096)), dim3(256), 0, s,
                       a);
  }
  bwd_products<T>(a, s);
  return (a.dw || a.dbias) && a.splits > 1 ? reduce(a, s) : hipGetLastError();
}

// Splits of the rows for dW: as many workgroups as the CUs hold at once beside those of dx in the
// same launch (LDS and registers allow two or three on a CU, one of fp32 in tiles of 128, and one
// of ragged bf16 in tiles of 128 without planes, whose 193 + 64 registers are a few too many for
// the two that are counted here: its grid runs in two turns), each of at least 128 rows; none,
// which needs no further sum, for up to 256 rows.
template <typename T>
int dw_splits(int64_t m, int k, int n, int act) {
  const bool ww = wide_w(m, k, n), smooth = act > TRIATTN_ACT_RELU;
  const int64_t tiles = tiles_of(k, n, ww ? 128 : 64);
  const int64_t fit = 256 * (ww ? (sizeof(T) == 4 ? 1 : 2) : sizeof(T) == 2 && smooth ? 2 : 3);
  const int64_t ndx = wide<T>(m, k, n) ? 0 : tiles_of(m, k, 64);
  int64_t s = (ndx < fit * 3 / 4 ? fit - ndx : fit) / tiles, most = (m + 127) / 128;
  if (s > most) s = most;
  if (s < 1 || m <= 256) s = 1;
  const int64_t per = split_rows(m, (int)s);
  return (int)((m + per - 1) / per);  // no split without rows
}

}  // namespace

LinBwdPlan lin_bwd_plan(int dtype, int64_t m, int k, int n, int act) {
  LinBwdPlan p{};
  p.splits = narrow(dtype, k, n) ? narrow_parts(m, k, n, act)
             : dtype == TRIATTN_BF16 ? dw_splits<bf16>(m, k, n, act)
                                     : dw_splits<float>(m, k, n, act);
  if (p.splits > 1) p.part = (size_t)p.splits * (size_t)slab_floats(k, n) * sizeof(float);
  if (make_dz(act, k) && !narrow(dtype, k, n)) p.dz = (size_t)m * n * sizeof(float);
  return p;
}

hipError_t launch_lin_fwd(int dtype, const LinArgs& a, hipStream_t s) {
  return dtype == TRIATTN_BF16 ? fwd<bf16>(a, s) : fwd<float>(a, s);
}
hipError_t launch_lin_bwd(int dtype, const LinBwdArgs& a, hipStream_t s) {
  return dtype == TRIATTN_BF16 ? bwd<bf16>(a, s) : bwd<float>(a, s);
}

}  // namespace triattn
