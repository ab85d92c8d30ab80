// Cross attention: device pieces shared by its forward and backward kernels.
//
// For every sample and key head, the rows of the problem are the (query, head) pairs whose
// heads read that key head: row r = query r / group, head hk * group + r % group.  So the
// heads that share keys share the key tiles too, and the sums over them that dK and dV need
// are sums over rows.
//
// Channels are padded to DP = 32, 64 or 128 in LDS and registers with zeros (exact: they add
// nothing); memory is read and written as it is.
#pragma once

#include "dma.h"
#include "ops.h"
#include "triattn.h"

namespace triattn {

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

// Eight consecutive elements as they lie in memory.
template <typename T>
struct Chunk {
  static constexpr int N = (int)sizeof(T) / 2;  // 16-byte words
  u32x4 v[N];
};

// A tile of rows x DP channels in LDS, read along rows (a fragment holds channels of one row
// a lane) and across them (channels of 4 or 8 rows a lane).
//
// bf16: 16-byte chunks of a line permuted by XOR with a value s of the line's low bits (l0 ..
// l3).  Both reads are free of bank conflicts whether the LDS serves 128 or 256 bytes a
// cycle: s differs between any 8 consecutive lines that share banks, and between any 16; and
// lines of a transposing read (4 lines x 2 or 4 chunks) that share banks differ in s's high
// bits.  fp32: lines of DP + 4 floats, so that 8 consecutive lines start 4 banks apart; the
// reads across take one float a lane, 32 lanes of a line.
template <typename T, int DP>
struct XTile;

template <int DP>
struct XTile<bf16, DP> {
  static constexpr int LINE = DP * 2;
  static constexpr int N = DP / 16;  // fragments of a row
  using Row = bf16x8[N];
  __device__ static inline int at(int line, int c) {
    int s;
    if constexpr (DP == 32) {
      s = swz(line);
    } else if constexpr (DP == 64) {
      s = ((((line >> 1) & 1) << 2) | ((line & 1) << 1) | ((line >> 2) & 1)) ^
          (((line >> 3) & 1) << 1);
    } else {
      const int e = line & 3;
      s = ((e ^ (e << 1)) << 1) ^ ((line >> 2) & 3);
    }
    return line * LINE + 16 * (c ^ s);
  }
  __device__ static inline void put(char* t, int line, int c, const Chunk<bf16>& x) {
    *(u32x4*)(t + at(line, c)) = x.v[0];
  }
  // sum over the channels of (line r0 + accumulator row) times (the row in `b`)
  __device__ static inline f32x16 dot(const char* t, int r0, const Row& b, f32x16 acc) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const bf16x8 a = *(const bf16x8*)(t + at(r0 + (lane & 31), 2 * i + (lane >> 5)));
      acc = Mma<bf16>::mma(a, b[i], acc);
    }
    return acc;
  }
  // The 8 indices of a fragment of channels 32 n + lane % 32, lines r0 + 16 i + 4 g .. and
  // r0 + 16 i + 8 + 4 g ..: the order of an accumulator fed back (acc_frags).
  __device__ static inline bf16x8 across(const char* t, int r0, int n) {
    const int lane = threadIdx.x & 63, i = lane & 15;
    const int line = r0 + (i >> 2) + 4 * (lane >> 5), ch = 32 * n + (lane & 16) + 4 * (i & 3);
    typedef TRIATTN_LDS s16x4* lds4;
    const char* a = t + at(line, ch >> 3) + (ch & 4) * 2;
    const char* b = t + at(line + 8, ch >> 3) + (ch & 4) * 2;
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(uintptr_t)lds_addr(a));
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(uintptr_t)lds_addr(b));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  }
  // out[n] += (lines r0 .. r0 + 31)^T p, contraction over the lines
  using Frag = bf16x8[2];
  __device__ static inline void add(const char* t, int r0, const Frag& p, f32x16 (&out)[DP / 32]) {
#pragma unroll
    for (int n = 0; n < DP / 32; ++n)
#pragma unroll
      for (int i = 0; i < 2; ++i) out[n] = Mma<bf16>::mma(across(t, r0 + 16 * i, n), p[i], out[n]);
  }
  // two products with the same lines
  __device__ static inline void add2(const char* t, int r0, const Frag& p, f32x16 (&out)[DP / 32],
                                     const Frag& p2, f32x16 (&out2)[DP / 32]) {
#pragma unroll
    for (int n = 0; n < DP / 32; ++n)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const bf16x8 a = across(t, r0 + 16 * i, n);
        out[n] = Mma<bf16>::mma(a, p[i], out[n]);
        out2[n] = Mma<bf16>::mma(a, p2[i], out2[n]);
      }
  }
  // The row's channels in registers; `p` its first, d a multiple of 8; zeros if !real.  All
  // loads at once, without conditions: one inside a branch is waited for at its end.
  __device__ static inline void row(const bf16* p, int d, bool real, Row& r) {
    const int g = (threadIdx.x & 63) >> 5;
#pragma unroll
    for (int i = 0; i < N; ++i) r[i] = *(const bf16x8*)(p + min(16 * i + 8 * g, d - 8));
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (!real || 16 * i + 8 * g >= d) r[i] = bf16x8{};
  }
  __device__ static inline float dot_regs(const Row& a, const Row& b) {  // this half's channels
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) s = fmaf((float)a[i][e], (float)b[i][e], s);
    return s;
  }
};

template <int DP>
struct XTile<float, DP> {
  static constexpr int LINE = (DP + 4) * 4;
  static constexpr int N = DP / 2;
  using Row = float[N];
  __device__ static inline void put(char* t, int line, int c, const Chunk<float>& x) {
    u32x4* p = (u32x4*)(t + line * LINE + 32 * c);
    p[0] = x.v[0];
    p[1] = x.v[1];
  }
  __device__ static inline f32x16 dot(const char* t, int r0, const Row& b, f32x16 acc) {
    const int lane = threadIdx.x & 63;
    const char* p = t + (r0 + (lane & 31)) * LINE + (lane >> 5) * N * 4;
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
      const f32x4 a = *(const f32x4*)(p + 16 * i);
#pragma unroll
      for (int e = 0; e < 4; ++e) acc = Mma<float>::mma(a[e], b[4 * i + e], acc);
    }
    return acc;
  }
  using Frag = float[16];
  __device__ static inline float across(const char* t, int r0, int v, int n) {
    const int lane = threadIdx.x & 63;
    return *(const float*)(t + (r0 + acc_row(v, lane >> 5)) * LINE + (32 * n + (lane & 31)) * 4);
  }
  __device__ static inline void add(const char* t, int r0, const Frag& p, f32x16 (&out)[DP / 32]) {
#pragma unroll
    for (int n = 0; n < DP / 32; ++n)
#pragma unroll
      for (int v = 0; v < 16; ++v) out[n] = Mma<float>::mma(across(t, r0, v, n), p[v], out[n]);
  }
  __device__ static inline void add2(const char* t, int r0, const Frag& p, f32x16 (&out)[DP / 32],
                                     const Frag& p2, f32x16 (&out2)[DP / 32]) {
#pragma unroll
    for (int n = 0; n < DP / 32; ++n)
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        const float a = across(t, r0, v, n);
        out[n] = Mma<float>::mma(a, p[v], out[n]);
        out2[n] = Mma<float>::mma(a, p2[v], out2[n]);
      }
  }
  __device__ static inline void row(const float* p, int d, bool real, Row& r) {
    const int g = (threadIdx.x & 63) >> 5;
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
      const f32x4 x = *(const f32x4*)(p + min(N * g + 4 * i, d - 4));
#pragma unroll
      for (int e = 0; e < 4; ++e) r[4 * i + e] = x[e];
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (!real || N * g + i >= d) r[i] = 0.f;
  }
  __device__ static inline float dot_regs(const Row& a, const Row& b) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) s = fmaf(a[i], b[i], s);
    return s;
  }
};

// Quotient and remainder by the number of heads that share a key head; inv = 2^32 / group
// rounded up, exact for r * group < 2^32.
__device__ inline int row_query(const XatArgs& a, int r) {
  return a.group == 1 ? r : (int)(((uint64_t)(uint32_t)r * a.inv_group) >> 32);
}
// First element of row r of sample b, key head kh in a tensor [batch][nq][h][c].
__device__ inline int64_t row_at(const XatArgs& a, int64_t b, int kh, int r, int c) {
  const int q = row_query(a, r);
  return ((b * a.nq + q) * a.h + kh * a.group + (r - q * a.group)) * c;
}

// Chunks of `LINES` lines of DP channels, by the threads of NW waves: line() and col() of a
// thread's chunk u.
template <int DP, int LINES, int NW>
struct Share {
  static constexpr int PER = DP / 8, C = LINES * PER / (64 * NW);
  static_assert(LINES * PER % (64 * NW) == 0, "whole chunks");
  __device__ static inline int id(int u) { return (int)(threadIdx.x % (64 * NW)) + 64 * NW * u; }
  __device__ static inline int line(int u) { return id(u) / PER; }
  __device__ static inline int col(int u) { return id(u) % PER; }
};

// Chunk at byte `off` of a resource (zeros past its end).
template <typename T>
__device__ inline Chunk<T> load_chunk(rsrc_t rs, uint32_t off) {
  Chunk<T> x;
#pragma unroll
  for (int i = 0; i < Chunk<T>::N; ++i)
    x.v[i] = __builtin_bit_cast(
        u32x4, __builtin_amdgcn_raw_buffer_load_b128(rs, (int)(off + 16 * i), 0, 0));
  return x;
}
constexpr uint32_t NOWHERE = 0x80000000u;  // past the end of any resource here

// Staging of tiles of BK keys, keys and values: through registers, into LDS with the rows of
// masked keys zeroed, so that nothing in them reaches a product.
template <typename T, int DP, int BK, int NW>
struct KvStage {
  using S = Share<DP, BK, NW>;
  using L = XTile<T, DP>;
  static constexpr int BYTES = BK * L::LINE;
  Chunk<T> k[S::C], v[S::C];
  int valid;  // of key k0 + lane
  __device__ inline void load(const XatArgs& a, int64_t b, int kh, int k0) {
    const int rows = a.nk - k0 < BK ? a.nk - k0 : BK, stride = a.hk * a.d;
    const uint32_t n = rows > 0 ? (uint32_t)((rows - 1) * stride + a.d) * sizeof(T) : 0u;
    const int64_t at = ((b * a.nk + k0) * a.hk + kh) * a.d;
    const rsrc_t rk = buf_rsrc_n((const T*)a.k + at, n), rv = buf_rsrc_n((const T*)a.v + at, n);
#pragma unroll
    for (int u = 0; u < S::C; ++u) {
      const int line = S::line(u), c = 8 * S::col(u);
      const uint32_t off =
          c < a.d && line < rows ? (uint32_t)(line * stride + c) * sizeof(T) : NOWHERE;
      k[u] = load_chunk<T>(rk, off);
      v[u] = load_chunk<T>(rv, off);
    }
    const int lane = threadIdx.x & 63, in = rows > 0 ? rows : 0;
    valid = lane < in;
    if (a.mask)  // bytes past the tile's keys read as zeros
      valid = __builtin_amdgcn_raw_buffer_load_b8(buf_rsrc_n(a.mask + b * a.nk + k0, (uint32_t)in),
                                                  lane, 0, 0);
  }
  // Which of the tile's keys are valid.
  __device__ inline uint64_t bits() const { return __ballot(valid != 0); }
  __device__ inline void store(char* tk, char* tv, uint64_t ok) const {
    constexpr uint64_t ALL = BK == 64 ? ~0ull : (1ull << BK) - 1;
#pragma unroll
    for (int u = 0; u < S::C; ++u) {
      const int line = S::line(u), c = S::col(u);
      Chunk<T> x = k[u], y = v[u];
      if (ok != ALL && !((ok >> line) & 1)) x = Chunk<T>{}, y = Chunk<T>{};
      L::put(tk, line, c, x);
      L::put(tv, line, c, y);
    }
  }
};

// Where the bias comes from: none; planes of it, a head each, that a launch before made; or, for
// four heads at a time, as it lies (heads fastest).  In the last case a workgroup's four waves
// take four heads of the same 32 rows (or keys): each stages its own head's tiles, and they
// share the bias tile of 32 queries x 32 keys x 4 heads, whose 4 heads are one load.
enum XatBias { XB_NONE, XB_PLANES, XB_HEADS };

// Keys of a tile: 64 for workgroups of four waves where the two buffers leave room for several
// on a CU, else 32.
template <typename T, int DP, int NW>
constexpr int xat_keys() {
  return NW == 4 && (sizeof(T) == 2 || DP == 32) ? 64 : 32;
}

// Waves of a workgroup that share staged tiles: 32 rows each.  Few rows take a wave to
// themselves, which needs no barrier.
// (fp32 rows of more than 64 channels would take it too many registers.)
inline int xat_waves_for(int dtype, const XatArgs& a, int64_t rows) {
  return rows <= 32 && (dtype == TRIATTN_BF16 || a.d <= 64) ? 1 : 4;
}
inline int xat_row_waves(int dtype, const XatArgs& a) {
  return xat_waves_for(dtype, a, (int64_t)a.nq * a.group);
}
inline int xat_key_waves(int dtype, const XatArgs& a) { return xat_waves_for(dtype, a, a.nk); }
// (with the heads side by side, a wave has 32 rows or keys and a workgroup's others the same)
inline int xat_row_tiles(const XatArgs& a, int nw) {
  return (int)(((int64_t)a.nq * a.group + 32 * nw - 1) / (32 * nw));
}
inline int xat_key_tiles(const XatArgs& a, int nw) { return (a.nk + 32 * nw - 1) / (32 * nw); }

constexpr int XAT_SPLITS = 128;

// Tiles whose loads are in flight: two where a wave stages for itself rows of at most `most`
// bytes (for its registers: 128 forward, 64 backward).
template <typename T, int DP>
constexpr int xat_ahead(int sharing, int most) {
  return sharing == 1 && DP * (int)sizeof(T) <= most ? 2 : 1;
}

// Splits of a long loop: so that the workgroups (of nw waves) fill the GPU, each of at least
// `least` steps.  (768 x 768, 16 heads of 24, training: 2 splits 73 us with their joins, none 83.)
inline int xat_splits(int64_t wgs, int nw, int64_t steps, int64_t least) {
  const int64_t want = nw == 1 ? 2048 : 512;
  int64_t s = (want + wgs - 1) / wgs;
  if (wgs >= want) s = 1;
  if (s > steps / least) s = steps / least;
  return s < 1 ? 1 : (s > XAT_SPLITS ? XAT_SPLITS : (int)s);
}
// Whether a bias is taken as it lies, four heads a workgroup: 4 heads a load, and the heads'
// tiles and the bias tile fit LDS.  Otherwise launches before and after turn it (and dS) into
// planes: 768 x 768 with 16 heads of 24, training, kernels 147 us by planes and 75 so; 737 windows
// of 32 x 128 with 4 heads of 32, 229 and 88.
inline bool xat_by_heads(int dtype, const XatArgs& a) {
  const int64_t e = dtype == TRIATTN_BF16 ? 2 : 4;
  return a.bias_batch > 0 && a.group == 1 && a.h % 4 == 0 && a.d <= (e == 2 ? 128 : 64) &&
         32 * e * a.nk * a.h < (int64_t)1 << 31;  // offsets within a tile
}

// Groups of waves of a workgroup that take the tiles of its loop in turn (and join their sums in
// LDS), where few workgroups have long loops: fewer partial results cross memory (one query of 3
// samples to 30,011 keys: joining the splits 14 us, 5.5 with four groups).  Four where a wave
// stages for itself.  With four heads side by side two, for 256 registers a lane, and one where the
// tiles would not fit LDS.
inline bool xat_groups(int64_t wgs, int64_t steps) { return wgs < 512 && steps >= 8; }
template <typename T, int DP, int NW, int MODE>
constexpr int xat_most_groups() {
  return NW == 1 ? 4 : MODE == XB_HEADS && DP <= (sizeof(T) == 2 ? 64 : 32) ? 2 : 1;
}
inline int xat_most_groups(int dtype, const XatArgs& a, int nw) {
  if (xat_by_heads(dtype, a)) return a.d <= (dtype == TRIATTN_BF16 ? 64 : 32) ? 2 : 1;
  return nw == 1 ? 4 : 1;
}

// Splits of a loop over `steps` tiles of 32 by `wgs` workgroups of nw waves.
inline int xat_loop_splits(int dtype, const XatArgs& a, int64_t wgs, int nw, int64_t steps) {
  const int groups = xat_groups(wgs, steps) ? xat_most_groups(dtype, a, nw) : 1;
  if (xat_by_heads(dtype, a)) return xat_splits(wgs * groups * 2, 4, steps, 6 * groups);
  return xat_splits(wgs * groups, nw, steps, 8 * groups);
}
inline int64_t xat_row_wgs(int dtype, const XatArgs& a) {
  if (xat_by_heads(dtype, a)) return a.batch * (a.h / 4) * xat_row_tiles(a, 1);
  return a.batch * a.hk * xat_row_tiles(a, xat_row_waves(dtype, a));
}
inline int64_t xat_key_wgs(int dtype, const XatArgs& a) {
  if (xat_by_heads(dtype, a)) return a.batch * (a.h / 4) * xat_key_tiles(a, 1);
  return a.batch * a.hk * xat_key_tiles(a, xat_key_waves(dtype, a));
}
inline int64_t xat_key_steps(const XatArgs& a) { return (a.nk + 31) / 32; }
inline int64_t xat_row_steps(const XatArgs& a) { return ((int64_t)a.nq * a.group + 31) / 32; }
inline int xat_key_splits(int dtype, const XatArgs& a) {
  return xat_loop_splits(dtype, a, xat_row_wgs(dtype, a), xat_row_waves(dtype, a),
                         xat_key_steps(a));
}
inline int xat_row_splits(int dtype, const XatArgs& a) {
  return xat_loop_splits(dtype, a, xat_key_wgs(dtype, a), xat_key_waves(dtype, a),
                         xat_row_steps(a));
}


// Waves a SIMD that a kernel's registers have to leave room for: backward, forward.  (bf16, 64
// channels, 2 x 2048 x 4099: dkv 360 us at one wave, 218 at two; dq 212 and 138.)
template <typename T, int DP, int NW>
constexpr int xat_waves() {
  return DP <= (sizeof(T) == 2 || NW == 4 ? 64 : 32) ? 2 : 1;
}
template <typename T, int DP, int NW, int MODE>
constexpr int xat_fwd_waves() {
  const int most = DP == 32 ? 4 : DP == 64 ? 3 : 2;  // without a bias, tiles shared
  return sizeof(T) == 4 ? 1 : NW == 1 || MODE != XB_NONE ? most - 1 : most;
}

// The logits' (or weights') values of a tile's masked keys set to `value`, for the few tiles that
// need it.  The empty statement keeps it in a branch of its own: without, its comparisons and
// selects run for every tile.  The caller has used every value it passes in ordinary
// instructions before the branch: the compiler counts the wait states after a matrix instruction
// along one path to a join only, and that may be the longer one.
__device__ inline void mask_tile(f32x16& s, uint32_t bits, int g, float value) {
  asm volatile("");
  const uint32_t b = bits >> (4 * g);
#pragma unroll
  for (int v = 0; v < 16; ++v)
    if (!((b >> (8 * (v >> 2) + (v & 3))) & 1u)) s[v] = value;
}

template <typename T>
struct BiasTile {
  typedef T V __attribute__((__vector_size__(4 * sizeof(T))));
  // lines of 32 keys x 4 heads, 8 or 16 bytes apart from the banks of the next: reads of a
  // head of one key a line (32 lanes, bf16) fall on distinct banks, those of a line's keys too
  static constexpr int LINE = 32 * 4 * (int)sizeof(T) + 4 * (int)sizeof(T), BYTES = 32 * LINE;
  static constexpr int C = 4;  // entries of a thread
  V x[C];
  __device__ static inline int q(int u) { return (int)(threadIdx.x & 255) / 32 + 8 * u; }
  __device__ static inline int k() { return threadIdx.x % 32; }
  __device__ static inline int64_t at(const XatArgs& a, int64_t b, int q, int k) {
    return ((b * a.nq + q) * a.nk + k) * a.h;
  }
  // The tile at query q0, key k0, heads h0 .. h0 + 3; 0 past the ends.
  __device__ inline void load(const XatArgs& a, int64_t b, int h0, int q0, int k0) {
    const rsrc_t rs = buf_rsrc_n((const T*)a.bias + at(a, b, q0, k0) + h0, 0x7fffffffu);
#pragma unroll
    for (int u = 0; u < C; ++u) {
      const uint32_t off = q0 + q(u) < a.nq && k0 + k() < a.nk
                               ? (uint32_t)((q(u) * a.nk + k()) * a.h) * sizeof(T)
                               : NOWHERE;
      if constexpr (sizeof(T) == 2)
        x[u] = __builtin_bit_cast(V, __builtin_amdgcn_raw_buffer_load_b64(rs, (int)off, 0, 0));
      else
        x[u] = __builtin_bit_cast(V, __builtin_amdgcn_raw_buffer_load_b128(rs, (int)off, 0, 0));
    }
  }
  __device__ inline void store(char* t) const {
#pragma unroll
    for (int u = 0; u < C; ++u) *(V*)(t + q(u) * LINE + k() * 4 * (int)sizeof(T)) = x[u];
  }
  __device__ static inline T* entry(char* t, int q, int k, int head) {
    return (T*)(t + q * LINE + (k * 4 + head) * (int)sizeof(T));
  }
  // Writes the tile (as T holds it) to `to`, of the bias's layout.
  __device__ static inline void write(const XatArgs& a, T* to, int64_t b, int h0, int q0, int k0,
                                      const char* t) {
#pragma unroll
    for (int u = 0; u < C; ++u)
      if (q0 + q(u) < a.nq && k0 + k() < a.nk)
        *(V*)(to + at(a, b, q0 + q(u), k0 + k()) + h0) =
            *(const V*)(t + q(u) * LINE + k() * 4 * (int)sizeof(T));
  }
};

// The wave's number, known to the compiler to be the same for its lanes: what goes by it stays in
// scalar registers, buffer resources among them (one that may differ between lanes costs a
// loop over its values at each load: kernels of 2 x 2048 x 4099, 16 heads of 64, 448 us; 420 so).
__device__ inline int wave_id() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }

// Work items are numbered so that the ones that read the same keys (or rows) are neighbours.
struct Item {
  int64_t b;
  int kh, tile, split;
};
__device__ inline Item item_of(const XatArgs& a, int wg, int tiles, int splits) {
  Item t;
  t.split = wg % splits;
  wg /= splits;
  t.tile = wg % tiles;
  wg /= tiles;
  t.kh = wg % a.hk;
  t.b = wg / a.hk;
  return t;
}
// The same of four heads side by side: neighbours read the same bias lines.
__device__ inline Item heads_item(const XatArgs& a, int wg, int tiles, int splits) {
  Item t;
  const int quads = a.h / 4;
  t.kh = 4 * (wg % quads) + (wave_id() & 3);
  wg /= quads;
  t.split = wg % splits;
  wg /= splits;
  t.tile = wg % tiles;
  t.b = wg / tiles;
  return t;
}

// Adds the groups' accumulators to the first group's, in order, through the waves' places in LDS
// (`bytes` each); for all waves of a workgroup.
template <int DP, int NW, int KW>
__device__ inline void add_groups(char* lds, int bytes, f32x16 (&acc)[DP / 32]) {
  const int lane = threadIdx.x & 63, wave = wave_id();
  __syncthreads();
  if (wave >= NW) {
    f32x4* p = (f32x4*)(lds + wave * bytes) + lane;
#pragma unroll
    for (int i = 0; i < DP / 8; ++i)
      p[64 * i] = f32x4{acc[i / 4][i % 4 * 4], acc[i / 4][i % 4 * 4 + 1], acc[i / 4][i % 4 * 4 + 2],
                        acc[i / 4][i % 4 * 4 + 3]};
  }
  __syncthreads();
  if (wave < NW) {
#pragma unroll
    for (int k = 1; k < KW; ++k) {
      const f32x4* p = (const f32x4*)(lds + (wave + NW * k) * bytes) + lane;
#pragma unroll
      for (int i = 0; i < DP / 8; ++i) {
        const f32x4 x = p[64 * i];
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[i / 4][i % 4 * 4 + e] += x[e];
      }
    }
  }
}

// Waits for a wave's own LDS stores (others' where a tile is shared).
template <bool SHARED>
__device__ inline void tile_barrier() {
  if (SHARED) __syncthreads();
  else __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
}

}  // namespace triattn
