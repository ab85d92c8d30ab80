// Cross attention, backward.  With P and dP = dO V^T recomputed from the saved maximum and sum
// of each row:
//   D = sum over keys of P dP,  dS = P (dP - D),
//   dQ = scale dS K,  dK = scale dS^T Q,  dV = P^T dO,  dbias = dS.
//
// Two passes, neither of which writes P or dS but for dbias:
//   dq   a wave owns 32 rows and walks the keys, as the forward does;
//   dkv  a wave owns 32 keys and walks the rows (of all heads that share them).
//
// D: the row's sum of P dP equals dO . out, but out is rounded.  Taken from it as it is, D
// would leave sum(dS) off zero by that rounding: where one key takes all the weight, that is all
// there is of dS.  So the first pass takes d = dO . out only as a shift, dS' = P (dP - d), sums
// dS' in fp32 (e), and ends with
//   dQ = scale (dS' K - e P K),  D = d + e,
// one more product for an exact D, where a pass of its own over the keys would take two and the
// exponentials again.  A sample with one valid key has P = 1 and dS = 0 whatever its logits, which
// no rounded P and D give exactly: its dS are set to 0 (the keys are counted over all splits).
//
// dS and P are rounded to bf16 for the second products (bf16 tensors), half a step of each: dq, dk
// and dv are off by 2.4e-3 of their norms, where their own rounding alone makes 1.7e-3.  With what
// the roundings leave as products of their own it is 1.7e-3, but 432 us for 315 at 2 x 2048 x 4099
// (first passes; windows 71 for 66, 768 x 768 with 16 heads of 24 46 for 42).
//
// 2 x 2048 x 4099, 16 heads of 64, a quarter of the keys masked: dq 123 us, dkv 147 (840 and 700
// TFLOP/s of the valid keys' four products each; 137 and 168 in the first passes), as the forward
// with no unit busy all the time: two waves a SIMD for their registers, vector issue 53 and 46% of
// the cycles, the matrix cores 41 and 36%.  737 windows of 32 x 128: 22 and 43 us, 5 and 3.5 TB/s.
#include "timing.h"
#include "triattn.h"
#include "xat.h"

namespace triattn {
namespace {

// P of logits s (accumulator values): exp2(s c + add), or with a bias exp2((s - m) c + add).
template <bool BIAS>
__device__ inline float weight(float s, float c, float m, float add) {
  return __builtin_amdgcn_exp2f(BIAS ? fmaf(s - m, c, add) : fmaf(s, c, add));
}

// A row's statistics as weight() takes them: its maximum (with a bias), and the addend, -inf
// for a row without keys (P = 0).
template <bool BIAS>
__device__ inline void row_stat(f32x2 x, float& m, float& add) {
  const bool none = x[0] == neg_inf();
  m = none ? 0.f : x[0];
  add = none ? neg_inf() : -LOG2E * (BIAS ? x[1] : x[0] + x[1]);
}

// Partial results of a split of the keys: dS' K and P K of every row, then e.
__device__ inline float* part_ab(const XatArgs& a, int split, int64_t R, int which) {
  const int64_t all = a.batch * a.nq * a.h;
  return a.part + (((int64_t)split * all + R) * 2 + which) * a.d;
}
__device__ inline float* part_e(const XatArgs& a, int split, int64_t R) {
  const int64_t all = a.batch * a.nq * a.h;
  return a.part + (int64_t)a.splits * all * 2 * a.d + (int64_t)split * all + R;
}

template <typename T, int DP, int NW, int MODE, int KW>
__global__ __launch_bounds__(64 * NW * KW, (xat_waves<T, DP, NW>())) void xat_dq_kernel(XatArgs a,
                                                                                   int tiles) {
  constexpr bool BIAS = MODE != XB_NONE, HEADS = MODE == XB_HEADS;
  constexpr int SW = HEADS ? 1 : NW;  // waves that share a tile
  constexpr int BK = xat_keys<T, DP, SW>(), J = BK / 32;
  constexpr uint64_t ALL = BK == 64 ? ~0ull : (1ull << BK) - 1;
  using St = KvStage<T, DP, BK, SW>;
  using Bt = BiasTile<T>;
  using L = XTile<T, DP>;
  __shared__ __attribute__((aligned(16))) char lds[2 * St::BYTES * (SW == 1 ? NW * KW : 2)];
  __shared__ __attribute__((aligned(16))) char blds[HEADS ? 2 * KW * Bt::BYTES : 16];
  const int wg = xcd_swizzle(blockIdx.x, gridDim.x);
  const Item w = HEADS ? heads_item(a, wg, tiles, a.splits) : item_of(a, wg, tiles, a.splits);
  const int lane = threadIdx.x & 63, wave = wave_id(), g = lane >> 5;
  const int head = wave % NW, group = wave / NW;  // head: or the tile of rows (keys)
  const int rows = a.nq * a.group, first = (w.tile * SW + (HEADS ? 0 : head)) * 32;
  const int64_t bb = a.bias_batch == 1 ? 0 : w.b;
  const int r = first + (lane & 31), in = r < rows ? r : rows - 1;
  const int64_t R = row_at(a, w.b, w.kh, in, 1);
  typename L::Row q, dy;
  L::row((const T*)a.q + R * a.d, a.d, r < rows, q);
  L::row((const T*)a.dout + R * a.d, a.d, r < rows, dy);
  float shift;
  {
    typename L::Row o;
    L::row((const T*)a.out + R * a.d, a.d, r < rows, o);
    shift = wave_xor32_sum(L::dot_regs(dy, o));
  }
  float m, add;
  row_stat<BIAS>(*(const f32x2*)(a.stat + 2 * R), m, add);
  const T* bias = nullptr;
  if (MODE == XB_PLANES)
    bias = (const T*)a.planes + ((bb * a.hk + w.kh) * rows + in) * a.nkp + 4 * g;
  const int nt = (a.nk + BK - 1) / BK;
  const int t0 = (int)((int64_t)nt * w.split / a.splits);
  const int t1 = (int)((int64_t)nt * (w.split + 1) / a.splits);
  const float c = BIAS ? LOG2E : a.scale * LOG2E;
  f32x16 sk[DP / 32] = {}, pk[DP / 32] = {};
  float e = 0.f;
  int valid = 0;  // keys
  constexpr int D = xat_ahead<T, DP>(SW, 64);  // loads run D tiles ahead
  St st[D];
  Bt bt[D];
  const int n = (t1 - t0 + KW - 1) / KW;  // steps, in each the next KW tiles
  auto load = [&](int d, int i) {
    const int t = t0 + i * KW + group, k0 = t < t1 ? t * BK : nt * BK;
    st[d].load(a, w.b, w.kh, k0);
    if (HEADS) bt[d].load(a, bb, w.kh & ~3, first, k0);
  };
  auto step = [&](int d, int i) {
    const int t = t0 + i * KW + group;
    char* tk = lds + (SW == 1 ? wave : i & 1) * 2 * St::BYTES;
    char* tv = tk + St::BYTES;
    char* tb = blds + (HEADS ? (2 * group + (i & 1)) * Bt::BYTES : 0);
    const uint64_t ok = st[d].bits();
    st[d].store(tk, tv, ok);
    if (HEADS) bt[d].store(tb);
    valid += __popcll(ok);
    load(d, i + D);
    tile_barrier<(SW > 1 || HEADS)>();
    if (ok == 0 || first >= rows) return;
#pragma unroll
    for (int j = 0; j < J; ++j) {
      f32x16 s = L::dot(tk, 32 * j, q, f32x16{});
      f32x16 dp = L::dot(tv, 32 * j, dy, f32x16{});
      if constexpr (BIAS) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          f32x4 x;
          if constexpr (HEADS) {
#pragma unroll
            for (int u = 0; u < 4; ++u)
              x[u] = (float)*Bt::entry(tb, lane & 31, 8 * i + 4 * g + u, head);
          } else {
            x = load4(bias + (int64_t)t * BK + 32 * j + 8 * i);
          }
#pragma unroll
          for (int u = 0; u < 4; ++u) s[4 * i + u] = fmaf(s[4 * i + u], a.scale, x[u]);
        }
      }
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        s[v] = weight<BIAS>(s[v], c, m, add);
        dp[v] -= shift;
        asm volatile("" : "+v"(s[v]), "+v"(dp[v]));  // made before the branch
      }
      if (ok != ALL) mask_tile(s, (uint32_t)(ok >> (32 * j)), g, 0.f);
      dp *= s;
      typename L::Frag fp, fs;
      acc_frags(s, fp);
      acc_frags(dp, fs);
      e += sum16(dp);
      L::add2(tk, 32 * j, fs, sk, fp, pk);
    }
  };
#pragma unroll
  for (int d = 0; d < D; ++d) load(d, d);
  for (int i = 0; i < n; i += D) {
    step(0, i);
    if (D == 2 && i + 1 < n) step(D - 1, i + 1);
  }
  float sum = wave_xor32_sum(e);
  if constexpr (KW > 1) {
    __shared__ float part[NW * KW][32];
    __shared__ int count[NW * KW];
    if (g == 0) part[wave][lane] = sum;
    if (lane == 0) count[wave] = valid;
    add_groups<DP, NW, KW>(lds, 2 * St::BYTES, sk);
    add_groups<DP, NW, KW>(lds, 2 * St::BYTES, pk);
    if (group > 0) return;
#pragma unroll
    for (int k = 1; k < KW; ++k) {
      sum += part[head + NW * k][lane & 31];
      valid += count[head + NW * k];
    }
  }
  // (of split keys, the sample's are known to the join)
  const bool single = a.splits == 1 && valid <= 1;
  if (w.tile == 0 && w.kh == 0 && threadIdx.x == 0) {
    if (a.splits > 1) a.valid[w.b * a.splits + w.split] = valid;
    else a.single[w.b] = single;
  }
  if (r >= rows) return;
  if (a.splits > 1) {
    float *ps = part_ab(a, w.split, R, 0), *pp = part_ab(a, w.split, R, 1);
#pragma unroll
    for (int n = 0; n < DP / 32; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int ch = 32 * n + 8 * i + 4 * g;
        if (ch < a.d) {
          const f32x16 &x = sk[n], &y = pk[n];
          store4(ps + ch, f32x4{x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]});
          store4(pp + ch, f32x4{y[4 * i], y[4 * i + 1], y[4 * i + 2], y[4 * i + 3]});
        }
      }
    if (g == 0) {
      *part_e(a, w.split, R) = sum;
      if (w.split == 0) a.dsum[R] = shift;
    }
    return;
  }
  T* dq = (T*)a.dq + R * a.d;
#pragma unroll
  for (int n = 0; n < DP / 32; ++n)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int ch = 32 * n + 8 * i + 4 * g;
      f32x4 x;
#pragma unroll
      for (int u = 0; u < 4; ++u)
        x[u] = single ? 0.f : a.scale * fmaf(-sum, pk[n][4 * i + u], sk[n][4 * i + u]);
      if (ch < a.d) store4(dq + ch, x);
    }
  if (g == 0) a.dsum[R] = shift + sum;
}

// Joins the splits of the keys: four channels of a row a thread.
template <typename T>
__global__ __launch_bounds__(256) void xat_dq_join_kernel(XatArgs a) {
  const int64_t all = a.batch * a.nq * a.h, quads = a.d / 4;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= all * quads) return;
  const int64_t R = i / quads;
  const int ch = 4 * (int)(i % quads);
  const uint32_t rows = (uint32_t)a.nq * a.h, b = (uint32_t)R / rows;  // (at most 2^31 rows)
  f32x4 sk{}, pk{};
  float e = 0.f;
  int valid = 0;
  for (int s = 0; s < a.splits; ++s) {
    sk += *(const f32x4*)(part_ab(a, s, R, 0) + ch);
    pk += *(const f32x4*)(part_ab(a, s, R, 1) + ch);
    e += *part_e(a, s, R);
    valid += a.valid[(int64_t)b * a.splits + s];
  }
  const bool single = valid <= 1;
  f32x4 x;
#pragma unroll
  for (int u = 0; u < 4; ++u) x[u] = single ? 0.f : a.scale * fmaf(-e, pk[u], sk[u]);
  store4((T*)a.dq + R * a.d + ch, x);
  if (ch == 0) {
    a.dsum[R] += e;
    if ((uint32_t)R == b * rows) a.single[b] = single;
  }
}

// Tiles of BQ rows of q and dout, and the rows' statistics.
template <typename T, int DP, int BQ, int NW, bool BIAS>
struct RowStage {
  using S = Share<DP, BQ, NW>;
  using L = XTile<T, DP>;
  static constexpr int TILE = BQ * L::LINE, BYTES = 2 * TILE + 3 * BQ * 4;
  Chunk<T> q[S::C], dy[S::C];
  f32x2 stat;
  float d;
  bool real;
  __device__ inline void load(const XatArgs& a, int64_t b, int kh, int r0) {
    const int rows = a.nq * a.group, q0 = row_query(a, r0 < rows ? r0 : 0);
    const int64_t at = ((b * a.nq + q0) * a.h + kh * a.group) * a.d;
    const uint32_t n = 0x7fffffffu;  // rows are checked here
    const rsrc_t rq = buf_rsrc_n((const T*)a.q + at, n), rd = buf_rsrc_n((const T*)a.dout + at, n);
#pragma unroll
    for (int u = 0; u < S::C; ++u) {
      const int r = r0 + S::line(u), c = 8 * S::col(u), qi = row_query(a, r);
      const uint32_t off =
          r < rows && c < a.d
              ? (uint32_t)(((qi - q0) * a.h + r - qi * a.group) * a.d + c) * sizeof(T)
              : NOWHERE;
      q[u] = load_chunk<T>(rq, off);
      dy[u] = load_chunk<T>(rd, off);
    }
    const int id = threadIdx.x % (64 * NW), r = r0 + id, qi = row_query(a, r);
    real = id < BQ && r < rows;
    const int64_t R0 = (b * a.nq + q0) * a.h + kh * a.group;
    const uint32_t i = (uint32_t)((qi - q0) * a.h + r - qi * a.group);
    stat = __builtin_bit_cast(
        f32x2, __builtin_amdgcn_raw_buffer_load_b64(buf_rsrc_n(a.stat + 2 * R0, n),
                                                    (int)(real ? 8 * i : NOWHERE), 0, 0));
    d = __builtin_bit_cast(
        float, __builtin_amdgcn_raw_buffer_load_b32(buf_rsrc_n(a.dsum + R0, n),
                                                    (int)(real ? 4 * i : NOWHERE), 0, 0));
  }
  __device__ inline void store(char* t) const {
#pragma unroll
    for (int u = 0; u < S::C; ++u) {
      L::put(t, S::line(u), S::col(u), q[u]);
      L::put(t + TILE, S::line(u), S::col(u), dy[u]);
    }
    const int id = threadIdx.x % (64 * NW);
    if (id < BQ) {
      float m, add;
      row_stat<BIAS>(real ? stat : f32x2{neg_inf(), 0.f}, m, add);
      float* p = (float*)(t + 2 * TILE) + id;
      p[0] = m;
      p[BQ] = add;
      p[2 * BQ] = d;
    }
  }
};

template <typename T, int DP, int NW, int MODE, int KW, typename DS = float>
__global__ __launch_bounds__(64 * NW * KW, (xat_waves<T, DP, NW>())) void xat_dkv_kernel(XatArgs a,
                                                                                    int tiles) {
  constexpr bool BIAS = MODE != XB_NONE, HEADS = MODE == XB_HEADS;
  constexpr int SW = HEADS ? 1 : NW;  // waves that share a tile
  constexpr int BQ = xat_keys<T, DP, SW>(), J = BQ / 32;
  using St = RowStage<T, DP, BQ, SW, BIAS>;
  using Bt = BiasTile<T>;
  using Dt = BiasTile<DS>;
  using L = XTile<T, DP>;
  // dS of the four heads leaves through LDS: in the bias's place where it has the bias's type
  constexpr bool SAME = sizeof(T) == sizeof(DS);
  __shared__ __attribute__((aligned(16))) char lds[St::BYTES * (SW == 1 ? NW * KW : 2)];
  __shared__ __attribute__((aligned(16))) char blds[HEADS ? 2 * KW * Bt::BYTES : 16];
  __shared__ __attribute__((aligned(16))) char dlds[HEADS && !SAME ? 2 * KW * Dt::BYTES : 16];
  const int wg = xcd_swizzle(blockIdx.x, gridDim.x);
  const Item w = HEADS ? heads_item(a, wg, tiles, a.splits_q) : item_of(a, wg, tiles, a.splits_q);
  const int lane = threadIdx.x & 63, wave = wave_id(), g = lane >> 5;
  const int head = wave % NW, group = wave / NW;  // head: or the tile of rows (keys)
  const int rows = a.nq * a.group, first = (w.tile * SW + (HEADS ? 0 : head)) * 32;
  const int key = first + (lane & 31);
  const int64_t bb = a.bias_batch == 1 ? 0 : w.b;
  const bool valid = key < a.nk && (a.mask == nullptr || a.mask[w.b * a.nk + key] != 0);
  const int64_t K = (w.b * a.nk + (key < a.nk ? key : a.nk - 1)) * a.hk + w.kh;
  typename L::Row kf, vf;
  L::row((const T*)a.k + K * a.d, a.d, valid, kf);
  L::row((const T*)a.v + K * a.d, a.d, valid, vf);
  const T* bias = nullptr;
  float* ds = nullptr;
  if (MODE == XB_PLANES) {
    bias = (const T*)a.planes + (bb * a.hk + w.kh) * rows * a.nkp + key;
    if (a.dbias) ds = a.dplanes + (w.b * a.hk + w.kh) * rows * a.nkp + key;
  }
  const int nt = (rows + BQ - 1) / BQ;
  const int t0 = (int)((int64_t)nt * w.split / a.splits_q);
  const int t1 = (int)((int64_t)nt * (w.split + 1) / a.splits_q);
  const float c = BIAS ? LOG2E : a.scale * LOG2E;
  f32x16 dv[DP / 32] = {}, dk[DP / 32] = {};
  const bool single = a.single[w.b] != 0;
  constexpr int D = HEADS ? xat_ahead<T, DP>(SW, 64) : 1;  // loads run D tiles ahead
  St st[D];
  Bt bt[D];
  const int n = (t1 - t0 + KW - 1) / KW;  // steps, in each the next KW tiles
  auto load = [&](int d, int i) {
    const int t = t0 + i * KW + group, r0 = t < t1 ? t * BQ : nt * BQ;
    st[d].load(a, w.b, w.kh, r0);
    if (HEADS) bt[d].load(a, bb, w.kh & ~3, r0, first);
  };
  const bool any = __any(valid);  // the wave has a valid key
  auto step = [&](int d, int i) {
    const int t = t0 + i * KW + group;
    char* tq = lds + (SW == 1 ? wave : i & 1) * St::BYTES;
    char* td = tq + St::TILE;
    char* tb = blds + (HEADS ? (2 * group + (i & 1)) * Bt::BYTES : 0);
    char* ts = SAME ? tb : dlds + (HEADS ? (2 * group + (i & 1)) * Dt::BYTES : 0);
    const float* stat = (const float*)(tq + 2 * St::TILE);
    st[d].store(tq);
    if (HEADS) bt[d].store(tb);
    load(d, i + D);
    tile_barrier<(SW > 1 || HEADS)>();
    if (!any && !BIAS) return;
    if (first >= a.nk) return;
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const int r0 = t * BQ + 32 * j;
      // (with the heads side by side every wave comes to the barrier below: a tile past the
      // group's last is zeros, and its dS go nowhere)
      if (!HEADS && (t >= t1 || r0 >= rows)) break;
      float x[16];
      if constexpr (BIAS) {
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          const int r = r0 + acc_row(v, g);
          if (HEADS) x[v] = (float)*Bt::entry(tb, acc_row(v, g), lane & 31, head);
          else x[v] = key < a.nk && r < rows ? (float)bias[(int64_t)r * a.nkp] : 0.f;
        }
      }
      f32x16 s = L::dot(tq, 32 * j, kf, f32x16{});
      f32x16 dp = L::dot(td, 32 * j, vf, f32x16{});
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int line = 32 * j + 8 * i + 4 * g;
        f32x4 m{};
        if (BIAS) m = *(const f32x4*)(stat + line);
        const f32x4 add = *(const f32x4*)(stat + BQ + line);
        const f32x4 sum = *(const f32x4*)(stat + 2 * BQ + line);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const int v = 4 * i + u;
          if constexpr (BIAS) s[v] = fmaf(s[v], a.scale, x[v]);
          s[v] = weight<BIAS>(s[v], c, m[u], add[u]);
          dp[v] = s[v] * (dp[v] - sum[u]);
        }
      }
      if (single) dp = f32x16{};
      if (HEADS && a.dbias) {
        // a wave writes where it alone has read; all four before the entries leave
#pragma unroll
        for (int v = 0; v < 16; ++v)
          *Dt::entry(ts, acc_row(v, g), lane & 31, head) = (DS)(valid ? dp[v] : 0.f);
        __syncthreads();
        Dt::write(a, a.bias_batch == a.batch ? (DS*)a.dbias : (DS*)a.dplanes, w.b, w.kh & ~3,
                  t < t1 ? r0 : rows, first, ts);
      }
      if (MODE == XB_PLANES && ds) {
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          const int r = r0 + acc_row(v, g);
          if (key < a.nk && r < rows) ds[(int64_t)r * a.nkp] = valid ? dp[v] : 0.f;
        }
      }
      typename L::Frag f;
      acc_frags(s, f);
      L::add(td, 32 * j, f, dv);
      acc_frags(dp, f);
      L::add(tq, 32 * j, f, dk);
    }
  };
  // a workgroup whose keys are all masked has nothing to sum
  if (BIAS || __syncthreads_or(valid)) {
#pragma unroll
    for (int d = 0; d < D; ++d) load(d, d);
    for (int i = 0; i < n; i += D) {
      step(0, i);
      if (D == 2 && i + 1 < n) step(D - 1, i + 1);
    }
  }
  if constexpr (KW > 1) {
    add_groups<DP, NW, KW>(lds, St::BYTES, dv);
    add_groups<DP, NW, KW>(lds, St::BYTES, dk);
    if (group > 0) return;
  }
  if (key >= a.nk) return;
  // whatever the column of a masked key holds, its gradients are zeros
  const int64_t all = a.batch * a.nk * a.hk * a.d;
  float* part = a.part_q + (int64_t)w.split * 2 * all + K * a.d;
#pragma unroll
  for (int n = 0; n < DP / 32; ++n)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int ch = 32 * n + 8 * i + 4 * g;
      f32x4 x{}, y{};
      if (valid) {
#pragma unroll
        for (int u = 0; u < 4; ++u) x[u] = a.scale * dk[n][4 * i + u], y[u] = dv[n][4 * i + u];
      }
      if (ch >= a.d) continue;
      if (a.splits_q > 1) {
        store4(part + ch, x);
        store4(part + all + ch, y);
      } else {
        store4((T*)a.dk + K * a.d + ch, x);
        store4((T*)a.dv + K * a.d + ch, y);
      }
    }
}

// Sums of the splits of the rows: four channels of dk and of dv a thread.
template <typename T>
__global__ __launch_bounds__(256) void xat_dkv_join_kernel(XatArgs a) {
  const int64_t all = a.batch * a.nk * a.hk * a.d;
  const int64_t i = 4 * ((int64_t)blockIdx.x * 256 + threadIdx.x);
  if (i >= all) return;
  f32x4 x{}, y{};
  for (int s = 0; s < a.splits_q; ++s) {
    x += *(const f32x4*)(a.part_q + (int64_t)s * 2 * all + i);
    y += *(const f32x4*)(a.part_q + (int64_t)s * 2 * all + all + i);
  }
  store4((T*)a.dk + i, x);
  store4((T*)a.dv + i, y);
}

template <typename T, int DP, int NW, int MODE>
void dq_launch(const XatArgs& a, hipStream_t s) {
  constexpr int KW = xat_most_groups<T, DP, NW, MODE>();
  const int tiles = xat_row_tiles(a, MODE == XB_HEADS ? 1 : NW);
  const int64_t wgs = xat_row_wgs(sizeof(T) == 2 ? TRIATTN_BF16 : TRIATTN_F32, a);
  const dim3 grid((unsigned)(wgs * a.splits));
  if (KW > 1 && xat_groups(wgs, xat_key_steps(a)))
    hipLaunchKernelGGL((xat_dq_kernel<T, DP, NW, MODE, KW>), grid, dim3(64 * NW * KW), 0, s, a,
                       tiles);
  else
    hipLaunchKernelGGL((xat_dq_kernel<T, DP, NW, MODE, 1>), grid, dim3(64 * NW), 0, s, a, tiles);
}
// DS: dbias as it leaves the kernel, the tensors' type, or fp32 to be summed over the samples.
template <typename T, int DP, int NW, int MODE, typename DS = float>
void dkv_launch(const XatArgs& a, hipStream_t s) {
  constexpr int KW = xat_most_groups<T, DP, NW, MODE>();
  // (fp32 tiles of dS beside bf16 ones of the bias leave no room for two groups of 64 channels)
  constexpr int GROUPS = MODE == XB_HEADS && sizeof(DS) > sizeof(T) && DP == 64 ? 1 : KW;
  const int tiles = xat_key_tiles(a, MODE == XB_HEADS ? 1 : NW);
  const int64_t wgs = xat_key_wgs(sizeof(T) == 2 ? TRIATTN_BF16 : TRIATTN_F32, a);
  const dim3 grid((unsigned)(wgs * a.splits_q));
  if (GROUPS > 1 && xat_groups(wgs, xat_row_steps(a)))
    hipLaunchKernelGGL((xat_dkv_kernel<T, DP, NW, MODE, GROUPS, DS>), grid, dim3(64 * NW * GROUPS),
                       0, s, a, tiles);
  else
    hipLaunchKernelGGL((xat_dkv_kernel<T, DP, NW, MODE, 1, DS>), grid, dim3(64 * NW), 0, s, a,
                       tiles);
}
template <typename T, int DP>
void dq_width(const XatArgs& a, bool heads, hipStream_t s) {
  constexpr int ONE = sizeof(T) == 2 || DP <= 64 ? 1 : 4;
  const int nw = xat_row_waves(sizeof(T) == 2 ? TRIATTN_BF16 : TRIATTN_F32, a);
  if constexpr (sizeof(T) == 2 || DP <= 64)
    if (heads) return dq_launch<T, DP, 4, XB_HEADS>(a, s);
  if (a.bias)
    nw == 1 ? dq_launch<T, DP, ONE, XB_PLANES>(a, s) : dq_launch<T, DP, 4, XB_PLANES>(a, s);
  else nw == 1 ? dq_launch<T, DP, ONE, XB_NONE>(a, s) : dq_launch<T, DP, 4, XB_NONE>(a, s);
}
template <typename T, int DP>
void dkv_width(const XatArgs& a, bool heads, hipStream_t s) {
  constexpr int ONE = sizeof(T) == 2 || DP <= 64 ? 1 : 4;
  const int nw = xat_key_waves(sizeof(T) == 2 ? TRIATTN_BF16 : TRIATTN_F32, a);
  if constexpr (sizeof(T) == 2 || DP <= 64) {
    if (heads && a.bias_batch == a.batch) return dkv_launch<T, DP, 4, XB_HEADS, T>(a, s);
    if (heads) return dkv_launch<T, DP, 4, XB_HEADS, float>(a, s);
  }
  if (a.bias)
    nw == 1 ? dkv_launch<T, DP, ONE, XB_PLANES>(a, s) : dkv_launch<T, DP, 4, XB_PLANES>(a, s);
  else nw == 1 ? dkv_launch<T, DP, ONE, XB_NONE>(a, s) : dkv_launch<T, DP, 4, XB_NONE>(a, s);
}

template <typename T>
hipError_t bwd(const XatArgs& a, hipStream_t s) {
  const int dtype = sizeof(T) == 2 ? TRIATTN_BF16 : TRIATTN_F32;
  const bool heads = xat_by_heads(dtype, a);
  if (a.bias && !heads) {
    const hipError_t e = launch_xat_planes(dtype, a, s);
    if (e != hipSuccess) return e;
  }
  {
    KernelTimer t(K_XAT_DQ, s);
    if (a.d <= 32) dq_width<T, 32>(a, heads, s);
    else if (a.d <= 64) dq_width<T, 64>(a, heads, s);
    else dq_width<T, 128>(a, heads, s);
  }
  if (a.splits > 1) {
    KernelTimer t(K_XAT_JOIN, s);
    const int64_t n = a.batch * a.nq * a.h * (a.d / 4);
    hipLaunchKernelGGL(xat_dq_join_kernel<T>, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, s,
                       a);
  }
  {
    KernelTimer t(K_XAT_DKV, s);
    if (a.d <= 32) dkv_width<T, 32>(a, heads, s);
    else if (a.d <= 64) dkv_width<T, 64>(a, heads, s);
    else dkv_width<T, 128>(a, heads, s);
  }
  if (a.splits_q > 1) {
    KernelTimer t(K_XAT_JOIN, s);
    const int64_t n = a.batch * a.nk * a.hk * (a.d / 4);
    hipLaunchKernelGGL(xat_dkv_join_kernel<T>, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, s,
                       a);
  }
  if (a.dbias && !(heads && a.bias_batch == a.batch)) return launch_xat_dbias(dtype, a, heads, s);
  return hipGetLastError();
}

}  // namespace

XatPlan xat_bwd_plan(int dtype, const XatArgs& a) {
  XatPlan p{};
  const int64_t all = a.batch * a.nq * a.h, keys = a.batch * a.nk * a.hk;
  p.nkp = (a.nk + 63) / 64 * 64;
  p.splits = xat_key_splits(dtype, a);
  p.splits_q = xat_row_splits(dtype, a);
  const size_t e = dtype == TRIATTN_BF16 ? 2 : 4;
  if (a.bias_batch) {
    const bool heads = xat_by_heads(dtype, a);
    const size_t maps = (size_t)a.batch * a.h * a.nq;
    if (!heads) p.planes = (size_t)a.bias_batch * a.h * a.nq * p.nkp * e;
    // (unused without dbias)
    if (!heads) p.dplanes = maps * p.nkp * sizeof(float);
    else if (a.bias_batch != a.batch) p.dplanes = maps * a.nk * sizeof(float);
  }
  p.dsum = (size_t)all * sizeof(float);
  p.single = (size_t)a.batch * sizeof(int);
  if (p.splits > 1) p.valid = (size_t)a.batch * p.splits * sizeof(int);
  if (p.splits > 1) p.part = (size_t)p.splits * all * (2 * a.d + 1) * sizeof(float);
  if (p.splits_q > 1) p.part_q = (size_t)p.splits_q * keys * 2 * a.d * sizeof(float);
  return p;
}

hipError_t launch_xat_bwd(int dtype, const XatArgs& a, hipStream_t s) {
  return dtype == TRIATTN_BF16 ? bwd<bf16>(a, s) : bwd<float>(a, s);
}

}  // namespace triattn
