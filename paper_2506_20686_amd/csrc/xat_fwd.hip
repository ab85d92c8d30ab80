// Cross attention, forward: out = softmax(scale q k^T + bias over the valid keys) v.
//
// One pass over the keys with a running maximum and sum a row.  A wave owns 32 rows (a row a
// lane, its keys over the accumulator's registers: S^T = K Q^T), so the row's statistics are a
// lane's own; P^T feeds back as an operand of O^T = V^T P^T.  Tiles of keys and values go
// through registers into LDS, the next tile's loads in flight while one is multiplied.
//
// Logits stay in natural units where there is a bias: a bias of the type's lowest value would
// overflow in base 2.  P is rounded to bf16 for its product (bf16 tensors), half a step of each
// weight: an output is off by 1.9e-3 to 2.3e-3 of its norm, where its own rounding alone makes
// 1.7e-3.  With what the rounding leaves as a second product, 16 bits of P, it is 1.7e-3, but 137
// us for 107 at 2 x 2048 x 4099 (first passes; windows 21.3 for 20.7).
//
// With long loops no unit is busy all the time: vector issue (an exponential a logit, a quarter of
// the rate, and some 100 other instructions a 32 x 32 tile) takes 55% of the cycles, the matrix
// cores 26%, LDS 21%, one after the other in each of the two waves a SIMD that 512 workgroups
// make.  2 x 2048 x 4099, 16 heads of 64, a quarter of the keys masked: 89 us (770 TFLOP/s of all
// keys, 580 of the valid ones; 105 us in the first passes, before the card has settled).  One
// query to 30,011 keys: 22 us, 4.1 TB/s.  737 windows of 32 x 128 with a bias: 20 us, 4.3 TB/s.
#include "timing.h"
#include "triattn.h"
#include "xat.h"

namespace triattn {
namespace {

template <typename T, int DP, int NW, int MODE, int KW>
__global__ __launch_bounds__(64 * NW * KW, (xat_fwd_waves<T, DP, NW, MODE>())) void xat_fwd_kernel(
    XatArgs a, int tiles) {
  constexpr bool BIAS = MODE != XB_NONE, HEADS = MODE == XB_HEADS;
  constexpr int SW = HEADS ? 1 : NW;  // waves that share a tile
  constexpr int BK = xat_keys<T, DP, SW>(), J = BK / 32;
  constexpr uint64_t ALL = BK == 64 ? ~0ull : (1ull << BK) - 1;
  using St = KvStage<T, DP, BK, SW>;
  using Bt = BiasTile<T>;
  using L = XTile<T, DP>;
  // K and V of each wave, or two buffers of all waves'; the groups' bias tiles, two buffers each
  __shared__ __attribute__((aligned(16))) char lds[2 * St::BYTES * (SW == 1 ? NW * KW : 2)];
  __shared__ __attribute__((aligned(16))) char blds[HEADS ? 2 * KW * Bt::BYTES : 16];
  const int wg = xcd_swizzle(blockIdx.x, gridDim.x);
  const Item w = HEADS ? heads_item(a, wg, tiles, a.splits) : item_of(a, wg, tiles, a.splits);
  const int lane = threadIdx.x & 63, wave = wave_id(), g = lane >> 5;
  const int head = wave % NW, group = wave / NW;  // head: or the tile of rows
  const int rows = a.nq * a.group, first = (w.tile * SW + (HEADS ? 0 : head)) * 32;
  const int r = first + (lane & 31), in = r < rows ? r : rows - 1;
  const int64_t bb = a.bias_batch == 1 ? 0 : w.b;
  typename L::Row q;
  L::row((const T*)a.q + row_at(a, w.b, w.kh, in, a.d), a.d, r < rows, q);
  const T* bias = nullptr;
  if (MODE == XB_PLANES)
    bias = (const T*)a.planes + ((bb * a.hk + w.kh) * rows + in) * a.nkp + 4 * g;
  const int nt = (a.nk + BK - 1) / BK;
  const int t0 = (int)((int64_t)nt * w.split / a.splits);
  const int t1 = (int)((int64_t)nt * (w.split + 1) / a.splits);
  const float c = BIAS ? LOG2E : a.scale * LOG2E;
  float m = neg_inf(), l = 0.f;
  f32x16 o[DP / 32] = {};
  // loads run D tiles ahead; past the end they touch no memory
  constexpr int D = xat_ahead<T, DP>(SW, 128);
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
    load(d, i + D);
    // what waves share was last read two steps ago, before the barrier of the last step
    tile_barrier<(SW > 1 || HEADS)>();
    if (ok == 0 || first >= rows) return;
    f32x16 s[J];
#pragma unroll
    for (int j = 0; j < J; ++j) {
      s[j] = L::dot(tk, 32 * j, q, f32x16{});
      if constexpr (BIAS) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          f32x4 x;
          if constexpr (HEADS) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              x[e] = (float)*Bt::entry(tb, lane & 31, 8 * i + 4 * g + e, head);
          } else {
            x = load4(bias + (int64_t)t * BK + 32 * j + 8 * i);
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) s[j][4 * i + e] = fmaf(s[j][4 * i + e], a.scale, x[e]);
        }
      }
    }
    float top = max16(s[0]);
    if constexpr (J == 2) top = fmaxf(top, max16(s[J - 1]));
    asm volatile("" : "+v"(top));  // made before the branch
    if (ok != ALL) {
#pragma unroll
      for (int j = 0; j < J; ++j) mask_tile(s[j], (uint32_t)(ok >> (32 * j)), g, neg_inf());
      top = max16(s[0]);
      if constexpr (J == 2) top = fmaxf(top, max16(s[J - 1]));
    }
    top = fmaxf(m, wave_xor32_max(top));
    if (__any(top > m)) {
      const float f = top > m ? __builtin_amdgcn_exp2f((m - top) * c) : 1.f;
      l *= f;
#pragma unroll
      for (int n = 0; n < DP / 32; ++n)
#pragma unroll
        for (int v = 0; v < 16; ++v) o[n][v] *= f;
      m = top;
    }
    const float base = m == neg_inf() ? 0.f : m, shift = -base * c;
#pragma unroll
    for (int j = 0; j < J; ++j) {
#pragma unroll
      for (int v = 0; v < 16; ++v)
        s[j][v] = __builtin_amdgcn_exp2f(BIAS ? (s[j][v] - base) * c : fmaf(s[j][v], c, shift));
      l += sum16(s[j]);
      typename L::Frag p;
      acc_frags(s[j], p);
      L::add(tv, 32 * j, p, o);
    }
  };
#pragma unroll
  for (int d = 0; d < D; ++d) load(d, d);
  for (int i = 0; i < n; i += D) {
    step(0, i);
    if (D == 2 && i + 1 < n) step(D - 1, i + 1);
  }
  l = wave_xor32_sum(l);
  if constexpr (KW > 1) {  // all groups to the maximum of theirs, then their sums
    __shared__ f32x2 ml[NW * KW][32];
    if (g == 0) ml[wave][lane] = f32x2{m, l};
    __syncthreads();
    float top = m;
#pragma unroll
    for (int k = 0; k < KW; ++k) top = fmaxf(top, ml[head + NW * k][lane & 31][0]);
    const float f = top > m ? __builtin_amdgcn_exp2f((m - top) * c) : 1.f;
#pragma unroll
    for (int n = 0; n < DP / 32; ++n)
#pragma unroll
      for (int v = 0; v < 16; ++v) o[n][v] *= f;
    l = 0.f;
#pragma unroll
    for (int k = 0; k < KW; ++k) {
      const f32x2 x = ml[head + NW * k][lane & 31];
      l = fmaf(x[1], top > x[0] ? __builtin_amdgcn_exp2f((x[0] - top) * c) : 1.f, l);
    }
    m = top;
    add_groups<DP, NW, KW>(lds, 2 * St::BYTES, o);
    if (group > 0) return;
  }
  if (r >= rows) return;
  if (!BIAS) m *= a.scale;  // scale > 0: -inf stays
  const int64_t R = row_at(a, w.b, w.kh, r, 1);
  const int64_t all = a.batch * a.nq * a.h;
  if (a.splits > 1) {
    float* po = a.part + ((int64_t)w.split * all + R) * a.d;
    float* pm = a.part + (int64_t)a.splits * all * a.d + ((int64_t)w.split * all + R) * 2;
#pragma unroll
    for (int n = 0; n < DP / 32; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int ch = 32 * n + 8 * i + 4 * g;
        if (ch < a.d) store4(po + ch, f32x4{o[n][4 * i], o[n][4 * i + 1], o[n][4 * i + 2],
                                            o[n][4 * i + 3]});
      }
    if (g == 0) *(f32x2*)pm = f32x2{m, l};
    return;
  }
  const float inv = l > 0.f ? 1.f / l : 0.f;
  T* out = (T*)a.out + R * a.d;
#pragma unroll
  for (int n = 0; n < DP / 32; ++n)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int ch = 32 * n + 8 * i + 4 * g;
      if (ch < a.d) store4(out + ch, f32x4{o[n][4 * i] * inv, o[n][4 * i + 1] * inv,
                                           o[n][4 * i + 2] * inv, o[n][4 * i + 3] * inv});
    }
  if (g == 0) *(f32x2*)(a.stat + 2 * R) = f32x2{m, l > 0.f ? __logf(l) : 0.f};
}

// Joins the splits: a wave a row, its lanes over channels (in fours) and over splits.
template <typename T>
__global__ __launch_bounds__(256) void xat_join_kernel(XatArgs a) {
  const int64_t all = a.batch * a.nq * a.h;
  const int64_t R = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (R >= all) return;
  const int lane = threadIdx.x & 63;
  const float* pm = a.part + (int64_t)a.splits * all * a.d;
  // the weights of splits lane and lane + 64
  static_assert(XAT_SPLITS <= 128, "two splits a lane");
  f32x2 x[2];
  float m = neg_inf();
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int s = lane + 64 * u;
    x[u] = f32x2{neg_inf(), 0.f};
    if (s < a.splits) x[u] = *(const f32x2*)(pm + ((int64_t)s * all + R) * 2);
    m = fmaxf(m, x[u][0]);
  }
  for (int i = 1; i < 64; i *= 2) m = fmaxf(m, __shfl_xor(m, i));
  const float base = m == neg_inf() ? 0.f : m;
  float f[2], l = 0.f;
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    f[u] = __builtin_amdgcn_exp2f((x[u][0] - base) * LOG2E);
    l = fmaf(x[u][1], f[u], l);
  }
  for (int i = 1; i < 64; i *= 2) l += __shfl_xor(l, i);
  const int per = a.d <= 32 ? 8 : a.d <= 64 ? 16 : 32, ch = 4 * (lane % per);
  f32x4 o{};
#pragma unroll 4
  for (int s0 = 0; s0 < a.splits; s0 += 64 / per) {
    const int s = s0 + lane / per;
    const float w = __shfl(s < 64 ? f[0] : f[1], s & 63);
    if (s < a.splits && ch < a.d)
      o += *(const f32x4*)(a.part + ((int64_t)s * all + R) * a.d + ch) * w;
  }
  for (int i = per; i < 64; i *= 2)
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] += __shfl_xor(o[e], i);
  const float inv = l > 0.f ? 1.f / l : 0.f;
  if (lane < per && ch < a.d) store4((T*)a.out + R * a.d + ch, o * inv);
  if (lane == 0) *(f32x2*)(a.stat + 2 * R) = f32x2{m, l > 0.f ? __logf(l) : 0.f};
}

template <typename T, int DP, int NW, int MODE>
void fwd_launch(const XatArgs& a, hipStream_t s) {
  constexpr int KW = xat_most_groups<T, DP, NW, MODE>();
  const int tiles = xat_row_tiles(a, MODE == XB_HEADS ? 1 : NW);
  const int64_t wgs = xat_row_wgs(sizeof(T) == 2 ? TRIATTN_BF16 : TRIATTN_F32, a);
  const dim3 grid((unsigned)(wgs * a.splits));
  if (KW > 1 && xat_groups(wgs, xat_key_steps(a)))
    hipLaunchKernelGGL((xat_fwd_kernel<T, DP, NW, MODE, KW>), grid, dim3(64 * NW * KW), 0, s, a,
                       tiles);
  else
    hipLaunchKernelGGL((xat_fwd_kernel<T, DP, NW, MODE, 1>), grid, dim3(64 * NW), 0, s, a, tiles);
}
template <typename T, int DP>
void fwd_width(const XatArgs& a, bool heads, hipStream_t s) {
  constexpr int ONE = sizeof(T) == 2 || DP <= 64 ? 1 : 4;
  const int nw = xat_row_waves(sizeof(T) == 2 ? TRIATTN_BF16 : TRIATTN_F32, a);
  if constexpr (sizeof(T) == 2 || DP <= 64)
    if (heads) return fwd_launch<T, DP, 4, XB_HEADS>(a, s);
  if (a.bias)
    nw == 1 ? fwd_launch<T, DP, ONE, XB_PLANES>(a, s) : fwd_launch<T, DP, 4, XB_PLANES>(a, s);
  else nw == 1 ? fwd_launch<T, DP, ONE, XB_NONE>(a, s) : fwd_launch<T, DP, 4, XB_NONE>(a, s);
}

template <typename T>
hipError_t fwd(const XatArgs& a, hipStream_t s) {
  const int dtype = sizeof(T) == 2 ? TRIATTN_BF16 : TRIATTN_F32;
  const bool heads = xat_by_heads(dtype, a);
  if (a.bias && !heads) {
    const hipError_t e = launch_xat_planes(dtype, a, s);
    if (e != hipSuccess) return e;
  }
  {
    KernelTimer t(K_XAT_FWD, s);
    if (a.d <= 32) fwd_width<T, 32>(a, heads, s);
    else if (a.d <= 64) fwd_width<T, 64>(a, heads, s);
    else fwd_width<T, 128>(a, heads, s);
  }
  if (a.splits > 1) {
    KernelTimer t(K_XAT_JOIN, s);
    const int64_t n = a.batch * a.nq * a.h;
    hipLaunchKernelGGL(xat_join_kernel<T>, dim3((unsigned)((n + 3) / 4)), dim3(256), 0, s, a);
  }
  return hipGetLastError();
}

}  // namespace

bool xat_needs_planes(int dtype, const XatArgs& a) {
  return a.bias_batch > 0 && !xat_by_heads(dtype, a);
}

XatPlan xat_fwd_plan(int dtype, const XatArgs& a) {
  XatPlan p{};
  const int64_t all = a.batch * a.nq * a.h;
  p.nkp = (a.nk + 63) / 64 * 64;
  p.splits = xat_key_splits(dtype, a);
  const size_t e = dtype == TRIATTN_BF16 ? 2 : 4;
  if (xat_needs_planes(dtype, a))
    p.planes = (size_t)a.bias_batch * a.h * a.nq * p.nkp * e;
  if (p.splits > 1) p.part = (size_t)p.splits * all * (a.d + 2) * sizeof(float);
  return p;
}

hipError_t launch_xat_fwd(int dtype, const XatArgs& a, hipStream_t s) {
  return dtype == TRIATTN_BF16 ? fwd<bf16>(a, s) : fwd<float>(a, s);
}

}  // namespace triattn
