// Gated linear projection: [a | b] = x W + bias, out = act(a) b, W [k][2 f].
//
// Both projections are one product (lin_tile.h): a tile of W holds the same columns of both
// halves, 8 and 8 in turn, so that a thread ends with a and b of the same outputs and neither is
// written.  The backward forms them again, with
//   da = dout b act'(a),  db = dout act(a)
// in the product's epilogue, as dz = [da | db] in fp32; dx = dz W^T, dW = x^T dz and the sums of
// dz are the linear projection's products.
#include "lin_tile.h"
#include "timing.h"

namespace triattn {
namespace {

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
  } else {
    sigmoid<sizeof(T) == 4>(z, p, q);
    value = act == TRIATTN_ACT_SILU ? z * p : p;
    slope = act == TRIATTN_ACT_SILU ? p * (1.f + z * q) : p * q;
  }
}
template <typename T>
__device__ inline float gate_value(float z, int act) {
  if (act != TRIATTN_ACT_SIGMOID) return act_value<T>(z, act);
  float p, q;
  sigmoid<sizeof(T) == 4>(z, p, q);
  return p;
}

template <typename T, int R, bool ALIGNED, bool DZ>
__global__ __launch_bounds__(256, sizeof(T) == 2 ? 2 : 1) void glu_kernel(GluArgs a) {
  using G = Product<T, T, R, step_k(R, 2 * planes<T>()), true, false, planes<T>(), planes<T>(), DZ_X,
                    DZ_X, ALIGNED, false, true>;
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
  G::run(lds, Mat<T>{(const T*)a.x, a.m, a.k}, nullptr, Mat<T>{(const T*)a.w, a.k, 2 * a.f}, nullptr,
         0, i0, j0, 0, a.k, false, none, acc);
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
      float* dz = a.dz + i * 2 * a.f + j;
      put8<float, ALIGNED>(dz, have, za);
      put8<float, ALIGNED>(dz + a.f, have, zb);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) za[e] = gate_value<T>(za[e], a.act) * zb[e];
      put8<T, ALIGNED>((T*)a.out + i * a.f + j, have, za);
    }
  });
}

template <typename T, bool DZ>
hipError_t launch(const GluArgs& a, hipStream_t s) {
  KernelTimer t(DZ ? K_GLU_DZ : K_GLU_FWD, s);
  const bool al = a.k % WORD<T> == 0 && a.f % WORD<T> == 0;
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
  return dtype == TRIATTN_BF16 ? launch<bf16, false>(a, s) : launch<float, false>(a, s);
}
hipError_t launch_glu_dz(int dtype, const GluArgs& a, hipStream_t s) {
  return dtype == TRIATTN_BF16 ? launch<bf16, true>(a, s) : launch<float, true>(a, s);
}

}  // namespace triattn
