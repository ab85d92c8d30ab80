// Internal launch interface between the C ABI (api_ops.hip) and the kernels of the operators
// beside the attention.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "common.h"

namespace triattn {

// ---- layer norm (ln.hip) ----------------------------------------------------------------
constexpr int LN_MAX_C = 8192;

struct LnArgs {
  int64_t m;
  int c;
  float eps;
  const void *x, *gamma, *beta;  // x [m][c]; gamma and beta [c] or null
  void* out;                     // [m][c]
  float *mean, *rstd;            // [m]
};

struct LnBwdArgs {
  int64_t m;
  int c;
  const void *x, *gamma, *dout;
  const float *mean, *rstd;
  void* dx;                // [m][c]
  float *dgamma, *dbeta;   // [c] or null
  float* part;             // workspace: [nwg][2][c] partial sums (dgamma's, dbeta's)
  int nwg;
};

int ln_bwd_parts(int dtype, int64_t m, int c);  // nwg
hipError_t launch_ln_fwd(int dtype, const LnArgs& a, hipStream_t s);
hipError_t launch_ln_bwd(int dtype, const LnBwdArgs& a, hipStream_t s);

// ---- linear projection with epilogue (lin.hip) --------------------------------------------
constexpr int LIN_MAX_K = 8192;

struct LinArgs {
  int64_t m;
  int k, n;
  int act;                                // triattn_act
  const void *x, *w, *bias, *residual;    // x [m][k], w [k][n]; bias, residual or null
  void *out, *z;                          // [m][n]; z or null
};

struct LinBwdArgs {
  int64_t m;
  int k, n;
  int act;
  const void *x, *w, *z, *dout;
  void* dx;                // [m][k] or null
  float *dw, *dbias;       // [k][n], [n], or null
  float* part;             // workspace: [splits] partial sums (dw, dbias); none for 1 split
  int splits;
  float* dz;               // workspace: dz [m][n], or null
};

struct LinBwdPlan {
  int splits;
  size_t part, dz;  // bytes of workspace, 0 for none
};
LinBwdPlan lin_bwd_plan(int dtype, int64_t m, int k, int n, int act);
hipError_t launch_lin_fwd(int dtype, const LinArgs& a, hipStream_t s);
hipError_t launch_lin_bwd(int dtype, const LinBwdArgs& a, hipStream_t s);

// ---- relative position bias (rel.hip) -------------------------------------------------------
constexpr int REL_MAX_EDGES = 255;
constexpr int REL_MAX_H = 256;

// Differences the edges may span to be looked up by difference (a byte of LDS each).
constexpr int REL_SPAN = 8192;
constexpr int REL_LUT = 2048;  // those whose table the arguments hold

struct RelArgs {
  int64_t batch;
  int n, h;
  int ne, rows;               // edges; table rows
  const int32_t *pos, *chain; // [batch][n]; chain or null
  const void *table, *base;   // [rows][h]; [batch][n][n][h] or null
  void* out;                  // [batch][n][n][h]
  const void* dout;           // backward
  float* dtable;              // backward: [rows][h]
  float* part;                // backward, workspace: slabs of [rows][h] partial sums
  uint32_t inv_h;             // 2^32 / h rounded up (0 for h = 1)
  int32_t low, span;          // looked up: differences low .. low + span
  union {
    int32_t edges[REL_MAX_EDGES + 1];
    uint8_t lut[REL_LUT];     // bucket of difference low + i
  };
};

size_t rel_bwd_ws(int64_t batch, int n, int h, int rows);  // bytes of workspace
hipError_t launch_rel_fwd(int dtype, const RelArgs& a, hipStream_t s);
hipError_t launch_rel_bwd(int dtype, const RelArgs& a, hipStream_t s);

}  // namespace triattn
