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

// The products of a backward whose dz [m][n] is made already (a.dz; act, z and dout unused), in
// fp32 or, for rows of whole 16-byte words, as three planes of bf16 one after the other.
LinBwdPlan lin_made_plan(int dtype, int64_t m, int k, int n, bool planes);
hipError_t launch_lin_made(int dtype, const LinBwdArgs& a, bool planes, hipStream_t s);
// Slabs of partial sums (dw, then dbias) and their sum.
size_t lin_slab_bytes(int k, int n, int splits);
hipError_t launch_lin_reduce(const LinBwdArgs& a, hipStream_t s);

// ---- gated linear projection (glu.hip) -------------------------------------------------------
constexpr int GLU_MAX_F = 4096;  // 2 f columns of W: the linear projection's 8192, whose products
                                 // the backward runs

struct GluArgs {
  int64_t m;
  int k, f;
  int act;                      // triattn_act
  const void *x, *w, *bias;     // x [m][k], w [k][2 f], bias [2 f] or null
  void* out;                    // [m][f]
  const void* dout;             // backward
  float* dz;                    // backward, workspace: [m][2 f]
};
hipError_t launch_glu_fwd(int dtype, const GluArgs& a, hipStream_t s);
// The backward: b holds its results (n = 2 f), slabs and dz, as the plan sizes them.
LinBwdPlan glu_bwd_plan(int dtype, int64_t m, int k, int f);
hipError_t launch_glu_bwd(int dtype, const GluArgs& a, const LinBwdArgs& b, hipStream_t s);

// ---- norm and clipping of gradients (grad.hip) ------------------------------------------------
// Tensors of a launch: their addresses and sizes travel in its arguments.
constexpr int GRAD_MAX = 96;

struct GradArgs {
  int count;
  const void* src[GRAD_MAX];
  void* dst[GRAD_MAX];
  int64_t size[GRAD_MAX];
  int first[GRAD_MAX + 1];      // first workgroup of each
  uint8_t dtype[GRAD_MAX];
  double* part;                 // workspace: a sum of squares a workgroup
  int wg0;                      // workgroups of earlier launches
  const float* norm;
  float limit;
  int64_t span;                 // elements of a workgroup
};
hipError_t launch_grad_squares(const GradArgs& a, hipStream_t s);
hipError_t launch_grad_root(const double* part, int64_t count, float* norm, hipStream_t s);
hipError_t launch_grad_scale(const GradArgs& a, hipStream_t s);

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

// ---- cross attention (xat_fwd.hip, xat_bwd.hip) ----------------------------------------------
struct XatArgs {
  int64_t batch;
  int nq, nk, h, hk, d;
  int group;                  // heads that share a key head: h / hk
  uint32_t inv_group;         // 2^32 / group rounded up
  float scale;
  const void *q, *k, *v;      // [batch][nq][h][d], [batch][nk][hk][d]
  const void* bias;           // [nq][nk][h] or [batch][nq][nk][h], or null
  int64_t bias_batch;         // 1 or batch
  const uint8_t* mask;        // [batch][nk] or null
  void* out;                  // [batch][nq][h][d]
  float* stat;                // [batch][nq][h][2]
  const void* dout;           // backward
  void *dq, *dk, *dv, *dbias;
  // workspace
  void* planes;               // bias, [bias_batch][hk][nq * group][nkp] (dtype)
  int nkp;                    // nk rounded up to whole tiles
  int splits, splits_q;       // of the keys (forward, dq), of the rows (dk, dv)
  float* part;                // partial results of the splits of the keys
  float* part_q;              // and of the rows
  float* dsum;                // [batch][nq][h]
  int* single;                // [batch]: whether it has one valid key at most
  int* valid;                 // [batch][splits]: a split's valid keys
  float* dplanes;             // dbias of every sample, [batch][hk][nq * group][nkp] or as dbias
};

struct XatPlan {
  int nkp, splits, splits_q;
  size_t planes, part, part_q, dsum, single, valid, dplanes;  // bytes of workspace, 0 for none
};
bool xat_needs_planes(int dtype, const XatArgs& a);  // of its bias
XatPlan xat_fwd_plan(int dtype, const XatArgs& a);
XatPlan xat_bwd_plan(int dtype, const XatArgs& a);
hipError_t launch_xat_fwd(int dtype, const XatArgs& a, hipStream_t s);
hipError_t launch_xat_bwd(int dtype, const XatArgs& a, hipStream_t s);
// Bias to planes, one row of a plane after the other (xat_bias.hip).
hipError_t launch_xat_planes(int dtype, const XatArgs& a, hipStream_t s);
// The other way; heads: from [batch][nq][nk][h] as it is, summed over the samples.
hipError_t launch_xat_dbias(int dtype, const XatArgs& a, bool heads, hipStream_t s);

}  // namespace triattn
