// C ABI of the operators beside the attention: layer norm, linear projection with
// epilogue, relative position bias.  Argument checks, workspace layout and launch;
// every check runs before the first HIP call.
#include <math.h>
#include <stdint.h>

#include "ops.h"
#include "triattn.h"

namespace {

constexpr int64_t MAX_M = (int64_t)1 << 31;

size_t round256(size_t x) { return (x + 255) & ~(size_t)255; }
bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }
bool aligned4(const void* p) { return ((uintptr_t)p & 3u) == 0; }
bool bad_dtype(int dtype) { return dtype != TRIATTN_F32 && dtype != TRIATTN_BF16; }

// All of `ptrs` present and aligned, and those of `maybe` aligned (null is).
template <size_t N, size_t M>
bool bad_pointers(const void* const (&ptrs)[N], const void* const (&maybe)[M]) {
  for (const void* p : ptrs)
    if (p == nullptr || !aligned16(p)) return true;
  for (const void* p : maybe)
    if (!aligned16(p)) return true;
  return false;
}

int ln_check(int dtype, int64_t m, int64_t c) {
  if (bad_dtype(dtype) || m < 1 || m > MAX_M || c < 1) return TRIATTN_ERR_INVALID_ARG;
  return c > triattn::LN_MAX_C ? TRIATTN_ERR_UNSUPPORTED : TRIATTN_OK;
}

size_t ln_ws(int dtype, int64_t m, int64_t c) {
  return round256((size_t)triattn::ln_bwd_parts(dtype, m, (int)c) * 2 * c * sizeof(float));
}

// `width`: of the widest result, n or (backward) the larger of k and n.
int lin_check(int dtype, int64_t m, int64_t k, int64_t n, int act, int64_t width) {
  if (bad_dtype(dtype) || m < 1 || m > MAX_M || k < 1 || n < 1) return TRIATTN_ERR_INVALID_ARG;
  if (act < TRIATTN_ACT_NONE || act > TRIATTN_ACT_SILU) return TRIATTN_ERR_INVALID_ARG;
  if (k > triattn::LIN_MAX_K || n > triattn::LIN_MAX_K) return TRIATTN_ERR_UNSUPPORTED;
  // a launch holds fewer than 2^32 threads
  const int64_t tiles = (m + 63) / 64 * ((width + 63) / 64);
  return tiles >= (int64_t)1 << 24 ? TRIATTN_ERR_UNSUPPORTED : TRIATTN_OK;
}

// Partial sums, then dz; never 0, so that a workspace is always one.
size_t lin_ws(const triattn::LinBwdPlan& p) { return round256(p.part) + round256(p.dz) + 256; }

int rel_check(int dtype, int64_t batch, int64_t n, int64_t h, int n_edges) {
  if (bad_dtype(dtype) || batch < 1 || batch > ((int64_t)1 << 20) || n < 1 || n > 8192 || h < 1 ||
      n_edges < 1)
    return TRIATTN_ERR_INVALID_ARG;
  if (h > triattn::REL_MAX_H || n_edges > triattn::REL_MAX_EDGES) return TRIATTN_ERR_UNSUPPORTED;
  return batch * n * n * h >= (int64_t)1 << 39 ? TRIATTN_ERR_UNSUPPORTED : TRIATTN_OK;
}

// The workspace does not depend on whether there are chains: the larger need counts.
size_t rel_ws(int64_t batch, int64_t n, int64_t h, int n_edges) {
  const size_t one = triattn::rel_bwd_ws(batch, (int)n, (int)h, n_edges + 1);
  const size_t two = triattn::rel_bwd_ws(batch, (int)n, (int)h, n_edges + 2);
  return round256(one > two ? one : two);
}

int rel_args(int64_t batch, int64_t n, int64_t h, int n_edges, const int32_t* edges,
             const int32_t* pos, const int32_t* chain, triattn::RelArgs* a) {
  if (edges == nullptr || pos == nullptr || !aligned4(pos) || !aligned4(chain))
    return TRIATTN_ERR_INVALID_ARG;
  a->batch = batch;
  a->n = (int)n;
  a->h = (int)h;
  a->ne = n_edges;
  a->rows = n_edges + 1 + (chain != nullptr ? 1 : 0);
  a->pos = pos;
  a->chain = chain;
  for (int i = 0; i < n_edges; ++i) {
    if (i > 0 && edges[i] <= edges[i - 1]) return TRIATTN_ERR_INVALID_ARG;
    a->edges[i] = edges[i];
  }
  return TRIATTN_OK;
}

int launched(hipError_t e) { return e == hipSuccess ? TRIATTN_OK : TRIATTN_ERR_HIP; }

}  // namespace

extern "C" {

// ---- layer norm -----------------------------------------------------------------------

int tri_layer_norm_fwd(int dtype, int64_t m, int64_t c, float eps, const void* x,
                       const void* gamma, const void* beta, void* out, float* mean, float* rstd,
                       void* stream) {
  const int st = ln_check(dtype, m, c);
  if (st != TRIATTN_OK) return st;
  if (!(isfinite(eps) && eps >= 0.f)) return TRIATTN_ERR_INVALID_ARG;
  if (bad_pointers({x, out, mean, rstd}, {gamma, beta})) return TRIATTN_ERR_INVALID_ARG;
  triattn::LnArgs a{};
  a.m = m;
  a.c = (int)c;
  a.eps = eps;
  a.x = x;
  a.gamma = gamma;
  a.beta = beta;
  a.out = out;
  a.mean = mean;
  a.rstd = rstd;
  return launched(triattn::launch_ln_fwd(dtype, a, (hipStream_t)stream));
}

int tri_layer_norm_bwd_workspace_bytes(int dtype, int64_t m, int64_t c, size_t* bytes) {
  const int st = ln_check(dtype, m, c);
  if (st != TRIATTN_OK) return st;
  if (bytes == nullptr) return TRIATTN_ERR_INVALID_ARG;
  *bytes = ln_ws(dtype, m, c);
  return TRIATTN_OK;
}

int tri_layer_norm_bwd(int dtype, int64_t m, int64_t c, const void* x, const void* gamma,
                       const float* mean, const float* rstd, const void* dout, void* dx,
                       float* dgamma, float* dbeta, void* workspace, size_t workspace_bytes,
                       void* stream) {
  const int st = ln_check(dtype, m, c);
  if (st != TRIATTN_OK) return st;
  if (bad_pointers({x, mean, rstd, dout, dx}, {gamma, dgamma, dbeta}))
    return TRIATTN_ERR_INVALID_ARG;
  if ((dgamma != nullptr || dbeta != nullptr) &&
      (workspace == nullptr || !aligned16(workspace) || workspace_bytes < ln_ws(dtype, m, c)))
    return TRIATTN_ERR_WORKSPACE;
  triattn::LnBwdArgs a{};
  a.m = m;
  a.c = (int)c;
  a.x = x;
  a.gamma = gamma;
  a.dout = dout;
  a.mean = mean;
  a.rstd = rstd;
  a.dx = dx;
  a.dgamma = dgamma;
  a.dbeta = dbeta;
  a.part = (float*)workspace;
  a.nwg = triattn::ln_bwd_parts(dtype, m, (int)c);
  return launched(triattn::launch_ln_bwd(dtype, a, (hipStream_t)stream));
}

// ---- linear projection with epilogue -----------------------------------------------------

int tri_linear_fwd(int dtype, int64_t m, int64_t k, int64_t n, int act, const void* x,
                   const void* w, const void* bias, const void* residual, void* out, void* z,
                   void* stream) {
  const int st = lin_check(dtype, m, k, n, act, n);
  if (st != TRIATTN_OK) return st;
  if (bad_pointers({x, w, out}, {bias, residual, z})) return TRIATTN_ERR_INVALID_ARG;
  triattn::LinArgs a{};
  a.m = m;
  a.k = (int)k;
  a.n = (int)n;
  a.act = act;
  a.x = x;
  a.w = w;
  a.bias = bias;
  a.residual = residual;
  a.out = out;
  a.z = z;
  return launched(triattn::launch_lin_fwd(dtype, a, (hipStream_t)stream));
}

int tri_linear_bwd_workspace_bytes(int dtype, int64_t m, int64_t k, int64_t n, int act,
                                   size_t* bytes) {
  const int st = lin_check(dtype, m, k, n, act, k > n ? k : n);
  if (st != TRIATTN_OK) return st;
  if (bytes == nullptr) return TRIATTN_ERR_INVALID_ARG;
  *bytes = lin_ws(triattn::lin_bwd_plan(dtype, m, (int)k, (int)n, act));
  return TRIATTN_OK;
}

int tri_linear_bwd(int dtype, int64_t m, int64_t k, int64_t n, int act, const void* x,
                   const void* w, const void* z, const void* dout, void* dx, float* dw,
                   float* dbias, void* workspace, size_t workspace_bytes, void* stream) {
  const int st = lin_check(dtype, m, k, n, act, k > n ? k : n);
  if (st != TRIATTN_OK) return st;
  if (bad_pointers({x, w, dout}, {z, dx, dw, dbias})) return TRIATTN_ERR_INVALID_ARG;
  if (act != TRIATTN_ACT_NONE && z == nullptr) return TRIATTN_ERR_INVALID_ARG;
  if (dx == nullptr && dw == nullptr && dbias == nullptr) return TRIATTN_ERR_INVALID_ARG;
  const triattn::LinBwdPlan plan = triattn::lin_bwd_plan(dtype, m, (int)k, (int)n, act);
  if (workspace == nullptr || !aligned16(workspace) || workspace_bytes < lin_ws(plan))
    return TRIATTN_ERR_WORKSPACE;
  triattn::LinBwdArgs a{};
  a.m = m;
  a.k = (int)k;
  a.n = (int)n;
  a.act = act;
  a.x = x;
  a.w = w;
  a.z = z;
  a.dout = dout;
  a.dx = dx;
  a.dw = dw;
  a.dbias = dbias;
  a.part = (float*)workspace;
  a.splits = plan.splits;
  if (plan.dz > 0) a.dz = (float*)((char*)workspace + round256(plan.part));
  return launched(triattn::launch_lin_bwd(dtype, a, (hipStream_t)stream));
}

// ---- relative position bias ----------------------------------------------------------------

int tri_rel_bias_fwd(int dtype, int64_t batch, int64_t n, int64_t h, int n_edges,
                     const int32_t* edges, const int32_t* pos, const int32_t* chain,
                     const void* table, const void* base, void* out, void* stream) {
  int st = rel_check(dtype, batch, n, h, n_edges);
  if (st != TRIATTN_OK) return st;
  triattn::RelArgs a{};
  st = rel_args(batch, n, h, n_edges, edges, pos, chain, &a);
  if (st != TRIATTN_OK) return st;
  if (bad_pointers({table, out}, {base})) return TRIATTN_ERR_INVALID_ARG;
  a.table = table;
  a.base = base;
  a.out = out;
  return launched(triattn::launch_rel_fwd(dtype, a, (hipStream_t)stream));
}

int tri_rel_bias_bwd_workspace_bytes(int dtype, int64_t batch, int64_t n, int64_t h, int n_edges,
                                     size_t* bytes) {
  const int st = rel_check(dtype, batch, n, h, n_edges);
  if (st != TRIATTN_OK) return st;
  if (bytes == nullptr) return TRIATTN_ERR_INVALID_ARG;
  *bytes = rel_ws(batch, n, h, n_edges);
  return TRIATTN_OK;
}

int tri_rel_bias_bwd(int dtype, int64_t batch, int64_t n, int64_t h, int n_edges,
                     const int32_t* edges, const int32_t* pos, const int32_t* chain,
                     const void* dout, float* dtable, void* workspace, size_t workspace_bytes,
                     void* stream) {
  int st = rel_check(dtype, batch, n, h, n_edges);
  if (st != TRIATTN_OK) return st;
  triattn::RelArgs a{};
  st = rel_args(batch, n, h, n_edges, edges, pos, chain, &a);
  if (st != TRIATTN_OK) return st;
  if (bad_pointers({(const void*)dout, (const void*)dtable}, {(const void*)nullptr}))
    return TRIATTN_ERR_INVALID_ARG;
  if (workspace == nullptr || !aligned16(workspace) ||
      workspace_bytes < rel_ws(batch, n, h, n_edges))
    return TRIATTN_ERR_WORKSPACE;
  a.dout = dout;
  a.dtable = dtable;
  a.part = (float*)workspace;
  return launched(triattn::launch_rel_bwd(dtype, a, (hipStream_t)stream));
}

}  // extern "C"
