// C ABI of the cross attention, the gated linear projection and the clipping of gradients.
// Argument checks, workspace layout and launch; every check runs before the first HIP call.
#include <math.h>
#include <stdint.h>

#include <algorithm>
#include <memory>
#include <new>

#include "ops.h"
#include "triattn.h"

namespace {

constexpr int64_t MAX_M = (int64_t)1 << 31, MAX_WGS = (int64_t)1 << 24;

size_t round256(size_t x) { return (x + 255) & ~(size_t)255; }
bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }
bool bad_dtype(int dtype) { return dtype != TRIATTN_F32 && dtype != TRIATTN_BF16; }
int launched(hipError_t e) { return e == hipSuccess ? TRIATTN_OK : TRIATTN_ERR_HIP; }

// All of `ptrs` present and aligned, and those of `maybe` aligned (null is).
template <size_t N, size_t M>
bool bad_pointers(const void* const (&ptrs)[N], const void* const (&maybe)[M]) {
  for (const void* p : ptrs)
    if (p == nullptr || !aligned16(p)) return true;
  for (const void* p : maybe)
    if (!aligned16(p)) return true;
  return false;
}

// ---- cross attention --------------------------------------------------------------------

int xat_sizes(int dtype, int64_t batch, int64_t nq, int64_t nk, int64_t h, int64_t hk, int64_t d,
              int64_t bias_batch, triattn::XatArgs* a) {
  if (bad_dtype(dtype) || batch < 1 || batch > ((int64_t)1 << 20) || nq < 1 || nk < 1 ||
      nq > ((int64_t)1 << 22) || nk > ((int64_t)1 << 22) || h < 1 || hk < 1 || h < hk ||
      h % hk != 0 || d < 1)
    return TRIATTN_ERR_INVALID_ARG;
  if (bias_batch != 0 && bias_batch != 1 && bias_batch != batch) return TRIATTN_ERR_INVALID_ARG;
  if (h > 256 || d > 128 || d % 8 != 0) return TRIATTN_ERR_UNSUPPORTED;
  const int64_t g = h / hk;
  if ((nq * g + 256) * g >= (int64_t)1 << 32) return TRIATTN_ERR_UNSUPPORTED;
  const int64_t most = (int64_t)1 << 34;
  if (batch * nq > most / (h * d) || batch * nk > most / (hk * d)) return TRIATTN_ERR_UNSUPPORTED;
  // at most one workgroup for 32 rows or keys, times the splits of few
  if (batch * hk * ((nq * g + 31) / 32) >= MAX_WGS || batch * hk * ((nk + 31) / 32) >= MAX_WGS)
    return TRIATTN_ERR_UNSUPPORTED;
  if (bias_batch > 0 && nq * (nk + 64) >= most / h) return TRIATTN_ERR_UNSUPPORTED;
  a->batch = batch;
  a->nq = (int)nq;
  a->nk = (int)nk;
  a->h = (int)h;
  a->hk = (int)hk;
  a->d = (int)d;
  a->group = (int)g;
  a->inv_group = g == 1 ? 0 : (uint32_t)((((uint64_t)1 << 32) + g - 1) / g);
  a->bias_batch = bias_batch;
  // of a bias that is turned into planes, at most one for 16 keys of a row of its maps
  if (triattn::xat_needs_planes(dtype, *a) && bias_batch * nq * ((nk + 63) / 64 * 4) >= MAX_WGS)
    return TRIATTN_ERR_UNSUPPORTED;
  return TRIATTN_OK;
}

size_t xat_ws(const triattn::XatPlan& p) {
  return round256(p.planes) + round256(p.part) + round256(p.part_q) + round256(p.dsum) +
         round256(p.single) + round256(p.valid) + round256(p.dplanes) + 256;
}
void xat_place(const triattn::XatPlan& p, void* workspace, triattn::XatArgs* a) {
  char* w = (char*)workspace;
  a->nkp = p.nkp;
  a->splits = p.splits;
  a->splits_q = p.splits_q;
  a->planes = w;
  w += round256(p.planes);
  a->part = (float*)w;
  w += round256(p.part);
  a->part_q = (float*)w;
  w += round256(p.part_q);
  a->dsum = (float*)w;
  w += round256(p.dsum);
  a->single = (int*)w;
  w += round256(p.single);
  a->valid = (int*)w;
  w += round256(p.valid);
  a->dplanes = (float*)w;
}

// ---- gated linear projection ---------------------------------------------------------------

int glu_check(int dtype, int64_t m, int64_t k, int64_t f, int64_t width) {
  if (bad_dtype(dtype) || m < 1 || m > MAX_M || k < 1 || f < 1) return TRIATTN_ERR_INVALID_ARG;
  if (k > triattn::LIN_MAX_K || f > triattn::GLU_MAX_F) return TRIATTN_ERR_UNSUPPORTED;
  return (m + 63) / 64 * ((width + 63) / 64) >= MAX_WGS ? TRIATTN_ERR_UNSUPPORTED : TRIATTN_OK;
}
bool bad_act(int act) { return act < TRIATTN_ACT_NONE || act > TRIATTN_ACT_SIGMOID; }
int64_t wider(int64_t k, int64_t f) { return k > 2 * f ? k : 2 * f; }
size_t glu_ws(const triattn::LinBwdPlan& p) { return round256(p.part) + round256(p.dz) + 256; }

// ---- norm and clipping of gradients -----------------------------------------------------------

struct GradPlan {
  int64_t span, wgs;
};
int64_t grad_wgs(int64_t size, int64_t span) { return (size + span - 1) / span; }
// A workgroup's elements: 32768 (16 words of 16 bytes a thread in bf16, 32 in fp32, four at a
// time), fewer where that leaves CUs idle, down to 2048 (130,000 elements of 14 tensors: one or two
// words a thread).
int grad_plan(int64_t count, const int64_t* sizes, GradPlan* p) {
  if (count < 1 || count > ((int64_t)1 << 20) || sizes == nullptr) return TRIATTN_ERR_INVALID_ARG;
  int64_t total = 0;
  for (int64_t i = 0; i < count; ++i) {
    if (sizes[i] < 0) return TRIATTN_ERR_INVALID_ARG;
    const int64_t room = ((int64_t)1 << 39) - 1 - total;
    if (sizes[i] > room) return TRIATTN_ERR_UNSUPPORTED;
    total += sizes[i];
  }
  p->span = 2048;
  while (p->span < 32768 && total / p->span > 2048) p->span *= 2;
  p->wgs = 0;
  for (int64_t i = 0; i < count; ++i) p->wgs += grad_wgs(sizes[i], p->span);
  return p->wgs >= MAX_WGS ? TRIATTN_ERR_UNSUPPORTED : TRIATTN_OK;
}
int grad_list(int64_t count, const int32_t* dtypes, const int64_t* sizes,
              const void* const* list) {
  if (dtypes == nullptr || list == nullptr) return TRIATTN_ERR_INVALID_ARG;
  for (int64_t i = 0; i < count; ++i)
    if (bad_dtype(dtypes[i]) || (sizes[i] > 0 && (list[i] == nullptr || !aligned16(list[i]))))
      return TRIATTN_ERR_INVALID_ARG;
  return TRIATTN_OK;
}
// TRIATTN_OK if the results are apart from each other and from every gradient that is not
// clipped in its place: workgroups would write what others have still to read.
int grad_apart(int64_t count, const int32_t* dtypes, const int64_t* sizes,
               const void* const* grads, void* const* outs) {
  struct Span {
    uintptr_t at, end;
  };
  Span few[64];
  std::unique_ptr<Span[]> many;
  if (count > 64) many.reset(new (std::nothrow) Span[count]);
  Span* s = count > 64 ? many.get() : few;
  if (s == nullptr) return TRIATTN_ERR_UNSUPPORTED;
  auto bytes = [&](int64_t i) { return (uintptr_t)sizes[i] * (dtypes[i] == TRIATTN_BF16 ? 2 : 4); };
  int64_t n = 0;
  for (int64_t i = 0; i < count; ++i)
    if (sizes[i] > 0) s[n++] = Span{(uintptr_t)outs[i], (uintptr_t)outs[i] + bytes(i)};
  std::sort(s, s + n, [](const Span& a, const Span& b) { return a.at < b.at; });
  for (int64_t i = 1; i < n; ++i)
    if (s[i - 1].end > s[i].at) return TRIATTN_ERR_INVALID_ARG;
  for (int64_t i = 0; i < count; ++i) {
    if (sizes[i] == 0 || grads[i] == outs[i]) continue;
    const uintptr_t at = (uintptr_t)grads[i];
    // the first result that ends behind the gradient's start
    const Span* x =
        std::upper_bound(s, s + n, at, [](uintptr_t v, const Span& a) { return v < a.end; });
    if (x != s + n && x->at < at + bytes(i)) return TRIATTN_ERR_INVALID_ARG;
  }
  return TRIATTN_OK;
}
size_t grad_ws(int64_t wgs) { return round256((size_t)wgs * sizeof(double)) + 256; }

// Calls `launch` with as many tensors at a time as a launch takes.
template <typename F>
int grad_each(int64_t count, const int32_t* dtypes, const int64_t* sizes,
              const void* const* grads, void* const* outs, triattn::GradArgs& a, F launch) {
  a.wg0 = 0;
  int64_t i = 0;
  while (i < count) {
    a.count = 0;
    a.first[0] = 0;
    for (; i < count && a.count < triattn::GRAD_MAX; ++i) {
      if (sizes[i] == 0) continue;
      const int n = a.count++;
      a.src[n] = grads[i];
      a.dst[n] = outs ? outs[i] : nullptr;
      a.size[n] = sizes[i];
      a.dtype[n] = (uint8_t)dtypes[i];
      a.first[n + 1] = a.first[n] + (int)grad_wgs(sizes[i], a.span);
    }
    if (a.count == 0) break;
    if (launch(a) != hipSuccess) return TRIATTN_ERR_HIP;
    a.wg0 += a.first[a.count];
  }
  return TRIATTN_OK;
}

}  // namespace

extern "C" {

int tri_cross_attn_fwd_workspace_bytes(int dtype, int64_t batch, int64_t nq, int64_t nk,
                                       int64_t heads, int64_t key_heads, int64_t d,
                                       int64_t bias_batch, size_t* bytes) {
  triattn::XatArgs a{};
  const int st = xat_sizes(dtype, batch, nq, nk, heads, key_heads, d, bias_batch, &a);
  if (st != TRIATTN_OK) return st;
  if (bytes == nullptr) return TRIATTN_ERR_INVALID_ARG;
  *bytes = xat_ws(triattn::xat_fwd_plan(dtype, a));
  return TRIATTN_OK;
}

int tri_cross_attn_fwd(int dtype, int64_t batch, int64_t nq, int64_t nk, int64_t heads,
                       int64_t key_heads, int64_t d, int64_t bias_batch, float scale,
                       const void* q, const void* k, const void* v, const void* bias,
                       const uint8_t* mask, void* out, float* stat, void* workspace,
                       size_t workspace_bytes, void* stream) {
  triattn::XatArgs a{};
  const int st = xat_sizes(dtype, batch, nq, nk, heads, key_heads, d, bias_batch, &a);
  if (st != TRIATTN_OK) return st;
  if (!(isfinite(scale) && scale > 0.f)) return TRIATTN_ERR_INVALID_ARG;
  if (bad_pointers({q, k, v, out, stat}, {bias})) return TRIATTN_ERR_INVALID_ARG;
  if ((bias == nullptr) != (bias_batch == 0)) return TRIATTN_ERR_INVALID_ARG;
  const triattn::XatPlan plan = triattn::xat_fwd_plan(dtype, a);
  if (workspace == nullptr || !aligned16(workspace) || workspace_bytes < xat_ws(plan))
    return TRIATTN_ERR_WORKSPACE;
  xat_place(plan, workspace, &a);
  a.scale = scale;
  a.q = q;
  a.k = k;
  a.v = v;
  a.bias = bias;
  a.mask = mask;
  a.out = out;
  a.stat = stat;
  return launched(triattn::launch_xat_fwd(dtype, a, (hipStream_t)stream));
}

int tri_cross_attn_bwd_workspace_bytes(int dtype, int64_t batch, int64_t nq, int64_t nk,
                                       int64_t heads, int64_t key_heads, int64_t d,
                                       int64_t bias_batch, size_t* bytes) {
  triattn::XatArgs a{};
  const int st = xat_sizes(dtype, batch, nq, nk, heads, key_heads, d, bias_batch, &a);
  if (st != TRIATTN_OK) return st;
  if (bytes == nullptr) return TRIATTN_ERR_INVALID_ARG;
  *bytes = xat_ws(triattn::xat_bwd_plan(dtype, a));
  return TRIATTN_OK;
}

int tri_cross_attn_bwd(int dtype, int64_t batch, int64_t nq, int64_t nk, int64_t heads,
                       int64_t key_heads, int64_t d, int64_t bias_batch, float scale,
                       const void* q, const void* k, const void* v, const void* bias,
                       const uint8_t* mask, const void* out, const float* stat,
                       const void* dout, void* dq, void* dk, void* dv, void* dbias,
                       void* workspace, size_t workspace_bytes, void* stream) {
  triattn::XatArgs a{};
  const int st = xat_sizes(dtype, batch, nq, nk, heads, key_heads, d, bias_batch, &a);
  if (st != TRIATTN_OK) return st;
  if (!(isfinite(scale) && scale > 0.f)) return TRIATTN_ERR_INVALID_ARG;
  if (bad_pointers({q, k, v, out, stat, dout, dq, dk, dv}, {bias, dbias}))
    return TRIATTN_ERR_INVALID_ARG;
  if ((bias == nullptr) != (bias_batch == 0) || (bias == nullptr && dbias != nullptr))
    return TRIATTN_ERR_INVALID_ARG;
  const triattn::XatPlan plan = triattn::xat_bwd_plan(dtype, a);
  if (workspace == nullptr || !aligned16(workspace) || workspace_bytes < xat_ws(plan))
    return TRIATTN_ERR_WORKSPACE;
  xat_place(plan, workspace, &a);
  a.scale = scale;
  a.q = q;
  a.k = k;
  a.v = v;
  a.bias = bias;
  a.mask = mask;
  a.out = const_cast<void*>(out);
  a.stat = const_cast<float*>(stat);
  a.dout = dout;
  a.dq = dq;
  a.dk = dk;
  a.dv = dv;
  a.dbias = dbias;
  return launched(triattn::launch_xat_bwd(dtype, a, (hipStream_t)stream));
}

int tri_gated_linear_fwd(int dtype, int64_t m, int64_t k, int64_t f, int act, const void* x,
                         const void* w, const void* bias, void* out, void* stream) {
  const int st = glu_check(dtype, m, k, f, 2 * f);
  if (st != TRIATTN_OK) return st;
  if (bad_act(act) || bad_pointers({x, w, out}, {bias})) return TRIATTN_ERR_INVALID_ARG;
  triattn::GluArgs a{};
  a.m = m;
  a.k = (int)k;
  a.f = (int)f;
  a.act = act;
  a.x = x;
  a.w = w;
  a.bias = bias;
  a.out = out;
  return launched(triattn::launch_glu_fwd(dtype, a, (hipStream_t)stream));
}

int tri_gated_linear_bwd_workspace_bytes(int dtype, int64_t m, int64_t k, int64_t f,
                                         size_t* bytes) {
  const int st = glu_check(dtype, m, k, f, wider(k, f));
  if (st != TRIATTN_OK) return st;
  if (bytes == nullptr) return TRIATTN_ERR_INVALID_ARG;
  *bytes = glu_ws(triattn::glu_bwd_plan(dtype, m, (int)k, (int)f));
  return TRIATTN_OK;
}

int tri_gated_linear_bwd(int dtype, int64_t m, int64_t k, int64_t f, int act, const void* x,
                         const void* w, const void* bias, const void* dout, void* dx, float* dw,
                         float* dbias, void* workspace, size_t workspace_bytes, void* stream) {
  const int st = glu_check(dtype, m, k, f, wider(k, f));
  if (st != TRIATTN_OK) return st;
  if (bad_act(act) || bad_pointers({x, w, dout}, {bias, dx, dw, dbias}))
    return TRIATTN_ERR_INVALID_ARG;
  if (dx == nullptr && dw == nullptr && dbias == nullptr) return TRIATTN_ERR_INVALID_ARG;
  const triattn::LinBwdPlan plan = triattn::glu_bwd_plan(dtype, m, (int)k, (int)f);
  if (workspace == nullptr || !aligned16(workspace) || workspace_bytes < glu_ws(plan))
    return TRIATTN_ERR_WORKSPACE;
  float* dz = (float*)((char*)workspace + round256(plan.part));
  triattn::GluArgs a{};
  a.m = m;
  a.k = (int)k;
  a.f = (int)f;
  a.act = act;
  a.x = x;
  a.w = w;
  a.bias = bias;
  a.dout = dout;
  a.dz = dz;
  triattn::LinBwdArgs b{};
  b.m = m;
  b.k = (int)k;
  b.n = (int)(2 * f);
  b.x = x;
  b.w = w;
  b.dx = dx;
  b.dw = dw;
  b.dbias = dbias;
  b.part = (float*)workspace;
  b.splits = plan.splits;
  b.dz = dz;
  return launched(triattn::launch_glu_bwd(dtype, a, b, (hipStream_t)stream));
}

int tri_grad_norm_workspace_bytes(int64_t count, const int64_t* sizes, size_t* bytes) {
  GradPlan plan;
  const int st = grad_plan(count, sizes, &plan);
  if (st != TRIATTN_OK) return st;
  if (bytes == nullptr) return TRIATTN_ERR_INVALID_ARG;
  *bytes = grad_ws(plan.wgs);
  return TRIATTN_OK;
}

int tri_grad_norm(int64_t count, const int32_t* dtypes, const int64_t* sizes,
                  const void* const* grads, float* norm, void* workspace, size_t workspace_bytes,
                  void* stream) {
  GradPlan plan;
  int st = grad_plan(count, sizes, &plan);
  if (st == TRIATTN_OK) st = grad_list(count, dtypes, sizes, grads);
  if (st != TRIATTN_OK) return st;
  if (norm == nullptr || ((uintptr_t)norm & 3u) != 0) return TRIATTN_ERR_INVALID_ARG;
  if (workspace == nullptr || !aligned16(workspace) || workspace_bytes < grad_ws(plan.wgs))
    return TRIATTN_ERR_WORKSPACE;
  triattn::GradArgs a{};
  a.part = (double*)workspace;
  a.span = plan.span;
  const hipStream_t s = (hipStream_t)stream;
  st = grad_each(count, dtypes, sizes, grads, nullptr, a,
                 [&](const triattn::GradArgs& x) { return triattn::launch_grad_squares(x, s); });
  if (st != TRIATTN_OK) return st;
  return launched(triattn::launch_grad_root(a.part, plan.wgs, norm, s));
}

int tri_grad_clip(int64_t count, const int32_t* dtypes, const int64_t* sizes,
                  const void* const* grads, const float* norm, float max_norm,
                  void* const* outs, void* stream) {
  GradPlan plan;
  int st = grad_plan(count, sizes, &plan);
  if (st == TRIATTN_OK) st = grad_list(count, dtypes, sizes, grads);
  if (st == TRIATTN_OK) st = grad_list(count, dtypes, sizes, outs);
  if (st != TRIATTN_OK) return st;
  if (norm == nullptr || ((uintptr_t)norm & 3u) != 0) return TRIATTN_ERR_INVALID_ARG;
  if (!(isfinite(max_norm) && max_norm > 0.f)) return TRIATTN_ERR_INVALID_ARG;
  st = grad_apart(count, dtypes, sizes, grads, outs);
  if (st != TRIATTN_OK) return st;
  triattn::GradArgs a{};
  a.norm = norm;
  a.span = plan.span;
  a.limit = max_norm;
  const hipStream_t s = (hipStream_t)stream;
  return grad_each(count, dtypes, sizes, grads, outs, a,
                   [&](const triattn::GradArgs& x) { return triattn::launch_grad_scale(x, s); });
}

}  // extern "C"
