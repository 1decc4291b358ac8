// C ABI of the mixture-of-experts calls (include/bnn.h): host-side checks and
// dispatch, in the manner of api.cpp.
#include "bnn.h"

#include <math.h>

#include "dtypes.hpp"
#include "experts.hpp"
#include "kernels.hpp"
#include "status.hpp"

namespace {

using bnn::fail;
using bnn::hip_status;
using bnn::ok;

constexpr int64_t kMaxRows = int64_t{1} << 24;
// Rows times 64-output tiles: a grid's work-items stay below 2^32.
constexpr int64_t kMaxTiles = int64_t{1} << 28;

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

bool real_type(int32_t t) { return t == BNN_F32 || t == BNN_F16 || t == BNN_BF16; }

bnn_status route_check(const bnn_route_desc* d, int64_t T, int64_t stride) {
  if (!d) return fail(BNN_ERR_NULL, "route: descriptor is NULL");
  if (d->E < 1 || d->E > BNN_MAX_EXPERTS)
    return fail(BNN_ERR_SHAPE, "route: %d experts, not in 1..%d", d->E, BNN_MAX_EXPERTS);
  if (d->top_k < 1 || d->top_k > BNN_MAX_TOP_K || d->top_k > d->E)
    return fail(BNN_ERR_SHAPE, "route: top_k %d, not in 1..min(%d, E)", d->top_k, BNN_MAX_TOP_K);
  if (d->groups < 1 || d->groups > BNN_MAX_ROUTE_GROUPS || d->E % d->groups != 0)
    return fail(BNN_ERR_SHAPE, "route: %d groups of %d experts", d->groups, d->E);
  if (d->top_groups < 1 || d->top_groups > d->groups)
    return fail(BNN_ERR_SHAPE, "route: top_groups %d, not in 1..%d", d->top_groups, d->groups);
  if (d->group_top != 1 && d->group_top != 2)
    return fail(BNN_ERR_SHAPE, "route: group_top %d, not 1 or 2", d->group_top);
  if (d->score != BNN_SCORE_SOFTMAX && d->score != BNN_SCORE_SIGMOID)
    return fail(BNN_ERR_SHAPE, "route: unknown score %d", d->score);
  if (d->renorm != 0 && d->renorm != 1)
    return fail(BNN_ERR_SHAPE, "route: renorm %d, not 0 or 1", d->renorm);
  if (!real_type(d->dtype) && d->dtype != BNN_I32)
    return fail(BNN_ERR_SHAPE, "route: unknown dtype %d", d->dtype);
  if (!(d->logit_scale > 0.0f) || !isfinite(d->logit_scale) || !isfinite(d->scale))
    return fail(BNN_ERR_SHAPE, "route: scale must be finite and logit_scale positive and finite");
  if (T < 0 || T >= kMaxRows || stride < d->E || stride > (int64_t{1} << 31))
    return fail(BNN_ERR_SHAPE, "route: T=%lld rows of stride %lld (E=%d)", (long long)T,
                (long long)stride, d->E);
  return BNN_OK;
}

bnn_status group_check(int64_t M, int32_t G) {
  if (M < 0 || M >= kMaxRows || G < 1 || G > BNN_MAX_EXPERTS)
    return fail(BNN_ERR_SHAPE, "group_rows: M=%lld rows, %d groups", (long long)M, G);
  return BNN_OK;
}

bnn_status workspace_check(const char* what, const void* ws, size_t bytes, size_t need) {
  if (bytes < need || (need && !ws))
    return fail(BNN_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu needed", what, bytes, need);
  if (need && !aligned16(ws))
    return fail(BNN_ERR_ALIGN, "%s: the workspace must be 16-byte aligned", what);
  return BNN_OK;
}

bnn_status experts_check(const bnn_experts_desc* d, const char* what) {
  if (!d) return fail(BNN_ERR_NULL, "%s: descriptor is NULL", what);
  if (d->E < 1 || d->E > BNN_MAX_EXPERTS)
    return fail(BNN_ERR_SHAPE, "%s: %d experts, not in 1..%d", what, d->E, BNN_MAX_EXPERTS);
  if (d->top_k < 1 || d->top_k > BNN_MAX_TOP_K)
    return fail(BNN_ERR_SHAPE, "%s: top_k %d, not in 1..%d", what, d->top_k, BNN_MAX_TOP_K);
  if (d->N < 1 || d->N > 65536 || d->K < 1 || d->K > 65535)
    return fail(BNN_ERR_SHAPE, "%s: N=%d K=%d out of range", what, d->N, d->K);
  if (d->share != 0 && d->share != 1)
    return fail(BNN_ERR_SHAPE, "%s: share %d, not 0 or 1", what, d->share);
  if (d->T < 0 || d->T >= kMaxRows || d->T * d->top_k >= kMaxRows)
    return fail(BNN_ERR_SHAPE, "%s: %lld rows of %d experts", what, (long long)d->T, d->top_k);
  if (d->T * d->top_k * ((d->N + 63) / 64) > kMaxTiles)
    return fail(BNN_ERR_SHAPE, "%s: %lld rows of %d outputs are too large for one launch", what,
                (long long)(d->T * d->top_k), d->N);
  return BNN_OK;
}

bnn::ExpertsArgs experts_args(const bnn_experts_desc& d, const uint32_t* x, const uint32_t* w,
                              const int32_t* offsets, const int32_t* order) {
  bnn::ExpertsArgs a = {};
  a.x = x;
  a.w = w;
  a.offsets = offsets;
  a.order = order;
  a.T = d.T;
  a.M = static_cast<int32_t>(d.T * d.top_k);
  a.E = d.E;
  a.N = d.N;
  a.K = d.K;
  a.top_k = d.top_k;
  a.share = d.share ? d.top_k : 1;
  return a;
}

bnn_status lora_check(const bnn_lora_desc* d) {
  if (!d) return fail(BNN_ERR_NULL, "lora: descriptor is NULL");
  if (d->M < 0 || d->M >= kMaxRows)
    return fail(BNN_ERR_SHAPE, "lora: M=%lld rows", (long long)d->M);
  if (d->N < 1 || d->N > 65536 || d->K < 1 || d->K > 65536)
    return fail(BNN_ERR_SHAPE, "lora: N=%d K=%d out of range", d->N, d->K);
  if (d->M * ((d->N + 63) / 64) > kMaxTiles)
    return fail(BNN_ERR_SHAPE, "lora: %lld rows of %d outputs are too large for one launch",
                (long long)d->M, d->N);
  if (d->adapters < 1 || d->adapters > BNN_MAX_EXPERTS)
    return fail(BNN_ERR_SHAPE, "lora: %d adapters, not in 1..%d", d->adapters, BNN_MAX_EXPERTS);
  if (d->rank < 1) return fail(BNN_ERR_SHAPE, "lora: rank %d < 1", d->rank);
  if (d->rank > BNN_MAX_RANK || d->rank % 8 != 0)
    return fail(BNN_ERR_UNSUPPORTED, "lora: rank %d is not a multiple of 8 up to %d", d->rank,
                BNN_MAX_RANK);
  if (!real_type(d->dtype) || !real_type(d->out_dtype))
    return fail(BNN_ERR_SHAPE, "lora: unknown dtype %d or out_dtype %d", d->dtype, d->out_dtype);
  return BNN_OK;
}

}  // namespace

extern "C" {

bnn_status bnn_route(const bnn_route_desc* d, int64_t T, const void* logits, int64_t stride,
                     const float* bias, int32_t* ids, float* weights, hipStream_t stream) {
  try {
    const bnn_status st = route_check(d, T, stride);
    if (st != BNN_OK) return st;
    if (T == 0) return ok();
    if (!logits || !ids || !weights)
      return fail(BNN_ERR_NULL, "route: logits, ids and weights must be non-NULL");
    if (reinterpret_cast<uintptr_t>(logits) % bnn::dtype_bytes(d->dtype) != 0)
      return fail(BNN_ERR_SHAPE, "route: logits are not aligned to their element");
    return hip_status(bnn::launch_route(*d, T, logits, stride, bias, ids, weights, stream),
                      "route launch");
  } catch (...) {
    return fail(BNN_ERR_HIP, "route: unexpected C++ exception");
  }
}

bnn_status bnn_group_rows_workspace_size(int64_t M, int32_t G, size_t* bytes) {
  try {
    const bnn_status st = group_check(M, G);
    if (st != BNN_OK) return st;
    if (!bytes) return fail(BNN_ERR_NULL, "group_rows: bytes is NULL");
    *bytes = bnn::group_rows_workspace(M, G);
    return ok();
  } catch (...) {
    return fail(BNN_ERR_HIP, "group_rows: unexpected C++ exception");
  }
}

bnn_status bnn_group_rows(int64_t M, int32_t G, const int32_t* ids, int32_t* offsets,
                          int32_t* order, void* workspace, size_t ws_bytes, hipStream_t stream) {
  try {
    const bnn_status st = group_check(M, G);
    if (st != BNN_OK) return st;
    if (!offsets || (M > 0 && (!ids || !order)))
      return fail(BNN_ERR_NULL, "group_rows: ids, offsets and order must be non-NULL");
    const bnn_status ws = workspace_check("group_rows", workspace, ws_bytes,
                                          bnn::group_rows_workspace(M, G));
    if (ws != BNN_OK) return ws;
    return hip_status(bnn::launch_group_rows(M, G, ids, offsets, order, workspace, stream),
                      "group_rows launch");
  } catch (...) {
    return fail(BNN_ERR_HIP, "group_rows: unexpected C++ exception");
  }
}

bnn_status bnn_experts_fc(const bnn_experts_desc* d, const uint32_t* x, const uint32_t* w,
                          const int32_t* offsets, const int32_t* order, const int32_t* thr,
                          const uint32_t* flip, uint32_t* out_bits, hipStream_t stream) {
  try {
    const bnn_status st = experts_check(d, "experts_fc");
    if (st != BNN_OK) return st;
    if (d->T == 0) return ok();
    if (!x || !w || !offsets || !order || !thr || !out_bits)
      return fail(BNN_ERR_NULL,
                  "experts_fc: x, w, offsets, order, thr and out_bits must be non-NULL");
    if (!aligned16(x) || !aligned16(w) || !aligned16(out_bits))
      return fail(BNN_ERR_ALIGN, "experts_fc: x, w and out_bits must be 16-byte aligned");
    bnn::ExpertsArgs a = experts_args(*d, x, w, offsets, order);
    a.thr = thr;
    a.flip = flip;
    a.bits = out_bits;
    return hip_status(bnn::launch_experts_fc(a, stream), "experts_fc launch");
  } catch (...) {
    return fail(BNN_ERR_HIP, "experts_fc: unexpected C++ exception");
  }
}

bnn_status bnn_experts_sum_workspace_size(const bnn_experts_desc* d, size_t* bytes) {
  try {
    const bnn_status st = experts_check(d, "experts_sum");
    if (st != BNN_OK) return st;
    if (!bytes) return fail(BNN_ERR_NULL, "experts_sum: bytes is NULL");
    *bytes = bnn::experts_sum_workspace(*d);
    return ok();
  } catch (...) {
    return fail(BNN_ERR_HIP, "experts_sum: unexpected C++ exception");
  }
}

bnn_status bnn_experts_sum(const bnn_experts_desc* d, const uint32_t* x, const uint32_t* w,
                           const int32_t* ids, const float* weights, const int32_t* offsets,
                           const int32_t* order, const float* alpha, int32_t dtype, void* y,
                           void* workspace, size_t ws_bytes, hipStream_t stream) {
  try {
    const bnn_status st = experts_check(d, "experts_sum");
    if (st != BNN_OK) return st;
    if (!real_type(dtype)) return fail(BNN_ERR_SHAPE, "experts_sum: unknown dtype %d", dtype);
    if (d->T == 0) return ok();
    if (!x || !w || !ids || !weights || !offsets || !order || !y)
      return fail(BNN_ERR_NULL,
                  "experts_sum: x, w, ids, weights, offsets, order and y must be non-NULL");
    if (!aligned16(x) || !aligned16(w) || !aligned16(y))
      return fail(BNN_ERR_ALIGN, "experts_sum: x, w and y must be 16-byte aligned");
    const bnn_status ws = workspace_check("experts_sum", workspace, ws_bytes,
                                          bnn::experts_sum_workspace(*d));
    if (ws != BNN_OK) return ws;
    bnn::ExpertsArgs a = experts_args(*d, x, w, offsets, order);
    a.ids = ids;
    a.weights = weights;
    a.alpha = alpha;
    a.dtype = dtype;
    a.y = y;
    a.ws = workspace;
    return hip_status(bnn::launch_experts_sum(a, stream), "experts_sum launch");
  } catch (...) {
    return fail(BNN_ERR_HIP, "experts_sum: unexpected C++ exception");
  }
}

bnn_status bnn_bgemm_lora_workspace_size(const bnn_lora_desc* d, size_t* bytes) {
  try {
    const bnn_status st = lora_check(d);
    if (st != BNN_OK) return st;
    if (!bytes) return fail(BNN_ERR_NULL, "lora: bytes is NULL");
    *bytes = bnn::lora_workspace(*d);
    return ok();
  } catch (...) {
    return fail(BNN_ERR_HIP, "lora: unexpected C++ exception");
  }
}

bnn_status bnn_bgemm_lora(const bnn_lora_desc* d, const void* x, int64_t x_stride,
                          const float* offset, const uint32_t* w, const float* alpha,
                          const int32_t* ids, const void* a, const void* b, const float* scale,
                          const int32_t* order, void* y, void* workspace, size_t ws_bytes,
                          hipStream_t stream) {
  try {
    const bnn_status st = lora_check(d);
    if (st != BNN_OK) return st;
    if (x_stride < d->K || x_stride > (int64_t{1} << 31))
      return fail(BNN_ERR_SHAPE, "lora: x_stride %lld (K=%d)", (long long)x_stride, d->K);
    if (d->M == 0) return ok();
    if (!x || !w || !ids || !a || !b || !y)
      return fail(BNN_ERR_NULL, "lora: x, w, ids, a, b and y must be non-NULL");
    if (!aligned16(x) || !aligned16(w) || !aligned16(a) || !aligned16(b) || !aligned16(y))
      return fail(BNN_ERR_ALIGN, "lora: x, w, a, b and y must be 16-byte aligned");
    const bnn_status ws = workspace_check("lora", workspace, ws_bytes, bnn::lora_workspace(*d));
    if (ws != BNN_OK) return ws;
    bnn::LoraArgs g = {};
    g.x = x;
    g.offset = offset;
    g.w = w;
    g.alpha = alpha;
    g.ids = ids;
    g.a = a;
    g.b = b;
    g.scale = scale;
    g.order = order;
    g.y = y;
    g.ws = workspace;
    g.x_stride = x_stride;
    g.M = static_cast<int32_t>(d->M);
    g.N = d->N;
    g.K = d->K;
    g.adapters = d->adapters;
    g.rank = d->rank;
    g.dtype = d->dtype;
    g.out_dtype = d->out_dtype;
    return hip_status(bnn::launch_bgemm_lora(g, stream), "lora launch");
  } catch (...) {
    return fail(BNN_ERR_HIP, "lora: unexpected C++ exception");
  }
}

}  // extern "C"
