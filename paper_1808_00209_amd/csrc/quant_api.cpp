// C ABI of the 8-bit layers and the answers' log probabilities (include/bnn.h):
// host-side checks and dispatch, in the manner of api.cpp.
#include "bnn.h"

#include <math.h>

#include "dtypes.hpp"
#include "quant.hpp"
#include "status.hpp"

namespace {

using bnn::fail;
using bnn::hip_status;
using bnn::ok;

constexpr int64_t kMaxRows = int64_t{1} << 24;
constexpr int64_t kMaxStride = int64_t{1} << 31;

bool real_type(int32_t t) { return t == BNN_F32 || t == BNN_F16 || t == BNN_BF16; }

bool aligned_to(const void* p, size_t bytes) {
  return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0;
}

bnn_status norm_check(const bnn_rmsnorm_desc* d) {
  if (!d) return fail(BNN_ERR_NULL, "rmsnorm: descriptor is NULL");
  if (d->M < 0 || d->M >= kMaxRows)
    return fail(BNN_ERR_SHAPE, "rmsnorm: M=%lld rows", (long long)d->M);
  if (d->D < 1 || d->D > BNN_MAX_NORM_SIZE)
    return fail(BNN_ERR_SHAPE, "rmsnorm: D=%d, not in 1..%d", d->D, BNN_MAX_NORM_SIZE);
  if (!real_type(d->dtype)) return fail(BNN_ERR_SHAPE, "rmsnorm: unknown dtype %d", d->dtype);
  if (d->weight_dtype != d->dtype && d->weight_dtype != BNN_F32)
    return fail(BNN_ERR_SHAPE, "rmsnorm: weight_dtype %d, neither the rows' nor fp32",
                d->weight_dtype);
  if (!(d->eps >= 0.0f) || !isfinite(d->eps))
    return fail(BNN_ERR_SHAPE, "rmsnorm: eps must be finite and not negative");
  return BNN_OK;
}

bnn_status q8_check(const bnn_q8gemm_desc* d, int64_t x_stride, int64_t w_stride) {
  if (!d) return fail(BNN_ERR_NULL, "q8gemm: descriptor is NULL");
  if (d->M < 0 || d->M >= kMaxRows)
    return fail(BNN_ERR_SHAPE, "q8gemm: M=%lld rows", (long long)d->M);
  if (d->N < 1 || d->N > (1 << 20) || d->K < 1 || d->K > 131071)
    return fail(BNN_ERR_SHAPE, "q8gemm: N=%d K=%d out of range", d->N, d->K);
  if (d->M * d->N > int64_t{1} << 35)
    return fail(BNN_ERR_SHAPE, "q8gemm: %lld rows of %d outputs are too large for one launch",
                (long long)d->M, d->N);
  if (!real_type(d->dtype)) return fail(BNN_ERR_SHAPE, "q8gemm: unknown dtype %d", d->dtype);
  if (x_stride < d->K || x_stride > kMaxStride || w_stride < d->K || w_stride > kMaxStride)
    return fail(BNN_ERR_SHAPE, "q8gemm: rows of stride %lld and %lld (K=%d)", (long long)x_stride,
                (long long)w_stride, d->K);
  return BNN_OK;
}

bnn_status logprobs_check(const bnn_logprobs_desc* d) {
  if (!d) return fail(BNN_ERR_NULL, "logprobs: descriptor is NULL");
  if (d->T < 0 || d->T >= kMaxRows)
    return fail(BNN_ERR_SHAPE, "logprobs: T=%lld rows", (long long)d->T);
  if (d->V < 1 || d->V > (1 << 24))
    return fail(BNN_ERR_SHAPE, "logprobs: V=%d, not in 1..2^24", d->V);
  if (d->n < 0 || d->n > BNN_MAX_GIVEN)
    return fail(BNN_ERR_SHAPE, "logprobs: n=%d, not in 0..%d", d->n, BNN_MAX_GIVEN);
  if (d->top_k < 0 || d->top_k > BNN_MAX_ALTERNATIVES || d->top_k > d->V)
    return fail(BNN_ERR_SHAPE, "logprobs: top_k %d, not in 0..min(%d, V)", d->top_k,
                BNN_MAX_ALTERNATIVES);
  if (!real_type(d->dtype) && d->dtype != BNN_I32)
    return fail(BNN_ERR_SHAPE, "logprobs: unknown dtype %d", d->dtype);
  if (!(d->logit_scale > 0.0f) || !(d->logit_scale <= 0x1p100f))
    return fail(BNN_ERR_SHAPE, "logprobs: logit_scale must be positive and at most 2^100");
  return BNN_OK;
}

}  // namespace

extern "C" {

bnn_status bnn_rmsnorm(const bnn_rmsnorm_desc* d, const void* x, int64_t x_stride,
                       const void* residual, int64_t residual_stride, const void* weight,
                       void* sum, void* y, int8_t* q, int64_t q_stride, float* scale,
                       hipStream_t stream) {
  try {
    const bnn_status st = norm_check(d);
    if (st != BNN_OK) return st;
    if (x_stride < d->D || x_stride > kMaxStride ||
        (residual && (residual_stride < d->D || residual_stride > kMaxStride)) ||
        (q && (q_stride < d->D || q_stride > kMaxStride)))
      return fail(BNN_ERR_SHAPE, "rmsnorm: rows of stride %lld, %lld and %lld (D=%d)",
                  (long long)x_stride, (long long)residual_stride, (long long)q_stride, d->D);
    if (d->M == 0) return ok();
    if (!sum && !y && !q) return fail(BNN_ERR_NULL, "rmsnorm: one of sum, y and q must be non-NULL");
    if (!q != !scale) return fail(BNN_ERR_NULL, "rmsnorm: q and scale go together");
    if (!x) return fail(BNN_ERR_NULL, "rmsnorm: x must be non-NULL");
    if (sum && sum == y) return fail(BNN_ERR_SHAPE, "rmsnorm: sum and y are the same rows");
    const size_t size = bnn::dtype_bytes(d->dtype);
    if (!aligned_to(x, size) || !aligned_to(residual, size) || !aligned_to(sum, size) ||
        !aligned_to(y, size) || !aligned_to(weight, bnn::dtype_bytes(d->weight_dtype)) ||
        !aligned_to(scale, 4))
      return fail(BNN_ERR_SHAPE, "rmsnorm: a pointer is not aligned to its element");
    for (const void* out : {static_cast<const void*>(sum), static_cast<const void*>(y)})
      if (out && ((out == x && x_stride != d->D && d->M > 1) ||
                  (out == residual && residual_stride != d->D && d->M > 1)))
        return fail(BNN_ERR_SHAPE, "rmsnorm: rows written in place must be contiguous");
    bnn::NormArgs a = {};
    a.x = x;
    a.residual = residual;
    a.weight = weight;
    a.sum = sum;
    a.y = y;
    a.q = q;
    a.scale = scale;
    a.x_stride = x_stride;
    a.r_stride = residual_stride;
    a.q_stride = q_stride;
    a.M = d->M;
    a.D = d->D;
    a.dtype = d->dtype;
    a.weight_dtype = d->weight_dtype;
    a.eps = d->eps;
    return hip_status(bnn::launch_rmsnorm(a, stream), "rmsnorm launch");
  } catch (...) {
    return fail(BNN_ERR_HIP, "rmsnorm: unexpected C++ exception");
  }
}

bnn_status bnn_q8gemm(const bnn_q8gemm_desc* d, const int8_t* x, int64_t x_stride,
                      const float* x_scale, const int8_t* w, int64_t w_stride,
                      const float* w_scale, const float* bias, void* y, hipStream_t stream) {
  try {
    const bnn_status st = q8_check(d, x_stride, w_stride);
    if (st != BNN_OK) return st;
    if (d->M == 0) return ok();
    if (!x || !w || !y) return fail(BNN_ERR_NULL, "q8gemm: x, w and y must be non-NULL");
    if (!aligned_to(y, 16)) return fail(BNN_ERR_ALIGN, "q8gemm: y must be 16-byte aligned");
    if (!aligned_to(x_scale, 4) || !aligned_to(w_scale, 4) || !aligned_to(bias, 4))
      return fail(BNN_ERR_SHAPE, "q8gemm: scales or bias are not aligned to their element");
    bnn::Q8Args a = {};
    a.x = x;
    a.w = w;
    a.x_scale = x_scale;
    a.w_scale = w_scale;
    a.bias = bias;
    a.y = y;
    a.x_stride = x_stride;
    a.w_stride = w_stride;
    a.M = d->M;
    a.N = d->N;
    a.K = d->K;
    a.dtype = d->dtype;
    return hip_status(bnn::launch_q8gemm(a, stream), "q8gemm launch");
  } catch (...) {
    return fail(BNN_ERR_HIP, "q8gemm: unexpected C++ exception");
  }
}

bnn_status bnn_logprobs_workspace_size(const bnn_logprobs_desc* d, size_t* bytes) {
  try {
    const bnn_status st = logprobs_check(d);
    if (st != BNN_OK) return st;
    if (!bytes) return fail(BNN_ERR_NULL, "logprobs: bytes is NULL");
    *bytes = bnn::logprobs_workspace(d->T, d->V, d->top_k);
    return ok();
  } catch (...) {
    return fail(BNN_ERR_HIP, "logprobs: unexpected C++ exception");
  }
}

bnn_status bnn_logprobs(const bnn_logprobs_desc* d, const void* logits, int64_t stride,
                        const int32_t* ids, float* logp, float* entropy, int32_t* top_ids,
                        float* top_logp, void* workspace, size_t ws_bytes, hipStream_t stream) {
  try {
    const bnn_status st = logprobs_check(d);
    if (st != BNN_OK) return st;
    if (stride < d->V || stride > kMaxStride)
      return fail(BNN_ERR_SHAPE, "logprobs: rows of stride %lld (V=%d)", (long long)stride, d->V);
    if (d->T == 0) return ok();
    if (!logits) return fail(BNN_ERR_NULL, "logprobs: logits must be non-NULL");
    if (d->n > 0 && (!ids || !logp))
      return fail(BNN_ERR_NULL, "logprobs: ids and logp must be non-NULL");
    if (d->top_k > 0 && (!top_ids || !top_logp))
      return fail(BNN_ERR_NULL, "logprobs: top_ids and top_logp must be non-NULL");
    if (d->n == 0 && !entropy && d->top_k == 0)
      return fail(BNN_ERR_NULL, "logprobs: nothing is asked for");
    if (!aligned_to(logits, bnn::dtype_bytes(d->dtype)) || !aligned_to(ids, 4) ||
        !aligned_to(logp, 4) || !aligned_to(entropy, 4) || !aligned_to(top_ids, 4) ||
        !aligned_to(top_logp, 4))
      return fail(BNN_ERR_SHAPE, "logprobs: a pointer is not aligned to its element");
    const size_t need = bnn::logprobs_workspace(d->T, d->V, d->top_k);
    if (ws_bytes < need || (need && !workspace))
      return fail(BNN_ERR_WORKSPACE, "logprobs: workspace of %zu bytes, %zu needed", ws_bytes,
                  need);
    if (need && !aligned_to(workspace, 16))
      return fail(BNN_ERR_ALIGN, "logprobs: the workspace must be 16-byte aligned");
    bnn::LogprobsArgs a = {};
    a.logits = logits;
    a.ids = ids;
    a.logp = logp;
    a.entropy = entropy;
    a.top_ids = top_ids;
    a.top_logp = top_logp;
    a.workspace = workspace;
    a.stride = stride;
    a.T = d->T;
    a.V = d->V;
    a.n = d->n;
    a.top_k = d->top_k;
    a.dtype = d->dtype;
    a.scale = d->logit_scale;
    return hip_status(bnn::launch_logprobs(a, stream), "logprobs launch");
  } catch (...) {
    return fail(BNN_ERR_HIP, "logprobs: unexpected C++ exception");
  }
}

}  // extern "C"
