// Launchers of the 8-bit layers and the answers' log probabilities
// (rmsnorm.hip, q8gemm.hip, q8gemm_skinny.hip, logprobs.hip).
#pragma once

#include <hip/hip_runtime_api.h>
#include <stddef.h>
#include <stdint.h>

#include "bnn.h"

namespace bnn {

struct NormArgs {
  const void* x;
  const void* residual;  // or NULL
  const void* weight;    // or NULL
  void* sum;             // or NULL
  void* y;               // or NULL
  int8_t* q;             // or NULL, with scale
  float* scale;
  int64_t x_stride, r_stride, q_stride;
  int64_t M;
  int32_t D, dtype, weight_dtype;
  float eps;
};
hipError_t launch_rmsnorm(const NormArgs& a, hipStream_t s);

struct Q8Args {
  const int8_t* x;
  const int8_t* w;
  const float* x_scale;  // or NULL
  const float* w_scale;  // or NULL
  const float* bias;     // or NULL
  void* y;
  int64_t x_stride, w_stride;
  int64_t M;
  int32_t N, K, dtype;
};
hipError_t launch_q8gemm(const Q8Args& a, hipStream_t s);

struct LogprobsArgs {
  const void* logits;
  const int32_t* ids;  // or NULL
  float* logp;         // or NULL
  float* entropy;      // or NULL
  int32_t* top_ids;    // NULL with top_k == 0
  float* top_logp;
  void* workspace;
  int64_t stride;
  int64_t T;
  int32_t V, n, top_k, dtype;
  float scale;
};
size_t logprobs_workspace(int64_t T, int32_t V, int32_t top_k);
hipError_t launch_logprobs(const LogprobsArgs& a, hipStream_t s);

}  // namespace bnn
