// Launchers of the kernels behind the mixture-of-experts calls of
// include/bnn.h.  The C-ABI layer (experts_api.cpp) validates every argument
// first; the launchers assume valid sizes and non-empty work.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "bnn.h"

namespace bnn {

hipError_t launch_route(const bnn_route_desc& d, int64_t T, const void* logits, int64_t stride,
                        const float* bias, int32_t* ids, float* weights, hipStream_t s);

size_t group_rows_workspace(int64_t M, int32_t G);
hipError_t launch_group_rows(int64_t M, int32_t G, const int32_t* ids, int32_t* offsets,
                             int32_t* order, void* ws, hipStream_t s);

struct ExpertsArgs {
  const uint32_t* x;       // [T or M][Kw]
  const uint32_t* w;       // [E][N][Kw]
  const int32_t* offsets;  // [E + 1]
  const int32_t* order;    // [M]
  const int32_t* thr;      // [E][N] (bits)
  const uint32_t* flip;    // [E][Nw] or null (bits)
  uint32_t* bits;          // [M][Nw] (bits)
  const int32_t* ids;      // [T][top_k] (sum)
  const float* weights;    // [T][top_k] (sum)
  const float* alpha;      // [E][N] or null (sum)
  void* y;                 // [T][N] (sum)
  void* ws;                // (sum)
  int64_t T;
  int32_t M, E, N, K, top_k;
  int32_t share;           // pairs per row of x: top_k or 1
  int32_t dtype;           // of y (sum)
};

hipError_t launch_experts_fc(const ExpertsArgs& a, hipStream_t s);

// The experts' products on the matrix cores (experts_tile.hip): bits, or with
// counts [M][counts_stride(N)] the numbers of equal bits (S + K) / 2.  x of at most 4 GiB.
bool experts_tile_supported(const ExpertsArgs& a);
hipError_t launch_experts_tile(const ExpertsArgs& a, uint16_t* counts, hipStream_t s);
// The same for few rows per expert (experts_skinny.hip).
hipError_t launch_experts_skinny(const ExpertsArgs& a, uint16_t* counts, hipStream_t s);
// Outputs from one row of counts to the next: N rounded up to 16 bytes.
inline __host__ __device__ int32_t counts_stride(int32_t N) { return (N + 7) / 8 * 8; }
// bnn_experts_sum for few rows in one launch (experts_sum_rows.hip).
hipError_t launch_experts_sum_rows(const ExpertsArgs& a, hipStream_t s);
// y from the counts (experts_combine.hip).
hipError_t launch_experts_combine(const ExpertsArgs& a, const uint16_t* counts, hipStream_t s);

size_t experts_sum_workspace(const bnn_experts_desc& d);
hipError_t launch_experts_sum(const ExpertsArgs& a, hipStream_t s);

struct LoraArgs {
  const void* x;        // [M] rows of K, x_stride elements apart
  const float* offset;  // [K] or null
  const uint32_t* w;    // [N][Kw]
  const float* alpha;   // [N] or null
  const int32_t* ids;   // [M]
  const void* a;        // [adapters][rank][K]
  const void* b;        // [adapters][N][rank]
  const float* scale;   // [adapters] or null
  const int32_t* order; // [M] or null
  void* y;              // [M][N]
  void* ws;
  int64_t x_stride;
  int32_t M, N, K, adapters, rank;
  int32_t dtype, out_dtype;
};

size_t lora_workspace(const bnn_lora_desc& d);
hipError_t launch_bgemm_lora(const LoraArgs& a, hipStream_t s);

// The same on the matrix cores (lora_tile.hip); sign bits of at most 4 GiB.
size_t lora_tile_workspace(int64_t M, int32_t K, int32_t rank);
bool lora_tile_supported(const LoraArgs& a);
hipError_t launch_lora_tile(const LoraArgs& a, hipStream_t s);
// Its two steps for few rows (lora_skinny.hip): u [M][rank] and sign bits, and
// y from them (u as `slices` partial sums).
void launch_lora_down_rows(const LoraArgs& a, float* u, uint32_t* bits, hipStream_t s);
void launch_lora_up_skinny(const LoraArgs& a, const float* u, const uint32_t* bits, int slices,
                           hipStream_t s);

}  // namespace bnn
