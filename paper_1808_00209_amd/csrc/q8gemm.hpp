// What the kernels of the 8-bit matrix product share.
#pragma once

#include <hip/hip_runtime.h>

#include <type_traits>

#include "dtypes.hpp"
#include "q8_plans.hpp"
#include "quant.hpp"

namespace bnn {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v16i __attribute__((ext_vector_type(16)));
typedef int v4i_any __attribute__((ext_vector_type(4), aligned(1)));

// The 16 bytes of v with the first n (0: none, 16 and more: all) zeroed.
__device__ __forceinline__ v4i low_bytes_cleared(v4i v, int n) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int left = n - 4 * i;  // of this word
    const uint32_t keep = left <= 0 ? ~0u : left >= 4 ? 0u : ~0u << (8 * left);
    v[i] = static_cast<int>(static_cast<uint32_t>(v[i]) & keep);
  }
  return v;
}

template <class T>
__device__ __forceinline__ T q8_output(int32_t sum, float xs, float ws, float bias) {
  return from_f32<T>(static_cast<float>(sum) * xs * ws + bias);
}

// Few rows: every weight read once (q8gemm_skinny.hip).
hipError_t launch_q8_skinny(const Q8Args& a, hipStream_t s);

// Many rows on 16-byte steps (q8gemm_tile.hip): one of the tile forms.
hipError_t launch_q8_tile(const Q8Args& a, Q8Form form, hipStream_t s);

}  // namespace bnn
