// Real-valued element types of the C ABI (bnn_dtype) in device code.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "bnn.h"

namespace bnn {

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(_Float16 x) { return static_cast<float>(x); }
__device__ __forceinline__ float to_f32(__bf16 x) { return static_cast<float>(x); }
__device__ __forceinline__ float to_f32(int32_t x) { return static_cast<float>(x); }

// One rounding to the output type, to nearest even.
template <class T>
__device__ __forceinline__ T from_f32(float x) {
  return static_cast<T>(x);
}

// Calls f with a value of the C++ type of a bnn_dtype (not BNN_I32).
template <class F>
auto with_real_type(int32_t dtype, F&& f) {
  switch (dtype) {
    case BNN_F16: return f(_Float16{});
    case BNN_BF16: return f(__bf16{});
    default: return f(float{});
  }
}

inline size_t dtype_bytes(int32_t dtype) { return dtype == BNN_F32 || dtype == BNN_I32 ? 4 : 2; }

}  // namespace bnn
