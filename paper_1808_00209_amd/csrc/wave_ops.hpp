// Reductions over a wave's 64 lanes on the vector ALU: DPP inside rows of 16,
// gfx950's v_permlane16/32_swap between them.  Every lane gets the result.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace bnn {

template <int kCtrl>
__device__ __forceinline__ uint32_t dpp_move(uint32_t x) {
  return static_cast<uint32_t>(
      __builtin_amdgcn_update_dpp(0, static_cast<int>(x), kCtrl, 0xF, 0xF, false));
}

// x of the lane before (lane 0: unspecified).
__device__ __forceinline__ uint32_t lane_before(uint32_t x) {
  return static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(x), 0x138, 0xF, 0xF, false));
}

// op over the wave, op commutative.  swap(x, x) leaves the lower of two halves
// (rows) in both places of its first result and the upper in its second.
template <class T, class Op>
__device__ __forceinline__ T wave_reduce(T v, Op&& op) {
  static_assert(sizeof(T) == 4, "one register");
  auto f = [](uint32_t b) { return __builtin_bit_cast(T, b); };
  auto b = [](T x) { return __builtin_bit_cast(uint32_t, x); };
  v = op(v, f(dpp_move<0xB1>(b(v))));   // lane ^ 1
  v = op(v, f(dpp_move<0x4E>(b(v))));   // lane ^ 2
  v = op(v, f(dpp_move<0x141>(b(v))));  // 7 - lane in each 8
  v = op(v, f(dpp_move<0x140>(b(v))));  // 15 - lane in each row
  auto r = __builtin_amdgcn_permlane16_swap(b(v), b(v), false, false);
  v = op(f(r[0]), f(r[1]));
  r = __builtin_amdgcn_permlane32_swap(b(v), b(v), false, false);
  return op(f(r[0]), f(r[1]));
}

template <class Op>
__device__ __forceinline__ double wave_reduce(double v, Op&& op) {
  auto join = [](uint32_t lo, uint32_t hi) {
    return __builtin_bit_cast(double, static_cast<uint64_t>(hi) << 32 | lo);
  };
  auto lo = [](double x) { return static_cast<uint32_t>(__builtin_bit_cast(uint64_t, x)); };
  auto hi = [](double x) { return static_cast<uint32_t>(__builtin_bit_cast(uint64_t, x) >> 32); };
  v = op(v, join(dpp_move<0xB1>(lo(v)), dpp_move<0xB1>(hi(v))));
  v = op(v, join(dpp_move<0x4E>(lo(v)), dpp_move<0x4E>(hi(v))));
  v = op(v, join(dpp_move<0x141>(lo(v)), dpp_move<0x141>(hi(v))));
  v = op(v, join(dpp_move<0x140>(lo(v)), dpp_move<0x140>(hi(v))));
  auto l = __builtin_amdgcn_permlane16_swap(lo(v), lo(v), false, false);
  auto h = __builtin_amdgcn_permlane16_swap(hi(v), hi(v), false, false);
  v = op(join(l[0], h[0]), join(l[1], h[1]));
  l = __builtin_amdgcn_permlane32_swap(lo(v), lo(v), false, false);
  h = __builtin_amdgcn_permlane32_swap(hi(v), hi(v), false, false);
  return op(join(l[0], h[0]), join(l[1], h[1]));
}

template <class T>
__device__ __forceinline__ T wave_sum(T v) {
  return wave_reduce(v, [](T a, T b) { return a + b; });
}
__device__ __forceinline__ float wave_max(float v) {
  return wave_reduce(v, [](float a, float b) { return __builtin_fmaxf(a, b); });
}
__device__ __forceinline__ int32_t wave_max(int32_t v) {
  return wave_reduce(v, [](int32_t a, int32_t b) { return a > b ? a : b; });
}
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
  return wave_reduce(v, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
}
__device__ __forceinline__ uint32_t wave_min(uint32_t v) {
  return wave_reduce(v, [](uint32_t a, uint32_t b) { return a < b ? a : b; });
}
__device__ __forceinline__ double wave_max(double v) {
  return wave_reduce(v, [](double a, double b) { return __builtin_fmax(a, b); });
}

}  // namespace bnn
