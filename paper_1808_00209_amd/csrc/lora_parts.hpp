// Pieces that the kernels of the layer with adapters share: rows by position,
// and u b^T on the bf16 matrix cores at fp32's precision.
#pragma once

#include <type_traits>

#include "dtypes.hpp"
#include "experts.hpp"
#include "fp32_split.hpp"
#include "fp4_expand.hpp"

namespace bnn {

// The row at position p of the order (p itself without one).
__device__ __forceinline__ int lora_row(const LoraArgs& a, int p) {
  p = min(p, a.M - 1);
  return a.order ? static_cast<int>(min(static_cast<uint32_t>(a.order[p]),
                                        static_cast<uint32_t>(a.M - 1)))
                 : p;
}

// The adapter of a row, -1 for none.
__device__ __forceinline__ int lora_adapter(const LoraArgs& a, int row) {
  const int l = a.ids[row];
  return l >= 0 && l < a.adapters ? l : -1;
}

// Parts of a value on the bf16 matrix cores: 1 (bf16), 2 (fp16: 11 significant
// bits) or 3 (fp32), each product of u's three parts and these exact.
template <class T>
constexpr int kParts = sizeof(T) == 4 ? 3 : std::is_same<T, _Float16>::value ? 2 : 1;

// Eight values of u (or b) as bf16 operands, one per part.
template <int P>
__device__ __forceinline__ void split_frag(const float (&v)[8], bool keep, v8bf (&out)[P]) {
  uint16_t b[3][8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const Split3 s = split3(keep ? v[e] : 0.0f);
    b[0][e] = bf16_bits(s.p0);
    b[1][e] = bf16_bits(s.p1);
    b[2][e] = bf16_bits(s.p2);
  }
#pragma unroll
  for (int i = 0; i < P; ++i) out[i] = bf16x8(b[i]);
}

// Lane (h, c)'s share of 16 ranks: b[l][n][r .. r + 7] of an output n (past the
// rank or N: other values, dropped by split_b), as it lies in memory.
template <class T>
struct RawB {
  T v[8];
};

template <class T>
__device__ __forceinline__ RawB<T> load_b(const LoraArgs& a, int l, int n, int r) {
  const bool in = n < a.N && r < a.rank;
  const T* src = static_cast<const T*>(a.b) +
                 (in ? (static_cast<size_t>(l) * a.N + n) * a.rank + r : size_t{0});
  RawB<T> x;
  __builtin_memcpy(x.v, __builtin_assume_aligned(src, 16), sizeof(x.v));
  return x;
}

template <class T>
__device__ __forceinline__ void split_b(const RawB<T>& x, bool keep, v8bf (&out)[kParts<T>]) {
  if constexpr (kParts<T> == 1) {
    uint32_t w[4];
    __builtin_memcpy(w, x.v, sizeof(w));
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = keep ? w[i] : 0u;
    __builtin_memcpy(&out[0], w, sizeof(w));
  } else {
    float f[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = to_f32(x.v[e]);
    split_frag<kParts<T>>(f, keep, out);
  }
}

// acc (32 outputs x 32 rows) += 16 ranks of b u^T, the smallest products first,
// in the rows (a lane's sums are of one) that are `mine`; the others keep
// theirs, whatever b and their u hold.
template <class T>
__device__ __forceinline__ void add_rows(v16f& acc, const v8bf (&b)[kParts<T>],
                                         const v8bf (&u)[3], bool mine) {
  v16f sum = acc;
#pragma unroll
  for (int i = kParts<T> - 1; i >= 0; --i)
#pragma unroll
    for (int j = 2; j >= 0; --j)
      if (i + j < 4) sum = __builtin_amdgcn_mfma_f32_32x32x16_bf16(b[i], u[j], sum, 0, 0, 0);
#pragma unroll
  for (int e = 0; e < 16; ++e) acc[e] = mine ? sum[e] : acc[e];
}

}  // namespace bnn
