// A shared binary FC layer with low-rank adapters (bnn_bgemm_lora), in two
// launches: x is read for its sign bits and for u = scale (x a^T), then every
// output adds u b^T to its binary dot product.
#include "dtypes.hpp"
#include "experts.hpp"
#include "kernels.hpp"

namespace bnn {
namespace {

constexpr int kNT = 256;

// The workspace: u [M][rank] fp32, then the sign bits [M][Kw].
struct LoraWs {
  float* u;
  uint32_t* bits;
};

LoraWs split_ws(const LoraArgs& a) {
  LoraWs w;
  w.u = static_cast<float*>(a.ws);
  w.bits = reinterpret_cast<uint32_t*>(w.u + static_cast<size_t>(a.M) * a.rank);
  return w;
}

// A wave per (row, rank component), and one per row for its sign bits.
template <class T>
__global__ __launch_bounds__(64) void lora_down_valu_kernel(LoraArgs a, LoraWs ws) {
  const int m = blockIdx.x, r = static_cast<int>(blockIdx.y) - 1, lane = threadIdx.x;
  const T* x = static_cast<const T*>(a.x) + m * a.x_stride;
  if (r < 0) {
    const int kw = (a.K + 31) / 32;
    for (int k0 = 0; k0 < a.K; k0 += 64) {
      const int k = k0 + lane;
      const bool on = k < a.K && to_f32(x[k]) + (a.offset ? a.offset[k] : 0.0f) > 0.0f;
      const uint64_t word = __ballot(on);
      if ((lane & 31) == 0 && k < a.K)
        ws.bits[static_cast<size_t>(m) * kw + k / 32] =
            __brev(static_cast<uint32_t>(lane ? word >> 32 : word));
    }
    return;
  }
  const int l = a.ids[m];
  if (l < 0 || l >= a.adapters) return;
  const T* row = static_cast<const T*>(a.a) + (static_cast<size_t>(l) * a.rank + r) * a.K;
  float sum = 0.0f;
  for (int k = lane; k < a.K; k += 64) sum += to_f32(x[k]) * to_f32(row[k]);
#pragma unroll
  for (int s = 32; s > 0; s >>= 1) sum += __shfl_xor(sum, s);
  if (lane == 0) ws.u[static_cast<size_t>(m) * a.rank + r] = sum * (a.scale ? a.scale[l] : 1.0f);
}

template <class T, class Y>
__global__ __launch_bounds__(kNT) void lora_up_valu_kernel(LoraArgs a, LoraWs ws) {
  const int m = blockIdx.x;
  const int n = blockIdx.y * kNT + threadIdx.x;
  const int kw = (a.K + 31) / 32;
  if (n >= a.N) return;
  const uint32_t* x = ws.bits + static_cast<size_t>(m) * kw;
  const uint32_t* w = a.w + static_cast<size_t>(n) * kw;
  int pop = 0;
  for (int i = 0; i < kw; ++i)
    pop += __popc((x[i] ^ w[i]) & (i == kw - 1 ? tail_mask(a.K) : ~0u));
  float y = static_cast<float>(a.K - 2 * pop) * (a.alpha ? a.alpha[n] : 1.0f);
  const int l = a.ids[m];
  if (l >= 0 && l < a.adapters) {
    const float* u = ws.u + static_cast<size_t>(m) * a.rank;
    const T* b = static_cast<const T*>(a.b) + (static_cast<size_t>(l) * a.N + n) * a.rank;
    for (int r = 0; r < a.rank; ++r) y += u[r] * to_f32(b[r]);
  }
  static_cast<Y*>(a.y)[static_cast<size_t>(m) * a.N + n] = from_f32<Y>(y);
}

}  // namespace

size_t lora_workspace(const bnn_lora_desc& d) {
  const size_t valu = static_cast<size_t>(d.M) * (d.rank + (d.K + 31) / 32) * 4;
  const size_t tile = lora_tile_workspace(d.M, d.K, d.rank);
  return valu > tile ? valu : tile;
}

hipError_t launch_bgemm_lora(const LoraArgs& a, hipStream_t s) {
  if (options().algo != BNN_ALGO_VALU && lora_tile_supported(a)) return launch_lora_tile(a, s);
  const LoraWs ws = split_ws(a);
  with_real_type(a.dtype, [&](auto v) {
    using T = decltype(v);
    lora_down_valu_kernel<T><<<dim3(static_cast<unsigned>(a.M), static_cast<unsigned>(a.rank + 1)),
                               64, 0, s>>>(a, ws);
    const dim3 grid(static_cast<unsigned>(a.M), static_cast<unsigned>((a.N + kNT - 1) / kNT));
    with_real_type(a.out_dtype, [&](auto y) {
      lora_up_valu_kernel<T, decltype(y)><<<grid, kNT, 0, s>>>(a, ws);
    });
  });
  return hipGetLastError();
}

}  // namespace bnn
