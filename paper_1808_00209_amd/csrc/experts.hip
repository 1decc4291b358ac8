// Binary FC layers of experts (bnn_experts_fc, bnn_experts_sum): the choice of
// kernel, the vector-ALU kernels (a thread per output, XOR + popcount over the
// row's words, Eq. 4; option algo = BNN_ALGO_VALU and rows of over 4 GiB).
#include "dtypes.hpp"
#include "expert_plans.hpp"
#include "experts.hpp"
#include "kernels.hpp"

namespace bnn {
namespace {

constexpr int kNT = 256;

// K - 2 popcount(x xor w) over K valid bits.
__device__ __forceinline__ int dot_words(const uint32_t* __restrict__ x,
                                         const uint32_t* __restrict__ w, int K, int kw,
                                         uint32_t last) {
  int pop = 0;
  for (int i = 0; i < kw - 1; ++i) pop += __popc(x[i] ^ w[i]);
  pop += __popc((x[kw - 1] ^ w[kw - 1]) & last);
  return K - 2 * pop;
}

// Block (position in the order, 256 outputs).
__global__ __launch_bounds__(kNT) void experts_fc_valu_kernel(ExpertsArgs a) {
  const int pos = blockIdx.x;
  const int n = blockIdx.y * kNT + threadIdx.x;
  const int kw = (a.K + 31) / 32, nw = (a.N + 31) / 32;
  const int m = min(static_cast<uint32_t>(a.order[pos]), static_cast<uint32_t>(a.M - 1));
  // The group of the position: the number of group ends at or before it.
  int e = 0;
  for (int hi = a.E; e < hi;) {
    const int mid = (e + hi) / 2;
    if (a.offsets[mid + 1] <= pos)
      e = mid + 1;
    else
      hi = mid;
  }
  bool bit = false;
  if (e < a.E && n < a.N) {
    const size_t wrow = static_cast<size_t>(e) * a.N + n;
    const int S = dot_words(a.x + static_cast<size_t>(m / a.share) * kw, a.w + wrow * kw, a.K, kw,
                            tail_mask(a.K));
    const uint32_t fl = a.flip ? a.flip[static_cast<size_t>(e) * nw + n / 32] : 0u;
    bit = (S >= a.thr[wrow]) != ((fl >> (31 - n % 32)) & 1u);
  }
  const uint64_t word = __ballot(bit);
  const int lane = threadIdx.x & 63;
  if ((lane & 31) == 0 && n < a.N)
    a.bits[static_cast<size_t>(m) * nw + n / 32] =
        __brev(static_cast<uint32_t>(lane ? word >> 32 : word));
}

// Block (row, 256 outputs).
template <class Y>
__global__ __launch_bounds__(kNT) void experts_sum_valu_kernel(ExpertsArgs a) {
  const int t = blockIdx.x;
  const int n = blockIdx.y * kNT + threadIdx.x;
  const int kw = (a.K + 31) / 32;
  if (n >= a.N) return;
  float y = 0.0f;
  for (int j = 0; j < a.top_k; ++j) {
    const int m = t * a.top_k + j;
    const int e = a.ids[m];
    if (e < 0 || e >= a.E) continue;
    const size_t wrow = static_cast<size_t>(e) * a.N + n;
    const int S = dot_words(a.x + static_cast<size_t>(m / a.share) * kw, a.w + wrow * kw, a.K, kw,
                            tail_mask(a.K));
    y += a.weights[m] * (a.alpha ? a.alpha[wrow] : 1.0f) * static_cast<float>(S);
  }
  static_cast<Y*>(a.y)[static_cast<size_t>(t) * a.N + n] = from_f32<Y>(y);
}

bool use_tiles(const ExpertsArgs& a) {
  return options().algo != BNN_ALGO_VALU && experts_tile_supported(a);
}

hipError_t launch_products(const ExpertsArgs& a, uint16_t* counts, hipStream_t s) {
  return experts_skinny(a.M, a.E, a.N) ? launch_experts_skinny(a, counts, s)
                                       : launch_experts_tile(a, counts, s);
}

}  // namespace

hipError_t launch_experts_fc(const ExpertsArgs& a, hipStream_t s) {
  if (use_tiles(a)) return launch_products(a, nullptr, s);
  const dim3 grid(static_cast<unsigned>(a.M), static_cast<unsigned>((a.N + kNT - 1) / kNT));
  experts_fc_valu_kernel<<<grid, kNT, 0, s>>>(a);
  return hipGetLastError();
}

// The counts of every pair.
size_t experts_sum_workspace(const bnn_experts_desc& d) {
  const int64_t M = d.T * d.top_k;
  return experts_sum_by_rows(M, d.N, d.K) ? 0 : static_cast<size_t>(M) * counts_stride(d.N) * sizeof(uint16_t);
}

hipError_t launch_experts_sum(const ExpertsArgs& a, hipStream_t s) {
  if (use_tiles(a) && experts_sum_by_rows(a.M, a.N, a.K)) return launch_experts_sum_rows(a, s);
  if (use_tiles(a)) {
    uint16_t* counts = static_cast<uint16_t*>(a.ws);
    const hipError_t err = launch_products(a, counts, s);
    if (err != hipSuccess) return err;
    return launch_experts_combine(a, counts, s);
  }
  const dim3 grid(static_cast<unsigned>(a.T), static_cast<unsigned>((a.N + kNT - 1) / kNT));
  with_real_type(a.dtype, [&](auto v) {
    experts_sum_valu_kernel<decltype(v)><<<grid, kNT, 0, s>>>(a);
  });
  return hipGetLastError();
}

}  // namespace bnn
