// Binary FC layers of experts (bnn_experts_fc, bnn_experts_sum): the choice of
// kernel, the vector-ALU kernels (a thread per output, XOR + popcount over the
// row's words, Eq. 4; option algo = BNN_ALGO_VALU and rows of over 4 GiB).
#include "dtypes.hpp"
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

// The skinny kernel has a workgroup per 32 rows of an expert and 32 outputs,
// and splits K over its waves: quicker while the whole chip takes about one
// round of them, several times slower at many (measured, skinny against tile
// kernel, rows x experts per row of E, K -> N: 1 x 8 of 64, 1024 -> 4096: 5.7
// and 6.4 us, 4 x 8: 12.1 and 8.7; 4 x 8, 4096 -> 1024: 8.3 and 10.7, 64 x 8: 19.2
// and 11.4; 1 of 4, 4096 -> 4096: 4.6 and 10.6; 1000 x 2 of 8, 512 -> 512: 4.5 and
// 5.7; 301 x 3 of 24, 1000 -> 1500: 10.3 and 6.9).
hipError_t launch_products(const ExpertsArgs& a, uint16_t* counts, hipStream_t s) {
  const int64_t tiles = (a.M + 31) / 32 + (a.E < a.M ? a.E : a.M);
  return tiles * words_of(a.N) <= 1200 ? launch_experts_skinny(a, counts, s)
                                       : launch_experts_tile(a, counts, s);
}

}  // namespace

hipError_t launch_experts_fc(const ExpertsArgs& a, hipStream_t s) {
  if (use_tiles(a)) return launch_products(a, nullptr, s);
  const dim3 grid(static_cast<unsigned>(a.M), static_cast<unsigned>((a.N + kNT - 1) / kNT));
  experts_fc_valu_kernel<<<grid, kNT, 0, s>>>(a);
  return hipGetLastError();
}

namespace {

// Few rows: every row reads its experts' weights by itself, up to 32 MiB of
// them in all (one launch; rows x 8 of 64 experts, 4096 -> 1024, against
// products and combine: 4 rows 6.0 and 13.1 us, 8 8.1 and 20.0, 32 28.5 and 21.3;
// 32 rows 1024 -> 1024 13.4 and 12.9).
bool few_rows(int64_t M, int32_t N, int32_t K) {
  return M * N * words_of(K) <= (int64_t{8} << 20);
}

}  // namespace

// The counts of every pair.
size_t experts_sum_workspace(const bnn_experts_desc& d) {
  const int64_t M = d.T * d.top_k;
  return few_rows(M, d.N, d.K) ? 0 : static_cast<size_t>(M) * counts_stride(d.N) * sizeof(uint16_t);
}

hipError_t launch_experts_sum(const ExpertsArgs& a, hipStream_t s) {
  if (use_tiles(a) && few_rows(a.M, a.N, a.K)) return launch_experts_sum_rows(a, s);
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
