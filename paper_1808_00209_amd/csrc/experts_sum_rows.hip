// The weighted sum of the experts (bnn_experts_sum) for few rows, in one
// launch and without the rows' order: a workgroup per row and 16 outputs, a
// wave per expert of the row.  A lane compares 4 words of one output's weights
// with the row's at a time (XOR + popcount, Eq. 4: 8 vector instructions for
// 16 bytes, where the matrix cores' operands for the one row would take
// eleven times as many), all loads in flight.  The sums meet in LDS and are
// weighted and added in the order of the row's experts.
// 1 row x 8 experts, 4096 -> 1024: 5.8 us, a launch and two chains of loads (8.7
// us on the matrix cores in the same shape); 8 rows: 34 MB of weights in 8.1 us.
#include "dtypes.hpp"
#include "experts.hpp"
#include "kernels.hpp"

namespace bnn {
namespace {

typedef uint32_t v4u __attribute__((ext_vector_type(4)));

constexpr int kOuts = 16;   // outputs per workgroup: lane (q, c) has output c
constexpr int kStep = 16;   // words of a row per load: lane (q, c) has words 4 q ..
constexpr int kAhead = 8;   // loads in flight

template <class Y>
__global__ __launch_bounds__(64 * BNN_MAX_TOP_K) void experts_sum_rows_kernel(ExpertsArgs a) {
  __shared__ int32_t sums[BNN_MAX_TOP_K][kOuts];
  const int tid = threadIdx.x, lane = tid & 63, q = lane >> 4, c = lane & 15;
  const int j = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int kw = (a.K + 31) >> 5, tiles = (a.N + kOuts - 1) / kOuts;
  const int t = blockIdx.x / tiles, n0 = kOuts * (blockIdx.x - t * tiles);
  const int m = t * a.top_k + j;
  const int e = a.ids[m];
  if (e >= 0 && e < a.E) {  // (uniform over the wave)
    const uint32_t* x = a.x + static_cast<size_t>(m / a.share) * kw;
    const uint32_t* w =
        a.w + (static_cast<size_t>(e) * a.N + min(n0 + c, a.N - 1)) * kw;
    int pop = 0;
    const int fours = a.K >> 7 << 2;  // words in whole groups of 4
    for (int i0 = 0; i0 < fours; i0 += kStep * kAhead) {
      v4u u[kAhead], v[kAhead];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        u[k] = v[k] = v4u{};
        const int i = i0 + kStep * k + 4 * q;
        if (i < fours) {
          __builtin_memcpy(&u[k], x + i, sizeof(u[k]));
          __builtin_memcpy(&v[k], w + i, sizeof(v[k]));
        }
      }
#pragma unroll
      for (int k = 0; k < kAhead; ++k)
#pragma unroll
        for (int r = 0; r < 4; ++r) pop += __popc(u[k][r] ^ v[k][r]);
    }
    // Up to 4 words more, the last one by its valid bits.
    const int i = fours + q;
    if (i < kw) pop += __popc((x[i] ^ w[i]) & (i == kw - 1 ? tail_mask(a.K) : ~0u));
    pop += __shfl_xor(pop, 16);
    pop += __shfl_xor(pop, 32);
    if (q == 0) sums[j][c] = a.K - 2 * pop;
  }
  // The factors of the sums, loaded by the threads that add them up.
  const bool out = tid < kOuts && n0 + tid < a.N;
  float f[BNN_MAX_TOP_K];
  uint32_t used = 0;  // bit i: the row's place i has an expert
#pragma unroll
  for (int i = 0; i < BNN_MAX_TOP_K; ++i) {
    if (i >= a.top_k) break;
    const int at = t * a.top_k + i, id = a.ids[at];
    if (id < 0 || id >= a.E) continue;
    used |= 1u << i;
    if (out)
      f[i] = a.weights[at] *
             (a.alpha ? a.alpha[static_cast<size_t>(id) * a.N + n0 + tid] : 1.0f);
  }
  __syncthreads();
  if (!out) return;
  float y = 0.0f;
#pragma unroll
  for (int i = 0; i < BNN_MAX_TOP_K; ++i)
    if (used >> i & 1) y += f[i] * static_cast<float>(sums[i][tid]);
  static_cast<Y*>(a.y)[static_cast<size_t>(t) * a.N + n0 + tid] = from_f32<Y>(y);
}

}  // namespace

hipError_t launch_experts_sum_rows(const ExpertsArgs& a, hipStream_t s) {
  const unsigned grid = static_cast<unsigned>(a.T * ((a.N + kOuts - 1) / kOuts));
  with_real_type(a.dtype, [&](auto v) {
    experts_sum_rows_kernel<decltype(v)><<<grid, 64 * a.top_k, 0, s>>>(a);
  });
  return hipGetLastError();
}

}  // namespace bnn
