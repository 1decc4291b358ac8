// The weighted sum of the experts' products (bnn_experts_sum): y[t][n] = sum
// over j of weight[t][j] alpha[e][n] S, with S = 2 c - K from the counts c of
// equal bits that the product kernels left, 16 bits each (exact up to K =
// 65535, and half of what fp32 products would take).  Added in fp32 in the
// order of j, rounded once.
//
// A thread computes 8 outputs of a row.  The bytes are the counts, top_k N 2
// per row, and y; but every pair also reads its expert's alpha, twice the
// bytes of its counts, from the L2: 8192 rows x 8 experts, 1024 outputs, 122 us
// with one read after another.  Two forms avoid that: a row's reads are all in
// flight (36 us, 168 MB at 4.6 TB/s, at 64, 128 and 256 experts), or the alphas
// of all experts for 256 outputs are staged in LDS for many rows (combine_rows
// in expert_plans.hpp).
#include "dtypes.hpp"
#include "expert_plans.hpp"
#include "experts.hpp"

namespace bnn {
namespace {

constexpr int kNT = 256;
constexpr int kCols = kCombineCols;  // outputs per block of the staged form
constexpr int kColThreads = kCols / 8;
constexpr int kTokens = kNT / kColThreads;
constexpr int kAhead = 8;            // pairs in flight

// alpha of 8 outputs from n on.
__device__ __forceinline__ void load_alpha(const float* row, int n, int N, float (&f)[8]) {
  if (n + 8 <= N) {
    __builtin_memcpy(f, row + n, sizeof(f));
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = n + i < N ? row[n + i] : 0.0f;
  }
}

__device__ __forceinline__ void add_pair(float (&y)[8], const uint4& c, const float (&f)[8],
                                         float w, int K) {
  const uint32_t v[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int n = static_cast<int>(v[i / 2] >> (16 * (i & 1)) & 0xFFFFu);
    y[i] += w * f[i] * static_cast<float>(2 * n - K);
  }
}

template <class Y>
__device__ __forceinline__ void store_outputs(Y* row, int n, int N, const float (&y)[8]) {
  Y out[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) out[i] = from_f32<Y>(y[i]);
  if (n + 8 <= N) {
    __builtin_memcpy(row + n, out, sizeof(out));
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (n + i < N) row[n + i] = out[i];
  }
}

// STAGED: block (256 outputs, a range of rows), alphas in LDS; else block
// (row, 8 blockDim outputs).
template <class Y, bool STAGED>
__global__ __launch_bounds__(kNT) void experts_combine_kernel(ExpertsArgs a,
                                                              const uint16_t* __restrict__ counts,
                                                              int rows) {
  extern __shared__ __attribute__((aligned(16))) float alphas[];  // [E][kCols]
  int n, t, end, step;
  const int tid = threadIdx.x;
  if constexpr (STAGED) {
    const int n0 = blockIdx.x * kCols;
    for (int v = tid; v < a.E * kColThreads; v += kNT) {
      const int e = v / kColThreads, col = 8 * (v % kColThreads);
      float f[8] = {1.0f, 1.0f, 1.0f, 1.0f, 1.0f, 1.0f, 1.0f, 1.0f};
      if (a.alpha && n0 + col < a.N)
        load_alpha(a.alpha + static_cast<size_t>(e) * a.N, n0 + col, a.N, f);
      __builtin_memcpy(__builtin_assume_aligned(alphas + e * kCols + col, 16), f, sizeof(f));
    }
    __syncthreads();
    n = n0 + 8 * (tid % kColThreads);
    t = blockIdx.y * rows + tid / kColThreads;
    end = min(static_cast<int>(blockIdx.y + 1) * rows, static_cast<int>(a.T));
    step = kTokens;
  } else {
    t = blockIdx.x;
    end = t + 1;
    step = 1;
    n = 8 * (blockIdx.y * static_cast<int>(blockDim.x) + tid);
  }
  if (n >= a.N) return;
  const int ns = counts_stride(a.N);
  for (; t < end; t += step) {
    float y[8] = {};
    for (int j0 = 0; j0 < a.top_k; j0 += kAhead) {
      int id[kAhead];
      float w[kAhead];
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        const int m = t * a.top_k + min(j0 + j, a.top_k - 1);
        id[j] = j0 + j < a.top_k ? a.ids[m] : -1;
        w[j] = a.weights[m];
      }
      uint4 c[kAhead];
      float f[STAGED ? 1 : kAhead][8];
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        const bool in = id[j] >= 0 && id[j] < a.E;
        if (!in) id[j] = -1;
        const int m = t * a.top_k + min(j0 + j, a.top_k - 1);
        if (in)
          c[j] = *reinterpret_cast<const uint4*>(counts + static_cast<size_t>(m) * ns + n);
        if constexpr (!STAGED) {
#pragma unroll
          for (int i = 0; i < 8; ++i) f[j][i] = 1.0f;
          if (in && a.alpha) load_alpha(a.alpha + static_cast<size_t>(id[j]) * a.N, n, a.N, f[j]);
        }
      }
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        if (id[j] < 0) continue;
        if constexpr (STAGED) {
          float s[8];
          __builtin_memcpy(
              s, __builtin_assume_aligned(alphas + id[j] * kCols + 8 * (tid % kColThreads), 16),
              sizeof(s));
          add_pair(y, c[j], s, w[j], a.K);
        } else {
          add_pair(y, c[j], f[j], w[j], a.K);
        }
      }
    }
    store_outputs<Y>(static_cast<Y*>(a.y) + static_cast<size_t>(t) * a.N, n, a.N, y);
  }
}

template <class Y>
void launch_typed(const ExpertsArgs& a, const uint16_t* counts, hipStream_t s) {
  if (const int rows = combine_rows(a.T, a.E, a.N)) {
    const int cols = (a.N + kCols - 1) / kCols;
    const size_t lds = static_cast<size_t>(a.E) * kCols * sizeof(float);
    const dim3 grid(static_cast<unsigned>(cols), static_cast<unsigned>((a.T + rows - 1) / rows));
    experts_combine_kernel<Y, true><<<grid, kNT, lds, s>>>(a, counts, rows);
  } else {
    const int threads = a.N >= 8 * kNT ? kNT : ((a.N + 7) / 8 + 63) / 64 * 64;
    const dim3 grid(static_cast<unsigned>(a.T),
                    static_cast<unsigned>((a.N + 8 * threads - 1) / (8 * threads)));
    experts_combine_kernel<Y, false><<<grid, threads, 0, s>>>(a, counts, 1);
  }
}

}  // namespace

hipError_t launch_experts_combine(const ExpertsArgs& a, const uint16_t* counts, hipStream_t s) {
  with_real_type(a.dtype, [&](auto v) { launch_typed<decltype(v)>(a, counts, s); });
  return hipGetLastError();
}

}  // namespace bnn
