// 8-bit matrix product of few rows (bnn_q8gemm, up to 64 rows): every weight is
// read once, straight into the int8 matrix cores' registers.
//
// A workgroup's 8 waves split K among KW of them (a wave's share of x stays in
// its registers) and 16-output tiles among the others; they walk over the
// tiles, the next one's weights in flight while the present one's sums are
// added up over the KW waves in LDS.
//
// Bound by the weights: 65536 outputs, K 4096: one row in 53.1 us, 5.05 TB/s (a
// large copy reaches 5.1), 16 rows in 58.0, 4.6 TB/s; 4096 outputs, one row: 7.3
// us, of which the weights take 3.3.
#include "dtypes.hpp"
#include "q8gemm.hpp"

namespace bnn {
namespace {

constexpr int kWaves = 8;
constexpr int kNT = 64 * kWaves;
constexpr int kStep = 64;  // bytes of K per matrix instruction

// MT: 16-row tiles of x.  P: a wave's steps along K, at most.
template <class T, int MT, int P>
__global__ __launch_bounds__(kNT) void q8_skinny_kernel(Q8Args a, int kw_log, int steps) {
  __shared__ v4i part[2][kWaves][MT][64];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r = lane & 15, g = lane >> 4;
  const int KW = 1 << kw_log, NW = kWaves >> kw_log;
  const int wk = wave & (KW - 1), wn = wave >> kw_log;
  const int first = wk * steps;  // the wave's first step
  // Where a chunk of 16 bytes would pass the row's end, the last 16 bytes are
  // loaded, and x's that belong to other chunks (or to none) are zeroed.
  auto chunk_at = [&](int s) { return min((first + s) * kStep + 16 * g, a.K - 16); };

  const int tiles = (a.N + 15) / 16;
  v4i w[P];
  auto load_w = [&](int tile) {
    const int8_t* row =
        a.w + static_cast<int64_t>(min(16 * tile + r, a.N - 1)) * a.w_stride;
#pragma unroll
    for (int s = 0; s < P; ++s)
      if (s < steps) w[s] = *reinterpret_cast<const v4i_any*>(row + chunk_at(s));
  };
  load_w(blockIdx.x * NW + wn);  // (on their way before x's)
  __builtin_amdgcn_sched_barrier(0);
  v4i x[MT][P];
#pragma unroll
  for (int t = 0; t < MT; ++t) {
    const int8_t* row = a.x + min(static_cast<int64_t>(16 * t + r), a.M - 1) * a.x_stride;
#pragma unroll
    for (int s = 0; s < P; ++s) {
      v4i v = {0, 0, 0, 0};
      if (s < steps) {
        const int k = (first + s) * kStep + 16 * g;
        v = low_bytes_cleared(*reinterpret_cast<const v4i_any*>(row + chunk_at(s)), k - chunk_at(s));
      }
      x[t][s] = v;
    }
  }

  T* y = static_cast<T*>(a.y);
  int buf = 0;
  const int jump = gridDim.x * NW;
  for (int tile0 = blockIdx.x * NW; tile0 < tiles; tile0 += jump, buf ^= 1) {
    v4i acc[MT] = {};
#pragma unroll
    for (int s = 0; s < P; ++s)
      if (s < steps) {
#pragma unroll
        for (int t = 0; t < MT; ++t)
          acc[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[s], x[t][s], acc[t], 0, 0, 0);
      }
    if (tile0 + jump < tiles) load_w(tile0 + jump + wn);
#pragma unroll
    for (int t = 0; t < MT; ++t) part[buf][wave][t][lane] = acc[t];
    __syncthreads();
    // NW x MT tiles of 16 outputs x 16 rows; lane (g, r) has outputs 4 g .. of
    // row r.
    for (int i = wave; i < NW * MT; i += kWaves) {
      const int n_tile = i / MT, t = i % MT;
      v4i sum = part[buf][n_tile << kw_log][t][lane];
      for (int k = 1; k < KW; ++k) {
        const v4i p = part[buf][(n_tile << kw_log) + k][t][lane];
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[e] += p[e];
      }
      const int m = 16 * t + r, n = 16 * (tile0 + n_tile) + 4 * g;
      if (m < a.M && n < a.N) {
        const float xs = a.x_scale ? a.x_scale[m] : 1.0f;
        T out[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int nc = min(n + e, a.N - 1);
          out[e] = q8_output<T>(sum[e], xs, a.w_scale ? a.w_scale[nc] : 1.0f,
                                a.bias ? a.bias[nc] : 0.0f);
        }
        T* at = y + static_cast<int64_t>(m) * a.N + n;
        if (a.N % 4 == 0) {
          typedef uint32_t out_words __attribute__((ext_vector_type(sizeof(T)), aligned(8)));
          out_words v;
          __builtin_memcpy(&v, out, sizeof(v));
          *reinterpret_cast<out_words*>(at) = v;
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (n + e < a.N) at[e] = out[e];
        }
      }
    }
  }
}

}  // namespace

hipError_t launch_q8_skinny(const Q8Args& a, hipStream_t s) {
  const int all = (a.K + kStep - 1) / kStep;  // steps of a row
  const int kw_log = all >= 16 ? 3 : all >= 8 ? 2 : all >= 4 ? 1 : 0;
  const int steps = (all + (1 << kw_log) - 1) >> kw_log;
  const int tiles = (a.N + 15) / 16;
  const int sets = (tiles + (kWaves >> kw_log) - 1) / (kWaves >> kw_log);
  // Two workgroups per CU (16 x 65536 outputs, K 4096: 58.0 us, one per CU 61.3);
  // with more rows, whose x each of them reads, one (64 x 16384: 25.0 us, two 36.2).
  const int most = a.M <= 16 ? 512 : 256;
  const int grid = sets < most ? sets : most;
  with_real_type(a.dtype, [&](auto t) {
    using T = decltype(t);
    auto go = [&](auto mc, auto pc) {
      q8_skinny_kernel<T, decltype(mc)::value, decltype(pc)::value>
          <<<grid, kNT, 0, s>>>(a, kw_log, steps);
    };
    using std::integral_constant;
    auto rows = [&](auto pc) {
      if (a.M <= 16) return go(integral_constant<int, 1>{}, pc);
      if (a.M <= 32) return go(integral_constant<int, 2>{}, pc);
      if constexpr (decltype(pc)::value <= 8) go(integral_constant<int, 4>{}, pc);
    };
    if (steps <= 4) rows(integral_constant<int, 4>{});
    else if (steps <= 8) rows(integral_constant<int, 8>{});
    else rows(integral_constant<int, 16>{});
  });
  return hipGetLastError();
}

}  // namespace bnn
