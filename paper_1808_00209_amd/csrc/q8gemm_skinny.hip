// 8-bit matrix product of few rows (bnn_q8gemm, up to 16 rows): every weight is
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

// P: a wave's steps along K, at most.
template <class T, int P>
__global__ __launch_bounds__(kNT) void q8_skinny_kernel(Q8Args a, int kw_log, int steps) {
  __shared__ v4i part[2][kWaves][64];
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
  v4i x[P];
  const int8_t* row = a.x + min(static_cast<int64_t>(r), a.M - 1) * a.x_stride;
#pragma unroll
  for (int s = 0; s < P; ++s) {
    v4i v = {0, 0, 0, 0};
    if (s < steps) {
      const int k = (first + s) * kStep + 16 * g;
      v = low_bytes_cleared(*reinterpret_cast<const v4i_any*>(row + chunk_at(s)), k - chunk_at(s));
    }
    x[s] = v;
  }
  T* y = static_cast<T*>(a.y);
  const float xs = a.x_scale ? a.x_scale[min(static_cast<int64_t>(r), a.M - 1)] : 1.0f;
  int buf = 0;
  const int jump = gridDim.x * NW;
  for (int tile0 = blockIdx.x * NW; tile0 < tiles; tile0 += jump, buf ^= 1) {
    // the factors of the outputs that this wave will write, asked for early
    const int n = 16 * (tile0 + wave) + 4 * g;
    float ws[4], bias[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int nc = min(n + e, a.N - 1);
      ws[e] = wave < NW && a.w_scale ? a.w_scale[nc] : 1.0f;
      bias[e] = wave < NW && a.bias ? a.bias[nc] : 0.0f;
    }
    v4i acc = {0, 0, 0, 0};
#pragma unroll
    for (int s = 0; s < P; ++s)
      if (s < steps) acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[s], x[s], acc, 0, 0, 0);
    if (tile0 + jump < tiles) load_w(tile0 + jump + wn);
    part[buf][wave][lane] = acc;
    __syncthreads();
    // NW tiles of 16 outputs x 16 rows; lane (g, r) has outputs 4 g .. of row r.
    if (wave < NW) {
      v4i sum = part[buf][wave << kw_log][lane];
      for (int k = 1; k < KW; ++k) {
        const v4i p = part[buf][(wave << kw_log) + k][lane];
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[e] += p[e];
      }
      if (r < a.M && n < a.N) {
        T out[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) out[e] = q8_output<T>(sum[e], xs, ws[e], bias[e]);
        T* at = y + static_cast<int64_t>(r) * a.N + n;
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
  // two workgroups per CU (16 x 65536 outputs, K 4096: 58.0 us, one per CU 61.3)
  const int grid = sets < 512 ? sets : 512;
  with_real_type(a.dtype, [&](auto t) {
    using T = decltype(t);
    if (steps <= 4) q8_skinny_kernel<T, 4><<<grid, kNT, 0, s>>>(a, kw_log, steps);
    else if (steps <= 8) q8_skinny_kernel<T, 8><<<grid, kNT, 0, s>>>(a, kw_log, steps);
    else q8_skinny_kernel<T, 16><<<grid, kNT, 0, s>>>(a, kw_log, steps);
  });
  return hipGetLastError();
}

}  // namespace bnn
