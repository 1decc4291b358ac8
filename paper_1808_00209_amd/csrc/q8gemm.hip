// Matrix product of 8-bit integers with a scale per row and per output
// (bnn_q8gemm): the choice of kernel, and the one for operands that lie anywhere
// (rows that are not on 16-byte steps, K below 16).  Its tiles go through
// registers into two LDS buffers in turn: unaligned 16-byte loads, K's end masked
// on the way, the next stage's on their way while one is multiplied.
// 256 x 4096 outputs, K 4095: 30 us, 8192 x 16384 1205 (the tiles of
// q8gemm_tile.hip, K 4096: 9.9 and 500; one buffer and no load ahead 133 and
// 1290): weights that are used often are worth laying out 16 bytes apart.
#include "q8gemm.hpp"

namespace bnn {
namespace {

constexpr int kNT = 256;
constexpr int kBK = 128;         // bytes of K per step
constexpr int kChunks = kBK / 16;

// 16 bytes of a row of K from byte k on, 0 past its end.  Nothing past K is
// read: the last chunk is loaded from 16 bytes before the end and shifted.
__device__ __forceinline__ v4i load16(const int8_t* row, int k, int K) {
  if (k + 16 <= K) return *reinterpret_cast<const v4i_any*>(row + k);
  v4i r = {0, 0, 0, 0};
  if (k >= K) return r;
  const int n = K - k;  // 1..15
  if (K >= 16) {
    const v4i v = *reinterpret_cast<const v4i_any*>(row + K - 16);
    unsigned __int128 u = __builtin_bit_cast(unsigned __int128, v);
    u >>= 8 * (16 - n);
    return __builtin_bit_cast(v4i, u);
  }
  uint32_t b[4] = {0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < 15; ++i)
    if (i < n) b[i / 4] |= static_cast<uint32_t>(static_cast<uint8_t>(row[k + i])) << (8 * (i % 4));
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = static_cast<int>(b[i]);
  return r;
}

// A workgroup of 2 x 2 waves, 64 TM rows x 64 TN outputs.
template <class T, int TM, int TN>
__global__ __launch_bounds__(kNT) void q8_any_kernel(Q8Args a) {
  constexpr int BM = 64 * TM, BN = 64 * TN;
  constexpr int kLoads = (BM + BN) * kChunks / kNT;
  __shared__ v4i lds[2][(BM + BN) * kChunks];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int h = lane >> 5, c = lane & 31;
  const unsigned cols = (a.N + BN - 1) / BN;
  const int64_t m0 = static_cast<int64_t>(blockIdx.x / cols) * BM;
  const int n0 = static_cast<int>(blockIdx.x % cols) * BN;
  const int j = tid % kChunks;  // the thread's chunk of its rows
  const int8_t* rows[kLoads];
#pragma unroll
  for (int l = 0; l < kLoads; ++l) {
    const int row = (l * kNT + tid) / kChunks;
    rows[l] = row < BM ? a.x + min(m0 + row, a.M - 1) * a.x_stride
                       : a.w + static_cast<int64_t>(min(n0 + row - BM, a.N - 1)) * a.w_stride;
  }
  v4i next[kLoads];
  auto load = [&](int k0) {
    if (k0 + kBK <= a.K) {
#pragma unroll
      for (int l = 0; l < kLoads; ++l)
        next[l] = *reinterpret_cast<const v4i_any*>(rows[l] + k0 + 16 * j);
    } else {
#pragma unroll
      for (int l = 0; l < kLoads; ++l) next[l] = load16(rows[l], k0 + 16 * j, a.K);
    }
  };
  v16i acc[TM][TN] = {};
  const int wm = (wave >> 1) * 32 * TM, wn = BM + (wave & 1) * 32 * TN;
  load(0);
  for (int k0 = 0, buf = 0; k0 < a.K; k0 += kBK, buf ^= 1) {
#pragma unroll
    for (int l = 0; l < kLoads; ++l) {
      const int row = (l * kNT + tid) / kChunks;
      lds[buf][row * kChunks + (j ^ (row & 7))] = next[l];
    }
    __syncthreads();  // (the other buffer's readers are past the barrier before)
    if (k0 + kBK < a.K) load(k0 + kBK);
    auto chunk = [&](int row, int s) { return lds[buf][row * kChunks + ((2 * s + h) ^ (row & 7))]; };
#pragma unroll
    for (int s = 0; s < kBK / 32; ++s) {
      v4i x[TM], w[TN];
#pragma unroll
      for (int t = 0; t < TM; ++t) x[t] = chunk(wm + 32 * t + c, s);
#pragma unroll
      for (int t = 0; t < TN; ++t) w[t] = chunk(wn + 32 * t + c, s);
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int k = 0; k < TN; ++k)
          acc[i][k] = __builtin_amdgcn_mfma_i32_32x32x32_i8(x[i], w[k], acc[i][k], 0, 0, 0);
    }
  }
  T* y = static_cast<T*>(a.y);
#pragma unroll
  for (int k = 0; k < TN; ++k) {
    const int n = n0 + wn - BM + 32 * k + c;
    const int nc = min(n, a.N - 1);
    const float ws = a.w_scale ? a.w_scale[nc] : 1.0f;
    const float bias = a.bias ? a.bias[nc] : 0.0f;
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int64_t m = m0 + wm + 32 * i + 8 * (e / 4) + 4 * h + e % 4;
        if (m < a.M && n < a.N) {
          const float xs = a.x_scale ? a.x_scale[m] : 1.0f;
          y[m * a.N + n] = q8_output<T>(acc[i][k][e], xs, ws, bias);
        }
      }
  }
}

}  // namespace

hipError_t launch_q8gemm(const Q8Args& a, hipStream_t s) {
  const bool on16 = q8_on16(reinterpret_cast<uintptr_t>(a.x), a.x_stride, a.M) &&
                    q8_on16(reinterpret_cast<uintptr_t>(a.w), a.w_stride, a.N);
  const Q8Form form = q8_form(a.M, a.N, a.K, on16);
  if (form == kQ8Skinny) return launch_q8_skinny(a, s);
  if (form != kQ8Any) return launch_q8_tile(a, form, s);
  auto any = [&](auto size) {
    constexpr int TS = decltype(size)::value;
    const int64_t tiles = q8_tiles(a.M, a.N, 64 * TS);  // M * N <= 2^35: below 2^24
    with_real_type(a.dtype, [&](auto t) {
      q8_any_kernel<decltype(t), TS, TS><<<static_cast<unsigned>(tiles), kNT, 0, s>>>(a);
    });
  };
  if (q8_any_tile(a.M, a.N) == 128) any(std::integral_constant<int, 2>{});
  else any(std::integral_constant<int, 1>{});
  return hipGetLastError();
}

}  // namespace bnn
