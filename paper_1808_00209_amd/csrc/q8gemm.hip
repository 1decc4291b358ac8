// Matrix product of 8-bit integers with a scale per row and per output
// (bnn_q8gemm): the choice of kernel, and the one for operands that lie anywhere
// (rows that are not on 16-byte steps, K below 16).  Its 128 x 128 tiles are
// staged through registers, where K's end is masked, one stage at a time: 256 x
// 4096 outputs, K 4096 in 129 us where the tiles of q8gemm_tile.hip take 9.9, so
// that rows worth a second look are worth laying out 16 bytes apart.
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
  extern __shared__ v4i lds[];
  constexpr int BM = 64 * TM, BN = 64 * TN;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int h = lane >> 5, c = lane & 31;
  const unsigned cols = (a.N + BN - 1) / BN;
  const int64_t m0 = static_cast<int64_t>(blockIdx.x / cols) * BM;
  const int n0 = static_cast<int>(blockIdx.x % cols) * BN;
  v4i* lx = lds;
  v4i* lw = lds + BM * kChunks;
  v16i acc[TM][TN] = {};
  const int wm = (wave >> 1) * 32 * TM, wn = (wave & 1) * 32 * TN;
  for (int k0 = 0; k0 < a.K; k0 += kBK) {
    for (int i = tid; i < (BM + BN) * kChunks; i += kNT) {
      const int row = i / kChunks, j = i % kChunks;
      const int8_t* p;
      if (row < BM) p = a.x + min(m0 + row, a.M - 1) * a.x_stride;
      else p = a.w + static_cast<int64_t>(min(n0 + row - BM, a.N - 1)) * a.w_stride;
      lds[row * kChunks + (j ^ (row & 7))] = load16(p, k0 + 16 * j, a.K);
    }
    __syncthreads();
#pragma unroll
    for (int s = 0; s < kBK / 32; ++s) {
      v4i x[TM], w[TN];
#pragma unroll
      for (int t = 0; t < TM; ++t) {
        const int row = wm + 32 * t + c;
        x[t] = lx[row * kChunks + ((2 * s + h) ^ (row & 7))];
      }
#pragma unroll
      for (int t = 0; t < TN; ++t) {
        const int row = wn + 32 * t + c;
        w[t] = lw[row * kChunks + ((2 * s + h) ^ (row & 7))];
      }
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(x[i], w[j], acc[i][j], 0, 0, 0);
    }
    __syncthreads();
  }
  T* y = static_cast<T*>(a.y);
#pragma unroll
  for (int j = 0; j < TN; ++j) {
    const int n = n0 + wn + 32 * j + c;
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
          y[m * a.N + n] = from_f32<T>(static_cast<float>(acc[i][j][e]) * xs * ws + bias);
        }
      }
  }
}

}  // namespace

hipError_t launch_q8gemm(const Q8Args& a, hipStream_t s) {
  auto on16 = [](const void* p, int64_t stride) {
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride % 16 == 0;
  };
  const Q8Form form = q8_form(a.M, a.N, a.K, on16(a.x, a.x_stride) && on16(a.w, a.w_stride));
  if (form == kQ8Skinny) return launch_q8_skinny(a, s);
  if (form != kQ8Any) return launch_q8_tile(a, form, s);
  constexpr int TM = 2, TN = 2;
  const int64_t cols = (a.N + 64 * TN - 1) / (64 * TN), rows = (a.M + 64 * TM - 1) / (64 * TM);
  const unsigned grid = static_cast<unsigned>(rows * cols);  // M * N <= 2^35: below 2^23 + 2^18
  with_real_type(a.dtype, [&](auto t) {
    using T = decltype(t);
    q8_any_kernel<T, TM, TN><<<grid, kNT, size_t{64} * (TM + TN) * kBK, s>>>(a);
  });
  return hipGetLastError();
}

}  // namespace bnn
