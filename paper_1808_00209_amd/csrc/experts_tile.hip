// Binary FC layers of experts on the fp4 matrix cores (bnn_experts_fc, and the
// products of bnn_experts_sum): one GEMM tile of fp4_tile.hpp per row tile of
// an expert and 64, 128 or 256 outputs, the rows gathered through the order.
//
// 65536 pairs of 64 experts, 1024 -> 4096 to bits: 125-137 us from card to card,
// 4.1e15 operations a second; 4096 -> 1024 to counts 113-122 us (the FC kernel
// without experts reaches 5.5e15 at the clock that load allows).  The difference
// is row tiles that experts do not fill and each block's start and end, at 1024
// bits as long as its four chunks: there the matrix cores are busy in 47 % of
// the cycles, and 6.3 vector instructions issue per MFMA.  One launch bound for
// all: the grid holds the most tiles that there can be, blocks past the last one
// end at once.
#include "expert_plans.hpp"
#include "experts.hpp"
#include "fp4_tile.hpp"
#include "group_tiles.hpp"

namespace bnn {
namespace {

constexpr int kCountStride = 72;  // LDS halfwords per row of a counts tile (144 bytes)

struct EtArgs {
  const uint32_t* x;
  const uint32_t* w;
  const int32_t* offsets;
  const int32_t* order;
  const int32_t* thr;
  const uint32_t* flip;
  uint32_t* bits;
  uint16_t* counts;
  uint32_t x_bytes, w_bytes;  // of x; of one expert's weights
  uint32_t cols;
  int32_t M, E, N, Nw, Kw, K, share;
  int32_t chunks;             // of 8 words
  uint32_t tmask;             // valid bits of word Kw - 1
  int32_t wfl;                // log2 of the waves along the outputs
  int32_t rlog;               // log2 of the rows per tile
};

// PT: 32-row tiles per wave.  COUNTS: (S + K) / 2, the number of equal bits,
// as 16-bit words of row m; else bits.
template <int PT, bool COUNTS>
__global__ __launch_bounds__(kTileNT, 2) void experts_tile_kernel(EtArgs a) {
  extern __shared__ v4i act[];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int h = lane >> 5, c = lane & 31;
  const GroupTile gt = group_tile(a.offsets, a.E, a.M, !COUNTS, a.rlog, a.cols, blockIdx.x);
  if (gt.group < 0) return;
  const int rows = min(gt.end - gt.begin, 1 << a.rlog);
  auto pair_at = [&](int i) {  // the pair at row i of the tile (rows past it: the last one)
    return static_cast<int>(min(static_cast<uint32_t>(a.order[gt.begin + min(i, rows - 1)]),
                                static_cast<uint32_t>(a.M - 1)));
  };
  if (!COUNTS && gt.group == a.E) {  // pairs without an expert: bits 0
    const int w0 = static_cast<int>(gt.col) << (1 + a.wfl);
    const int nw = min(a.Nw - w0, 2 << a.wfl);
    for (int i = tid; i < rows * nw; i += kTileNT)
      a.bits[static_cast<size_t>(pair_at(i / nw)) * a.Nw + w0 + i % nw] = 0;
    return;
  }
  const int wfi = wave & ((1 << a.wfl) - 1);
  const int f0 = (static_cast<int>(gt.col) << (6 + a.wfl)) + wfi * 64;  // wave's first output
  const int wi = f0 / 32 + h;  // this lane half's output word

  TileLoop t;
  t.ra = tile_rsrc(a.x, a.x_bytes);
  t.rb = tile_rsrc(a.w + static_cast<size_t>(gt.group) * a.N * a.Kw, a.w_bytes);
#pragma unroll
  for (int tf = 0; tf < 2; ++tf)
    t.woff[tf] = (static_cast<uint32_t>(f0 + 32 * tf + c) * a.Kw + 4 * h) * 4;
  t.K = a.K;
  t.Kw = a.Kw;
  t.chunks = a.chunks;
  t.tmask = a.tmask;
  t.wpi = wave >> a.wfl;
  int32_t thv[2] = {0, 0};
  uint32_t fl = 0;
  if constexpr (!COUNTS) {
    const __amdgpu_buffer_rsrc_t rthr =
        tile_rsrc(a.thr + static_cast<size_t>(gt.group) * a.N, a.N * 4);
    const __amdgpu_buffer_rsrc_t rflip = tile_rsrc(
        a.flip + (a.flip ? static_cast<size_t>(gt.group) * a.Nw : 0), a.flip ? a.Nw * 4 : 0);
#pragma unroll
    for (int tf = 0; tf < 2; ++tf)
      thv[tf] = static_cast<int32_t>(
          __builtin_amdgcn_raw_buffer_load_b32(rthr, (f0 + 32 * tf + c) * 4, 0, 0));
    fl = __builtin_amdgcn_raw_buffer_load_b32(rflip, wi * 4, 0, 0);
  }

  // Bits: S + 0.5 - thr, thresholds clamped to [-K-1, K+1], which keeps the
  // comparison (|S| <= K).  Counts: S + K.
  v16f acc[2][PT];
#pragma unroll
  for (int tf = 0; tf < 2; ++tf) {
    const float from = COUNTS ? static_cast<float>(a.K)
                              : 0.5f - static_cast<float>(min(max(thv[tf], -a.K - 1), a.K + 1));
    tile_start<PT>(acc[tf], h == 0 ? from : 0.0f);
  }
  tile_loop<PT>(acc, act, t, [&] {
    return (static_cast<uint32_t>(pair_at(tid >> 1) / a.share) * a.Kw + 4 * (tid & 1)) * 4;
  });
  int pair[PT];  // (read here: kept through the loop they cost registers that it spills)
#pragma unroll
  for (int pt = 0; pt < PT; ++pt) pair[pt] = pair_at((t.wpi * PT + pt) * 32 + c);

  if constexpr (COUNTS) {
    // 32 rows x 64 outputs at a time through LDS (a region per wave), so that
    // a row's 64 counts are stored as one run of 128 bytes.
    uint16_t* ts = reinterpret_cast<uint16_t*>(act) + wave * (32 * kCountStride);
#pragma unroll
    for (int pt = 0; pt < PT; ++pt) {
#pragma unroll
      for (int tf = 0; tf < 2; ++tf)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          uint32_t v[4];
#pragma unroll
          for (int r = 0; r < 4; ++r)
            v[r] = static_cast<uint32_t>(0.5f * acc[tf][pt][4 * g + r]);
          *reinterpret_cast<uint2*>(&ts[c * kCountStride + 32 * tf + 8 * g + 4 * h]) =
              uint2{v[0] | v[1] << 16, v[2] | v[3] << 16};
        }
      const int f = f0 + 8 * (lane & 7);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int row = 8 * q + (lane >> 3);
        const int m = __shfl(pair[pt], row);
        const uint4 v = *reinterpret_cast<const uint4*>(&ts[row * kCountStride + 8 * (lane & 7)]);
        if ((t.wpi * PT + pt) * 32 + row < rows) {
          const int ns = counts_stride(a.N);
          if (f < ns)
            *reinterpret_cast<uint4*>(a.counts + static_cast<size_t>(m) * ns + f) = v;
        }
      }
    }
  } else {
    const uint32_t fm = wi == a.Nw - 1 ? tail_mask(a.N) : ~0u;
#pragma unroll
    for (int pt = 0; pt < PT; ++pt) {
      // one v_permlane32_swap of the two output tiles' words leaves lane half
      // h with the whole word of tile h; output bit = sign xor ~flip
      const auto sw = __builtin_amdgcn_permlane32_swap(sign_word(acc[0][pt], h),
                                                       sign_word(acc[1][pt], h), false, false);
      if ((t.wpi * PT + pt) * 32 + c < rows && wi < a.Nw)
        a.bits[static_cast<size_t>(pair[pt]) * a.Nw + wi] = ((sw[0] | sw[1]) ^ ~fl) & fm;
    }
  }
}

}  // namespace

bool experts_tile_supported(const ExpertsArgs& a) {
  const int64_t kw = words_of(a.K);
  return a.M / a.share * kw * 4 < (int64_t{1} << 32) - 64;
}

hipError_t launch_experts_tile(const ExpertsArgs& a, uint16_t* counts, hipStream_t s) {
  EtArgs e;
  e.x = a.x;
  e.w = a.w;
  e.offsets = a.offsets;
  e.order = a.order;
  e.thr = a.thr;
  e.flip = a.flip;
  e.bits = a.bits;
  e.counts = counts;
  e.M = a.M;
  e.E = a.E;
  e.N = a.N;
  e.Nw = static_cast<int32_t>(words_of(a.N));
  e.K = a.K;
  e.Kw = static_cast<int32_t>(words_of(a.K));
  e.chunks = (e.Kw + 7) / 8;
  e.tmask = tail_mask(a.K);
  e.share = a.share;
  e.x_bytes = static_cast<uint32_t>(static_cast<int64_t>(a.M / a.share) * e.Kw * 4);
  e.w_bytes = static_cast<uint32_t>(static_cast<int64_t>(a.N) * e.Kw * 4);
  const TileShape shape = experts_shape(a.M, a.E, a.N, e.chunks);
  e.wfl = shape.wfl;
  const int rows = shape.rows();
  e.rlog = rows == 128 ? 7 : rows == 64 ? 6 : 5;
  e.cols = static_cast<uint32_t>((a.N + shape.outputs() - 1) / shape.outputs());
  const int64_t tiles = group_tiles_bound(a.M, a.E + 1, rows) * e.cols;
  const unsigned grid = static_cast<unsigned>((tiles + 7) / 8 * 8);
  static_assert(kTileLds >= size_t{4} * 32 * kCountStride * 2, "the counts tiles fit");
  auto launch = [&](auto p) {
    constexpr int PT = decltype(p)::value;
    if (counts)
      experts_tile_kernel<PT, true><<<grid, kTileNT, kTileLds, s>>>(e);
    else
      experts_tile_kernel<PT, false><<<grid, kTileNT, kTileLds, s>>>(e);
  };
  switch (shape.pt) {
    case 4: launch(std::integral_constant<int, 4>{}); break;
    case 2: launch(std::integral_constant<int, 2>{}); break;
    default: launch(std::integral_constant<int, 1>{}); break;
  }
  return hipGetLastError();
}

}  // namespace bnn
