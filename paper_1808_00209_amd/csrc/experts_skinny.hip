// Binary FC layers of experts for few rows per expert: a 32 x 32 tile of
// fp4_skinny.hpp per row tile of an expert and 32 outputs.  The time is that of
// reading the weights and of one tile's chain of loads: offsets, order, rows.
// One row x 8 of 64 experts, 1024 -> 4096: 5.7 us (4 MB of weights); 1 of 4,
// 4096 -> 4096: 4.6 us, in the larger tiles 10.6.
#include "experts.hpp"
#include "fp4_skinny.hpp"
#include "group_tiles.hpp"
#include "lane_ops.hpp"

namespace bnn {
namespace {

struct EsArgs {
  const uint32_t* x;
  const uint32_t* w;
  const int32_t* offsets;
  const int32_t* order;
  const int32_t* thr;
  const uint32_t* flip;
  uint32_t* bits;
  uint16_t* counts;
  uint32_t x_bytes, w_bytes;  // of x; of one expert's weights
  uint32_t tmask;
  int32_t M, E, N, Nw, Kw, K, share, chunks;
};

template <int NW, bool COUNTS>
__global__ __launch_bounds__(64 * NW) void experts_skinny_kernel(EsArgs a) {
  __shared__ __attribute__((aligned(16))) float part[(NW - 1) * 64 * kSkinnyStride];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int h = lane >> 5, c = lane & 31;
  const GroupTile gt = group_tile(a.offsets, a.E, a.M, !COUNTS, 5, static_cast<uint32_t>(a.Nw),
                                  blockIdx.x);
  if (gt.group < 0) return;
  const int rows = min(gt.end - gt.begin, 32);
  const int pair = static_cast<int>(min(static_cast<uint32_t>(a.order[gt.begin + min(c, rows - 1)]),
                                        static_cast<uint32_t>(a.M - 1)));
  const int wi = static_cast<int>(gt.col), n0 = 32 * wi;
  if (!COUNTS && gt.group == a.E) {  // pairs without an expert: bits 0
    if (wave == 0 && h == 0 && c < rows) a.bits[static_cast<size_t>(pair) * a.Nw + wi] = 0;
    return;
  }
  SkinnyTile t;
  t.ra = tile_rsrc(a.x, a.x_bytes);
  t.rb = tile_rsrc(a.w + static_cast<size_t>(gt.group) * a.N * a.Kw, a.w_bytes);
  t.aoff = static_cast<uint32_t>(pair / a.share) * a.Kw * 4 + 16 * h;
  t.boff = static_cast<uint32_t>(n0 + c) * a.Kw * 4 + 16 * h;
  t.K = a.K;
  t.Kw = a.Kw;
  t.chunks = a.chunks;
  t.tmask = a.tmask;
  float thv[16] = {};
  uint32_t fl = 0;
  if constexpr (!COUNTS) {
    if (wave == 0) {
      const __amdgpu_buffer_rsrc_t rthr =
          tile_rsrc(a.thr + static_cast<size_t>(gt.group) * a.N, a.N * 4);
#pragma unroll
      for (int e = 0; e < 16; e += 4) {
        const v4i v = tile_load4(rthr, (n0 + 2 * e + 4 * h) * 4, 0);
        // Clamped to [-K-1, K+1], which keeps the comparison (|S| <= K).
#pragma unroll
        for (int i = 0; i < 4; ++i)
          thv[e + i] = 0.5f - static_cast<float>(min(max(v[i], -a.K - 1), a.K + 1));
      }
      if (a.flip) fl = a.flip[static_cast<size_t>(gt.group) * a.Nw + wi];
    }
  }
  v16f acc = skinny_part<NW>(t, wave, h);
  skinny_join<NW>(acc, part, wave, lane);
  if (wave > 0) return;
  if constexpr (COUNTS) {
    if (c >= rows) return;
    // Register e holds output 8 (e / 4) + 4 h + e % 4 of row c.
    const float half = 0.5f * static_cast<float>(a.K);
    const int ns = counts_stride(a.N);
    uint16_t* dst = a.counts + static_cast<size_t>(pair) * ns + n0;
#pragma unroll
    for (int e = 0; e < 16; e += 4) {
      const int n = 2 * e + 4 * h;
      uint32_t v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = static_cast<uint32_t>(0.5f * acc[e + i] + half);
      if (n0 + n < ns)
        *reinterpret_cast<uint2*>(dst + n) = uint2{v[0] | v[1] << 16, v[2] | v[3] << 16};
    }
  } else {
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[e] += thv[e];
    // output bit = (S >= thr) xor flip = sign xor ~flip
    const uint32_t word = (or_xor32(sign_word(acc, h)) ^ ~fl) &
                          (wi == a.Nw - 1 ? tail_mask(a.N) : ~0u);
    if (h == 0 && c < rows) a.bits[static_cast<size_t>(pair) * a.Nw + wi] = word;
  }
}

}  // namespace

hipError_t launch_experts_skinny(const ExpertsArgs& a, uint16_t* counts, hipStream_t s) {
  EsArgs e;
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
  e.share = a.share;
  e.chunks = (e.Kw + 7) / 8;
  e.tmask = tail_mask(a.K);
  e.x_bytes = static_cast<uint32_t>(static_cast<int64_t>(a.M / a.share) * e.Kw * 4);
  e.w_bytes = static_cast<uint32_t>(static_cast<int64_t>(a.N) * e.Kw * 4);
  const int64_t tiles = group_tiles_bound(a.M, a.E + 1, 32) * e.Nw;
  const unsigned grid = static_cast<unsigned>((tiles + 7) / 8 * 8);
  auto launch = [&](auto n) {
    constexpr int NW = decltype(n)::value;
    if (counts)
      experts_skinny_kernel<NW, true><<<grid, 64 * NW, 0, s>>>(e);
    else
      experts_skinny_kernel<NW, false><<<grid, 64 * NW, 0, s>>>(e);
  };
  switch (skinny_waves(e.chunks)) {
    case 8: launch(std::integral_constant<int, 8>{}); break;
    case 4: launch(std::integral_constant<int, 4>{}); break;
    default: launch(std::integral_constant<int, 2>{}); break;
  }
  return hipGetLastError();
}

}  // namespace bnn
