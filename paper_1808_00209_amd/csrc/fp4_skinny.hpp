// One 32 x 32 output tile of a binary GEMM on the fp4 matrix cores with K
// split over the NW waves of a workgroup, for few rows: the weights are read
// once, straight into registers, all of a wave's loads in flight, and the
// waves' parts meet in LDS (exact: whole numbers below 2^24).
#pragma once

#include "fp4_expand.hpp"
#include "fp4_tile.hpp"

namespace bnn {

constexpr int kSkinnyStride = 20;  // LDS floats per lane of a part (16-byte aligned)

// What a wave needs: lane half h of lane (h, c) takes words 4 h .. 4 h + 3 of
// every chunk of 8 words of data row c and weight row c.
struct SkinnyTile {
  __amdgpu_buffer_rsrc_t ra, rb;  // data rows and weight rows
  uint32_t aoff, boff;            // byte offsets of this lane's rows, + 16 h
  int32_t K, Kw, chunks;
  uint32_t tmask;                 // valid bits of word Kw - 1
};

// The wave's part of the tile: chunks wave, wave + NW, ...
template <int NW>
__device__ __forceinline__ v16f skinny_part(const SkinnyTile& t, int wave, int h) {
  constexpr int kRing = 4;  // chunks in flight
  const uint32_t smask = __builtin_amdgcn_readfirstlane(0x88888888u);
  uint32_t vfill;
  asm("v_mov_b32 %0, 0x22222222" : "=v"(vfill));
  v16f acc = {};
  for (int c0 = wave; c0 < t.chunks; c0 += NW * kRing) {
    v4i x[kRing], w[kRing];
#pragma unroll
    for (int r = 0; r < kRing; ++r) {
      const uint32_t at = static_cast<uint32_t>(min(c0 + r * NW, t.chunks - 1)) * 32;
      x[r] = tile_load4(t.ra, t.aoff, at);
      w[r] = tile_load4(t.rb, t.boff, at);
    }
#pragma unroll
    for (int r = 0; r < kRing; ++r) {
      const int ch = c0 + r * NW;
      if (ch >= t.chunks) break;
      v8i A[4], B[4];
#pragma unroll
      for (int s = 0; s < 4; s += 2) {
        expand_pair(static_cast<uint32_t>(w[r][s]), static_cast<uint32_t>(w[r][s + 1]), smask,
                    vfill, A[s], A[s + 1]);
        expand_pair(static_cast<uint32_t>(x[r][s]), static_cast<uint32_t>(x[r][s + 1]), smask,
                    vfill, B[s], B[s + 1]);
      }
      if (8 * ch + 8 > t.Kw - 1) {  // words and bits past K: fp4 0.0 in the data operand
#pragma unroll
        for (int s = 0; s < 4; ++s) {
          const int wi = 8 * ch + 4 * h + s;
          const uint32_t vm = wi < t.Kw - 1 ? ~0u : (wi == t.Kw - 1 ? t.tmask : 0u);
          const v8i keep = expand_fp4(vm, smask, 0u);  // sign bit of every kept nibble
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t k = static_cast<uint32_t>(keep[i]);
            B[s][i] &= static_cast<int>(k | (k >> 2));
          }
        }
      }
#pragma unroll
      for (int s = 0; s < 4; ++s)
        acc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(A[s], B[s], acc, 4, 4, 0, 127, 0,
                                                              127);
    }
  }
  return acc;
}

// Leaves the sum of all waves' parts with wave 0 (the others' are unspecified).
// `part`: NW - 1 regions of 64 kSkinnyStride floats.
template <int NW>
__device__ __forceinline__ void skinny_join(v16f& acc, float* part, int wave, int lane) {
  float* mine = part + ((wave - 1) * 64 + lane) * kSkinnyStride;
  if (wave > 0) {
#pragma unroll
    for (int e = 0; e < 16; e += 4)
      *reinterpret_cast<float4*>(mine + e) =
          float4{acc[e], acc[e + 1], acc[e + 2], acc[e + 3]};
  }
  __syncthreads();
  if (wave == 0) {
#pragma unroll
    for (int w = 0; w < NW - 1; ++w)
#pragma unroll
      for (int e = 0; e < 16; e += 4) {
        const float4 v =
            *reinterpret_cast<const float4*>(part + (w * 64 + lane) * kSkinnyStride + e);
        acc[e] += v.x;
        acc[e + 1] += v.y;
        acc[e + 2] += v.z;
        acc[e + 3] += v.w;
      }
  }
}

// Waves of a workgroup: one per chunk up to 8.
inline int skinny_waves(int32_t chunks) { return chunks > 4 ? 8 : chunks > 2 ? 4 : 2; }

}  // namespace bnn
