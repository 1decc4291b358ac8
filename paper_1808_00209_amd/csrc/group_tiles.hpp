// Row tiles of rows that lie in the order of their group (bnn_group_rows):
// which group and positions a workgroup's tile covers, found in the kernel
// from the groups' offsets, since only the device knows them.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace bnn {

struct GroupTile {
  int group;     // G for a tile of the rows of no group; -1: past the last tile
  int begin;     // first position
  int end;       // one past the group's last position
  uint32_t col;  // column tile
};

// Inclusive sum over the lanes of a wave (DPP row shifts and broadcasts).
__device__ __forceinline__ int wave_scan(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false);  // row_shr:1
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false);  // row_shr:2
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false);  // row_shr:4
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false);  // row_shr:8
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);  // row_bcast:15
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);  // row_bcast:31
  return v;
}

// The tile of block `block` of `grid` (a multiple of 8): every group's rows
// are cut into tiles of R = 1 << rlog positions, each with `cols` column
// tiles, column tiles fastest; groups 0 .. last are counted (last = G - 1, or G
// to cover the rows of no group too).  Block b runs on XCD b mod 8, and an XCD
// takes consecutive tiles, so that its L2 serves a row tile's rows and a
// group's weights to several of them.  Wave-uniform; every lane of a wave has
// to call it.  Offsets out of range are clamped.
__device__ __forceinline__ GroupTile group_tile(const int32_t* __restrict__ offsets, int G, int M,
                                                int last, int rlog, uint32_t cols, uint32_t block,
                                                uint32_t grid) {
  const int lane = threadIdx.x & 63;
  auto at = [&](int g) { return g > G ? M : min(max(offsets[g], 0), M); };
  auto tiles = [&](int g) {
    return g > last ? 0 : (max(at(g + 1) - at(g), 0) + (1 << rlog) - 1) >> rlog;
  };
  // One batch of 64 groups keeps its values; more are read again below.
  int mine = tiles(lane);
  int scan = wave_scan(mine);
  int total = __builtin_amdgcn_readlane(scan, 63);
  for (int g0 = 64; g0 <= last; g0 += 64)
    total += __builtin_amdgcn_readlane(wave_scan(tiles(g0 + lane)), 63);
  const uint32_t all = static_cast<uint32_t>(total) * cols;
  const uint32_t per = (all + 7) / 8;
  const uint32_t slot = block >> 3;
  const uint32_t t = (block & 7) * per + slot;
  GroupTile r = {-1, 0, 0, 0};
  if (slot >= per || t >= all) return r;
  int row = static_cast<int>(t / cols);
  r.col = t - static_cast<uint32_t>(row) * cols;
  for (int g0 = 0;;) {
    const uint64_t hit = __ballot(scan > row);
    if (hit) {
      const int l = __builtin_ctzll(hit);
      r.group = g0 + l;
      const int before = __builtin_amdgcn_readlane(scan - mine, l);
      r.begin = __builtin_amdgcn_readfirstlane(at(r.group)) + ((row - before) << rlog);
      r.end = __builtin_amdgcn_readfirstlane(at(r.group + 1));
      return r;
    }
    row -= __builtin_amdgcn_readlane(scan, 63);
    g0 += 64;
    if (g0 > last) return r;
    mine = tiles(g0 + lane);
    scan = wave_scan(mine);
  }
}

// Row tiles that M rows in G groups can come to, at most.
inline int64_t group_tiles_bound(int64_t M, int64_t groups, int64_t R) {
  return M / R + (groups < M ? groups : M);
}

}  // namespace bnn
