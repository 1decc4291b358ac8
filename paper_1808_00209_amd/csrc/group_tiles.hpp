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

// The tile of block `block` (of a grid that is a multiple of 8): every group's
// rows are cut into tiles of 1 << rlog positions, each with `cols` column
// tiles, column tiles fastest; with `rest`, the rows of no group come as tiles
// of group G after the others.  Block b runs on XCD b mod 8, and an XCD takes
// consecutive tiles, so that its L2 serves a row tile's rows and a group's
// weights to several of them.  Wave-uniform; every lane of a wave has to call
// it.  Offsets out of range are clamped.
__device__ __forceinline__ GroupTile group_tile(const int32_t* __restrict__ offsets, int G, int M,
                                                bool rest, int rlog, uint32_t cols,
                                                uint32_t block) {
  const int lane = threadIdx.x & 63;
  const int round = (1 << rlog) - 1;
  // 64 groups at a time, one per lane: first position, end and tiles.
  int b = 0, e = 0, mine = 0, scan = 0;
  auto batch = [&](int g0) {
    const int g = g0 + lane;
    b = offsets[min(g, G)];
    e = offsets[min(g + 1, G)];
    b = min(max(b, 0), M);
    e = min(max(e, b), M);
    mine = (e - b + round) >> rlog;  // (0 from group G on)
    scan = wave_scan(mine);
  };
  int total = 0, g0 = 0;
  for (;;) {
    batch(g0);
    total += __builtin_amdgcn_readlane(scan, 63);
    if (g0 + 64 >= G) break;
    g0 += 64;
  }
  const int done = __builtin_amdgcn_readlane(e, (G - 1) & 63);  // rows of all groups
  const int tail = rest ? (M - done + round) >> rlog : 0;
  const uint32_t all = static_cast<uint32_t>(total + tail) * cols;
  const uint32_t per = (all + 7) / 8;
  const uint32_t slot = block >> 3;
  const uint32_t t = (block & 7) * per + slot;
  GroupTile r = {-1, 0, 0, 0};
  if (slot >= per || t >= all) return r;
  int row = static_cast<int>(t / cols);
  r.col = t - static_cast<uint32_t>(row) * cols;
  if (row >= total) {
    r.group = G;
    r.begin = done + ((row - total) << rlog);
    r.end = M;
    return r;
  }
  if (g0 > 0) {  // (several batches: the last one is held)
    g0 = 0;
    batch(0);
  }
  for (;;) {
    const uint64_t hit = __ballot(scan > row);
    if (hit) {
      const int l = __builtin_ctzll(hit);
      r.group = g0 + l;
      r.begin = __builtin_amdgcn_readlane(b, l) +
                ((row - __builtin_amdgcn_readlane(scan - mine, l)) << rlog);
      r.end = __builtin_amdgcn_readlane(e, l);
      return r;
    }
    row -= __builtin_amdgcn_readlane(scan, 63);
    g0 += 64;
    if (g0 >= G) return r;  // (not reached: row < total)
    batch(g0);
  }
}

// Row tiles that M rows in G groups can come to, at most.
inline int64_t group_tiles_bound(int64_t M, int64_t groups, int64_t R) {
  return M / R + (groups < M ? groups : M);
}

}  // namespace bnn
