// Which kernels the experts' and adapters' calls take and how these cut their
// work.  Pure functions of the sizes, on the host, so that a choice can be
// looked at without a GPU.
#pragma once

#include <stdint.h>

#include "tile_plans.hpp"

namespace bnn {

// log2 of the waves along the outputs (64 each; the others lie along the rows)
// and 32-row tiles per wave.
struct TileShape {
  int wfl, pt;
  int rows() const { return (4 >> wfl) * pt * 32; }
  int outputs() const { return 64 << wfl; }
};

// The shape with the least estimated time, as fc_tile_plan (tile_plans.hpp)
// estimates it: rounds of two blocks per compute unit, each its chunks' MFMAs
// (8 PT per chunk and wave, at about 38 / 44 / 60 cycles for PT = 4 / 2 / 1; at
// least the latency of a chunk), plus `fixed` cycles of start and end and
// `tail` for every 32-row tile of a wave.  row_tiles(R): how many tiles of R
// rows there are.
template <class F>
TileShape tile_shape(int64_t N, int64_t chunks, double fixed, double tail, F row_tiles) {
  TileShape best = {0, 1};
  double least = -1;
  for (int wfl = 0; wfl <= 2; ++wfl)
    for (int pt = 4; pt >= 1; pt /= 2) {
      const TileShape s = {wfl, pt};
      if (s.rows() > 128) continue;
      const double tiles =
          static_cast<double>((N + s.outputs() - 1) / s.outputs()) * row_tiles(s.rows());
      const double one = 8 * pt * (pt == 4 ? 38 : pt == 2 ? 44 : 60);
      const double both = (tiles <= kCUs ? 1.25 : 1.9) * one;
      const double per = both > 1000 ? both : 1000.0;
      const double slots = 2.0 * kCUs;
      const double rounds = tiles <= slots ? 1.0 : tiles / slots;
      const double cost = rounds * (chunks * per + fixed + tail * pt);
      if (least < 0 || cost < least) {
        least = cost;
        best = s;
      }
    }
  return best;
}

// ---------------------------------------------------------------- experts ---

// bnn_experts_sum for few rows: every row reads its experts' weights by itself,
// up to 32 MiB of them in all (experts_sum_rows.hip, one launch; against
// products and combining pass, 4096 -> 1024, rows x 8 of 64 experts: 4 rows 6.3
// and 13.4 us, 8 8.4 and 14.6, 16 14.2 and 18.2, 32 27.2 and 18.3; 8 of 8: 8
// rows 8.4 and 9.2, 16 14.4 and 9.4; 2 of 8: 32 rows 7.8 and 8.5, 64 12.2 and
// 10.3; 1 of 2: 64 rows 7.4 and 8.4).  It does not look at the number of
// experts: between the limit and twice it, the form taken loses 4 us with many,
// and up to the limit 5 with few and short rows (8 of 8, 1024 -> 1024, 32 rows
// 13.2 and 8.2).
inline bool experts_sum_by_rows(int64_t M, int64_t N, int64_t K) {
  return M * N * ((K + 31) / 32) <= (int64_t{8} << 20);
}

// The skinny kernel (experts_skinny.hip) has a workgroup per 32 rows of an
// expert and 32 outputs and splits K over its waves: quicker while the whole
// chip takes about one round of them, several times slower at many (skinny
// against tile kernel, rows x experts per row of E, K -> N: 1 x 8 of 64, 1024 ->
// 4096: 5.7 and 6.4 us, 4 x 8: 12.1 and 8.7; 4 x 8, 4096 -> 1024: 8.3 and 10.7, 64 x
// 8: 19.2 and 11.4; 1 of 4, 4096 -> 4096: 4.6 and 10.6; 1000 x 2 of 8, 512 -> 512:
// 4.5 and 5.7; 301 x 3 of 24, 1000 -> 1500: 10.3 and 6.9).
inline bool experts_skinny(int64_t M, int64_t E, int64_t N) {
  return ((M + 31) / 32 + (E < M ? E : M)) * ((N + 31) / 32) <= 1200;
}

// Tiles of experts_tile.hip.  Row tiles: the whole ones and, for every expert
// that has rows, half a tile.
inline TileShape experts_shape(int64_t M, int64_t E, int64_t N, int64_t chunks) {
  const double some = static_cast<double>(E < M ? E : M);
  return tile_shape(N, chunks, 10000, 500, [&](int rows) {
    return static_cast<double>(M) / rows + some / 2 + (some < 2 ? 0.5 : 0.0);
  });
}

// The combining pass (experts_combine.hip) stages the alphas of all experts for
// 256 outputs in LDS (at most 64 KiB of them) where a block, two per compute
// unit, has 64 rows or more: fewer do not pay for the staging.  Rows per block,
// or 0 for the form that reads them as it goes.  Staged and not, rows x experts
// per row of E, outputs: 8192 x 8 of 64, 4096: 170 and 199 us; 3000 x 8 of 64,
// 4096: 48 and 51; 8192 x 8 of 64, 1024: 37.6 and 36.0; 8192 x 2 of 64, 1024: 22
// and 16; 32768 x 2 of 8, 512: 27 and 26.  Beyond 64 experts not, 35.6 us for
// 8192 x 8 of 128 or 256, 1024.
constexpr int kCombineCols = 256;
inline int combine_rows(int64_t T, int64_t E, int64_t N) {
  const int64_t cols = (N + kCombineCols - 1) / kCombineCols;
  const int64_t rows = (T * cols + 511) / 512;
  return E * kCombineCols * 4 <= (64 << 10) && rows >= 64 ? static_cast<int>(rows) : 0;
}

// ------------------------------------------------------------- with adapters ---

// A wave per row and rank component (lora_skinny.hip) while all of them are
// few rounds of the chip (both steps, rows and then k tiles, in us: 32 rows x
// 4096, rank 16, 28 adapters 14.2 and 38.1; 777 x 1100, rank 8 17.1 and 24.8; 512 x
// 4096, rank 16 23.5 and 26.3; 1024 x 4096, rank 16 27.4 and 24.6; 4096 x 1024,
// rank 8 28.2 and 20.7).
inline bool lora_down_by_rows(int64_t M, int64_t rank) { return M * (rank + 1) <= 16384; }

// Otherwise k slices of the down pass of lora_tile.hip (blocks of 32 rows and 8
// waves): a block per compute unit (two: 37 against 34 us for 8192 rows of
// 4096), at least one group of 128 k for every wave.
inline int lora_down_slices(int64_t M, int64_t K, int64_t rank) {
  if (M < 1 || lora_down_by_rows(M, rank)) return 1;
  const int64_t blocks = (M + 31) / 32 * ((rank + 63) / 64);
  const int64_t most = (K + 1023) / 1024;
  const int64_t want = (256 + blocks - 1) / blocks;
  return static_cast<int>(want < most ? want : most);
}

// Rows of u, over its slices, that M rows or any fewer can come to: at most
// (255 + blocks) / blocks slices of M <= 32 blocks rows, M + 255 x 32.
inline int64_t lora_u_rows(int64_t M, int64_t K, int64_t rank) {
  if (lora_down_by_rows(M, rank)) return M;
  const int64_t most = (K + 1023) / 1024 * M;
  const int64_t some = M + 255 * 32 / ((rank + 63) / 64);
  return most < some ? most : some;
}

// K split over a workgroup per 32 x 32 tile (lora_skinny.hip) while they are
// about three per compute unit (128 rows, 4096 -> 4096, many adapters 18.7 us,
// in the larger tiles 33.6; one per 16 rows, rank 64 21.8 and 25.5; 256 rows 27.1
// and 26.6).
inline bool lora_up_skinny(int64_t M, int64_t N) {
  return (M + 31) / 32 * ((N + 31) / 32) <= 800;
}

inline TileShape lora_shape(int64_t M, int64_t N, int64_t chunks) {
  return tile_shape(N, chunks, 7000, 2500, [&](int rows) {
    return static_cast<double>((M + rows - 1) / rows);
  });
}

}  // namespace bnn
