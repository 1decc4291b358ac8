// The shape of the fp4_tile.hpp tiles that the experts' and adapters' kernels
// cut their work into.  A pure function of the sizes, on the host.
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

}  // namespace bnn
