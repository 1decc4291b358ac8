// Which kernel and tile an 8-bit matrix product takes (q8gemm*.hip): rules on
// its sizes and where its operands lie, as host functions.
#pragma once

#include <stdint.h>

namespace bnn {

enum Q8Form {
  kQ8Any = 0,     // operands that lie anywhere, K below 16
  kQ8Skinny = 1,  // few rows: every weight read once
  kQ8Tile64 = 2,  // tiles of 64 x 64, 128 x 128 (two forms) and 256 x 256
  kQ8Tile128 = 3,
  kQ8Pair128 = 4,  // two workgroups per CU
  kQ8Tile256 = 5
};

// Tiles of n x n of an M x N product.
inline int64_t q8_tiles(int64_t M, int64_t N, int n) { return (M + n - 1) / n * ((N + n - 1) / n); }

// on16: x, w and their strides on 16-byte steps.
//
// Many rows: the tile whose estimated time is least, in us at K = 4096, from
// products of 256..8192 rows.  Tiles of 64 take 3 + 7 per 256 of them (256: 10.1,
// 1024: 30.8), at least 8; one round of up to 256 tiles of 128 takes 23 (two
// per CU and rounds of 512: 38), one of 256 tiles of 256 58 (up to half a round
// 46, the clock being higher).  Other K move all of them alike.
//
// Few rows (us, skinny : tiles of 64, K 4096): 16 rows of 4096 outputs 8.0 : 8.7
// and of 65536 58.0 : 59.4; 32 rows, in two operands of the skinny kernel, 10.6 :
// 8.9 and 19.7 : 13.6 (16384 outputs): there a workgroup's waves share the rows.
// x stays in the skinny kernel's registers up to K 8192.
inline Q8Form q8_form(int64_t M, int64_t N, int64_t K, bool on16) {
  if (K >= 16 && K <= 8192 && M <= 16) return kQ8Skinny;
  if (K < 16 || !on16) return kQ8Any;
  const int64_t t64 = q8_tiles(M, N, 64), t128 = q8_tiles(M, N, 128), t256 = q8_tiles(M, N, 256);
  const int64_t in64 = 3 + 7 * t64 / 256;
  const int64_t in128 = t128 <= 256 ? 23 : (t128 + 511) / 512 * 38;
  const int64_t in256 = t256 <= 128 ? 46 : (t256 + 255) / 256 * 58;
  if (in64 < 8 || (in64 <= in128 && in64 <= in256)) return kQ8Tile64;
  if (in128 <= in256) return t128 <= 256 ? kQ8Tile128 : kQ8Pair128;
  return kQ8Tile256;
}

}  // namespace bnn
