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

// Whether an operand's rows start on 16-byte steps.  (One row has no next one:
// its distance says nothing.)
inline bool q8_on16(uintptr_t address, int64_t stride, int64_t rows) {
  return address % 16 == 0 && (rows == 1 || stride % 16 == 0);
}

// on16: x's and w's rows on 16-byte steps.
//
// Many rows: the tile whose estimated time is least, in tenths of us at K = 4096,
// from products of 256..8192 rows.  Tiles of 64 take 3 + 7 per 256 of them (256:
// 10.1, 640: 21.6, 1128: 34.9); up to 256 tiles of 128 15 + 8 (160: 19.4, 256:
// 22.9); two per CU and more of these 28 + 10 (280: 29.6, 420: 36), then 38 per
// round of 512; tiles of 256 58 per round (up to half a round 46, the clock being
// higher).  Other K move all of them alike, but small ones favour fewer tiles
// (1500 x 3000, K 700: 64 13.6, two of 128 per CU 10.6 us; K 4096: 32.3, 27.1).  Of
// 46 products with K of 400 to 28672 two are off the best tile (64 x 20000, K 8000
// 1.16, 1500 x 1500, K 512 1.11), the others within 1.01.
//
// Few rows (us, skinny : tiles of 64, K 4096): 16 rows of 4096 outputs 8.0 : 8.7
// and of 65536 58.0 : 59.4; 32 rows, in two operands of the skinny kernel, 10.6 :
// 8.9 and 19.7 : 13.6 (16384 outputs): there a workgroup's waves share the rows.
// x stays in the skinny kernel's registers up to K 8192.
inline Q8Form q8_form(int64_t M, int64_t N, int64_t K, bool on16) {
  if (K >= 16 && K <= 8192 && M <= 16) return kQ8Skinny;
  if (K < 16 || !on16) return kQ8Any;
  const int64_t t64 = q8_tiles(M, N, 64), t128 = q8_tiles(M, N, 128), t256 = q8_tiles(M, N, 256);
  const int64_t in64 = 30 + 70 * t64 / 256;
  const int64_t in128 = t128 <= 256   ? 150 + 80 * t128 / 256
                        : t128 <= 512 ? 280 + 100 * (t128 - 256) / 256
                                      : (t128 + 511) / 512 * 380;
  const int64_t in256 = t256 <= 128 ? 460 : (t256 + 255) / 256 * 580;
  if (in64 <= in128 && in64 <= in256) return kQ8Tile64;
  if (in128 <= in256) return t128 <= 256 ? kQ8Tile128 : kQ8Pair128;
  return kQ8Tile256;
}

// kQ8Any's tiles: 128 x 128, or 64 x 64 where those leave CUs without one.
inline int q8_any_tile(int64_t M, int64_t N) { return q8_tiles(M, N, 128) >= 256 ? 128 : 64; }

}  // namespace bnn
