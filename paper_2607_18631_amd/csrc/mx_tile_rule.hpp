// Tile rules of the block-scaled grouped product (mx_gemm.hip): which tile, and which slices of K, a call runs on.  Plain
// host code, so that a test can evaluate them without a GPU.
#pragma once
#include <stdint.h>

namespace moe {

// Rows x weight rows of a tile, by the rows that a group has in the mean (the loads themselves stay on the device):
//   256 x 256  where groups have more than 64 rows and the tiles fill the chip.  The weights are read once for a group's
//              130 rows: 8192 rows on 64 experts of 2048 x 1408 in e2m1 120 us a call against 149 with 128 rows.
//   128 x 128  where such tiles fit on the chip at once: a tile waits for its slices' latency, so more compute units
//              asking is more memory at work.  501 rows on 8 experts of 2048 x 1408 in e4m3 26 us against 32 with
//              128 x 256; but 2048 rows on 4 of 2048 x 1024, which take a second round, 45 against 35.
//   128 x 256  elsewhere: that case 35 us against 51 with 256 rows; 512 rows on 32 experts of 7168 x 2048 in e2m1 153
//              against 168, as a low tile of 64 rows has more slices on their way.
// (Slower everywhere: 32 and 64 rows with 4 waves, which have nobody on their SIMD to multiply while they read.)
enum class MxTileId { k128x128, k128x256, k256x256 };

inline MxTileId mx_tile_rule(int64_t cus, int64_t max_rows, int64_t groups, int64_t weight_rows) {
  const int64_t per_group = max_rows / groups;
  // (a group ends half a tile early in the mean)
  const int64_t narrow = groups * ((per_group + 64 + 127) / 128) * ((weight_rows + 127) / 128);
  const int64_t large = groups * ((per_group + 255) / 256) * ((weight_rows + 255) / 256);
  if (narrow <= cus) return MxTileId::k128x128;
  return per_group > 64 && large >= cus ? MxTileId::k256x256 : MxTileId::k128x256;
}

// Whole slices: no slice has a row's end inside, and a row has the scales of a group (512 values).  Slices of 256 values
// where the token rows are e2m1 and tiles have 256 weight rows: rows of 128 bytes are one cache line each, rows of 64 cost
// as many accesses for half the bytes (2048 rows on 8 experts of 4096 x 14336: 395 us a call against 444; 8192 rows: 841
// against 874).  e4m3 rows have 128 bytes in slices of 128, and LDS has no room for two such stages of 256 rows.
enum class MxSlices { kRagged, kWhole128, kWhole256 };

inline MxSlices mx_slices(bool e2m1_rows, int tile_weight_rows, int64_t K) {
  if (K % 128 != 0 || K < 512) return MxSlices::kRagged;
  return e2m1_rows && tile_weight_rows == 256 && K % 256 == 0 ? MxSlices::kWhole256 : MxSlices::kWhole128;
}

}  // namespace moe
