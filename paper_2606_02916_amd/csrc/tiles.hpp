// Where tiles of rows by columns lie, for kernels whose neighbouring blocks share lines.
#pragma once

#include <stdint.h>

namespace gg {

// A tile's place: each of the 8 XCDs, which take blocks in turn, has a run of tiles,
// and in it bands of kBand tiles of rows, so that the blocks on one L2 at a time share
// rows and weights.
constexpr int32_t kXcds = 8, kBand = 4;

__device__ __forceinline__ uint32_t xcd_turn(uint32_t b, uint32_t total) {
  const uint32_t x = b % kXcds, q = total / kXcds, r = total % kXcds;
  return x * q + min(x, r) + b / kXcds;
}

__device__ __forceinline__ void tile_place(int32_t tiles_i, int32_t tiles_j, int32_t* ti, int32_t* tj) {
  const uint32_t t = xcd_turn(blockIdx.x, gridDim.x);
  const uint32_t width = kBand * tiles_j, band = t / width, first = band * kBand,
                 rows = min((uint32_t)tiles_i - first, (uint32_t)kBand), at = t - band * width;
  *ti = (int32_t)(first + at % rows);
  *tj = (int32_t)(at / rows);
}

}  // namespace gg
