// The order in which a matrix product's workgroups take the tiles of its output.
#pragma once
#include <cstdint>

namespace ep {

constexpr int kXcds = 8, kGroupRows = 4;

// Workgroups are dealt to the XCDs round-robin: spread the ids [0, count) so
// that each XCD takes a contiguous range of `per` indices.
__device__ __forceinline__ uint32_t xcd_spread(uint32_t id, uint32_t count) {
  const uint32_t per = count / kXcds;
  return id < per * kXcds ? (id % kXcds) * per + id / kXcds : id;
}

// Tile (row, column) of tile index `idx` among tm x tn tiles, taken in groups
// of kGroupRows tile rows, column by column within a group.
__device__ __forceinline__ void tile_of(uint32_t idx, uint32_t tm, uint32_t tn, uint32_t& ti,
                                        uint32_t& tj) {
  const uint32_t group = idx / (kGroupRows * tn), first = group * kGroupRows;
  const uint32_t rows = tm - first < kGroupRows ? tm - first : kGroupRows;
  const uint32_t q = idx - first * tn;
  ti = first + q % rows;
  tj = q / rows;
}

}  // namespace ep
