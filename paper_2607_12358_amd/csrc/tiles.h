// Order of a matrix product's output tiles over the device's XCDs.
#pragma once

#include "common.h"

namespace acid {

// Bijection from dispatch order to tile order giving XCD x (workgroups
// bid = x, x+8, ...) the contiguous tile range of its share.  Tile numbers
// are below 2^29 (the entry bounds the 256 x 256 tiles by 2^23) and divided in 32
// bits: the 64-bit divisions of a tile's coordinates were a chain that every
// workgroup waited for before its first load.
__device__ __forceinline__ uint32_t xcd_remap(uint32_t bid, uint32_t T) {
  constexpr uint32_t NX = 8;
  const uint32_t x = bid % NX, local = bid / NX;
  const uint32_t q = T / NX, r = T % NX;
  return (x < r) ? x * (q + 1) + local : r * (q + 1) + (x - r) * q + local;
}

// Tile t -> (tm, tn) in groups of GM token tiles, feature tiles inner.
// The 32 tiles an XCD runs at once then share few activation row blocks
// (streamed once from HBM) and many weight column blocks (re-read by every
// row block, so they come from the on-package cache): groups of 2 measured
// 3-6% faster than 8 on the model shapes here (4 and 3 within noise of 2).
template <uint32_t GM = 2>
__device__ __forceinline__ void tile_coords(uint32_t t, int64_t tiles_m, int tiles_n, int64_t& tm,
                                            int& tn) {
  const uint32_t per_group = GM * (uint32_t)tiles_n;
  const uint32_t g = t / per_group;
  const uint32_t first = g * GM;
  const uint32_t gsize = min(GM, (uint32_t)tiles_m - first);
  const uint32_t w = t - g * per_group;
  const uint32_t col = w / gsize;
  tm = first + (w - col * gsize);
  tn = (int)col;
}

}  // namespace acid
