// How work is cut into grids: arithmetic of the host alone, without CUDA.
#pragma once

#include <stdint.h>

#include <algorithm>

namespace rtopk {
namespace mat {

// Quotients of numbers below 2^31 by d: (k m / 2^32) / 2^shift with m = floor(2^(32 + shift) / d) + 1, 2^shift < d <= 2^(shift + 1); m is
// off by less than 1, which k times 2^-(32 + shift) keeps below 1 / d.
struct Divisor { uint32_t m, d; int shift; };
inline Divisor divisor(uint32_t d) {
  Divisor v = {0, d, 0};
  while (d > uint64_t(2) << v.shift) ++v.shift;
  v.m = (uint32_t)((uint64_t(1) << (32 + v.shift)) / d + 1);
  return v;
}

// Dropout takes four rows at a time, a quad, in `units` pieces along the columns, `per` of them a block.  31 bits count a band's pieces and those
// that its last block has no work for, so a band is of so many quads, along the grid's second side; one at least, since units
// <= 2^27 (2^30 columns by eight).
struct DropoutGrid {
  int64_t band, bands, blocks;      // rows of a band (a multiple of four), bands, blocks of each
  DropoutGrid(int64_t rows, int64_t units, int64_t per) {
    const int64_t most = std::max<int64_t>(1, ((int64_t(1) << 31) - 256) / units), quads = std::min((rows + 3) / 4, most);
    band = 4 * quads;
    bands = (rows + band - 1) / band;
    blocks = (quads * units + per - 1) / per;
  }
};

// Products whose contraction is cut: each tile has counters, each part room for its sums at the scratch's start.
constexpr int kSplitTiles = 1024;                      // tiles of a split product
constexpr int64_t kPartBytes = 128 * 256 * 4;          // the largest part of one block
constexpr int kPartBlocks = 160;                       // blocks with such a part, at most
constexpr int64_t kPartsBytes = kPartBlocks * kPartBytes;
inline bool parts_fit(int64_t tiles, int64_t split, int64_t tile_bytes) { return split == 1 || (tiles <= kSplitTiles && split <= kPartsBytes / tile_bytes / tiles); }

}  // namespace mat
}  // namespace rtopk
