// Internal: the arithmetic of 4-bit matrices that needs no GPU: their layout, and where the products' tiles are fetched from.  Plain C++
// without HIP, so that its limits can be tested without a GPU.
#ifndef FLASHOPTIM_MX4_H
#define FLASHOPTIM_MX4_H

#include <stdint.h>

#include "flashoptim_launch.h"

namespace fo {

constexpr int kBlock = 32;                  // values that share a scale
constexpr int kSegment = 256;               // a row of codes is filled up to a multiple of this many values
constexpr int kSegmentBytes = kSegment / 2;

// Quantisation along columns, or both ways: tiles of this many rows by 128 columns, over rows and columns filled up to whole segments.
// Rows of a tile, in us with 32 / 64 / 128: BF16, 1024 x 2304 4.4 / 4.8 / 6.1, 8192 x 4096 25.2 / 24.2 / 26.2, 14336 x 4096 38.7 / 36.5 / 38.4,
// stochastic 68 / 61 / 68; split weights, 1001 x 768 4.0 / 4.8 / 6.9, 14336 x 4096 45.2 / 45.4 / 56.4.
constexpr int kTileCols = 128, kTileLanes = 256;
constexpr int quantize_tile_rows(int64_t rows, int64_t cols) { return rows * cols < ((int64_t)1 << 25) ? 32 : 64; }
constexpr int64_t quantize_tiles(int64_t rows, int64_t cols) {
    return up(rows, kSegment) * (kSegment / quantize_tile_rows(rows, cols)) * up(cols, kSegment) * (kSegment / kTileCols);
}
// A launch has fewer than 2^32 lanes.
constexpr bool quantize_fits(int64_t rows, int64_t cols) { return quantize_tiles(rows, cols) < ((int64_t)1 << 32) / kTileLanes; }

// Tiles of the products come to LDS in copies of 16 bytes for each lane.  A step takes a segment of 256 terms, 128 bytes of codes of each row in eight
// pieces; of the scales, 1024 terms at a time, 32 bytes of each row in two.  In LDS, piece c of row r lies at c ^ swizzle(r), so that the 64
// lanes of a read, 32 rows of the same piece in each half, spread evenly over the banks.  A copy to LDS writes consecutive lanes to
// consecutive places, so the lanes ask memory for their pieces in that order.
constexpr int kScaleTerms = 1024, kScaleBytes = kScaleTerms / kBlock, kScaleSteps = kScaleTerms / kSegment;
constexpr int code_swizzle(int row) { return row >> 1 & 7; }
constexpr int scale_swizzle(int row) { return row >> 3 & 1; }

// Where a lane of wavefront `wave` finds what its i-th copy takes, from the tile's first row and the step's first byte on.  Rows begin `pitch` bytes
// apart; behind row `last`, the matrix's last one in the tile, it takes that row again.
constexpr int code_row(int copy, int lane) { return copy * 8 + lane / 8; }
constexpr uint32_t code_place(int copy, int lane, uint32_t last, uint32_t pitch) {
    const int row = code_row(copy, lane);
    return ((uint32_t)row < last ? (uint32_t)row : last) * pitch + (uint32_t)((lane % 8 ^ code_swizzle(row)) * 16);
}
constexpr int scale_row(int copy, int lane) { return copy * 32 + lane / 2; }
constexpr uint32_t scale_place(int copy, int lane, uint32_t last, uint32_t pitch) {
    const int row = scale_row(copy, lane);
    return ((uint32_t)row < last ? (uint32_t)row : last) * pitch + (uint32_t)((lane % 2 ^ scale_swizzle(row)) * 16);
}

// The buffer that a copy fetches from: the tile's `bytes` from `begin` on, none where there is no such step.  A lane whose place is `bytes` or more
// fetches nothing.  A step's first byte is in the buffer's address, so that a lane's place is the whole of what is compared with its
// size: how a separate offset would enter that comparison differs between descriptions of the hardware, and with an empty buffer, or in the last, half
// group of scales of the last row, one reading of it lets bytes behind the matrix be fetched.
struct CopyBuffer {
    uint64_t begin;
    uint32_t bytes;
};
constexpr CopyBuffer copy_buffer(uint32_t tile_bytes, uint32_t begin, bool there) {
    return {there ? begin : 0, there ? tile_bytes - begin : 0};
}

}  // namespace fo
#endif
