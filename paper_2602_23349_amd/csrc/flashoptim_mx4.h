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

// Where a lane finds what copy number `copy` of a tile takes, from the tile's first row and the step's first byte on.  Rows begin `pitch` bytes
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

// How a product of m by n sums over k terms is made: by the largest tiles of which there are enough.  In us, with tiles of 16 (the wavefronts of a
// workgroup share out the sum) / 64 / 128 / 256:
//   kTiny while they are at most 256 tiles: 33 x 64 x 7600 (m, n, k) 6.1 / 9.6 / 16 / 39, 200 x 200 x 14000 11.1 / 16.2 / 28 / 71, 40 x 500 x 300
//     2.4 / 3.1 / 4.0 / 6.2; 90 x 950 x 950, 360 of them, 3.5 / 3.6, 600 x 600 x 600, 1444, 5.2 / 3.5;
//   kTile256 from 192 tiles on, three quarters of the compute units: 3000 x 4096 x 4096 - / 53 / 39.5 / 36.1; with 128 of them, 2048 x 4096 x 4096,
//     - / 37 / 26.6 / 32.7;
//   kTile64 up to 512 tiles, which is two for each compute unit: 512 x 4096 x 4096 86 / 10.4 / 12.1, 2304 x 768 x 1024 - / 5.2 / 6.2, 768 x 768 x 8000 49 /
//     10.8 / 19.8; kTile128 beyond: 1001 x 2304 x 768, 576 of them, - / 7.0 / 6.2, 1024 x 4096 x 4096 - / 19.5 / 15.7, 8192 x 768 x 768 - / 12.1 / 9.9.
// Sums split over workgroups and joined by another launch: 768 x 768 x 8000 in two 13.5, in four 16.2.
constexpr int64_t kMaxTiledTerms = (int64_t)1 << 23;      // 256 rows of codes stay below 2^31 bytes, which a lane's offset reaches
enum Shape { kTiny, kTile64, kTile128, kTile256 };
constexpr Shape product_shape(int64_t m, int64_t n, int64_t k) {
    if (k > kMaxTiledTerms || up(m, 16) * up(n, 16) <= 256) return kTiny;
    if (up(m, 256) * up(n, 256) >= 192) return kTile256;
    return m > 64 && n > 64 && up(m, 64) * up(n, 64) > 512 ? kTile128 : kTile64;
}

// The wavefronts that share out a sum over this many segments.
constexpr int sum_waves(int64_t segments) { return segments <= 4 ? 4 : segments <= 16 ? 8 : 16; }

constexpr int64_t kFewRows = 16;
constexpr int kFewAhead = 2;      // segments of a wavefront's weights that are on their way at a time
constexpr int kFewBatch = 4;      // units of eight values of x that a lane asks for at a time, if there are more than one for each lane

// How linear_small goes about it: tiles of 16 columns to a workgroup, and wavefronts.  In us:
//   two tiles where one each would be more than one workgroup for each compute unit: 6000 x 6000 (n, k), 375 tiles, 1 row 8.4 with one, 8.0 with two, 16
//     rows 17.6, 12.5; 14336 x 4096 1 row 10.2, 9.2, 8 rows 14.1, 11.8; 8192 x 2048 1 row 4.4, 4.6, 16 rows 7.0, 6.2;
//   16 wavefronts where there is no more than one workgroup for each compute unit, and many segments or rows: 4096 x 4096 with 8 / 16, 1 row 4.3 / 4.5, 16 rows
//     8.0 / 6.9; 6000 x 6000 as above 8.4 / 8.0 and 14.4 / 12.5; 14336 x 4096 9.2 / 11.4;
//   4 for up to four segments and few rows: 12000 x 500 with 4 / 8, 1 row 3.9 / 4.0, 16 rows 4.8 / 4.4.
struct FewPlan {
    int tiles, waves;
    int64_t workgroups;
};
constexpr FewPlan plan_few(int64_t m, int64_t n, int64_t k) {
    const int64_t tiles = up(n, 16), segments = up(k, kSegment);
    FewPlan p = {tiles > 256 ? 2 : 1, 8, 0};
    p.workgroups = up(tiles, p.tiles);
    if (segments <= 4) p.waves = m >= 8 ? 8 : 4;
    else if (p.workgroups <= 256 && (m >= 4 || segments > 16)) p.waves = 16;
    return p;
}
// Whether x is quantised by every workgroup of linear_small, or once by a launch of its own: by the work on x that a compute unit then has.  One launch /
// two, us: 4096 x 4096 with 1 row 4.4 / 6.5, 16 rows 6.9 / 7.8; 4096 x 14336 4 rows 11.4 / 12.2, 8 rows 14.3 / 13.5; 14336 x 4096 8 rows 11.8 / 11.3, 16 rows
// 15.0 / 11.3; 6000 x 6000 16 rows 12.5 / 13.6.
constexpr int64_t kFewValues = 98304;

constexpr bool takes_few_rows(int64_t m, int64_t n, int64_t k) {
    return m >= 1 && m <= kFewRows && n >= 1 && k >= 1 && m * up(k, kSegment) * kSegment * up(plan_few(m, n, k).workgroups, 256) <= kFewValues;
}

}  // namespace fo
#endif
