// Internal: how the calls over a list of gradients (flashoptim_clip.hip) are cut into tiles, workgroups and launches.  Plain C++ without
// HIP, so that its limits can be tested without a GPU.
#ifndef FLASHOPTIM_CLIP_H
#define FLASHOPTIM_CLIP_H

#include <stdint.h>

#include "flashoptim_launch.h"

namespace fo {

// A tile is what a workgroup handles at a time: consecutive elements of one tensor.
constexpr int kGradThreads = 256;
constexpr int kGradTile = 8192;

// A launch's tensors, as they travel in its arguments.  `first[i]` is tensor i's first tile, counted within the launch, and behind the last
// tensor all its tiles; `lack[i]` the elements that its last tile is short of.  What is left of the tables is not used.
template <int N, bool DST>
struct GradTable {
    const void* src[N];
    void* dst[DST ? N : 1];
    uint32_t first[N + 1];
    uint16_t lack[N];
};
// As many as the 4 KB of a launch's arguments hold, or few, for which the host has fewer bytes to copy.
// (kGradSome and one more are a wavefront's lanes.)
constexpr int kGradFew = 16, kGradSome = 63, kGradMany = 280, kClipMany = 176;
constexpr int64_t kGradArgBytes = 4096 - 64;             // beside the other arguments
static_assert(sizeof(GradTable<kGradMany, false>) <= kGradArgBytes && sizeof(GradTable<kClipMany, true>) <= kGradArgBytes, "kernel arguments");

constexpr int64_t grad_tiles(int64_t numel) { return up(numel, kGradTile); }
// The most tiles of a launch: so many that their number fits 31 bits, and of a clipping launch, one workgroup each, that its lanes fit 32.
constexpr int64_t kMostTiles = kMaxWorkItems / kGradThreads;

// The workgroups of a launch that sums up: each takes every so many-th tile and leaves one sum.
constexpr int64_t kNormGroups = 2048;
constexpr int64_t norm_groups(int64_t tiles) { return tiles < kNormGroups ? tiles : kNormGroups; }
// Lists of up to so many tiles are summed up by one workgroup, whose four groups of wavefronts take a tile each: one launch against two.  The sums of
// squares, which are FP64, bind it, 0.25 us a tile.  (Called one after the other: 8 tiles 4.6 us against 7.1, 12 tiles 5.6 against 7.1, 16 tiles 6.5 against 7.1; in a
// graph, without the host's time for a launch, 4.1, 5.3 and 6.4 against 4.2.)
constexpr int64_t kSmallTiles = 12;
// What the sum leaves in the 256 MB memory-side cache.
constexpr int64_t kKeptBytes = (int64_t)160 << 20;

}  // namespace fo
#endif
