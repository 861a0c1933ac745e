// The global norm of a list of gradients and their clipping, for gfx950.
//
//   sum_squares = sum over all tensors of g^2,   norm = sqrt(sum_squares),   scale = norm > max_norm ? max_norm / norm : 1,   dst = round(src * scale)
// Bound: HBM for all but small lists: the norm reads a gradient once, clipping reads it again and writes it.  Squares are summed in FP64: no finite
// gradient overflows them and no order of the sum is visible in the FP32 norm, at one conversion and one multiply-add for each element, which
// hide behind the loads.

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <cstring>

#include "flashoptim.h"
#include "flashoptim_clip.h"
#include "flashoptim_host.h"
#include "flashoptim_layers.h"

namespace {

using fo::GradTable;
using fo::f32x4;
using fo::i32x4;
using fo::kGradThreads;
using fo::kGradTile;

constexpr int kJoinThreads = 1024;

// Where a tile lies: its tensor's memory, its first element there and how many elements it has.
struct Tile {
    const void* src;
    void* dst;
    int64_t begin;
    int left;
};
// A launch's table.  Of up to kGradSome tensors each lane holds one, fetched once and all together, so that a tile is found in registers; longer ones are
// searched in memory, one step after the other.  (25 tensors of 250 thousand elements together, searched in memory and held: norm 3.6 us and 2.8, clipping 4.3
// and 3.8; 21 tensors of 1.5 G elements, norm 447 us and 441.)
template <int N, bool DST>
struct Lookup {
    static constexpr bool kHeld = N <= fo::kGradSome;
    const GradTable<N, DST>& t;
    uint32_t n, first = 0xffffffffu, lack = 0;
    uint64_t src = 0, dst = 0;

    __device__ __forceinline__ Lookup(const GradTable<N, DST>& table, uint32_t tensors) : t(table), n(tensors) {
        if constexpr (kHeld) {
            const uint32_t lane = threadIdx.x & 63;
            if (lane <= n) first = t.first[lane];
            if (lane < n) {
                src = (uint64_t)t.src[lane];
                lack = t.lack[lane];
                if constexpr (DST) dst = (uint64_t)t.dst[lane];
            }
        }
    }
    static __device__ __forceinline__ uint32_t of_lane(uint32_t v, uint32_t lane) { return (uint32_t)__builtin_amdgcn_readlane((int)v, (int)lane); }
    static __device__ __forceinline__ uint64_t of_lane(uint64_t v, uint32_t lane) {
        return (uint64_t)of_lane((uint32_t)(v >> 32), lane) << 32 | of_lane((uint32_t)v, lane);
    }
    // (All lanes of the wavefront ask for the same tile.)
    __device__ __forceinline__ Tile operator()(uint32_t tile) const {
        if constexpr (kHeld) {
            const uint32_t i = (uint32_t)__builtin_popcountll(__builtin_amdgcn_ballot_w64(first <= tile)) - 1;
            const bool last = tile == of_lane(first, i + 1) - 1;
            return {(const void*)of_lane(src, i), DST ? (void*)of_lane(dst, i) : nullptr, (int64_t)(tile - of_lane(first, i)) * kGradTile,
                    last ? kGradTile - (int)of_lane(lack, i) : kGradTile};
        } else {
            const uint32_t i = fo::entry_of(tile, 0u, n - 1, [&](uint32_t k) { return t.first[k]; });
            void* d = nullptr;
            if constexpr (DST) d = t.dst[i];
            return {t.src[i], d, (int64_t)(tile - t.first[i]) * kGradTile, tile == t.first[i + 1] - 1 ? kGradTile - (int)t.lack[i] : kGradTile};
        }
    }
};

// Sixteen bytes of a gradient: eight BF16 values or four FP32 ones.  KEEP: they stay in the caches; else they go past them.
template <bool FP32>
constexpr int kValues = FP32 ? 4 : 8;
template <bool FP32, bool KEEP = false>
__device__ __forceinline__ i32x4 load_word(const void* p, int64_t at) {
    const i32x4* w = (const i32x4*)((const char*)p + at * (FP32 ? 4 : 2));
    return KEEP ? *w : __builtin_nontemporal_load(w);
}
template <bool FP32>
__device__ __forceinline__ void values(const i32x4& w, float (&v)[kValues<FP32>]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (FP32) v[i] = __int_as_float(w[i]);
        else {
            v[2 * i] = __uint_as_float((uint32_t)w[i] << 16);
            v[2 * i + 1] = __uint_as_float((uint32_t)w[i] & 0xffff0000u);
        }
    }
}
template <bool FP32>
__device__ __forceinline__ float value_at(const void* p, int64_t at) {
    return FP32 ? ((const float*)p)[at] : __uint_as_float((uint32_t)((const uint16_t*)p)[at] << 16);
}

// The sum over a workgroup, in lane 0, in a fixed order.
template <int THREADS>
__device__ __forceinline__ double group_sum(double s) {
    __shared__ double part[THREADS / 64];
    s = fo::sum_of_wave(s);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = s;
    __syncthreads();
    s = 0.0;
#pragma unroll
    for (int k = 0; k < THREADS / 64; ++k) s += part[k];
    return s;
}

__device__ __forceinline__ void set_factor(flashoptim_clip_factor* f, double sum, float max_norm) {
    const double norm = sqrt(sum);
    f->sum_squares = sum;
    f->norm = (float)norm;
    f->scale = !(sum < __builtin_inf()) ? __builtin_nanf("") : norm > (double)max_norm ? (float)((double)max_norm / norm) : 1.0f;
}

__device__ __forceinline__ void add_square(double& sum, float v) {
    const double d = (double)v;
    sum = fma(d, d, sum);
}

// What a lane holds of a tile that kGradThreads lanes share: every so many-th word, all fetched together, and behind a tensor's last whole word one value.
// Words and values that are not there are 0.
template <bool FP32, bool KEEP>
struct TileWords {
    static constexpr int kN = kValues<FP32>, kWords = kGradTile / (kGradThreads * kN);
    i32x4 w[kWords];
    float edge = 0.0f;

    __device__ __forceinline__ void load(const Tile& at, int lane) {
        if (at.left == kGradTile) {
#pragma unroll
            for (int p = 0; p < kWords; ++p) w[p] = load_word<FP32, KEEP>(at.src, at.begin + (p * kGradThreads + lane) * kN);
        } else {
            const int whole = at.left / kN, k = whole * kN + lane;
#pragma unroll
            for (int p = 0; p < kWords; ++p) {
                w[p] = i32x4{};
                if (p * kGradThreads + lane < whole) w[p] = load_word<FP32, KEEP>(at.src, at.begin + (p * kGradThreads + lane) * kN);
            }
            if (k < at.left) edge = value_at<FP32>(at.src, at.begin + k);
        }
    }
    __device__ __forceinline__ void add_to(double& sum) const {
#pragma unroll
        for (int p = 0; p < kWords; ++p) {
            float v[kN];
            values<FP32>(w[p], v);
#pragma unroll
            for (int i = 0; i < kN; ++i) add_square(sum, v[i]);
        }
        add_square(sum, edge);
    }
};
template <bool FP32, bool KEEP>
__device__ __forceinline__ void add_tile(double& sum, const Tile& at, int lane) {
    TileWords<FP32, KEEP> words;
    words.load(at, lane);
    words.add_to(sum);
}

// Each workgroup takes every so many-th tile.  The tiles from `keep` on, the list's last ones, stay in the memory-side cache for the clipping that begins with
// them (all past the caches -> these kept, norm and clipping of GPT-2's 124 M gradients BF16 128 -> 120 us, FP32 200 -> 194; all kept, the norm alone is 10 %
// slower: 300 M FP32 gradients 174 -> 197).
template <bool FP32, int N>
__global__ __launch_bounds__(kGradThreads) void norm_kernel(GradTable<N, false> t, uint32_t n, uint32_t tiles, uint32_t keep, double* part) {
    double sum = 0.0;
    const Lookup<N, false> locate(t, n);
    for (uint32_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const Tile at = locate(tile);
        if (tile < keep) add_tile<FP32, false>(sum, at, (int)threadIdx.x);
        else add_tile<FP32, true>(sum, at, (int)threadIdx.x);
    }
    sum = group_sum<kGradThreads>(sum);
    if (threadIdx.x == 0) part[blockIdx.x] = sum;
}

// A few tiles, by one workgroup that needs nobody to join its sum.
template <bool FP32, int N>
__global__ __launch_bounds__(kJoinThreads) void norm_small_kernel(GradTable<N, false> t, uint32_t n, uint32_t tiles, float max_norm, flashoptim_clip_factor* factor) {
    double sum = 0.0;
    const uint32_t group = (uint32_t)__builtin_amdgcn_readfirstlane((int)threadIdx.x / kGradThreads);
    const Lookup<N, false> locate(t, n);
    constexpr uint32_t kGroups = kJoinThreads / kGradThreads, kTogether = FP32 ? 2 : 4;      // (tiles of a group whose words are on their way together)
    for (uint32_t tile = group; tile < tiles; tile += kTogether * kGroups) {
        TileWords<FP32, true> words[kTogether];
#pragma unroll
        for (uint32_t k = 0; k < kTogether; ++k)
            if (tile + k * kGroups < tiles) words[k].load(locate(tile + k * kGroups), (int)threadIdx.x % kGradThreads);
#pragma unroll
        for (uint32_t k = 0; k < kTogether; ++k)
            if (tile + k * kGroups < tiles) words[k].add_to(sum);
    }
    sum = group_sum<kJoinThreads>(sum);
    if (threadIdx.x == 0) set_factor(factor, sum, max_norm);
}

__global__ __launch_bounds__(kJoinThreads) void norm_join_kernel(const double* part, uint32_t parts, float max_norm, flashoptim_clip_factor* factor) {
    double sum = 0.0;
    for (uint32_t i = threadIdx.x; i < parts; i += kJoinThreads) sum += part[i];
    sum = group_sum<kJoinThreads>(sum);
    if (threadIdx.x == 0) set_factor(factor, sum, max_norm);
}

__global__ void factor_kernel(flashoptim_clip_factor* factor, float max_norm) {
    if (threadIdx.x == 0) set_factor(factor, factor->sum_squares, max_norm);
}

// One value, and the values of one word of src, times the factor, at their place in dst.
template <bool DST32>
__device__ __forceinline__ void put(void* p, int64_t at, float v) {
    if constexpr (DST32) ((float*)p)[at] = v;
    else ((__bf16*)p)[at] = (__bf16)v;
}
template <bool SRC32, bool DST32>
__device__ __forceinline__ void put_word(void* p, int64_t at, const i32x4& w, float scale) {
    using f32x8 = float __attribute__((ext_vector_type(8)));
    using bf16x4 = __bf16 __attribute__((ext_vector_type(4)));
    using bf16x8 = __bf16 __attribute__((ext_vector_type(8)));
    using i32x2 = int __attribute__((ext_vector_type(2)));
    float v[kValues<SRC32>];
    values<SRC32>(w, v);
#pragma unroll
    for (int i = 0; i < kValues<SRC32>; ++i) v[i] *= scale;
    char* to = (char*)p + at * (DST32 ? 4 : 2);
    if constexpr (!SRC32) __builtin_nontemporal_store(__builtin_bit_cast(i32x4, __builtin_convertvector((f32x8){v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7]}, bf16x8)), (i32x4*)to);
    else if constexpr (DST32) __builtin_nontemporal_store(__builtin_bit_cast(i32x4, (f32x4){v[0], v[1], v[2], v[3]}), (i32x4*)to);
    else __builtin_nontemporal_store(__builtin_bit_cast(i32x2, __builtin_convertvector((f32x4){v[0], v[1], v[2], v[3]}, bf16x4)), (i32x2*)to);
}

// DST: dst differs from src (otherwise the same buffers, left alone where the factor is 1).
template <bool SRC32, bool DST32, bool DST, int N>
__global__ __launch_bounds__(kGradThreads) void clip_kernel(GradTable<N, DST> t, uint32_t n, uint32_t tiles, const flashoptim_clip_factor* factor) {
    constexpr int kN = kValues<SRC32>, kWords = kGradTile / (kGradThreads * kN);       // of a lane, of a whole tile
    const float scale = factor->scale;
    if (!DST && scale == 1.0f) return;
    const Lookup<N, DST> locate(t, n);
    for (uint32_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const Tile at = locate(tiles - 1 - tile);      // (the list's last ones first: the norm has left them in the memory-side cache)
        const void* src = at.src;
        void* dst = DST ? at.dst : const_cast<void*>(src);
        if (DST && dst == src && scale == 1.0f) continue;
        TileWords<SRC32, false> words;
        words.load(at, (int)threadIdx.x);
        if (at.left == kGradTile) {
#pragma unroll
            for (int p = 0; p < kWords; ++p) put_word<SRC32, DST32>(dst, at.begin + (p * kGradThreads + (int)threadIdx.x) * kN, words.w[p], scale);
            continue;
        }
        const int whole = at.left / kN, k = whole * kN + (int)threadIdx.x;
#pragma unroll
        for (int p = 0; p < kWords; ++p) {
            const int word = p * kGradThreads + (int)threadIdx.x;
            if (word < whole) put_word<SRC32, DST32>(dst, at.begin + word * kN, words.w[p], scale);
        }
        if (k < at.left) put<DST32>(dst, at.begin + k, words.edge * scale);
    }
}

bool known(int dtype) { return dtype == FLASHOPTIM_BF16 || dtype == FLASHOPTIM_FP32; }

int check_list(const flashoptim_gradient* g, int64_t n, int src_dtype) {
    if (n < 0 || (n > 0 && !g) || !known(src_dtype)) return FLASHOPTIM_ERR_INVALID_ARG;
    int64_t all = 0;
    for (int64_t i = 0; i < n; ++i) {
        if (g[i].numel < 0 || g[i].numel >= fo::kMaxElems) return FLASHOPTIM_ERR_NUMEL_RANGE;
        all += g[i].numel;
        if (all >= ((int64_t)1 << 43)) return FLASHOPTIM_ERR_NUMEL_RANGE;
    }
    return FLASHOPTIM_OK;
}
int check_factor(const flashoptim_clip_factor* f) {
    if (!f) return FLASHOPTIM_ERR_INVALID_ARG;
    return fo::aligned_to(f, 16) ? FLASHOPTIM_OK : FLASHOPTIM_ERR_MISALIGNED;
}

int64_t live_tensors(const flashoptim_gradient* g, int64_t n) {
    int64_t live = 0;
    for (int64_t i = 0; i < n; ++i) live += g[i].numel > 0;
    return live;
}

// The next launch's tensors: those of the list from *at on that fit, the empty ones left out.
struct Cut {
    uint32_t n = 0, tiles = 0;
};
template <int N, bool DST>
Cut fill(GradTable<N, DST>& t, const flashoptim_gradient* g, int64_t n, int64_t* at) {
    Cut c;
    for (; *at < n && c.n < (uint32_t)N; ++*at) {
        const flashoptim_gradient& x = g[*at];
        if (x.numel == 0) continue;
        const int64_t tiles = fo::grad_tiles(x.numel);
        if ((int64_t)c.tiles + tiles > 0x7fffffff) break;
        t.src[c.n] = x.src;
        if (DST) t.dst[c.n] = x.dst;
        t.first[c.n] = c.tiles;
        t.lack[c.n] = (uint16_t)(tiles * kGradTile - x.numel);
        c.tiles += (uint32_t)tiles;
        ++c.n;
    }
    t.first[c.n] = c.tiles;
    return c;
}

// The partial sums of a list's launches, which are cut as fill() and for_each_cut() do.
int64_t norm_parts(const flashoptim_gradient* g, int64_t n) {
    const int64_t live = live_tensors(g, n), most = live <= fo::kGradFew ? fo::kGradFew : live <= fo::kGradSome ? fo::kGradSome : fo::kGradMany;
    int64_t parts = 0, tensors = 0, tiles = 0;
    for (int64_t i = 0; i < n; ++i) {
        if (g[i].numel == 0) continue;
        const int64_t k = fo::grad_tiles(g[i].numel);
        if (tensors == most || tiles + k > 0x7fffffff) {
            parts += fo::norm_groups(tiles);
            tensors = tiles = 0;
        }
        ++tensors;
        tiles += k;
    }
    return parts + fo::norm_groups(tiles);
}

// launch(table, its cut) for each of a call's launches, with tables of up to MANY tensors, of fewer where the list is short.
template <int MANY, bool DST, typename F>
int for_each_cut(const flashoptim_gradient* g, int64_t n, F launch) {
    const int64_t live = live_tensors(g, n);
    const auto with = [&](auto& table, int64_t* at) {
        const Cut c = fill(table, g, n, at);
        return c.n ? launch(table, c) : (int)FLASHOPTIM_OK;
    };
    for (int64_t at = 0; at < n;) {
        if (live <= fo::kGradFew) {
            GradTable<fo::kGradFew, DST> t;
            FO_TRY(with(t, &at));
        } else if (live <= fo::kGradSome) {
            GradTable<fo::kGradSome, DST> t;
            FO_TRY(with(t, &at));
        } else {
            GradTable<MANY, DST> t;
            FO_TRY(with(t, &at));
        }
    }
    return FLASHOPTIM_OK;
}

template <bool SRC32, bool DST32, bool DST>
int clip_launches(const flashoptim_gradient* g, int64_t n, const flashoptim_clip_factor* factor, void* stream) {
    return for_each_cut<DST ? fo::kClipMany : fo::kGradMany, DST>(g, n, [&](auto& t, const Cut& c) {
        const unsigned blocks = (unsigned)(c.tiles < fo::kMostTiles ? c.tiles : fo::kMostTiles);
        constexpr int N = sizeof(t.lack) / sizeof(t.lack[0]);
        hipLaunchKernelGGL((clip_kernel<SRC32, DST32, DST, N>), dim3(blocks), dim3(kGradThreads), 0, (hipStream_t)stream, t, c.n, c.tiles, factor);
        return fo::hip_status(hipGetLastError());
    });
}

}  // namespace

extern "C" {

int64_t flashoptim_grad_norm_workspace(const flashoptim_gradient* grads, int64_t n_grads, int src_dtype) {
    FO_TRY(check_list(grads, n_grads, src_dtype));
    return norm_parts(grads, n_grads) * (int64_t)sizeof(double);
}

int flashoptim_grad_norm(const flashoptim_gradient* grads, int64_t n_grads, int src_dtype, float max_norm,
                         flashoptim_clip_factor* factor, void* workspace, int64_t workspace_bytes, void* stream) {
    FO_TRY(check_list(grads, n_grads, src_dtype));
    if (!(max_norm >= 0.0f)) return FLASHOPTIM_ERR_INVALID_ARG;
    FO_TRY(check_factor(factor));
    for (int64_t i = 0; i < n_grads; ++i) {
        if (grads[i].numel == 0) continue;
        if (!grads[i].src) return FLASHOPTIM_ERR_INVALID_ARG;
        if (!fo::aligned_to(grads[i].src, 16)) return FLASHOPTIM_ERR_MISALIGNED;
    }
    const int64_t need = flashoptim_grad_norm_workspace(grads, n_grads, src_dtype);
    if (need < 0) return (int)need;
    if (need > 0 && !workspace) return FLASHOPTIM_ERR_INVALID_ARG;
    if (workspace_bytes < need) return FLASHOPTIM_ERR_WORKSPACE;
    if (!fo::aligned_to(workspace, 16)) return FLASHOPTIM_ERR_MISALIGNED;
    double* part = (double*)workspace;
    uint32_t parts = 0;
    int64_t left = 0;                                    // tiles of this launch and of those behind it
    for (int64_t i = 0; i < n_grads; ++i) left += fo::grad_tiles(grads[i].numel);
    const int64_t kept = fo::kKeptBytes / (fo::kGradTile * fo::elem_bytes(src_dtype));
    const bool small = left > 0 && left <= fo::kSmallTiles;
    FO_TRY((for_each_cut<fo::kGradMany, false>(grads, n_grads, [&](auto& t, const Cut& c) {
        constexpr int N = sizeof(t.lack) / sizeof(t.lack[0]);
        if (small && c.tiles == left) {
            const dim3 one(1), block(kJoinThreads);
            if (src_dtype == FLASHOPTIM_FP32) hipLaunchKernelGGL((norm_small_kernel<true, N>), one, block, 0, (hipStream_t)stream, t, c.n, c.tiles, max_norm, factor);
            else hipLaunchKernelGGL((norm_small_kernel<false, N>), one, block, 0, (hipStream_t)stream, t, c.n, c.tiles, max_norm, factor);
            left = -1;
            return fo::hip_status(hipGetLastError());
        }
        const dim3 grid((unsigned)fo::norm_groups(c.tiles)), block(kGradThreads);
        const uint32_t keep = (uint32_t)(left <= kept ? 0 : left - kept < (int64_t)c.tiles ? left - kept : (int64_t)c.tiles);
        if (src_dtype == FLASHOPTIM_FP32) hipLaunchKernelGGL((norm_kernel<true, N>), grid, block, 0, (hipStream_t)stream, t, c.n, c.tiles, keep, part + parts);
        else hipLaunchKernelGGL((norm_kernel<false, N>), grid, block, 0, (hipStream_t)stream, t, c.n, c.tiles, keep, part + parts);
        parts += grid.x;
        left -= c.tiles;
        return fo::hip_status(hipGetLastError());
    })));
    if (left < 0) return FLASHOPTIM_OK;
    hipLaunchKernelGGL(norm_join_kernel, dim3(1), dim3(kJoinThreads), 0, (hipStream_t)stream, part, parts, max_norm, factor);
    return fo::hip_status(hipGetLastError());
}

int flashoptim_clip_factor_from_sum(flashoptim_clip_factor* factor, float max_norm, void* stream) {
    FO_TRY(check_factor(factor));
    if (!(max_norm >= 0.0f)) return FLASHOPTIM_ERR_INVALID_ARG;
    hipLaunchKernelGGL(factor_kernel, dim3(1), dim3(64), 0, (hipStream_t)stream, factor, max_norm);
    return fo::hip_status(hipGetLastError());
}

int flashoptim_clip_gradients(const flashoptim_gradient* grads, int64_t n_grads, int src_dtype, int dst_dtype,
                              const flashoptim_clip_factor* factor, void* stream) {
    FO_TRY(check_list(grads, n_grads, src_dtype));
    if (!known(dst_dtype) || (src_dtype == FLASHOPTIM_BF16 && dst_dtype == FLASHOPTIM_FP32)) return FLASHOPTIM_ERR_INVALID_ARG;
    FO_TRY(check_factor(factor));
    bool in_place = true;
    for (int64_t i = 0; i < n_grads; ++i) {
        const flashoptim_gradient& g = grads[i];
        if (g.numel == 0) continue;
        if (!g.src || !g.dst || (g.src == g.dst && src_dtype != dst_dtype)) return FLASHOPTIM_ERR_INVALID_ARG;
        if (!fo::aligned_to(g.src, 16) || !fo::aligned_to(g.dst, 16)) return FLASHOPTIM_ERR_MISALIGNED;
        in_place = in_place && g.src == g.dst;
    }
    const bool s = src_dtype == FLASHOPTIM_FP32, d = dst_dtype == FLASHOPTIM_FP32;
    if (in_place) return s ? clip_launches<true, true, false>(grads, n_grads, factor, stream) : clip_launches<false, false, false>(grads, n_grads, factor, stream);
    if (s) return d ? clip_launches<true, true, true>(grads, n_grads, factor, stream) : clip_launches<true, false, true>(grads, n_grads, factor, stream);
    return clip_launches<false, false, true>(grads, n_grads, factor, stream);
}

}  // extern "C"
