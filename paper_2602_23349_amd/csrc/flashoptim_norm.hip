// The norms before and after a block with its gate and residual scale, and their gradients, for gfx950.
//
// Forward, by row: u = f or norm(f) w + b;  h = a x + c act(gate) u;  y = norm(h) w' + b'.  Backward, with hat(v) = (v - mean) rstd:
//   dH = dh + rstd (g - hat(h) mean(g hat(h)) [- mean(g]),  g = dy w'           (the bracket: layer norms only)
//   dx = a dH,  dgate = sum c dH u act',  du = c dH act,  df = the same through the norm behind
//   dw' = sum dy hat(h),  db' = sum dy,  dw = sum du hat(f),  db = sum du       (over rows)
// Bound: HBM.  A row is loaded once, kept in registers through all its sums, which are FP32, and stored once (of the widest rows in the backward pass
// see norm_gradients).  RMS norms of 4096 BF16 values: 16384 rows forward with a branch as it is 91 us, 5.9 TB/s; 8192 rows backward with
// both norms and a gate 90 us with the sums over rows, 4.5 TB/s.  One row forward 3.2 us.  Forward, rows wider than 4096 with a branch, as it is / normalised: 4096
// rows of 8192 BF16 values 62 / 74 us (4.3 / 3.6 TB/s), layer norms on an FP32 stream 84 / 102 (4.8 / 3.9); 2000 of 12000 56 / 67; 8192 of 16384 210 / 254.

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "flashoptim.h"
#include "flashoptim_host.h"
#include "flashoptim_launch.h"
#include "flashoptim_layers.h"

namespace {

using fo::f32x4;
using fo::i32x4;
using fo::load_as;
using fo::store_as;
using fo::up;
using f32x8 = float __attribute__((ext_vector_type(8)));
using bf16x8 = __bf16 __attribute__((ext_vector_type(8)));


// A matrix as a kernel takes it; data NULL: left out.
struct Rows {
    char* data;
    int64_t stride;      // values
};
Rows to_dev(const flashoptim_matrix* m) { return m ? Rows{(char*)m->data, m->rows > 1 ? m->stride : 0} : Rows{nullptr, 0}; }

// Eight values as they lie in memory, so that loads can be issued well ahead of their first use.  `fp32` is a constant for the matrices and the
// same for all lanes for the weights.
struct Raw {
    i32x4 a, b;      // BF16: all in a
};
// The eight neighbouring columns that a lane loads, and which of them, from `first` on, are its own.  Every lane loads eight that exist: the last
// one of a ragged row the row's last eight, some of which are its neighbour's; those behind it the same, none of them theirs.  So a load is
// never a case distinction, at whose end the compiler has each wait for its data before the next is made (as such: 100 rows of 768,
// backward, 8.8 us of kernel time, so 7.4).  Rows of fewer than eight columns have kernels of their own (NARROW), in which lane 0 takes them
// one by one.
template <bool NARROW>
struct Place {
    int col, first, last;
    __device__ __forceinline__ Place() = default;
    __device__ __forceinline__ Place(int at, int cols) {
        col = NARROW ? 0 : min(at, cols - 8);
        first = min(at - col, 8);
        last = NARROW ? cols : 8;
    }
    __device__ __forceinline__ bool whole() const { return !NARROW && first == 0; }
    __device__ __forceinline__ f32x8 mask(f32x8 v) const {
        if (!whole()) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = i >= first && i < last ? v[i] : 0.0f;
        }
        return v;
    }
};

// `row`: where the row begins, in values.
template <bool NARROW>
__device__ __forceinline__ Raw load8(const void* p, bool fp32, int64_t row, const Place<NARROW>& at) {
    Raw r = {};
    if constexpr (NARROW) {
        uint32_t w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int64_t from = row + min(i, at.last - 1);
            w[i] = fp32 ? ((const uint32_t*)p)[from] : (uint32_t)((const uint16_t*)p)[from];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (fp32) { if (i < 4) r.a[i] = (int)w[i]; else r.b[i - 4] = (int)w[i]; }
            else r.a[i / 2] |= (int)(w[i] << (16 * (i % 2)));
        }
    } else {
        const char* f = (const char*)p + (row + at.col) * (fp32 ? 4 : 2);
        r.a = load_as<i32x4>(f);
        r.b = load_as<i32x4>(f + (fp32 ? 16 : 0));      // (of BF16 matrices, where fp32 is a constant, left out)
    }
    return r;
}
__device__ __forceinline__ f32x8 values(const Raw& r, bool fp32) {
    f32x8 v;
    if (fp32) {
#pragma unroll
        for (int i = 0; i < 4; ++i) { v[i] = __int_as_float(r.a[i]); v[4 + i] = __int_as_float(r.b[i]); }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float((uint32_t)r.a[i] << 16);
            v[2 * i + 1] = __uint_as_float((uint32_t)r.a[i] & 0xffff0000u);
        }
    }
    return v;
}
template <bool NARROW>
__device__ __forceinline__ void store8(void* p, bool fp32, int64_t row, const Place<NARROW>& at, f32x8 v) {
    if (fp32) {
        float* f = (float*)p + row + at.col;
        if (at.whole()) {
            store_as(f, f32x4{v[0], v[1], v[2], v[3]});
            store_as(f + 4, f32x4{v[4], v[5], v[6], v[7]});
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) if (i >= at.first && i < at.last) f[i] = v[i];
        }
    } else {
        __bf16* f = (__bf16*)p + row + at.col;
        const bf16x8 w = __builtin_convertvector(v, bf16x8);
        if (at.whole()) store_as(f, w);
        else {
#pragma unroll
            for (int i = 0; i < 8; ++i) if (i >= at.first && i < at.last) f[i] = w[i];
        }
    }
}

// The sum over a wavefront, in every lane, in a fixed order.
__device__ __forceinline__ float wave_sum(float v) {
#define FO_ADD(ctrl, rows) v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), ctrl, rows, 0xf, false))
    FO_ADD(0x111, 0xf);      // row_shr 1, 2, 4, 8: lane 15 of each row of 16 has the row's sum
    FO_ADD(0x112, 0xf);
    FO_ADD(0x114, 0xf);
    FO_ADD(0x118, 0xf);
    FO_ADD(0x142, 0xa);      // row_bcast 15, into the second and the fourth row
    FO_ADD(0x143, 0xc);      // row_bcast 31, into the upper half
#undef FO_ADD
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}

// Sums over the lanes that share a row.  With more than one wavefront through LDS: the two halves of `part` alternate, so that one barrier
// lies between a half's readers and its next writers.
template <int LANES>
struct RowSums {
    static constexpr int kWaves = LANES / 64;
    f32x4* part;             // [2][kWaves], the first two of each in use
    int turn;
    __device__ __forceinline__ void sum2(float& a, float& b) {
        a = wave_sum(a);
        b = wave_sum(b);
        if constexpr (kWaves > 1) {
            f32x4* p = part + turn * kWaves;
            turn ^= 1;
            if (threadIdx.x % 64 == 0) p[threadIdx.x / 64 % kWaves] = f32x4{a, b, 0.0f, 0.0f};
            __syncthreads();
            a = b = 0.0f;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) { a += p[w][0]; b += p[w][1]; }
        }
    }
    __device__ __forceinline__ float sum(float a) {
        float none = 0.0f;
        sum2(a, none);
        return a;
    }
};

// Has a kernel's arguments in scalar registers from here on.  Left to itself the compiler loads each where a path first needs it, one wait after the
// other: a dozen of them ahead of the first row.
#define FO_ROWS(r) "s"((r).data), "s"((r).stride)

// Rows that a workgroup handles side by side: where a wavefront has a row to itself, four (they need no barrier).
constexpr int lines_of(int lanes) { return lanes == 64 ? 4 : 1; }

// (The hardware's exponential and reciprocal, within a few units of the last place, where the sums around it are off by dozens.)
__device__ __forceinline__ float sigmoid(float v, float* rest) {      // *rest: 1 - sigmoid(v)
    const float e = __builtin_amdgcn_exp2f(v * -0x1.715476p+0f), s = __builtin_amdgcn_rcpf(1.0f + e);
    *rest = e > 1.0f ? 1.0f - s : e * s;        // (the difference of a sigmoid near 1 from 1 would keep few of its bits, beyond 17 none)
    return s;
}
__device__ __forceinline__ float sigmoid(float v) {
    float rest;
    return sigmoid(v, &rest);
}

struct NormArgs {
    Rows x, f, gate, h, y;
    const void *post_weight, *post_bias, *pre_weight, *pre_bias;
    float* stats;
    uint32_t rows, rows_per_gate;
    int32_t cols;
    float eps, residual_scale, branch_scale, inv_cols;
    uint8_t layer, post_norm, sigmoid, param_fp32;
};

// Mean and 1/sqrt(mean square distance + eps) of the row whose values the lanes have (0 where a lane has none).
template <int LANES, int CHUNKS, bool NARROW>
__device__ __forceinline__ void moments(RowSums<LANES>& sums, const f32x8 (&v)[CHUNKS], const Place<NARROW> (&at)[CHUNKS], const NormArgs& a, float* mean,
                                        float* rstd) {
    *mean = 0.0f;
    if (a.layer) {
        float s = 0.0f;
#pragma unroll
        for (int j = 0; j < CHUNKS; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) s += v[j][i];
        *mean = sums.sum(s) * a.inv_cols;
    }
    float s = 0.0f;
#pragma unroll
    for (int j = 0; j < CHUNKS; ++j) {
        const f32x8 d = at[j].mask(v[j] - *mean);
#pragma unroll
        for (int i = 0; i < 8; ++i) s = fmaf(d[i], d[i], s);
    }
    *rstd = 1.0f / sqrtf(fmaf(sums.sum(s), a.inv_cols, a.eps));
}

template <int CHUNKS>
struct Params {
    Raw weight[CHUNKS], bias[CHUNKS];
    template <bool NARROW>
    __device__ __forceinline__ void load(const void* w, const void* b, bool fp32, const Place<NARROW> (&at)[CHUNKS]) {
#pragma unroll
        for (int j = 0; j < CHUNKS; ++j) {
            if (w) weight[j] = load8(w, fp32, 0, at[j]);
            if (b) bias[j] = load8(b, fp32, 0, at[j]);
        }
    }
};

template <int CHUNKS>
__device__ __forceinline__ void affine(f32x8 (&v)[CHUNKS], const Params<CHUNKS>& p, bool weight, bool bias, bool fp32, float mean, float rstd) {
#pragma unroll
    for (int j = 0; j < CHUNKS; ++j) {
        v[j] = (v[j] - mean) * rstd;
        if (weight) v[j] *= values(p.weight[j], fp32);
        if (bias) v[j] += values(p.bias[j], fp32);
    }
}

// LANES lanes to a row, each CHUNKS times eight neighbouring values.  All that a row reads is asked for at once: a single row, whose time is
// latency, waits for memory once.
template <bool STREAM_FP32, bool BRANCH_FP32, int LANES, int CHUNKS, bool NARROW>
__global__ __launch_bounds__(LANES * lines_of(LANES)) void norm_rows(NormArgs a) {
    constexpr int kLines = lines_of(LANES);
    __shared__ f32x4 part[2 * (LANES / 64)];
    const uint32_t row = blockIdx.x * kLines + (kLines > 1 ? threadIdx.x / LANES : 0);
    const int lane = threadIdx.x % LANES;
    if (kLines > 1 && row >= a.rows) return;
    RowSums<LANES> sums = {part, 0};
    Place<NARROW> at[CHUNKS];
    Raw x[CHUNKS], f[CHUNKS], gate[CHUNKS];
    Params<CHUNKS> post, pre;
#pragma unroll
    for (int j = 0; j < CHUNKS; ++j) {
        at[j] = Place<NARROW>((j * LANES + lane) * 8, a.cols);
        if (a.f.data) f[j] = load8(a.f.data, BRANCH_FP32, (int64_t)row * a.f.stride, at[j]);
        x[j] = load8(a.x.data, STREAM_FP32, (int64_t)row * a.x.stride, at[j]);
        if (a.gate.data) gate[j] = load8(a.gate.data, BRANCH_FP32, (int64_t)(row / a.rows_per_gate) * a.gate.stride, at[j]);
    }
    post.load(a.post_weight, a.post_bias, a.param_fp32, at);
    pre.load(a.pre_weight, a.pre_bias, a.param_fp32, at);
    float post_mean = 0.0f, post_rstd = 0.0f, pre_mean = 0.0f, pre_rstd = 0.0f;
    f32x8 h[CHUNKS], u[CHUNKS];
#pragma unroll
    for (int j = 0; j < CHUNKS; ++j) h[j] = at[j].mask(values(x[j], STREAM_FP32));
    if (a.f.data) {
#pragma unroll
        for (int j = 0; j < CHUNKS; ++j) u[j] = at[j].mask(values(f[j], BRANCH_FP32));
        if (a.post_norm) {
            moments(sums, u, at, a, &post_mean, &post_rstd);
            affine(u, post, a.post_weight, a.post_bias, a.param_fp32, post_mean, post_rstd);
        }
#pragma unroll
        for (int j = 0; j < CHUNKS; ++j) {
            if (a.gate.data) {
                f32x8 g = values(gate[j], BRANCH_FP32);
                if (a.sigmoid) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) g[i] = sigmoid(g[i]);
                }
                u[j] *= g;
            }
            h[j] = at[j].mask(a.residual_scale * h[j] + a.branch_scale * u[j]);
            store8(a.h.data, STREAM_FP32, (int64_t)row * a.h.stride, at[j], h[j]);
        }
    }
    if (a.y.data) {
        moments(sums, h, at, a, &pre_mean, &pre_rstd);
        affine(h, pre, a.pre_weight, a.pre_bias, a.param_fp32, pre_mean, pre_rstd);
#pragma unroll
        for (int j = 0; j < CHUNKS; ++j) store8(a.y.data, BRANCH_FP32, (int64_t)row * a.y.stride, at[j], h[j]);
    }
    if (a.stats && lane == 0) {
        const int64_t rows = a.rows;
        a.stats[row] = post_mean;
        a.stats[rows + row] = post_rstd;
        a.stats[2 * rows + row] = pre_mean;
        a.stats[3 * rows + row] = pre_rstd;
    }
}

// ------------------------------------------------------------------------------------------------------- backward --

// Sums over rows are formed in two stages of fixed order: a workgroup adds up the rows of its part in registers and leaves one row
// of sums for each kind of them; sum_parts adds up the parts.  Of a gate that serves many rows no part crosses the boundary
// (units are then rows); of one that serves few a part takes whole groups (units are groups), and their sums are complete.
enum Sum { kPreWeight, kPreBias, kPostWeight, kPostBias, kGate, kSums };

struct GradArgs {
    Rows h, f, gate, dy, dh, dx, df, dgate;
    const void *post_weight, *post_bias, *pre_weight;
    const float* stats;
    float* part;                 // [kind in use][parts][cols]
    int32_t slot[kSums];         // which kind in use, or -1
    uint32_t rows, rows_per_gate, parts;
    uint32_t unit_rows, part_units, units_per_group;      // (units_per_group: units that parts may not reach beyond)
    uint32_t parts_per_group;
    int32_t cols;
    float residual_scale, branch_scale, inv_cols;
    uint8_t post_norm, sigmoid, param_fp32, gate_done;      // gate_done: a unit's sums of the gate are complete
};

// What a row reads.
template <int CHUNKS>
struct RowData {
    Raw h[CHUNKS], dy[CHUNKS], dh[CHUNKS], f[CHUNKS], gate[CHUNKS];
    float post_mean, post_rstd, pre_mean, pre_rstd;
};

template <bool STREAM_FP32, bool BRANCH_FP32, int LANES, int CHUNKS, bool NARROW, int LINES, bool LAYER, bool BRANCH>
__global__ __launch_bounds__(LANES * LINES) void norm_gradients(GradArgs a) {
    __shared__ f32x4 part_sums[LINES][2 * (LANES / 64)];
    __shared__ float joined[LINES > 1 ? LINES : 1][LINES > 1 ? LANES * 8 * CHUNKS : 1];
    asm volatile("" ::FO_ROWS(a.h), FO_ROWS(a.f), FO_ROWS(a.gate), FO_ROWS(a.dy), FO_ROWS(a.dh), FO_ROWS(a.dx), FO_ROWS(a.df), "s"(a.post_weight),
                 "s"(a.post_bias), "s"(a.pre_weight), "s"(a.stats), "s"(a.rows), "s"(a.rows_per_gate), "s"(a.unit_rows), "s"(a.part_units),
                 "s"(a.units_per_group), "s"(a.parts_per_group), "s"(a.cols), "s"(a.residual_scale));
    const int line = LINES > 1 ? threadIdx.x / LANES : 0, lane = threadIdx.x % LANES;
    RowSums<LANES> sums = {part_sums[line], 0};
    Place<NARROW> at[CHUNKS];
#pragma unroll
    for (int j = 0; j < CHUNKS; ++j) {
        at[j] = Place<NARROW>((j * LANES + lane) * 8, a.cols);
    }
    // What a row reads is held from its loads on, and the next row's with it.  Of rows of more than 4096 values that takes more registers than there
    // are, by what they hold: their weights, then all that is theirs, are read again where they are needed, from the L2.  us with all of it held
    // (spilled), the weights read again, all read again, for 4096 rows of 8192 of a branch: RMS in BF16 98, 126, 100; RMS on an FP32 stream 239, 159,
    // 193; layer in BF16 266, 138, 188; layer on an FP32 stream 609, 234, 202; 2000 rows of 12000, RMS in BF16: 1120, -, 179.
    constexpr bool kNarrow = CHUNKS == 1 || (CHUNKS == 2 && !BRANCH);
    constexpr bool kHold = kNarrow || (CHUNKS == 2 && (LAYER ? !STREAM_FP32 : !BRANCH_FP32));
    constexpr bool kHoldParams = kNarrow || (CHUNKS == 2 && !LAYER && !STREAM_FP32);
    Params<kHoldParams ? CHUNKS : 1> post, pre;
    if constexpr (kHoldParams) {
        pre.load(a.pre_weight, nullptr, a.param_fp32, at);
        if constexpr (BRANCH) post.load(a.post_weight, a.post_bias, a.param_fp32, at);
    }
    RowData<kHold ? CHUNKS : 1> d, next;
    auto load = [&](RowData<kHold ? CHUNKS : 1>& d, uint32_t row) {
        const int64_t rows = a.rows;
        if (a.dy.data) {
            d.pre_mean = a.stats[2 * rows + row];
            d.pre_rstd = a.stats[3 * rows + row];
        }
        if (BRANCH && a.post_norm) {
            d.post_mean = a.stats[row];
            d.post_rstd = a.stats[rows + row];
        }
        if constexpr (kHold) {
#pragma unroll
            for (int j = 0; j < CHUNKS; ++j) {
                if (a.dy.data) {
                    d.h[j] = load8(a.h.data, STREAM_FP32, (int64_t)row * a.h.stride, at[j]);
                    d.dy[j] = load8(a.dy.data, BRANCH_FP32, (int64_t)row * a.dy.stride, at[j]);
                }
                if (a.dh.data) d.dh[j] = load8(a.dh.data, STREAM_FP32, (int64_t)row * a.dh.stride, at[j]);
                if constexpr (BRANCH) {
                    d.f[j] = load8(a.f.data, BRANCH_FP32, (int64_t)row * a.f.stride, at[j]);
                    if (a.gate.data) d.gate[j] = load8(a.gate.data, BRANCH_FP32, (int64_t)(row / a.rows_per_gate) * a.gate.stride, at[j]);
                }
            }
        }
    };
    // Chunk j of matrix m, held as `held`, of row `row`; and of a weight or bias.
    auto chunk = [&](const Rows& m, const Raw* held, bool fp32, uint32_t row, int j) {
        if constexpr (kHold) return values(held[j], fp32);
        else return values(load8(m.data, fp32, (int64_t)row * m.stride, at[j]), fp32);
    };
    auto param = [&](const void* p, const Raw* held, int j) {
        if constexpr (kHoldParams) return values(held[j], a.param_fp32);
        else return values(load8(p, a.param_fp32, 0, at[j]), a.param_fp32);
    };
    f32x8 acc[kSums][CHUNKS] = {};
    const uint32_t group = blockIdx.x / a.parts_per_group, in_group = blockIdx.x - group * a.parts_per_group;
    const uint32_t begin = group * a.units_per_group + in_group * a.part_units;
    const uint32_t end = min(begin + a.part_units, min((group + 1) * a.units_per_group, (a.rows + a.unit_rows - 1) / a.unit_rows));
    uint32_t unit = begin + line, row = unit * a.unit_rows;
    if (unit < end) load(d, row);
    while (unit < end) {
        // the next row is on its way while this one goes through its sums
        uint32_t next_row = row + 1, next_unit = unit;
        if (next_row == (unit + 1) * a.unit_rows) {
            next_unit = unit + LINES;
            next_row = next_unit * a.unit_rows;
        }
        if (next_unit < end) load(next, next_row);
        auto pre_hat = [&](int j) { return (chunk(a.h, d.h, STREAM_FP32, row, j) - d.pre_mean) * d.pre_rstd; };
        auto pre_grad = [&](int j) { return at[j].mask(chunk(a.dy, d.dy, BRANCH_FP32, row, j)); };
        float pre_s0 = 0.0f, pre_s1 = 0.0f;
        f32x8 kept_hat, kept_g, kept_post;
        if (a.dy.data) {
#pragma unroll
            for (int j = 0; j < CHUNKS; ++j) {
                const f32x8 hat = pre_hat(j);
                f32x8 g = pre_grad(j);
                acc[kPreWeight][j] += g * hat;
                if (LAYER) acc[kPreBias][j] += g;
                if (a.pre_weight) g *= param(a.pre_weight, pre.weight, j);
                kept_hat = hat;
                kept_g = g;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    pre_s0 = fmaf(g[i], hat[i], pre_s0);
                    if (LAYER) pre_s1 += g[i];
                }
            }
            sums.sum2(pre_s0, pre_s1);
            pre_s0 *= a.inv_cols;
            pre_s1 *= a.inv_cols;
        }
        const float mean = BRANCH && a.post_norm ? d.post_mean : 0.0f, rstd = BRANCH && a.post_norm ? d.post_rstd : 1.0f;
        auto post_hat = [&](int j) { return (chunk(a.f, d.f, BRANCH_FP32, row, j) - mean) * rstd; };
        f32x8 du[CHUNKS];
        float s0 = 0.0f, s1 = 0.0f;
#pragma unroll
        for (int j = 0; j < CHUNKS; ++j) {
            f32x8 total = a.dh.data ? chunk(a.dh, d.dh, STREAM_FP32, row, j) : f32x8{};
            if (a.dy.data) {
                f32x8 hat = kept_hat, g = kept_g;
                if constexpr (CHUNKS > 1) {
                    hat = pre_hat(j);
                    g = pre_grad(j);
                    if (a.pre_weight) g *= param(a.pre_weight, pre.weight, j);
                }
                total += d.pre_rstd * (g - hat * pre_s0 - (LAYER ? pre_s1 : 0.0f));
            }
            if constexpr (BRANCH) {
                const f32x8 hat = kept_post = post_hat(j);
                du[j] = a.branch_scale * total;
                if (a.gate.data) {
                    const Rows gate_row = {a.gate.data, 0};
                    f32x8 act = kHold ? chunk(gate_row, d.gate, BRANCH_FP32, 0, j)
                                      : values(load8(a.gate.data, BRANCH_FP32, (int64_t)(row / a.rows_per_gate) * a.gate.stride, at[j]), BRANCH_FP32);
                    f32x8 u = hat;
                    if (a.post_weight) u *= param(a.post_weight, post.weight, j);
                    if (a.post_bias) u += param(a.post_bias, post.bias, j);
                    u *= du[j];
                    if (a.sigmoid) {
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            float rest;
                            act[i] = sigmoid(act[i], &rest);
                            u[i] *= act[i] * rest;
                        }
                    }
                    acc[kGate][j] += u;
                    du[j] *= act;
                }
                if (a.post_norm) {
                    acc[kPostWeight][j] += du[j] * hat;
                    if (LAYER) acc[kPostBias][j] += du[j];
                    if (a.post_weight) du[j] *= param(a.post_weight, post.weight, j);
                    const f32x8 own = at[j].mask(du[j]);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        s0 = fmaf(own[i], hat[i], s0);
                        if (LAYER) s1 += own[i];
                    }
                }
            }
            if (a.dx.data) store8(a.dx.data, STREAM_FP32, (int64_t)row * a.dx.stride, at[j], BRANCH ? a.residual_scale * total : total);
        }
        if constexpr (BRANCH) {
            if (a.post_norm) {
                sums.sum2(s0, s1);
                s0 *= a.inv_cols;
                s1 *= a.inv_cols;
            }
            if (a.df.data) {
#pragma unroll
                for (int j = 0; j < CHUNKS; ++j) {
                    if (a.post_norm) du[j] = rstd * (du[j] - (CHUNKS == 1 ? kept_post : post_hat(j)) * s0 - (LAYER ? s1 : 0.0f));
                    store8(a.df.data, BRANCH_FP32, (int64_t)row * a.df.stride, at[j], du[j]);
                }
            }
            if (next_unit != unit && a.gate_done && a.dgate.data) {
#pragma unroll
                for (int j = 0; j < CHUNKS; ++j) {
                    store8(a.dgate.data, BRANCH_FP32, (int64_t)unit * a.dgate.stride, at[j], acc[kGate][j]);
                    acc[kGate][j] = f32x8{};
                }
            }
        }
        d = next;
        row = next_row;
        unit = next_unit;
    }
    if constexpr (LINES > 1 && LANES > 64) {
        // a line that has no row left goes along with the barriers of those that have
        const uint32_t count = end - min(begin, end), own = count - min(count, (uint32_t)line);
        const uint32_t left = ((count + LINES - 1) / LINES - (own + LINES - 1) / LINES) * a.unit_rows;
        for (uint32_t i = 0; i < left; ++i) {
            if (a.dy.data) __syncthreads();
            if (BRANCH && a.post_norm) __syncthreads();
        }
    }
#pragma unroll
    for (int k = 0; k < kSums; ++k) {
        if (a.slot[k] < 0 || (!BRANCH && k >= kPostWeight) || (!LAYER && (k == kPreBias || k == kPostBias))) continue;
        float* out = a.part + ((int64_t)a.slot[k] * a.parts + blockIdx.x) * a.cols;
        if constexpr (LINES > 1) {
            __syncthreads();
#pragma unroll
            for (int j = 0; j < CHUNKS; ++j)
#pragma unroll
                for (int i = 0; i < 8; ++i) joined[line][(j * 8 + i) * LANES + lane] = acc[k][j][i];
            __syncthreads();
            if (line == 0) {
#pragma unroll
                for (int j = 0; j < CHUNKS; ++j) {
#pragma unroll
                    for (int i = 0; i < 8; ++i)
#pragma unroll
                        for (int l = 1; l < LINES; ++l) acc[k][j][i] += joined[l][(j * 8 + i) * LANES + lane];
                    store8(out, true, 0, at[j], acc[k][j]);
                }
            }
        } else {
#pragma unroll
            for (int j = 0; j < CHUNKS; ++j) store8(out, true, 0, at[j], acc[k][j]);
        }
    }
}

// out[group][col] = the sum of part[group * parts .. (group + 1) * parts)[col].  One entry for each kind of sum.
struct PartSum {
    const float* part;
    void* out;
    int64_t stride;
    uint32_t parts, groups;
    int32_t fp32;
};
struct PartSums {
    PartSum of[kSums];
    int32_t cols;
};

// A wavefront of the 16 adds up every 16th part, sixteen loads on their way at a time.
constexpr int kSumWaves = 16;
__global__ __launch_bounds__(64 * kSumWaves) void sum_parts(PartSums p) {
    __shared__ float joined[kSumWaves][64];
    const PartSum& s = p.of[blockIdx.z];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, col = blockIdx.x * 64 + lane;
    for (uint32_t group = blockIdx.y; group < s.groups; group += gridDim.y) {
        float v = 0.0f;
        if (col < p.cols) {
            const float* at = s.part + ((int64_t)group * s.parts) * p.cols + col;
            for (uint32_t i = wave; i < s.parts; i += 16 * kSumWaves) {
                float w[16];
#pragma unroll
                for (uint32_t j = 0; j < 16; ++j) w[j] = i + j * kSumWaves < s.parts ? at[(int64_t)(i + j * kSumWaves) * p.cols] : 0.0f;
#pragma unroll
                for (uint32_t j = 0; j < 16; ++j) v += w[j];
            }
        }
        __syncthreads();
        joined[wave][lane] = v;
        __syncthreads();
        if (wave == 0 && col < p.cols) {
#pragma unroll
            for (int w = 1; w < kSumWaves; ++w) v += joined[w][lane];
            const int64_t at = (int64_t)group * s.stride + col;
            if (s.fp32) ((float*)s.out)[at] = v;
            else ((__bf16*)s.out)[at] = (__bf16)v;
        }
    }
}

// ------------------------------------------------------------------------------------------------------------ host --

constexpr int64_t kMaxCols = 16384;

int check_spec(const flashoptim_block_norm_spec* s) {
    if (!s || s->cols < 1 || s->kind < 0 || s->kind > 1 || s->post_norm < 0 || s->post_norm > 1 || s->gate_act < 0 || s->gate_act > 1 ||
        (s->param_dtype != FLASHOPTIM_BF16 && s->param_dtype != FLASHOPTIM_FP32) || !(s->eps >= 0.0f))
        return FLASHOPTIM_ERR_INVALID_ARG;
    if (s->kind == FLASHOPTIM_RMS_NORM && (s->post_bias || s->pre_bias)) return FLASHOPTIM_ERR_INVALID_ARG;
    if (s->cols > kMaxCols) return FLASHOPTIM_ERR_NUMEL_RANGE;
    const uintptr_t unit = (uintptr_t)fo::elem_bytes(s->param_dtype);
    for (const void* p : {s->post_weight, s->post_bias, s->pre_weight, s->pre_bias})
        if (!fo::aligned_to(p, unit)) return FLASHOPTIM_ERR_MISALIGNED;
    return FLASHOPTIM_OK;
}

// A matrix that may be left out: rows by cols, of this type if it is there.
int check_rows(const flashoptim_matrix* m, int64_t rows, int64_t cols, int dtype) {
    if (!m) return FLASHOPTIM_OK;
    const int rc = fo::check_matrix(m);
    if (rc != FLASHOPTIM_OK) return rc;
    return m->rows == rows && m->cols == cols && m->dtype == dtype ? FLASHOPTIM_OK : FLASHOPTIM_ERR_INVALID_ARG;
}

// The gate's rows, 0 without a gate.
int check_gate(const flashoptim_matrix* gate, int64_t rows, int64_t cols, int dtype, int64_t* rows_per_gate) {
    *rows_per_gate = rows > 0 ? rows : 1;
    if (!gate) return FLASHOPTIM_OK;
    FO_TRY(check_rows(gate, gate->rows, cols, dtype));
    if (gate->rows < 1 || rows % gate->rows != 0) return FLASHOPTIM_ERR_INVALID_ARG;
    if (rows > 0) *rows_per_gate = rows / gate->rows;
    return FLASHOPTIM_OK;
}

// Calls launch(lanes, chunks) as integral constants with the shape for rows of this many values.
template <int LANES, int CHUNKS, bool NARROW = false>
struct Shape {
    static constexpr int kLanes = LANES, kChunks = CHUNKS;
    static constexpr bool kNarrow = NARROW;
};
// Eight values to a lane as far as 512 lanes reach.  The backward pass keeps up to five sums a value, for which 1024 lanes, of 128 registers each,
// have no room: it takes 512 lanes with 16 or 32 values, as the forward pass does.
template <typename F>
void with_shape(int64_t cols, F launch) {
    if (cols < 8) launch(Shape<64, 1, true>{});
    else if (cols <= 512) launch(Shape<64, 1>{});
    else if (cols <= 1024) launch(Shape<128, 1>{});
    else if (cols <= 2048) launch(Shape<256, 1>{});
    else if (cols <= 4096) launch(Shape<512, 1>{});
    else if (cols <= 8192) launch(Shape<512, 2>{});
    else launch(Shape<512, 4>{});
}

// How the rows of a backward call are cut into parts.
struct Parts {
    int64_t unit_rows, part_units, units_per_group, parts_per_group, parts;
    bool gate_done;
};
// Rows that a workgroup of the backward pass handles side by side.  What it sums over its rows, five values a column, is written and read again: with
// 2000 rows of 768 in 1000 workgroups as many bytes as the rows themselves.  So eight where a wavefront has a row to itself, and four of two
// wavefronts where there are few rows; their barriers hold up all four, which many rows do not pay for (us, one line / four, layer norms of 768
// values: 2048 rows 18.2 / 16.2, 4096 23.3 / 22.9, 8192 37 / 41; of two lines of 256 lanes: 4096 rows of 2048 36 / 41).
int lines_of_gradients(int64_t rows, int64_t cols) { return cols <= 512 ? 8 : cols <= 1024 && rows <= 4096 ? 4 : 1; }
Parts cut(int64_t rows, int64_t gates, int64_t cols) {
    const int64_t rows_per_gate = rows / gates, lines = lines_of_gradients(rows, cols);
    // As many parts as there are compute units times what one holds of them, from 1024 of 128 lanes to 256 of 512 (us, 256 / 512 / 1024 / 1536 parts: 16384
    // rows of 1024 values 116 / 74 / 48 / 47, 8192 of 4096 98 / 99 / 106 / 121, 4096 of 2048, layer norms, 42 / 33 / 41 / 47).
    const int64_t least = lines > 1 ? lines : 2, most = lines > 1 ? 256 : cols <= 1024 ? 1024 : cols <= 2048 ? 512 : 256;
    int64_t part_rows = up(rows, most);
    if (part_rows < least) part_rows = least;
    Parts p;
    if (gates == 1 || rows_per_gate >= part_rows) {
        p.unit_rows = 1;
        p.part_units = part_rows;
        p.units_per_group = rows_per_gate;
        p.parts_per_group = up(rows_per_gate, part_rows);
        p.parts = gates * p.parts_per_group;
        p.gate_done = false;
    } else {
        p.unit_rows = rows_per_gate;
        p.part_units = up(part_rows, rows_per_gate);
        p.units_per_group = gates;
        p.parts_per_group = p.parts = up(gates, p.part_units);
        p.gate_done = true;
    }
    return p;
}

// Which sums a call wants, at most (workspace) or of this call.
int64_t part_bytes(const flashoptim_block_norm_spec* spec, int64_t rows, int64_t gates) {
    if (rows == 0) return 0;
    const int64_t kinds = spec->kind == FLASHOPTIM_LAYER_NORM ? 5 : 3;
    return kinds * cut(rows, gates, spec->cols).parts * spec->cols * 4;
}

}  // namespace

extern "C" {

int flashoptim_block_norm(const flashoptim_block_norm_spec* spec, const flashoptim_matrix* x, const flashoptim_matrix* f,
                          const flashoptim_matrix* gate, const flashoptim_matrix* h, const flashoptim_matrix* y, float* stats,
                          void* stream) {
    FO_TRY(check_spec(spec));
    FO_TRY(fo::check_matrix(x));
    const int64_t rows = x->rows;
    if (x->cols != spec->cols || (!f && !y) || (!f) != (!h) || (gate && !f)) return FLASHOPTIM_ERR_INVALID_ARG;
    const int branch_type = f ? f->dtype : y->dtype;
    if (branch_type == FLASHOPTIM_FP32 && x->dtype != FLASHOPTIM_FP32) return FLASHOPTIM_ERR_INVALID_ARG;
    FO_TRY(check_rows(f, rows, spec->cols, branch_type));
    FO_TRY(check_rows(h, rows, spec->cols, x->dtype));
    FO_TRY(check_rows(y, rows, spec->cols, branch_type));
    int64_t rows_per_gate;
    FO_TRY(check_gate(gate, rows, spec->cols, branch_type, &rows_per_gate));
    if (!fo::aligned_to(stats, 4)) return FLASHOPTIM_ERR_MISALIGNED;
    if (rows == 0) return FLASHOPTIM_OK;
    bool fits = true;                        // a launch of fewer than 2^32 lanes
    with_shape(spec->cols, [&](auto shape) { fits = rows <= (((int64_t)1 << 32) - 512) / decltype(shape)::kLanes; });
    if (!fits) return FLASHOPTIM_ERR_NUMEL_RANGE;
    NormArgs a = {};
    a.x = to_dev(x); a.f = to_dev(f); a.gate = to_dev(gate); a.h = to_dev(h); a.y = to_dev(y);
    a.post_weight = spec->post_weight; a.post_bias = spec->post_bias; a.pre_weight = spec->pre_weight; a.pre_bias = spec->pre_bias;
    a.stats = stats;
    a.rows = (uint32_t)rows; a.rows_per_gate = (uint32_t)rows_per_gate; a.cols = (int32_t)spec->cols;
    a.eps = spec->eps; a.residual_scale = spec->residual_scale; a.branch_scale = spec->branch_scale;
    a.inv_cols = (float)(1.0 / (double)spec->cols);
    a.layer = spec->kind == FLASHOPTIM_LAYER_NORM; a.post_norm = f && spec->post_norm; a.sigmoid = spec->gate_act == FLASHOPTIM_GATE_SIGMOID;
    a.param_fp32 = spec->param_dtype == FLASHOPTIM_FP32;
    const bool sf = x->dtype == FLASHOPTIM_FP32, bf = branch_type == FLASHOPTIM_FP32;
    with_shape(spec->cols, [&](auto shape) {
        constexpr int L = decltype(shape)::kLanes, C = decltype(shape)::kChunks, T = L * lines_of(L);
        constexpr bool N = decltype(shape)::kNarrow;
        const dim3 grid((unsigned)up(rows, T / L)), block(T);
        if (bf) hipLaunchKernelGGL((norm_rows<true, true, L, C, N>), grid, block, 0, (hipStream_t)stream, a);
        else if (sf) hipLaunchKernelGGL((norm_rows<true, false, L, C, N>), grid, block, 0, (hipStream_t)stream, a);
        else hipLaunchKernelGGL((norm_rows<false, false, L, C, N>), grid, block, 0, (hipStream_t)stream, a);
    });
    return fo::hip_status(hipGetLastError());
}

int64_t flashoptim_block_norm_backward_workspace(const flashoptim_block_norm_spec* spec, int64_t rows, int64_t gates) {
    FO_TRY(check_spec(spec));
    if (rows < 0 || gates < 1 || rows % gates != 0) return FLASHOPTIM_ERR_INVALID_ARG;
    if (rows >= ((int64_t)1 << 31)) return FLASHOPTIM_ERR_NUMEL_RANGE;
    return part_bytes(spec, rows, gates);
}

int flashoptim_block_norm_backward(const flashoptim_block_norm_spec* spec, const flashoptim_matrix* h, const flashoptim_matrix* f,
                                   const flashoptim_matrix* gate, const float* stats, const flashoptim_block_norm_grads* grads,
                                   void* workspace, int64_t workspace_bytes, void* stream) {
    FO_TRY(check_spec(spec));
    FO_TRY(fo::check_matrix(h));
    if (!grads || (!grads->dy && !grads->dh)) return FLASHOPTIM_ERR_INVALID_ARG;
    const int64_t rows = h->rows, cols = spec->cols;
    const flashoptim_block_norm_grads& g = *grads;
    const bool post_norm = f && spec->post_norm, layer = spec->kind == FLASHOPTIM_LAYER_NORM;
    if (h->cols != cols || (!f && (gate || g.df)) || (!gate && g.dgate)) return FLASHOPTIM_ERR_INVALID_ARG;
    const int branch_type = f ? f->dtype : g.dy ? g.dy->dtype : h->dtype;
    if (branch_type == FLASHOPTIM_FP32 && h->dtype != FLASHOPTIM_FP32) return FLASHOPTIM_ERR_INVALID_ARG;
    FO_TRY(check_rows(f, rows, cols, branch_type));
    FO_TRY(check_rows(g.dy, rows, cols, branch_type));
    FO_TRY(check_rows(g.dh, rows, cols, h->dtype));
    FO_TRY(check_rows(g.dx, rows, cols, h->dtype));
    FO_TRY(check_rows(g.df, rows, cols, branch_type));
    int64_t rows_per_gate;
    FO_TRY(check_gate(gate, rows, cols, branch_type, &rows_per_gate));
    if (gate) FO_TRY(check_rows(g.dgate, gate->rows, cols, branch_type));
    // a gradient of what is not there
    if ((!g.dy && (g.dpre_weight || g.dpre_bias)) || (!post_norm && (g.dpost_weight || g.dpost_bias)) ||
        (!layer && (g.dpre_bias || g.dpost_bias)))
        return FLASHOPTIM_ERR_INVALID_ARG;
    if ((g.dy || post_norm) && rows > 0 && !stats) return FLASHOPTIM_ERR_INVALID_ARG;
    const uintptr_t unit = (uintptr_t)fo::elem_bytes(spec->param_dtype);
    void* const outs[kSums] = {g.dpre_weight, g.dpre_bias, g.dpost_weight, g.dpost_bias, g.dgate ? g.dgate->data : nullptr};
    for (int k = 0; k < kGate; ++k)
        if (!fo::aligned_to(outs[k], unit)) return FLASHOPTIM_ERR_MISALIGNED;
    const int64_t gates = gate ? gate->rows : 1;
    const int64_t need = part_bytes(spec, rows, gates);
    if (need > 0 && !workspace) return FLASHOPTIM_ERR_INVALID_ARG;
    if (workspace_bytes < need) return FLASHOPTIM_ERR_WORKSPACE;
    if (!fo::aligned_to(workspace, 16) || !fo::aligned_to(stats, 4)) return FLASHOPTIM_ERR_MISALIGNED;

    PartSums p = {};
    p.cols = (int32_t)cols;
    int kinds = 0;
    const Parts c = rows > 0 ? cut(rows, gates, cols) : Parts{1, 1, 1, 1, 0, false};
    GradArgs a = {};
    for (int k = 0; k < kSums; ++k) {
        a.slot[k] = -1;
        if (!outs[k] || (k == kGate && c.gate_done)) continue;
        a.slot[k] = kinds;
        PartSum& s = p.of[kinds];
        s.part = (const float*)workspace + (int64_t)kinds * c.parts * cols;
        s.out = outs[k];
        s.groups = k == kGate ? (uint32_t)gates : 1u;
        s.parts = k == kGate ? (uint32_t)c.parts_per_group : (uint32_t)c.parts;
        s.stride = k == kGate ? (gates > 1 ? g.dgate->stride : 0) : 0;
        if (rows == 0) s.parts = 0;
        s.fp32 = k == kGate ? branch_type == FLASHOPTIM_FP32 : spec->param_dtype == FLASHOPTIM_FP32;
        ++kinds;
    }
    if (rows > 0) {
        a.h = to_dev(h); a.f = to_dev(f); a.gate = to_dev(gate);
        a.dy = to_dev(g.dy); a.dh = to_dev(g.dh); a.dx = to_dev(g.dx); a.df = to_dev(g.df); a.dgate = to_dev(g.dgate);
        a.post_weight = post_norm ? spec->post_weight : nullptr; a.post_bias = post_norm ? spec->post_bias : nullptr;
        a.pre_weight = spec->pre_weight;
        a.stats = stats; a.part = (float*)workspace;
        a.rows = (uint32_t)rows; a.rows_per_gate = (uint32_t)rows_per_gate; a.parts = (uint32_t)c.parts;
        a.unit_rows = (uint32_t)c.unit_rows; a.part_units = (uint32_t)c.part_units; a.units_per_group = (uint32_t)c.units_per_group;
        a.parts_per_group = (uint32_t)c.parts_per_group;
        a.cols = (int32_t)cols;
        a.residual_scale = spec->residual_scale; a.branch_scale = spec->branch_scale; a.inv_cols = (float)(1.0 / (double)cols);
        a.post_norm = post_norm; a.sigmoid = spec->gate_act == FLASHOPTIM_GATE_SIGMOID; a.param_fp32 = spec->param_dtype == FLASHOPTIM_FP32;
        a.gate_done = c.gate_done;
        const bool sf = h->dtype == FLASHOPTIM_FP32, bf = branch_type == FLASHOPTIM_FP32;
        with_shape(cols, [&](auto shape) {
            constexpr int L = decltype(shape)::kLanes, C = decltype(shape)::kChunks;
            constexpr bool N = decltype(shape)::kNarrow;
            const dim3 grid((unsigned)c.parts);
            auto launch = [&](auto lines_c, auto layer_c, auto branch_c) {
                constexpr int K = decltype(lines_c)::value;
                constexpr bool LN = decltype(layer_c)::value, BR = decltype(branch_c)::value;
                const dim3 block(L * K);
                if (bf) hipLaunchKernelGGL((norm_gradients<true, true, L, C, N, K, LN, BR>), grid, block, 0, (hipStream_t)stream, a);
                else if (sf) hipLaunchKernelGGL((norm_gradients<true, false, L, C, N, K, LN, BR>), grid, block, 0, (hipStream_t)stream, a);
                else hipLaunchKernelGGL((norm_gradients<false, false, L, C, N, K, LN, BR>), grid, block, 0, (hipStream_t)stream, a);
            };
            using Yes = std::true_type;
            using No = std::false_type;
            auto with_lines = [&](auto k) {
                if (layer) { if (f) launch(k, Yes{}, Yes{}); else launch(k, Yes{}, No{}); }
                else { if (f) launch(k, No{}, Yes{}); else launch(k, No{}, No{}); }
            };
            if constexpr (L == 64) with_lines(std::integral_constant<int, 8>{});
            else if constexpr (L == 128) {
                if (lines_of_gradients(rows, cols) == 4) with_lines(std::integral_constant<int, 4>{});
                else with_lines(std::integral_constant<int, 1>{});
            } else with_lines(std::integral_constant<int, 1>{});
        });
        FO_TRY(fo::hip_status(hipGetLastError()));
    }
    if (kinds) {
        const unsigned groups = a.slot[kGate] >= 0 ? (unsigned)(gates < 1024 ? gates : 1024) : 1u;
        hipLaunchKernelGGL(sum_parts, dim3((unsigned)up(cols, 64), groups, (unsigned)kinds), dim3(64 * kSumWaves), 0, (hipStream_t)stream, p);
        FO_TRY(fo::hip_status(hipGetLastError()));
    }
    return FLASHOPTIM_OK;
}

}  // extern "C"
