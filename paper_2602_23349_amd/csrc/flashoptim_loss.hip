// The losses on the logits and their gradients, for gfx950: log-probabilities of tokens, the clipped policy loss, the preference loss.
//
// By row of logits x with the token t and temperature T:   lse = log sum_j exp(x_j / T),  logprob = x_t / T - lse,  and with d the loss's gradient
// with respect to logprob:   dx_j = d / T ([j = t] - exp(x_j / T - lse)).
// Exponentials are powers of two of (x - m) log2(e) / T with m the row's largest value (the difference first: logits of the type's lowest value, as
// masks set them, stay finite).  Bound: HBM; a row costs two exponentials an element.

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <cmath>
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

constexpr double kLog2e = 1.4426950408889634;
constexpr int kPairThreads = 1024;

// A matrix of logits as a kernel takes it.
struct Logits {
    const char* data;
    int64_t stride;      // values
    int32_t vocab;
};
template <bool FP32>
__device__ __forceinline__ const char* row_of(const Logits& m, uint32_t row) {
    return m.data + (int64_t)row * m.stride * (FP32 ? 4 : 2);
}
template <bool FP32>
__device__ __forceinline__ float value_at(const char* row, int32_t j) {
    return FP32 ? ((const float*)row)[j] : __uint_as_float((uint32_t)((const uint16_t*)row)[j] << 16);
}
// The logit of a token; one that is not there has none.
template <bool FP32>
__device__ __forceinline__ float logit_of(const char* row, int64_t token, int32_t vocab) {
    return token >= 0 && token < vocab ? value_at<FP32>(row, (int32_t)token) : __builtin_nanf("");
}

__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float minus_inf() { return -__builtin_inff(); }
// What the difference to a largest value is taken from: where there is none, any finite value will do.
__device__ __forceinline__ float base_of(float most) { return most == minus_inf() ? 0.0f : most; }

template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ float max_with(float v) {
    return fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(v), __float_as_int(v), CTRL, ROWS, 0xf, false)));
}
// The largest value of a wavefront, in every lane.
__device__ __forceinline__ float wave_max(float v) {
    v = max_with<0x111>(v);              // row_shr 1, 2, 4, 8: lane 15 of each row of 16 has the row's
    v = max_with<0x112>(v);
    v = max_with<0x114>(v);
    v = max_with<0x118>(v);
    v = max_with<0x142, 0xa>(v);         // row_bcast 15, into the second and the fourth row
    v = max_with<0x143, 0xc>(v);         // row_bcast 31, into the upper half
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}
__device__ __forceinline__ double wave_sum(double v) {
    for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off);
    return v;
}

// A part of a row: its largest value and the sum of 2^((x - most) c), FP64.
struct Sum {
    double sum;
    float most;
};
__device__ __forceinline__ Sum join(const Sum& a, const Sum& b, float c) {
    const float most = fmaxf(a.most, b.most), base = base_of(most);
    return {a.sum * (double)exp2_of((a.most - base) * c) + b.sum * (double)exp2_of((b.most - base) * c), most};
}

// What LANES lanes hold of a row in registers: the values from `begin` up to `end`, at most LANES * NV * 8 of them, lane l's i-th eight from begin +
// 8 (i LANES + l) on.  Every lane loads eight values that exist, so that no load is a case distinction: the last eight of a ragged row begin within
// their neighbours', and those behind the end are the last eight again.  What is not the lane's own becomes -infinity, which adds nothing.
// (NARROW: rows of fewer than eight values, which lane 0 takes one by one.)
template <bool FP32, int LANES, int NV, bool NARROW = false>
struct Held {
    static constexpr int kWords = FP32 ? 2 : 1;
    i32x4 raw[NV][kWords];
    int32_t begin, end;
    int lane;

    // Between two passes over what is held.  The values are unpacked again in each: kept from one to the next, they would take twice the registers.
    __device__ __forceinline__ void forget_values() {
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int k = 0; k < kWords; ++k) asm volatile("" : "+v"(raw[i][k]));
    }
    // (32 bits beside the row's address, which is a wavefront's: vocab < 2^30)
    static __device__ __forceinline__ uint32_t bytes(int32_t j) { return (uint32_t)j * (FP32 ? 4u : 2u); }
    __device__ __forceinline__ int32_t at(int i) const { return begin + 8 * (i * LANES + lane); }
    __device__ __forceinline__ void load(const char* row, int32_t begin_, int32_t end_, int lane_) {
        begin = begin_; end = end_; lane = lane_;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if constexpr (NARROW) {
                raw[i][0] = raw[i][kWords - 1] = i32x4{};
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    if (i > 0 || k >= end) continue;
                    if constexpr (FP32) raw[i][k / 4][k % 4] = ((const int*)row)[k];
                    else raw[i][0][k / 2] |= (int)((uint32_t)((const uint16_t*)row)[k] << (16 * (k % 2)));
                }
            } else {
                const uint32_t from = bytes(min(at(i), end - 8));
#pragma unroll
                for (int k = 0; k < kWords; ++k) raw[i][k] = load_as<i32x4>(row + from + 16 * k);
            }
        }
    }
    // Of the i-th eight, those that are the lane's own: [first, last).
    __device__ __forceinline__ void own(int i, int* first, int* last) const {
        const int32_t j = at(i);
        if (NARROW) { *first = 0; *last = j == 0 ? end : 0; }
        else { *first = min(max(j - (end - 8), 0), 8); *last = 8; }
    }
    // Puts -infinity where a value is not the lane's own.  (Before the first use.)
    __device__ __forceinline__ void settle(int i) {
        if (begin + 8 * (i + 1) * LANES <= end || at(i) + 8 <= end) return;
        int first, last;
        own(i, &first, &last);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const bool keep = k >= first && k < last;
            if constexpr (FP32) raw[i][k / 4][k % 4] = keep ? raw[i][k / 4][k % 4] : (int)0xff800000;
            else {
                const uint32_t shift = 16 * (k % 2);
                const uint32_t w = (uint32_t)raw[i][0][k / 2];
                raw[i][0][k / 2] = keep ? (int)w : (int)((w & ~(0xffffu << shift)) | 0xff80u << shift);
            }
        }
    }
    __device__ __forceinline__ void values(int i, float (&v)[8]) const {
        if constexpr (FP32) {
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = __int_as_float(raw[i][k / 4][k % 4]);
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                v[2 * k] = __uint_as_float((uint32_t)raw[i][0][k] << 16);
                v[2 * k + 1] = __uint_as_float((uint32_t)raw[i][0][k] & 0xffff0000u);
            }
        }
    }
    // The sum of the wavefront's part, in every lane.  A lane adds up in FP32, apart from eights that hold a value near the wavefront's largest, which go into
    // an FP64 sum: beside a token that is all but certain the others would be lost in its rounding, and with them its log-probability.
    __device__ __forceinline__ Sum wave_part(float c) {
        float most = minus_inf();
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            settle(i);
            float v[8];
            values(i, v);
#pragma unroll
            for (int k = 0; k < 8; k += 2) most = fmaxf(fmaxf(most, v[k]), v[k + 1]);
        }
        forget_values();
        most = wave_max(most);
        const float base = base_of(most);
        float sum = 0.0f;
        double near = 0.0;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            float v[8];
            values(i, v);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = exp2_of((v[k] - base) * c);
            const float largest = fmaxf(fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3])), fmaxf(fmaxf(v[4], v[5]), fmaxf(v[6], v[7])));
            if (__builtin_amdgcn_ballot_w64(largest >= 0.5f)) {
#pragma unroll
                for (int k = 0; k < 8; ++k) near += (double)v[k];
            } else {
#pragma unroll
                for (int k = 0; k < 8; ++k) sum += v[k];
            }
        }
        return {wave_sum(near + (double)sum), most};
    }
    // Stores -d p, or d (1 - p) for the token, of all that is held: p = 2^((x - base) c - shift).
    __device__ __forceinline__ void store_gradient(char* row, int64_t token, float d, float base, float c, float shift) {
        forget_values();
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int32_t j = at(i);
            if (j >= end) continue;
            float v[8];
            values(i, v);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = -d * exp2_of(fmaf(v[k] - base, c, -shift));
            const int32_t from = NARROW ? 0 : min(j, end - 8);
            if (token >= from && token < from + 8) {
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] = token == from + k ? v[k] + d : v[k];
            }
            store(row, i, v);
        }
    }
    __device__ __forceinline__ void store_zeros(char* row) const {
        const float v[8] = {};
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (at(i) < end) store(row, i, v);
    }
    __device__ __forceinline__ void store(char* row, int i, const float (&v)[8]) const {
        const int32_t j = at(i);
        if (j + 8 <= end) {
            char* p = row + bytes(j);
            if constexpr (FP32) {
                store_as(p, f32x4{v[0], v[1], v[2], v[3]});
                store_as(p + 16, f32x4{v[4], v[5], v[6], v[7]});
            } else {
                store_as(p, __builtin_convertvector((f32x8){v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7]}, bf16x8));
            }
            return;
        }
        int first, last;
        own(i, &first, &last);
        const int32_t from = NARROW ? 0 : end - 8;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            if (k < first || k >= last) continue;
            if constexpr (FP32) ((float*)row)[from + k] = v[k];
            else ((__bf16*)row)[from + k] = (__bf16)v[k];
        }
    }
};

// The sum over a workgroup's wavefronts, in every lane.
template <int WAVES>
__device__ __forceinline__ Sum join_waves(const Sum& s, float c) {
    if constexpr (WAVES == 1) return s;
    __shared__ Sum parts[WAVES];
    if ((threadIdx.x & 63) == 0) parts[threadIdx.x >> 6] = s;
    __syncthreads();
    Sum all = parts[0];
#pragma unroll
    for (int k = 1; k < WAVES; ++k) all.most = fmaxf(all.most, parts[k].most);
    const float base = base_of(all.most);
    all.sum = 0.0;
#pragma unroll
    for (int k = 0; k < WAVES; ++k) all.sum += parts[k].sum * (double)exp2_of((parts[k].most - base) * c);
    return all;
}

// log sum exp(x / T) and the token's log-probability; log_sum is what lse is beyond the largest value.
struct RowLog {
    double lse, logprob, log_sum;
};
__device__ __forceinline__ RowLog row_log(const Sum& s, float x, double inv_t) {
    // (a sum beyond FP32 is that of a row with +infinity)
    const double log_sum = s.most < __builtin_inff() ? log(s.sum) : (double)__builtin_nanf("");
    return {(double)s.most * inv_t + log_sum, ((double)x - (double)s.most) * inv_t - log_sum, log_sum};
}

// A row's part of the policy loss.
struct PolicyRow {
    float slope;                        // of the loss by logprob, weight and grad_scale in it
    double surrogate, kl, blocked;      // with their weight
};
struct PolicyArgs {
    flashoptim_policy_spec spec;
    flashoptim_policy_inputs in;
    double* terms;                      // [3, rows]
};
__device__ __forceinline__ PolicyRow policy_row(const PolicyArgs& a, uint32_t row, double logprob, float w) {
    const double adv = a.in.advantages[row];
    const double ratio = a.in.old_logprob ? exp(logprob - (double)a.in.old_logprob[row]) : logprob - logprob + 1.0;
    const double low = 1.0 - (double)a.spec.clip_low, high = 1.0 + (double)a.spec.clip_high;
    const bool blocked = (adv > 0.0 && ratio > high) || (adv < 0.0 && ratio < low);
    const double surrogate = blocked ? -adv * (adv > 0.0 ? high : low) : -adv * ratio;
    double slope = blocked ? 0.0 : -adv * ratio, kl = 0.0;
    if (a.in.ref_logprob) {
        const double d = (double)a.in.ref_logprob[row] - logprob, e = expm1(d);
        kl = e - d;
        slope -= (double)a.spec.kl_weight * e;
    }
    return {(float)(slope * (double)w * (double)a.spec.grad_scale), surrogate * w, kl * w, blocked ? (double)w : 0.0};
}
__device__ __forceinline__ void put_terms(const PolicyArgs& a, uint32_t rows, uint32_t row, const PolicyRow& r) {
    a.terms[row] = r.surrogate;
    a.terms[(int64_t)rows + row] = r.kl;
    a.terms[2 * (int64_t)rows + row] = r.blocked;
}

// What the row kernels take.
struct RowsArgs {
    Logits x;
    const int64_t* tokens;
    float *logprob, *lse;
    double inv_t;
    float c;
    uint32_t rows;
    char* dx;                // the gradient (policy loss; NULL: not wanted)
    int64_t dx_stride;
    float scale;             // 1 / T
    PolicyArgs policy;
};

// One row to LANES lanes, which hold it: the policy loss and its gradient in one pass over the logits.
template <bool FP32, int LANES, int NV, bool NARROW>
__global__ __launch_bounds__(LANES < 256 ? 256 : LANES) void policy_rows_kernel(RowsArgs a) {
    constexpr int LINES = LANES < 256 ? 256 / LANES : 1;
    static_assert(LANES == 64 || LINES == 1, "a row is a wavefront's or a workgroup's");
    const uint32_t row = LINES == 1 ? blockIdx.x : blockIdx.x * LINES + (uint32_t)__builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int lane = (int)threadIdx.x & (LANES - 1);
    if (row >= a.rows) return;
    const int64_t token = a.tokens[row];
    const float w = a.policy.in.weights ? a.policy.in.weights[row] : 1.0f;
    char* dx = a.dx ? a.dx + (int64_t)row * a.dx_stride * (FP32 ? 4 : 2) : nullptr;
    Held<FP32, LANES, NV, NARROW> h;
    if (token < 0 || w == 0.0f) {
        if (lane == 0) {
            if (a.logprob) a.logprob[row] = 0.0f;
            put_terms(a.policy, a.rows, row, {});
        }
        h.begin = 0; h.end = a.x.vocab; h.lane = lane;
        if (dx) h.store_zeros(dx);
        return;
    }
    const char* x = row_of<FP32>(a.x, row);
    h.load(x, 0, a.x.vocab, lane);
    const float logit = logit_of<FP32>(x, token, a.x.vocab);
    const Sum s = join_waves<LANES / 64>(h.wave_part(a.c), a.c);
    const RowLog l = row_log(s, logit, a.inv_t);
    const PolicyRow p = policy_row(a.policy, row, l.logprob, w);
    if (lane == 0) {
        if (a.logprob) a.logprob[row] = (float)l.logprob;
        put_terms(a.policy, a.rows, row, p);
    }
    if (!dx) return;
    const float d = p.slope * a.scale;
    if (d == 0.0f) h.store_zeros(dx);
    else h.store_gradient(dx, token, d, base_of(s.most), a.c, (float)(l.log_sum * kLog2e));
}

// Log-probabilities only, one workgroup of WAVES wavefronts to a row, through which the wavefronts go in turn.
template <bool FP32, int WAVES, bool NARROW>
__global__ __launch_bounds__(WAVES * 64) void logprob_rows_kernel(RowsArgs a) {
    constexpr int NV = NARROW ? 1 : FP32 ? 4 : 8;
    const uint32_t row = blockIdx.x;
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int64_t token = a.tokens[row];
    if (token < 0) {
        if (threadIdx.x == 0) {
            if (a.logprob) a.logprob[row] = 0.0f;
            if (a.lse) a.lse[row] = 0.0f;
        }
        return;
    }
    const char* x = row_of<FP32>(a.x, row);
    const float logit = logit_of<FP32>(x, token, a.x.vocab);
    Sum s = {0.0, minus_inf()};
    for (int32_t begin = wave * 64 * NV * 8; begin < a.x.vocab; begin += WAVES * 64 * NV * 8) {
        Held<FP32, 64, NV, NARROW> h;
        h.load(x, begin, a.x.vocab, lane);
        s = join(s, h.wave_part(a.c), a.c);
    }
    s = join_waves<WAVES>(s, a.c);
    if (threadIdx.x != 0) return;
    const RowLog l = row_log(s, logit, a.inv_t);
    if (a.logprob) a.logprob[row] = (float)l.logprob;
    if (a.lse) a.lse[row] = (float)l.lse;
}

// ---- few rows, or rows that do not fit: each cut into parts, a workgroup to each, which leaves its sum; whoever needs a row's joins them.
constexpr int kPartThreads = 256;
template <bool FP32>
constexpr int part_vecs() { return FP32 ? 4 : 8; }
struct PartsArgs {
    RowsArgs r;
    Sum* sums;               // [rows, parts]
    float* logits;           // [rows]: of the tokens
    uint32_t parts;
    int32_t part;            // values
};
__device__ __forceinline__ bool counts(const PartsArgs& a, uint32_t row, int64_t token, float* w) {
    *w = a.r.policy.in.weights ? a.r.policy.in.weights[row] : 1.0f;
    return token >= 0 && *w != 0.0f;
}

template <bool FP32>
__global__ __launch_bounds__(kPartThreads) void parts_kernel(PartsArgs a) {
    const uint32_t row = blockIdx.x / a.parts, part = blockIdx.x % a.parts;
    const int64_t token = a.r.tokens[row];
    float w;
    if (!counts(a, row, token, &w)) return;
    const char* x = row_of<FP32>(a.r.x, row);
    const int32_t begin = (int32_t)part * a.part, end = min(a.r.x.vocab, begin + a.part);
    Held<FP32, kPartThreads, part_vecs<FP32>()> h;
    h.load(x, begin, end, (int)threadIdx.x);
    if (part == 0 && threadIdx.x == 0) a.logits[row] = logit_of<FP32>(x, token, a.r.x.vocab);
    const Sum s = join_waves<kPartThreads / 64>(h.wave_part(a.r.c), a.r.c);
    if (threadIdx.x == 0) a.sums[(int64_t)row * a.parts + part] = s;
}

// A row's sum from its parts', by a wavefront, in every lane.
__device__ __forceinline__ Sum join_parts(const PartsArgs& a, uint32_t row) {
    const Sum* parts = a.sums + (int64_t)row * a.parts;
    Sum s = {0.0, minus_inf()};
    for (uint32_t i = threadIdx.x & 63; i < a.parts; i += 64) s = join(s, parts[i], a.r.c);
    const float most = wave_max(s.most);
    return {wave_sum(s.sum * (double)exp2_of((s.most - base_of(most)) * a.r.c)), most};
}

constexpr int kJoinRows = 4;
__global__ __launch_bounds__(kJoinRows * 64) void logprob_join_kernel(PartsArgs a) {
    const uint32_t row = blockIdx.x * kJoinRows + (threadIdx.x >> 6);
    if (row >= a.r.rows) return;
    RowLog l = {0.0, 0.0, 0.0};
    if (a.r.tokens[row] >= 0) l = row_log(join_parts(a, row), a.logits[row], a.r.inv_t);
    if (threadIdx.x & 63) return;
    if (a.r.logprob) a.r.logprob[row] = (float)l.logprob;
    if (a.r.lse) a.r.lse[row] = (float)l.lse;
}

// The gradient of a part.  Every workgroup joins its row's sums and computes the row's slope for itself; the first of a row leaves what is kept of it.
template <bool FP32>
__global__ __launch_bounds__(kPartThreads) void policy_parts_kernel(PartsArgs a) {
    const uint32_t row = blockIdx.x / a.parts, part = blockIdx.x % a.parts;
    const int64_t token = a.r.tokens[row];
    float w;
    const bool there = counts(a, row, token, &w);
    char* dx = a.r.dx ? a.r.dx + (int64_t)row * a.r.dx_stride * (FP32 ? 4 : 2) : nullptr;
    const int32_t begin = (int32_t)part * a.part, end = min(a.r.x.vocab, begin + a.part);
    Held<FP32, kPartThreads, part_vecs<FP32>()> h;
    h.begin = begin; h.end = end; h.lane = (int)threadIdx.x;
    if (there && dx) h.load(row_of<FP32>(a.r.x, row), begin, end, (int)threadIdx.x);
    Sum s = {1.0, 0.0f};
    RowLog l = {0.0, 0.0, 0.0};
    PolicyRow p = {};
    if (there) {
        s = join_parts(a, row);
        l = row_log(s, a.logits[row], a.r.inv_t);
        p = policy_row(a.r.policy, row, l.logprob, w);
    }
    if (part == 0 && threadIdx.x == 0) {
        if (a.r.logprob) a.r.logprob[row] = (float)l.logprob;
        put_terms(a.r.policy, a.r.rows, row, p);
    }
    if (!dx) return;
    const float d = p.slope * a.r.scale;
    if (d == 0.0f) h.store_zeros(dx);
    else h.store_gradient(dx, token, d, base_of(s.most), a.r.c, (float)(l.log_sum * kLog2e));
}

// ---- the gradient of the logits from the lse of an earlier call
struct GradArgs {
    Logits x;
    char* dx;
    int64_t stride;
    const int64_t* tokens;
    const float *lse, *slope;
    float scale, c;          // of the slopes
    uint32_t parts;
    int32_t part;
};
template <bool FP32, bool NARROW>
__global__ __launch_bounds__(kPartThreads) void gradient_kernel(GradArgs a) {
    const uint32_t row = blockIdx.x / a.parts, part = blockIdx.x % a.parts;
    char* dx = a.dx + (int64_t)row * a.stride * (FP32 ? 4 : 2);
    const int32_t begin = (int32_t)part * a.part, end = min(a.x.vocab, begin + a.part);
    const int64_t token = a.tokens[row];
    float d = token < 0 ? 0.0f : a.slope[row] * a.scale;
    Held<FP32, kPartThreads, NARROW ? 1 : part_vecs<FP32>(), NARROW> h;
    if (d == 0.0f) {
        h.begin = begin; h.end = end; h.lane = (int)threadIdx.x;
        h.store_zeros(dx);
        return;
    }
    if (token >= a.x.vocab) d = __builtin_nanf("");
    const float shift = a.lse[row] * (float)kLog2e;
    h.load(row_of<FP32>(a.x, row), begin, end, (int)threadIdx.x);
    h.store_gradient(dx, token, d, 0.0f, a.c, shift);
}

// The sum over a workgroup, in every lane, in a fixed order.
template <int THREADS>
__device__ __forceinline__ double group_sum(double s) {
    __shared__ double part[THREADS / 64];
    s = wave_sum(s);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = s;
    __syncthreads();
    s = 0.0;
#pragma unroll
    for (int k = 0; k < THREADS / 64; ++k) s += part[k];
    return s;
}

__global__ __launch_bounds__(kPairThreads) void policy_stats_kernel(const double* terms, uint32_t rows, float kl_weight, float* stats) {
    double s[3] = {};
    for (uint32_t i = threadIdx.x; i < rows; i += kPairThreads)
        for (int k = 0; k < 3; ++k) s[k] += terms[(int64_t)k * rows + i];
    for (int k = 0; k < 3; ++k) s[k] = group_sum<kPairThreads>(s[k]);
    if (threadIdx.x == 0) {
        stats[0] = (float)(s[0] + (double)kl_weight * s[1]);
        for (int k = 0; k < 3; ++k) stats[1 + k] = (float)s[k];
    }
}

struct PairArgs {
    const float *logprob, *ref, *weights;
    const int64_t* offsets;
    float *loss, *margins, *dlogprob;
    int64_t rows, pairs;
    flashoptim_preference_spec spec;
};

__device__ __forceinline__ double softplus(double z) { return fmax(z, 0.0) + log1p(exp(-fabs(z))); }

// One workgroup for all pairs, so that the loss needs no second launch: there are a few bytes for each row of logits.
__global__ __launch_bounds__(kPairThreads) void preference_kernel(PairArgs a) {
    const auto bound = [&](int64_t i) { return min(max(a.offsets[i], (int64_t)0), a.rows); };
    const bool by_turns = a.spec.order == FLASHOPTIM_PAIRS_BY_TURNS;
    const double beta = a.spec.beta, e = a.spec.label_smoothing;
    double total = 0.0;
    for (int64_t p = 0; p < a.pairs; ++p) {
        const int64_t of[2] = {by_turns ? 2 * p : p, by_turns ? 2 * p + 1 : a.pairs + p};
        double gain = 0.0;
        for (int k = 0; k < 2; ++k) {
            const int64_t end = bound(of[k] + 1);
            double s = 0.0;
            for (int64_t i = bound(of[k]) + threadIdx.x; i < end; i += kPairThreads) {
                const float w = a.weights ? a.weights[i] : 1.0f;
                if (w != 0.0f) s += (double)w * ((double)a.logprob[i] - (a.ref ? (double)a.ref[i] : 0.0));
            }
            s = group_sum<kPairThreads>(s);
            gain += k ? -s : s;
        }
        const double z = beta * gain;
        double loss, d;
        if (a.spec.kind == FLASHOPTIM_PREFERENCE_SIGMOID) {
            loss = (1.0 - e) * softplus(-z) + (e > 0.0 ? e * softplus(z) : 0.0);      // (z may be infinite)
            d = e / (1.0 + exp(-z)) - (1.0 - e) / (1.0 + exp(z));
        } else if (a.spec.kind == FLASHOPTIM_PREFERENCE_HINGE) {
            loss = z < 1.0 ? 1.0 - z : z >= 1.0 ? 0.0 : z;                          // (z may be NaN)
            d = z < 1.0 ? -1.0 : z >= 1.0 ? 0.0 : z;
        } else {
            const double r = gain - 0.5 / beta;
            loss = r * r;
            d = 2.0 * r / beta;
        }
        total += loss;
        if (threadIdx.x == 0 && a.margins) a.margins[p] = (float)z;
        if (a.dlogprob) {
            d *= beta * (double)a.spec.grad_scale / (double)a.pairs;
            for (int k = 0; k < 2; ++k) {
                const int64_t end = bound(of[k] + 1);
                for (int64_t i = bound(of[k]) + threadIdx.x; i < end; i += kPairThreads) {
                    const float w = a.weights ? a.weights[i] : 1.0f;
                    a.dlogprob[i] = w == 0.0f ? 0.0f : (float)((k ? -d : d) * w);
                }
            }
        }
    }
    if (a.dlogprob) {
        const int64_t first = a.pairs ? bound(0) : a.rows, last = a.pairs ? bound(2 * a.pairs) : a.rows;
        for (int64_t i = threadIdx.x; i < first; i += kPairThreads) a.dlogprob[i] = 0.0f;
        for (int64_t i = last + threadIdx.x; i < a.rows; i += kPairThreads) a.dlogprob[i] = 0.0f;
    }
    if (threadIdx.x == 0) *a.loss = a.pairs ? (float)(total / (double)a.pairs) : 0.0f;
}

// --------------------------------------------------------------------------------------------------- host --

int check_sizes(int64_t rows, int64_t vocab) {
    if (rows < 0 || vocab < 0) return FLASHOPTIM_ERR_INVALID_ARG;
    if (rows >= ((int64_t)1 << 31) || vocab >= ((int64_t)1 << 30)) return FLASHOPTIM_ERR_NUMEL_RANGE;
    return FLASHOPTIM_OK;
}
int check_logits(const flashoptim_matrix* logits, const int64_t* tokens, float temperature) {
    FO_TRY(fo::check_matrix(logits));
    FO_TRY(check_sizes(logits->rows, logits->cols));
    if (!(temperature > 0.0f) || !std::isfinite(temperature) || !std::isfinite((float)(kLog2e / (double)temperature)) ||
        !std::isfinite(1.0f / temperature))
        return FLASHOPTIM_ERR_INVALID_ARG;
    if (logits->rows == 0) return FLASHOPTIM_OK;
    if (logits->cols == 0 || !tokens) return FLASHOPTIM_ERR_INVALID_ARG;
    return fo::aligned_to(tokens, 8) ? FLASHOPTIM_OK : FLASHOPTIM_ERR_MISALIGNED;
}
int check_gradient(const flashoptim_matrix* d, const flashoptim_matrix* logits) {
    if (!d) return FLASHOPTIM_OK;
    FO_TRY(fo::check_matrix(d));
    if (d->rows != logits->rows || d->cols != logits->cols || d->dtype != logits->dtype) return FLASHOPTIM_ERR_INVALID_ARG;
    if (d->data == logits->data && d->rows > 1 && d->stride != logits->stride) return FLASHOPTIM_ERR_INVALID_ARG;
    return FLASHOPTIM_OK;
}
Logits to_dev(const flashoptim_matrix* m) { return {(const char*)m->data, m->rows > 1 ? m->stride : 0, (int32_t)m->cols}; }

// How a row is cut: into parts of as many values as a workgroup holds, or of fewer where there are few rows, so that all compute units have one.
constexpr int64_t kHeldPart[2] = {kPartThreads * 8 * part_vecs<false>(), kPartThreads * 8 * part_vecs<true>()};     // by dtype
constexpr int64_t kLeastPart = 2048;
struct Parts {
    int32_t part;
    uint32_t parts;
};
Parts cut_rows(int64_t rows, int64_t vocab, int dtype) {
    int64_t part = kHeldPart[dtype];
    while (part > kLeastPart && rows * up(vocab, part) < 512) part /= 2;
    return {(int32_t)part, (uint32_t)up(vocab, part)};
}
bool known(int dtype) { return dtype == FLASHOPTIM_BF16 || dtype == FLASHOPTIM_FP32; }

// Calls launch(fp32, narrow) with the two as types.
template <typename F>
void with_types(bool fp32, bool narrow, F launch) {
    using Yes = std::true_type;
    using No = std::false_type;
    if (fp32) { if (narrow) launch(Yes{}, Yes{}); else launch(Yes{}, No{}); }
    else { if (narrow) launch(No{}, Yes{}); else launch(No{}, No{}); }
}

// Calls launch(shape) with the shape of the workgroups that hold rows of this many values, false if there is none.
template <int LANES, int NV, bool NARROW = false>
struct Shape {
    static constexpr int kLanes = LANES, kVecs = NV;
    static constexpr bool kNarrow = NARROW;
};
template <bool FP32, typename F>
bool with_held(int64_t vocab, F launch) {
    constexpr int K = FP32 ? 2 : 1;        // (eight FP32 values are twice the registers)
    if (vocab < 8) launch(Shape<64, 1, true>{});
    else if (vocab <= 64 * 8 * 4 / K) launch(Shape<64, 4 / K>{});
    else if (vocab <= 64 * 8 * 8 / K) launch(Shape<64, 8 / K>{});
    else if (vocab <= 256 * 8 * 8 / K) launch(Shape<256, 8 / K>{});
    else if (vocab <= 512 * 8 * 8 / K) launch(Shape<512, 8 / K>{});
    else if (vocab <= 512 * 8 * 16 / K) launch(Shape<512, 16 / K>{});
    else if (vocab <= 1024 * 8 * 16 / K) launch(Shape<1024, 16 / K>{});
    else return false;
    return true;
}
// Whether a call holds whole rows: those of a wavefront always, longer ones where there are as many as fill half the chip.
bool holds_rows(int64_t rows, int64_t vocab, int dtype) {
    const int64_t k = dtype == FLASHOPTIM_FP32 ? 2 : 1;
    return vocab <= 4096 / k || (vocab <= 131072 / k && rows >= 128);
}
bool streams_rows(int64_t rows, int64_t vocab) { return vocab <= 4096 || rows >= 512; }

int launch_parts(const PartsArgs& p, int dtype, void* stream) {
    const dim3 grid(p.r.rows * p.parts), block(kPartThreads);
    if (dtype == FLASHOPTIM_FP32) hipLaunchKernelGGL(parts_kernel<true>, grid, block, 0, (hipStream_t)stream, p);
    else hipLaunchKernelGGL(parts_kernel<false>, grid, block, 0, (hipStream_t)stream, p);
    return fo::hip_status(hipGetLastError());
}
// A call's parts in its workspace.
PartsArgs to_parts(const RowsArgs& a, const Parts& c, void* workspace) {
    PartsArgs p = {a, (Sum*)workspace, nullptr, c.parts, c.part};
    p.logits = (float*)(p.sums + (int64_t)a.rows * c.parts);
    return p;
}
int64_t parts_bytes(int64_t rows, const Parts& c) { return up(rows * (int64_t)c.parts * (int64_t)sizeof(Sum) + rows * 4, 16) * 16; }

template <bool FP32>
int launch_held(const RowsArgs& a, void* stream) {
    with_held<FP32>(a.x.vocab, [&](auto shape) {
        constexpr int L = decltype(shape)::kLanes, NV = decltype(shape)::kVecs, LINES = L < 256 ? 256 / L : 1;
        hipLaunchKernelGGL((policy_rows_kernel<FP32, L, NV, decltype(shape)::kNarrow>), dim3((unsigned)up(a.rows, LINES)), dim3(L * LINES), 0, (hipStream_t)stream, a);
    });
    return fo::hip_status(hipGetLastError());
}

int check_launch(const flashoptim_matrix* logits) {
    const int64_t blocks = logits->rows * (int64_t)cut_rows(logits->rows, logits->cols, logits->dtype).parts;
    return blocks > fo::kMaxWorkItems / kPartThreads || logits->rows > fo::kMaxWorkItems / 1024 ? FLASHOPTIM_ERR_NUMEL_RANGE : FLASHOPTIM_OK;
}
int check_workspace(int64_t need, const void* workspace, int64_t bytes) {
    if (need < 0) return (int)need;
    if (need > 0 && !workspace) return FLASHOPTIM_ERR_INVALID_ARG;
    if (bytes < need) return FLASHOPTIM_ERR_WORKSPACE;
    return fo::aligned_to(workspace, 16) ? FLASHOPTIM_OK : FLASHOPTIM_ERR_MISALIGNED;
}
RowsArgs rows_args(const flashoptim_matrix* logits, const int64_t* tokens, float temperature) {
    RowsArgs a = {};
    a.x = to_dev(logits);
    a.tokens = tokens;
    a.inv_t = 1.0 / (double)temperature;
    a.c = (float)(kLog2e / (double)temperature);
    a.scale = 1.0f / temperature;
    a.rows = (uint32_t)logits->rows;
    return a;
}

}  // namespace

extern "C" {

int64_t flashoptim_token_logprob_workspace(int64_t rows, int64_t vocab, int dtype) {
    if (!known(dtype)) return FLASHOPTIM_ERR_INVALID_ARG;
    FO_TRY(check_sizes(rows, vocab));
    return rows == 0 || streams_rows(rows, vocab) ? 0 : parts_bytes(rows, cut_rows(rows, vocab, dtype));
}

int flashoptim_token_logprob(const flashoptim_matrix* logits, const int64_t* tokens, float temperature, float* logprob, float* lse,
                             void* workspace, int64_t workspace_bytes, void* stream) {
    FO_TRY(check_logits(logits, tokens, temperature));
    const int64_t rows = logits->rows;
    if (rows == 0) return FLASHOPTIM_OK;
    if (!logprob && !lse) return FLASHOPTIM_ERR_INVALID_ARG;
    if (!fo::aligned_to(logprob, 4) || !fo::aligned_to(lse, 4)) return FLASHOPTIM_ERR_MISALIGNED;
    FO_TRY(check_launch(logits));
    FO_TRY(check_workspace(flashoptim_token_logprob_workspace(rows, logits->cols, logits->dtype), workspace, workspace_bytes));
    RowsArgs a = rows_args(logits, tokens, temperature);
    a.logprob = logprob;
    a.lse = lse;
    const bool fp32 = logits->dtype == FLASHOPTIM_FP32;
    if (streams_rows(rows, logits->cols)) {
        with_types(fp32, logits->cols < 8, [&](auto f, auto narrow) {
            hipLaunchKernelGGL((logprob_rows_kernel<decltype(f)::value, 4, decltype(narrow)::value>), dim3(a.rows), dim3(256), 0, (hipStream_t)stream, a);
        });
        return fo::hip_status(hipGetLastError());
    }
    const PartsArgs p = to_parts(a, cut_rows(rows, logits->cols, logits->dtype), workspace);
    FO_TRY(launch_parts(p, logits->dtype, stream));
    hipLaunchKernelGGL(logprob_join_kernel, dim3((unsigned)up(rows, kJoinRows)), dim3(kJoinRows * 64), 0, (hipStream_t)stream, p);
    return fo::hip_status(hipGetLastError());
}

int flashoptim_token_logprob_backward(const flashoptim_matrix* logits, const int64_t* tokens, float temperature, const float* lse,
                                      const float* dlogprob, const flashoptim_matrix* dlogits, void* stream) {
    FO_TRY(check_logits(logits, tokens, temperature));
    if (!dlogits) return FLASHOPTIM_ERR_INVALID_ARG;
    FO_TRY(check_gradient(dlogits, logits));
    if (logits->rows == 0) return FLASHOPTIM_OK;
    if (!lse || !dlogprob) return FLASHOPTIM_ERR_INVALID_ARG;
    if (!fo::aligned_to(lse, 4) || !fo::aligned_to(dlogprob, 4)) return FLASHOPTIM_ERR_MISALIGNED;
    FO_TRY(check_launch(logits));
    const Parts c = cut_rows(logits->rows, logits->cols, logits->dtype);
    const GradArgs g = {to_dev(logits), (char*)dlogits->data, dlogits->rows > 1 ? dlogits->stride : 0, tokens, lse, dlogprob, 1.0f / temperature,
                        (float)(kLog2e / (double)temperature), c.parts, c.part};
    const dim3 grid((unsigned)(logits->rows * (int64_t)c.parts)), block(kPartThreads);
    with_types(logits->dtype == FLASHOPTIM_FP32, logits->cols < 8, [&](auto f, auto narrow) {
        hipLaunchKernelGGL((gradient_kernel<decltype(f)::value, decltype(narrow)::value>), grid, block, 0, (hipStream_t)stream, g);
    });
    return fo::hip_status(hipGetLastError());
}

int64_t flashoptim_policy_loss_workspace(int64_t rows, int64_t vocab, int dtype) {
    if (!known(dtype)) return FLASHOPTIM_ERR_INVALID_ARG;
    FO_TRY(check_sizes(rows, vocab));
    const int64_t terms = up(rows * 24, 16) * 16;
    return terms + (rows == 0 || holds_rows(rows, vocab, dtype) ? 0 : parts_bytes(rows, cut_rows(rows, vocab, dtype)));
}

int flashoptim_policy_loss(const flashoptim_policy_spec* spec, const flashoptim_matrix* logits, const int64_t* tokens,
                           const flashoptim_policy_inputs* inputs, float* stats, float* logprob, const flashoptim_matrix* dlogits,
                           void* workspace, int64_t workspace_bytes, void* stream) {
    if (!spec || !inputs || !stats) return FLASHOPTIM_ERR_INVALID_ARG;
    FO_TRY(check_logits(logits, tokens, spec->temperature));
    if (!(spec->clip_low >= 0.0f) || !(spec->clip_high >= 0.0f) || !(spec->kl_weight >= 0.0f) || !std::isfinite(spec->clip_low) ||
        !std::isfinite(spec->kl_weight))
        return FLASHOPTIM_ERR_INVALID_ARG;
    FO_TRY(check_gradient(dlogits, logits));
    FO_TRY(check_launch(logits));
    const int64_t rows = logits->rows;
    if (rows > 0 && !inputs->advantages) return FLASHOPTIM_ERR_INVALID_ARG;
    for (const float* p : {inputs->advantages, inputs->old_logprob, inputs->ref_logprob, inputs->weights, (const float*)stats, (const float*)logprob})
        if (!fo::aligned_to(p, 4)) return FLASHOPTIM_ERR_MISALIGNED;
    FO_TRY(check_workspace(flashoptim_policy_loss_workspace(rows, logits->cols, logits->dtype), workspace, workspace_bytes));
    RowsArgs a = rows_args(logits, tokens, spec->temperature);
    a.logprob = logprob;
    a.policy = {*spec, *inputs, (double*)workspace};
    if (dlogits) {
        a.dx = (char*)dlogits->data;
        a.dx_stride = rows > 1 ? dlogits->stride : 0;
    }
    const bool fp32 = logits->dtype == FLASHOPTIM_FP32;
    if (rows > 0 && holds_rows(rows, logits->cols, logits->dtype)) {
        FO_TRY(fp32 ? launch_held<true>(a, stream) : launch_held<false>(a, stream));
    } else if (rows > 0) {
        const PartsArgs p = to_parts(a, cut_rows(rows, logits->cols, logits->dtype), (char*)workspace + up(rows * 24, 16) * 16);
        FO_TRY(launch_parts(p, logits->dtype, stream));
        const dim3 grid(p.r.rows * p.parts), block(kPartThreads);
        if (fp32) hipLaunchKernelGGL(policy_parts_kernel<true>, grid, block, 0, (hipStream_t)stream, p);
        else hipLaunchKernelGGL(policy_parts_kernel<false>, grid, block, 0, (hipStream_t)stream, p);
        FO_TRY(fo::hip_status(hipGetLastError()));
    }
    hipLaunchKernelGGL(policy_stats_kernel, dim3(1), dim3(kPairThreads), 0, (hipStream_t)stream, a.policy.terms, a.rows, spec->kl_weight, stats);
    return fo::hip_status(hipGetLastError());
}

int flashoptim_preference_loss(const flashoptim_preference_spec* spec, const float* logprob, const float* ref_logprob,
                               const float* weights, int64_t rows, const int64_t* offsets, int64_t pairs, float* loss, float* margins,
                               float* dlogprob, void* stream) {
    if (!spec || !loss || rows < 0 || pairs < 0 || spec->kind < 0 || spec->kind > 2 || spec->order < 0 || spec->order > 1)
        return FLASHOPTIM_ERR_INVALID_ARG;
    if (!(spec->beta > 0.0f) || !std::isfinite(spec->beta) || !(spec->label_smoothing >= 0.0f && spec->label_smoothing <= 0.5f) ||
        (spec->label_smoothing != 0.0f && spec->kind != FLASHOPTIM_PREFERENCE_SIGMOID))
        return FLASHOPTIM_ERR_INVALID_ARG;
    if (rows >= ((int64_t)1 << 31) || pairs >= ((int64_t)1 << 30)) return FLASHOPTIM_ERR_NUMEL_RANGE;
    if ((rows > 0 && !logprob) || (pairs > 0 && !offsets)) return FLASHOPTIM_ERR_INVALID_ARG;
    for (const float* p : {logprob, ref_logprob, weights, (const float*)loss, (const float*)margins, (const float*)dlogprob})
        if (!fo::aligned_to(p, 4)) return FLASHOPTIM_ERR_MISALIGNED;
    if (!fo::aligned_to(offsets, 8)) return FLASHOPTIM_ERR_MISALIGNED;
    const PairArgs a = {logprob, ref_logprob, weights, offsets, loss, margins, dlogprob, rows, pairs, *spec};
    hipLaunchKernelGGL(preference_kernel, dim3(1), dim3(kPairThreads), 0, (hipStream_t)stream, a);
    return fo::hip_status(hipGetLastError());
}

}  // extern "C"
