// The losses on the logits and their gradients, for gfx950: log-probabilities of tokens, the clipped policy loss, the preference loss.
//
// By row of logits x with the token t and temperature T:   lse = log sum_j exp(x_j / T),  logprob = x_t / T - lse,  and with d the loss's gradient
// with respect to logprob:   dx_j = d / T ([j = t] - exp(x_j / T - lse)).
// Exponentials are powers of two of (x - m) log2(e) / T with m the row's largest value (the difference first: logits of the type's lowest value, as
// masks set them, stay finite).  Bound: HBM; a row costs two exponentials an element.

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <cmath>

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

constexpr double kLog2e = 1.4426950408889634, kLn2 = 0.6931471805599453;
constexpr int kRowThreads = 256;
constexpr int kPairThreads = 1024;

// A matrix of logits as a kernel takes it.
struct Logits {
    const char* data;
    int64_t stride;      // values
    int32_t vocab;
};
struct Row {
    const char* data;
    int32_t vocab;
};
template <bool FP32>
__device__ __forceinline__ Row row_of(const Logits& m, uint32_t row) {
    return {m.data + (int64_t)row * m.stride * (FP32 ? 4 : 2), m.vocab};
}
template <bool FP32>
__device__ __forceinline__ float value_at(const char* row, int32_t j) {
    return FP32 ? ((const float*)row)[j] : __uint_as_float((uint32_t)((const uint16_t*)row)[j] << 16);
}
template <bool FP32>
__device__ __forceinline__ f32x8 load8(const char* row, int32_t j) {
    f32x8 v;
    if constexpr (FP32) {
        const f32x4 a = load_as<f32x4>(row + (int64_t)j * 4), b = load_as<f32x4>(row + (int64_t)j * 4 + 16);
#pragma unroll
        for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[4 + i] = b[i]; }
    } else {
        const i32x4 a = load_as<i32x4>(row + (int64_t)j * 2);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float((uint32_t)a[i] << 16);
            v[2 * i + 1] = __uint_as_float((uint32_t)a[i] & 0xffff0000u);
        }
    }
    return v;
}
template <bool FP32>
__device__ __forceinline__ void store8(char* row, int32_t j, f32x8 v) {
    if constexpr (FP32) {
        store_as(row + (int64_t)j * 4, f32x4{v[0], v[1], v[2], v[3]});
        store_as(row + (int64_t)j * 4 + 16, f32x4{v[4], v[5], v[6], v[7]});
    } else {
        store_as(row + (int64_t)j * 2, __builtin_convertvector(v, bf16x8));
    }
}
template <bool FP32>
__device__ __forceinline__ void store1(char* row, int32_t j, float v) {
    if constexpr (FP32) ((float*)row)[j] = v;
    else ((__bf16*)row)[j] = (__bf16)v;
}

__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

// A part of a row's sum of exponentials: its largest value, and the sum of 2^((x - most) c).
struct Sum {
    float most, sum;
};
// What the difference to a largest value is taken from: where there is none yet, any finite value will do.
__device__ __forceinline__ float base_of(float most) { return most == -__builtin_inff() ? 0.0f : most; }

template <int N, typename V>
__device__ __forceinline__ void add_values(Sum& s, const V& v, float c) {
    float most = s.most;
#pragma unroll
    for (int i = 0; i < N; ++i) most = fmaxf(most, v[i]);
    const float base = base_of(most);
    float sum = s.sum * exp2_of((s.most - base) * c);
#pragma unroll
    for (int i = 0; i < N; ++i) sum += exp2_of((v[i] - base) * c);
    s = {most, sum};
}

// The whole row's, in every lane: the largest value, and the sum in FP64, from the lanes' in a fixed order.
template <int THREADS>
__device__ __forceinline__ double join_lanes(Sum s, float c, float* most) {
    __shared__ float largest[THREADS / 64];
    __shared__ double sums[THREADS / 64];
    const int wave = (int)threadIdx.x >> 6;
    float m = s.most;
    for (int off = 32; off > 0; off >>= 1) m = fmaxf(m, __shfl_xor(m, off));
    if ((threadIdx.x & 63) == 0) largest[wave] = m;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < THREADS / 64; ++k) m = fmaxf(m, largest[k]);
    double d = (double)(s.sum * exp2_of((s.most - base_of(m)) * c));
    for (int off = 32; off > 0; off >>= 1) d += __shfl_xor(d, off);
    if ((threadIdx.x & 63) == 0) sums[wave] = d;
    __syncthreads();
    d = 0.0;
#pragma unroll
    for (int k = 0; k < THREADS / 64; ++k) d += sums[k];
    *most = m;
    return d;
}

// log sum exp(x / T) and the token's log-probability, in FP64.
struct RowLog {
    double lse, logprob, log_sum;     // log_sum: what lse is beyond the largest value
};
__device__ __forceinline__ RowLog row_log(float most, double sum, float x, double inv_t) {
    const double log_sum = log(sum);
    return {(double)most * inv_t + log_sum, ((double)x - (double)most) * inv_t - log_sum, log_sum};
}

struct RowsArgs {
    Logits x;
    const int64_t* tokens;
    float *logprob, *lse;
    double inv_t;
    float c;
    // policy loss
    flashoptim_policy_spec spec;
    flashoptim_policy_inputs in;
    float *slope, *most, *log_sum;
    double* terms;       // [3, rows]
    uint32_t rows;
    bool policy;
};

// One workgroup to a row.
template <bool FP32>
__global__ __launch_bounds__(kRowThreads) void rows_kernel(RowsArgs a) {
    const uint32_t row = blockIdx.x;
    const int64_t token = a.tokens[row];
    const float w = a.policy && a.in.weights ? a.in.weights[row] : 1.0f;
    if (token < 0 || w == 0.0f) {
        if (threadIdx.x == 0) {
            if (a.logprob) a.logprob[row] = 0.0f;
            if (a.lse) a.lse[row] = 0.0f;
            if (a.policy) {
                a.slope[row] = 0.0f;
                for (int k = 0; k < 3; ++k) a.terms[(int64_t)k * a.rows + row] = 0.0;
            }
        }
        return;
    }
    const Row r = row_of<FP32>(a.x, row);
    const int32_t whole = r.vocab & ~7;
    Sum s = {-__builtin_inff(), 0.0f};
    for (int32_t j = (int32_t)threadIdx.x * 8; j < whole; j += kRowThreads * 8) add_values<8>(s, load8<FP32>(r.data, j), a.c);
    if ((int32_t)threadIdx.x < r.vocab - whole) {
        const float v[1] = {value_at<FP32>(r.data, whole + (int32_t)threadIdx.x)};
        add_values<1>(s, v, a.c);
    }
    float most;
    const double sum = join_lanes<kRowThreads>(s, a.c, &most);
    if (threadIdx.x != 0) return;
    const float x = token < r.vocab ? value_at<FP32>(r.data, (int32_t)token) : __builtin_nanf("");
    const RowLog l = row_log(most, sum, x, a.inv_t);
    if (a.logprob) a.logprob[row] = (float)l.logprob;
    if (a.lse) a.lse[row] = (float)l.lse;
    if (!a.policy) return;
    const double adv = a.in.advantages[row];
    const double ratio = a.in.old_logprob ? exp(l.logprob - (double)a.in.old_logprob[row]) : l.logprob - l.logprob + 1.0;
    const double low = 1.0 - (double)a.spec.clip_low, high = 1.0 + (double)a.spec.clip_high;
    const bool blocked = (adv > 0.0 && ratio > high) || (adv < 0.0 && ratio < low);
    const double surrogate = blocked ? -adv * (adv > 0.0 ? high : low) : -adv * ratio;
    double slope = blocked ? 0.0 : -adv * ratio, kl = 0.0;
    if (a.in.ref_logprob) {
        const double d = (double)a.in.ref_logprob[row] - l.logprob;
        kl = expm1(d) - d;
        slope -= a.spec.kl_weight * expm1(d);
    }
    a.slope[row] = (float)(slope * w);
    a.most[row] = most;
    a.log_sum[row] = (float)l.log_sum;
    a.terms[row] = surrogate * w;
    a.terms[(int64_t)a.rows + row] = kl * w;
    a.terms[2 * (int64_t)a.rows + row] = blocked ? w : 0.0;
}

struct GradArgs {
    Logits x;
    char* dx;
    int64_t stride;
    const int64_t* tokens;
    const float *most, *log_sum, *slope;     // exp(x / T - lse) = exp((x - most) / T - log_sum); most NULL: 0
    float scale;         // of the slopes
    float c;
    uint32_t segments;
};
constexpr int32_t kSegment = 8192;

template <bool FP32>
__global__ __launch_bounds__(kRowThreads) void gradient_kernel(GradArgs a) {
    const uint32_t row = blockIdx.x / a.segments, segment = blockIdx.x % a.segments;
    const Row r = row_of<FP32>(a.x, row);
    char* dx = a.dx + (int64_t)row * a.stride * (FP32 ? 4 : 2);
    const int32_t begin = (int32_t)segment * kSegment, end = min(r.vocab, begin + kSegment), whole = end & ~7;
    const int64_t token = a.tokens[row];
    float d = token < 0 ? 0.0f : a.slope[row] * a.scale;
    if (token >= r.vocab && d != 0.0f) d = __builtin_nanf("");
    const float shift = d == 0.0f ? 0.0f : a.log_sum[row] * (float)kLog2e, most = a.most && d != 0.0f ? a.most[row] : 0.0f;
    auto of = [&](float x, int32_t j) { return d == 0.0f ? 0.0f : d * ((j == token ? 1.0f : 0.0f) - exp2_of(fmaf(x - most, a.c, -shift))); };
    for (int32_t j = begin + (int32_t)threadIdx.x * 8; j < whole; j += kRowThreads * 8) {
        f32x8 v = {};
        if (d != 0.0f) v = load8<FP32>(r.data, j);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = of(v[i], j + i);
        store8<FP32>(dx, j, v);
    }
    const int32_t j = whole + (int32_t)threadIdx.x;
    if (j < end) store1<FP32>(dx, j, of(d == 0.0f ? 0.0f : value_at<FP32>(r.data, j), j));
}

// The sum over a workgroup, in every lane, in a fixed order.
template <int THREADS>
__device__ __forceinline__ double group_sum(double s) {
    __shared__ double part[THREADS / 64];
    for (int off = 32; off > 0; off >>= 1) s += __shfl_xor(s, off);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = s;
    __syncthreads();
    s = 0.0;
#pragma unroll
    for (int k = 0; k < THREADS / 64; ++k) s += part[k];
    return s;
}

__global__ __launch_bounds__(kPairThreads) void policy_stats_kernel(const double* terms, uint32_t rows, float kl_weight, float* stats) {
    double s[3];
    for (int k = 0; k < 3; ++k) {
        double v = 0.0;
        for (uint32_t i = threadIdx.x; i < rows; i += kPairThreads) v += terms[(int64_t)k * rows + i];
        s[k] = group_sum<kPairThreads>(v);
    }
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
    if (rows >= ((int64_t)1 << 31) || vocab >= ((int64_t)1 << 31) - 4096) return FLASHOPTIM_ERR_NUMEL_RANGE;
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

int launch_rows(const RowsArgs& a, int dtype, void* stream) {
    if (dtype == FLASHOPTIM_FP32) hipLaunchKernelGGL(rows_kernel<true>, dim3(a.rows), dim3(kRowThreads), 0, (hipStream_t)stream, a);
    else hipLaunchKernelGGL(rows_kernel<false>, dim3(a.rows), dim3(kRowThreads), 0, (hipStream_t)stream, a);
    return fo::hip_status(hipGetLastError());
}

int launch_gradient(const flashoptim_matrix* logits, const int64_t* tokens, float temperature, const float* most, const float* log_sum,
                    const float* slope, float scale, const flashoptim_matrix* d, void* stream) {
    GradArgs g = {to_dev(logits), (char*)d->data, d->rows > 1 ? d->stride : 0, tokens, most, log_sum, slope, scale / temperature,
                  (float)(kLog2e / (double)temperature), (uint32_t)up(logits->cols, kSegment)};
    const int64_t blocks = logits->rows * (int64_t)g.segments;
    if (blocks > fo::kMaxWorkItems / kRowThreads) return FLASHOPTIM_ERR_NUMEL_RANGE;
    if (logits->dtype == FLASHOPTIM_FP32)
        hipLaunchKernelGGL(gradient_kernel<true>, dim3((unsigned)blocks), dim3(kRowThreads), 0, (hipStream_t)stream, g);
    else
        hipLaunchKernelGGL(gradient_kernel<false>, dim3((unsigned)blocks), dim3(kRowThreads), 0, (hipStream_t)stream, g);
    return fo::hip_status(hipGetLastError());
}
int check_launch(const flashoptim_matrix* logits) {
    const int64_t blocks = logits->rows * up(logits->cols, kSegment);
    return blocks > fo::kMaxWorkItems / kRowThreads ? FLASHOPTIM_ERR_NUMEL_RANGE : FLASHOPTIM_OK;
}

}  // namespace

extern "C" {

int64_t flashoptim_token_logprob_workspace(int64_t rows, int64_t vocab, int dtype) {
    if (dtype != FLASHOPTIM_BF16 && dtype != FLASHOPTIM_FP32) return FLASHOPTIM_ERR_INVALID_ARG;
    FO_TRY(check_sizes(rows, vocab));
    return 0;
}

int flashoptim_token_logprob(const flashoptim_matrix* logits, const int64_t* tokens, float temperature, float* logprob, float* lse,
                             void* workspace, int64_t workspace_bytes, void* stream) {
    FO_TRY(check_logits(logits, tokens, temperature));
    (void)workspace; (void)workspace_bytes;
    if (logits->rows == 0) return FLASHOPTIM_OK;
    if (!logprob && !lse) return FLASHOPTIM_ERR_INVALID_ARG;
    if (!fo::aligned_to(logprob, 4) || !fo::aligned_to(lse, 4)) return FLASHOPTIM_ERR_MISALIGNED;
    FO_TRY(check_launch(logits));
    RowsArgs a = {};
    a.x = to_dev(logits); a.tokens = tokens; a.logprob = logprob; a.lse = lse;
    a.inv_t = 1.0 / (double)temperature; a.c = (float)(kLog2e / (double)temperature);
    a.rows = (uint32_t)logits->rows;
    return launch_rows(a, logits->dtype, stream);
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
    return launch_gradient(logits, tokens, temperature, nullptr, lse, dlogprob, 1.0f, dlogits, stream);
}

int64_t flashoptim_policy_loss_workspace(int64_t rows, int64_t vocab, int dtype) {
    FO_TRY(flashoptim_token_logprob_workspace(rows, vocab, dtype));
    return rows * 40;       // three terms (FP64), slope, largest value and log of the sum of every row
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
    const int64_t need = flashoptim_policy_loss_workspace(rows, logits->cols, logits->dtype);
    if (need < 0) return (int)need;
    if (need > 0 && !workspace) return FLASHOPTIM_ERR_INVALID_ARG;
    if (workspace_bytes < need) return FLASHOPTIM_ERR_WORKSPACE;
    if (!fo::aligned_to(workspace, 16)) return FLASHOPTIM_ERR_MISALIGNED;
    RowsArgs a = {};
    a.x = to_dev(logits); a.tokens = tokens; a.logprob = logprob;
    a.inv_t = 1.0 / (double)spec->temperature; a.c = (float)(kLog2e / (double)spec->temperature);
    a.rows = (uint32_t)rows;
    a.spec = *spec; a.in = *inputs; a.policy = true;
    a.terms = (double*)workspace;
    a.slope = (float*)(a.terms + 3 * rows);
    a.most = a.slope + rows;
    a.log_sum = a.most + rows;
    if (rows > 0) FO_TRY(launch_rows(a, logits->dtype, stream));
    if (rows > 0 && dlogits)
        FO_TRY(launch_gradient(logits, tokens, spec->temperature, a.most, a.log_sum, a.slope, spec->grad_scale, dlogits, stream));
    hipLaunchKernelGGL(policy_stats_kernel, dim3(1), dim3(kPairThreads), 0, (hipStream_t)stream, a.terms, a.rows, spec->kl_weight, stats);
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
