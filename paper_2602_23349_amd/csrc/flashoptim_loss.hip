// The losses on the logits and their gradients, for gfx950: log-probabilities of tokens, the clipped policy loss, the preference loss.
//
// By row of logits x with the token t and temperature T:   lse = log sum_j exp(x_j / T),  logprob = x_t / T - lse,  and with d the loss's gradient
// with respect to logprob:   dx_j = d / T ([j = t] - exp(x_j / T - lse)).
// Exponentials are powers of two of (x - m) log2(e) / T with m the row's largest value (the difference first: logits of the type's lowest value, as
// masks set them, stay finite).  Bound: HBM; a row costs two exponentials an element.

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <cmath>
#include <limits>
#include <type_traits>

#include "flashoptim.h"
#include "flashoptim_host.h"
#include "flashoptim_launch.h"
#include "flashoptim_layers.h"

namespace {

using fo::f32x4;
using fo::i32x4;
using fo::load_as;
using fo::sum_of_wave;
using fo::up;
using f32x8 = float __attribute__((ext_vector_type(8)));
using bf16x8 = __bf16 __attribute__((ext_vector_type(8)));

typedef i32x4 anywhere __attribute__((aligned(2)));      // (the hardware takes global accesses at any byte)

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
// A token that is there as its place, one that is not as none that any lane holds.
__device__ __forceinline__ int32_t token_in(int64_t token, int32_t vocab) { return token < vocab ? (int32_t)token : 0x7fffffff; }
template <bool FP32>
__device__ __forceinline__ void put(char* row, int32_t j, float v) {
    if constexpr (FP32) ((float*)row)[j] = v;
    else ((__bf16*)row)[j] = (__bf16)v;
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

// log2(e) / T as the FP32 value below it and what that is short of it.  (The first alone is off by up to 2^-23, which goes into the log-probabilities of a
// sequence with the same sign for every token.)  Both are positive, so that -infinity times the factor is -infinity.
struct Factor {
    float high, low;
};
__device__ __forceinline__ float times(float x, Factor c) { return fmaf(x, c.high, x * c.low); }

// A part of a row: its largest value and the sum of 2^((x - most) c), FP64.
struct Sum {
    double sum;
    float most;
};
__device__ __forceinline__ Sum join(const Sum& a, const Sum& b, Factor c) {
    const float most = fmaxf(a.most, b.most), base = base_of(most);
    return {a.sum * (double)exp2_of(times(a.most - base, c)) + b.sum * (double)exp2_of(times(b.most - base, c)), most};
}

// A word of sixteen bytes: eight BF16 values or four FP32 ones.
template <bool FP32>
constexpr int kValues = FP32 ? 4 : 8;

// What LANES lanes hold of a row in registers.  A row is its words between 16-byte borders of memory and, ahead of the first and behind the last of these, up to
// kN - 1 values each, its edges.  (Words across such borders: log-probabilities of 8192 x 50257 BF16 logits 169 us, so 141.)  Lane l's i-th word is the row's
// first + i LANES + l-th; where there is none the row's last one is loaded, so that no load is a case distinction, and left out of the sum.  The edges belong to the part with the row's first word, a value to a lane.  Logits and gradients go past the caches: each is touched once, and
// there are more of them than the caches hold (with and without: the same log-probabilities 125 and 141 us, the gradient of 4096 x 128256 360 and 388).
// SKIP: words that none of a wavefront's lanes has are passed over, of the loads the upper half together (8192 rows of 8192 in 256 lanes of 8 words 68 -> 53 us;
// parts that are all full are not faster by it).
template <bool FP32, int LANES, int NV, bool SKIP = false>
struct Held {
    static constexpr int kN = kValues<FP32>, kSize = FP32 ? 4 : 2;
    i32x4 raw[NV];
    float edge;                          // -infinity: none
    int32_t first, words, head, vocab;   // words: the row's; head: values ahead of the first
    int lane, wave;                      // wave: the wavefront's first lane

    // The part of the row that begins with its `first_`-th word.
    __device__ __forceinline__ void place(const char* row, int32_t first_, int32_t vocab_, int lane_) {
        first = first_; vocab = vocab_; lane = lane_;
        head = min((int32_t)(-(uintptr_t)row & 15) / kSize, vocab);
        words = (vocab - head) / kN;
        wave = LANES == 64 ? 0 : __builtin_amdgcn_readfirstlane(lane_);
        asm volatile("" : "+v"(lane));       // (places are worked out where they are needed: kept through a loop, they take a register each)
    }
    // Whether the row has no word at all.  (SKIP: the rows of a workgroup are always longer.)
    __device__ __forceinline__ bool none() const { return (LANES == 64 || !SKIP) && words <= 0; }
    __device__ __forceinline__ int32_t word(int i) const { return first + i * LANES + lane; }
    // Whether the i-th words of the wavefront are there at all, and whether all are.
    __device__ __forceinline__ bool some(int i) const { return !SKIP || first + i * LANES + wave < words; }
    __device__ __forceinline__ bool all(int i) const { return first + i * LANES + wave + 64 <= words; }
    // Where a word is, in bytes.  (32 bits beside the row's address, which is a wavefront's: vocab < 2^30.)
    __device__ __forceinline__ uint32_t place_of(int32_t word) const { return (uint32_t)head * kSize + (uint32_t)word * 16u; }
    // The lane's value of the edges, if it has one: the head's are the first kN lanes', the others' behind the words the next kN.
    __device__ __forceinline__ bool edge_at(int32_t* j) const {
        *j = lane < kN ? lane : head + words * kN + lane - kN;
        return first == 0 && (lane < kN ? lane < head : lane < 2 * kN && *j < vocab);
    }
    template <bool PAST>
    __device__ __forceinline__ void load_word(int i, const char* row, i32x4& to) const {
        const i32x4* p = (const i32x4*)(row + place_of(min(word(i), words - 1)));
        to = PAST ? __builtin_nontemporal_load(p) : *p;
    }
    template <bool PAST = true>
    __device__ __forceinline__ void load(const char* row) {
        load_edge(row);
        if (none()) return;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (i >= NV / 2 && !some(NV / 2)) continue;
            load_word<PAST>(i, row, raw[i]);
        }
    }
    __device__ __forceinline__ void load_edge(const char* row) {
        int32_t j;
        edge = minus_inf();
        if (edge_at(&j)) edge = value_at<FP32>(row, j);
    }
    // How a pass over what is held unpacks it.  Each has numbers of its own, unknown to the compiler, so that it unpacks again: values kept from one pass to
    // the next would take twice the registers.
    struct Pass {
        uint32_t low, high;
        __device__ __forceinline__ Pass() : low(16), high(0xffff0000u) {
            if constexpr (!FP32) asm volatile("" : "+s"(low), "+s"(high));
        }
    };
    __device__ __forceinline__ void values(const Pass& pass, int i, float (&v)[kN]) const {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if constexpr (FP32) v[k] = __int_as_float(raw[i][k]);
            else {
                v[2 * k] = __uint_as_float((uint32_t)raw[i][k] << pass.low);
                v[2 * k + 1] = __uint_as_float((uint32_t)raw[i][k] & pass.high);
            }
        }
    }
    // The sum of the wavefront's part, in every lane.  A lane adds up in FP32, apart from words of some weight beside the wavefront's largest value, which go
    // into an FP64 sum: beside a token that is all but certain the others would be lost in its rounding, and with them its log-probability.
    __device__ __forceinline__ Sum wave_part(Factor c) {
        float most = edge;
        const Pass first_pass;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (none() || !some(i)) continue;      // (a word that is there twice is as good as one that is not)
            float v[kN];
            values(first_pass, i, v);
#pragma unroll
            for (int k = 0; k < kN; k += 2) most = fmaxf(fmaxf(most, v[k]), v[k + 1]);
        }
        most = wave_max(most);
        const float base = base_of(most);
        float sum = 0.0f;
        const Pass second_pass;
        double near = (double)exp2_of(times(edge - base, c));
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (none() || !some(i)) continue;
            float v[kN], eight = 0.0f;
            values(second_pass, i, v);
#pragma unroll
            for (int k = 0; k < kN; ++k) v[k] = exp2_of(times(v[k] - base, c));
            if (!all(i)) {
                const bool there = word(i) < words;
#pragma unroll
                for (int k = 0; k < kN; ++k) v[k] = there ? v[k] : 0.0f;
            }
#pragma unroll
            for (int k = 0; k < kN; k += 4) eight += (v[k] + v[k + 1]) + (v[k + 2] + v[k + 3]);
            if (__builtin_amdgcn_ballot_w64(eight >= 0.5f)) {
#pragma unroll
                for (int k = 0; k < kN; ++k) near += (double)v[k];
            } else {
                sum += eight;
            }
        }
        return {sum_of_wave(near + (double)sum), most};
    }
    // Stores -d p, or d (1 - p) for the token, of all that is held: p = 2^((x - base) c - shift).  (c is the factor in one part, off by 2^-24 of itself, or 2^-23 where it
    // is the sums' first part: p is off by as much of |x - base| / T.)
    __device__ __forceinline__ void store_gradient(char* row, int32_t token, float d, float base, float c, float shift) {
        const Pass pass;
        asm volatile("" : "+v"(lane));
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (all(i) || word(i) < words) {
                float v[kN];
                values(pass, i, v);
#pragma unroll
                for (int k = 0; k < kN; ++k) v[k] = -d * exp2_of(fmaf(v[k] - base, c, -shift));
                const int32_t j = head + word(i) * kN;
                if ((uint32_t)(token - j) < (uint32_t)kN) {
#pragma unroll
                    for (int k = 0; k < kN; ++k) v[k] = token == j + k ? v[k] + d : v[k];
                }
                i32x4 w;
                if constexpr (FP32) w = __builtin_bit_cast(i32x4, (f32x4){v[0], v[1], v[2], v[3]});
                else w = __builtin_bit_cast(i32x4, __builtin_convertvector((f32x8){v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7]}, bf16x8));
                __builtin_nontemporal_store(w, (anywhere*)(row + place_of(word(i))));
            }
        }
        int32_t j;
        if (edge_at(&j)) put<FP32>(row, j, (token == j ? d : 0.0f) - d * exp2_of(fmaf(edge - base, c, -shift)));
    }
    __device__ __forceinline__ void store_zeros(char* row) const {
#pragma unroll 1
        for (int i = 0; i < NV; ++i)
            if (word(i) < words) __builtin_nontemporal_store(i32x4{}, (anywhere*)(row + place_of(word(i))));
        int32_t j;
        if (edge_at(&j)) put<FP32>(row, j, 0.0f);
    }
};

// The sum over a workgroup's wavefronts, in every lane.  ALONG: loads on their way are not waited for, and of several calls in a row every other one takes the
// other slot (a wavefront that is one call ahead waits there).
template <int WAVES, bool ALONG = false>
__device__ __forceinline__ Sum join_waves(const Sum& s, Factor c, int slot = 0) {
    if constexpr (WAVES == 1) return s;
    __shared__ Sum slots[ALONG ? 2 : 1][WAVES];
    Sum* parts = slots[slot];
    if ((threadIdx.x & 63) == 0) parts[threadIdx.x >> 6] = s;
    if constexpr (ALONG) asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    else __syncthreads();
    Sum all = parts[0];
#pragma unroll
    for (int k = 1; k < WAVES; ++k) all.most = fmaxf(all.most, parts[k].most);
    const float base = base_of(all.most);
    all.sum = 0.0;
#pragma unroll
    for (int k = 0; k < WAVES; ++k) all.sum += parts[k].sum * (double)exp2_of(times(parts[k].most - base, c));
    return all;
}

// What is computed once for a row, in FP64, from the functions' series.  A coefficient is put into scalar registers where it is used: the compiler keeps those of
// the library's functions in vector registers all the time, in which a row is held.
template <int64_t BITS>
__device__ __forceinline__ double constant() {
    int low, high;
    asm volatile("s_mov_b32 %0, %1" : "=s"(low) : "i"((int)BITS));
    asm volatile("s_mov_b32 %0, %1" : "=s"(high) : "i"((int)(BITS >> 32)));
    return __hiloint2double(high, low);
}
#define FO_CONSTANT(value) constant<__builtin_bit_cast(int64_t, (double)(value))>()
constexpr double kLn2 = 0.69314718055994530942, kLn2Low = 2.3190468138462996e-17;      // (the sum is ln 2 to more than FP64)
constexpr double factorial(int n) { return n > 1 ? n * factorial(n - 1) : 1.0; }
// 1 / N! + r / (N + 1)! + ... up to r^(LAST - N) / LAST!, and 1 / N + r / (N + 2) + ... up to the power of 1 / LAST.
template <int N, int LAST>
__device__ __forceinline__ double exp_series(double r) {
    if constexpr (N == LAST) return FO_CONSTANT(1.0 / factorial(N));
    else return fma(r, exp_series<N + 1, LAST>(r), FO_CONSTANT(1.0 / factorial(N)));
}
template <int N, int LAST>
__device__ __forceinline__ double log_series(double r) {
    if constexpr (N == LAST) return FO_CONSTANT(1.0 / N);
    else return fma(r, log_series<N + 2, LAST>(r), FO_CONSTANT(1.0 / N));
}
// e^x - 1 and e^x.  With x = k ln 2 + r, |r| <= ln 2 / 2, the first term left out of e^r - 1, r^14 / 14!, is 2^-56 of it.
__device__ __forceinline__ double expm1_of(double x, double less = 1.0) {
    x = x > 800.0 ? 800.0 : x < -800.0 ? -800.0 : x;       // (NaN stays; beyond these the power of two gives infinity and 0)
    const double k = rint(x * FO_CONSTANT(kLog2e)), r = fma(-k, FO_CONSTANT(kLn2Low), fma(-k, FO_CONSTANT(kLn2), x));
    const double s = r * exp_series<1, 13>(r);
    return k == 0.0 ? s + (1.0 - less) : ldexp(1.0 + s, (int)k) - less;
}
__device__ __forceinline__ double exp_of(double x) { return expm1_of(x, 0.0); }
// log x for x >= 0: with x = 2^e m, sqrt(1/2) <= m < sqrt 2, and t = (m - 1) / (m + 1) it is e ln 2 + 2 t (1 + t^2 / 3 + t^4 / 5 + ...), whose first term left
// out, t^22 / 23, is 2^-60.
__device__ __forceinline__ double log_of(double x) {
    if (x == 0.0) return (double)minus_inf();
    double m = __builtin_amdgcn_frexp_mant(x);
    int e = __builtin_amdgcn_frexp_exp(x);
    if (m < FO_CONSTANT(0.70710678118654752440)) {
        m += m;
        --e;
    }
    const double n = m - 1.0, d = m + 1.0;
    double q = __builtin_amdgcn_rcp(d);
    q = fma(q, fma(-d, q, 1.0), q);
    q = fma(q, fma(-d, q, 1.0), q);
    double t = n * q;
    t = fma(q, fma(-d, t, n), t);
    const double s = 2.0 * t * log_series<1, 21>(t * t);
    return fma((double)e, FO_CONSTANT(kLn2), fma((double)e, FO_CONSTANT(kLn2Low), s));
}

// log sum exp(x / T) and the token's log-probability; log_sum is what lse is beyond the largest value.
struct RowLog {
    double lse, logprob, log_sum;
};
__device__ __forceinline__ RowLog row_log(const Sum& s, float x, double inv_t) {
    // (a sum beyond FP32 is that of a row with +infinity)
    const double log_sum = s.most < __builtin_inff() ? log_of(s.sum) : (double)__builtin_nanf("");
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
    double* terms;                      // [3, rows], or [3, workgroups]
};
struct PolicyIn {
    float w, advantage, old, ref;
};
__device__ __forceinline__ PolicyRow policy_row(const PolicyArgs& a, const PolicyIn& in, double logprob) {
    const double adv = in.advantage, w = in.w;
    // (of the policy to itself 1 whatever its logprob, also for a token of probability 0; NaN stays)
    const double ratio = a.in.old_logprob ? exp_of(logprob - (double)in.old) : logprob == logprob ? 1.0 : logprob;
    const double low = 1.0 - (double)a.spec.clip_low, high = 1.0 + (double)a.spec.clip_high;
    const bool blocked = (adv > 0.0 && ratio > high) || (adv < 0.0 && ratio < low);
    const double gain = adv == 0.0 && ratio == ratio ? 0.0 : adv * ratio;        // (the ratio may be infinite; NaN stays)
    const double surrogate = blocked ? -adv * (adv > 0.0 ? high : low) : -gain;
    double slope = blocked ? 0.0 : -gain, kl = 0.0;
    if (a.in.ref_logprob) {
        const double d = (double)in.ref - logprob, e = expm1_of(d);
        kl = d < __builtin_inf() ? e - d : d;
        if (a.spec.kl_weight != 0.0f) slope -= (double)a.spec.kl_weight * e;       // (0: watched only, and e may be infinite)
    }
    return {(float)(slope * w * (double)a.spec.grad_scale), surrogate * w, kl * w, blocked ? w : 0.0};
}
__device__ __forceinline__ PolicyRow policy_row(const PolicyArgs& a, uint32_t row, double logprob, float w) {
    const PolicyIn in = {w, a.in.advantages[row], a.in.old_logprob ? a.in.old_logprob[row] : 0.0f, a.in.ref_logprob ? a.in.ref_logprob[row] : 0.0f};
    return policy_row(a, in, logprob);
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
    double* wide;            // logprob in FP64
    double inv_t;
    Factor c;
    uint32_t rows;
    char* dx;                // the gradient (policy loss; NULL: not wanted)
    int64_t dx_stride;
    float scale;             // 1 / T
    PolicyArgs policy;
};

// The statistics from the sums of the three terms.  (A KL term without weight may be infinite.)
__device__ __forceinline__ void put_stats(const double (&s)[3], float kl_weight, float* stats) {
#pragma unroll
    for (int k = 0; k < 3; ++k) stats[1 + k] = (float)s[k];
    stats[0] = (float)(kl_weight != 0.0f ? s[0] + (double)kl_weight * s[1] : s[0]);
}

// One row to LANES lanes, which hold it: the policy loss and its gradient in one pass over the logits.  What the row's terms are, in lane 0.
template <bool FP32, int LANES, int NV>
__device__ __forceinline__ PolicyRow policy_of_row(const RowsArgs& a, uint32_t row, int lane) {
    const int64_t token = a.tokens[row];
    const float w = a.policy.in.weights ? a.policy.in.weights[row] : 1.0f;
    char* dx = a.dx ? a.dx + (int64_t)row * a.dx_stride * (FP32 ? 4 : 2) : nullptr;
    const char* x = row_of<FP32>(a.x, row);
    Held<FP32, LANES, NV, true> h;
    h.place(x, 0, a.x.vocab, lane);
    if (token < 0 || w == 0.0f) {
        if (lane == 0 && a.logprob) a.logprob[row] = 0.0f;
        if (dx) h.store_zeros(dx);
        return {};
    }
    h.load(x);
    const float logit = logit_of<FP32>(x, token, a.x.vocab);
    const Sum s = join_waves<LANES / 64>(h.wave_part(a.c), a.c);
    const RowLog l = row_log(s, logit, a.inv_t);
    const PolicyRow p = policy_row(a.policy, row, l.logprob, w);
    if (lane == 0 && a.logprob) a.logprob[row] = (float)l.logprob;
    const float d = p.slope * a.scale;
    if (!dx) return p;
    if (d == 0.0f) h.store_zeros(dx);
    else h.store_gradient(dx, token_in(token, a.x.vocab), d, base_of(s.most), a.c.high, (float)(l.log_sum * kLog2e));
    return p;
}
template <bool FP32, int LANES, int NV>
__global__ __launch_bounds__(LANES < 256 ? 256 : LANES) void policy_rows_kernel(RowsArgs a) {
    constexpr int LINES = LANES < 256 ? 256 / LANES : 1;
    static_assert(LANES == 64 || LINES == 1, "a row is a wavefront's or a workgroup's");
    const uint32_t row = LINES == 1 ? blockIdx.x : blockIdx.x * LINES + (uint32_t)__builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int lane = (int)threadIdx.x & (LANES - 1);
    if (row >= a.rows) return;
    const PolicyRow p = policy_of_row<FP32, LANES, NV>(a, row, lane);
    if (lane == 0) put_terms(a.policy, a.rows, row, p);
}

// A few short rows, a wavefront each, by one workgroup that adds up their terms itself: no second launch (12 rows of 1001 FP32 values
// 6.3 us against 7.8; 16 rows 7.0 and 17, by two launches, 7.8; rows of 8 words a lane are no faster so, 16 of 2000 values 8.9 us, 17 by two launches 8.7).
constexpr uint32_t kFewRows = 16;
constexpr int kFewVecs = 4;
template <bool FP32>
__global__ __launch_bounds__(kFewRows * 64) void policy_few_rows_kernel(RowsArgs a, float* stats) {
    __shared__ double terms[kFewRows][3];
    const uint32_t row = (uint32_t)__builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    if (row < a.rows) {
        const PolicyRow p = policy_of_row<FP32, 64, kFewVecs>(a, row, (int)threadIdx.x & 63);
        if ((threadIdx.x & 63) == 0) {
            terms[row][0] = p.surrogate;
            terms[row][1] = p.kl;
            terms[row][2] = p.blocked;
        }
    }
    __syncthreads();
    if (threadIdx.x != 0) return;
    double s[3] = {};
    for (uint32_t i = 0; i < a.rows; ++i)
#pragma unroll
        for (int k = 0; k < 3; ++k) s[k] += terms[i][k];
    put_stats(s, a.policy.spec.kl_weight, stats);
}

// Rows of which a compute unit holds one at a time.  Workgroups stay and take every so many-th row: of the next one the first kAhead words of each lane, as many as
// LDS holds, are on their way there while this one is worked on and stored, so that the memory is not idle between two rows.  (4096 rows of 128256 BF16 values
// 440-453 us without, 391-402 with; half as many words ahead 393-403.  Smaller shapes, of which a unit holds two or more rows, are no faster by it, or slower.)
// A wavefront fetches and reads its own words, so that nothing but the sums is shared.  Vector loads arrive in order: what is needed while the words are on their
// way comes as scalars or ahead of them.  A row's start waits for its own loads, and with them (one counter has both) for the stores of the row before.  What a workgroup leaves for the statistics are
// the sums of its rows' terms (4096 rows of 128256 BF16 values 392.7 us with each row's, 391.3 so; 1001 of 50257 FP32 values 85.1 and 84.6).
template <bool FP32>
__global__ __launch_bounds__(1024) void policy_long_rows_kernel(RowsArgs a) {
    constexpr int NV = 16, LANES = 1024, kAhead = 9;
    using Row = Held<FP32, LANES, NV, true>;
    __shared__ i32x4 ahead[kAhead][LANES];
    __shared__ double terms[3];          // lane 0's
    struct In {                          // what goes into a row's loss, as scalars
        int64_t token;
        PolicyIn p;
        bool there;
    };
    const auto scalar = [](auto p, uint32_t row) {
        using T = std::remove_cv_t<std::remove_pointer_t<decltype(p)>>;
        return ((const __attribute__((address_space(4))) T*)(uintptr_t)p)[row];
    };
    const auto inputs = [&](uint32_t row) {
        In in = {-1, {}, false};
        if (row >= a.rows) return in;
        in.token = scalar(a.tokens, row);
        in.p.w = a.policy.in.weights ? scalar(a.policy.in.weights, row) : 1.0f;
        in.p.advantage = scalar(a.policy.in.advantages, row);
        in.p.old = a.policy.in.old_logprob ? scalar(a.policy.in.old_logprob, row) : 0.0f;
        in.p.ref = a.policy.in.ref_logprob ? scalar(a.policy.in.ref_logprob, row) : 0.0f;
        in.there = in.token >= 0 && in.p.w != 0.0f;
        return in;
    };
    using Raw = std::conditional_t<FP32, uint32_t, uint16_t>;
    const auto fetch = [&](uint32_t row) {
        const char* x = row_of<FP32>(a.x, row);
        Row next;
        next.place(x, 0, a.x.vocab, (int)threadIdx.x);
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(x + next.place_of(min(next.word(i), next.words - 1))),
                                             (__attribute__((address_space(3))) void*)&ahead[i][next.wave], 16, 0, 2);
    };
    In in = inputs(blockIdx.x);
    if (in.there) fetch(blockIdx.x);
    if (threadIdx.x == 0) terms[0] = terms[1] = terms[2] = 0.0;
    int slot = 0;
    for (uint32_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const In next = inputs(row + gridDim.x);
        char* dx = a.dx ? a.dx + (int64_t)row * a.dx_stride * (FP32 ? 4 : 2) : nullptr;
        const char* x = row_of<FP32>(a.x, row);
        Row h;
        h.place(x, 0, a.x.vocab, (int)threadIdx.x);
        float d = 0.0f, shift = 0.0f;
        double logprob = 0.0;
        PolicyRow p = {};
        Sum s = {1.0, 0.0f};
        if (in.there) {
#pragma unroll
            for (int i = kAhead; i < NV; ++i) h.template load_word<true>(i, x, h.raw[i]);
            int32_t j;
            const bool has_edge = h.edge_at(&j);
            uint32_t edge = ((const Raw*)x)[has_edge ? j : 0], value = ((const Raw*)x)[in.token < a.x.vocab ? (int32_t)in.token : 0];
            __builtin_amdgcn_s_waitcnt(0x0f70);                     // vmcnt(0): this row is there
            asm volatile("" : "+v"(value), "+v"(edge)::"memory");
            h.edge = has_edge ? __uint_as_float(FP32 ? edge : edge << 16) : minus_inf();
            const float logit = in.token < a.x.vocab ? __uint_as_float(FP32 ? value : value << 16) : __builtin_nanf("");
#pragma unroll
            for (int i = 0; i < kAhead; ++i) h.raw[i] = ahead[i][threadIdx.x];
            __builtin_amdgcn_s_waitcnt(0xc07f);                     // lgkmcnt(0): and read, before the next one takes its place
            asm volatile("" ::: "memory");
            if (next.there) fetch(row + gridDim.x);
            s = join_waves<LANES / 64, true>(h.wave_part(a.c), a.c, slot);
            slot ^= 1;
            const RowLog l = row_log(s, logit, a.inv_t);
            logprob = l.logprob;
            p = policy_row(a.policy, in.p, l.logprob);
            d = p.slope * a.scale;
            shift = (float)(l.log_sum * kLog2e);
        } else if (next.there) {
            fetch(row + gridDim.x);
        }
        if (threadIdx.x == 0) {
            if (a.logprob) a.logprob[row] = (float)logprob;
            terms[0] += p.surrogate;
            terms[1] += p.kl;
            terms[2] += p.blocked;
        }
        if (dx) {
            if (d == 0.0f) h.store_zeros(dx);
            else h.store_gradient(dx, token_in(in.token, a.x.vocab), d, base_of(s.most), a.c.high, shift);
        }
        in = next;
    }
    if (threadIdx.x == 0) put_terms(a.policy, gridDim.x, blockIdx.x, {0.0f, terms[0], terms[1], terms[2]});
}

// Log-probabilities only, one workgroup of WAVES wavefronts to a row, through which the wavefronts go in turn.
template <bool FP32, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void logprob_rows_kernel(RowsArgs a) {
    constexpr int NV = 8, kPart = 64 * NV;
    const uint32_t row = blockIdx.x;
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int64_t token = a.tokens[row];
    if (token < 0) {
        if (threadIdx.x == 0) {
            if (a.logprob) a.logprob[row] = 0.0f;
            if (a.lse) a.lse[row] = 0.0f;
            if (a.wide) a.wide[row] = 0.0;
        }
        return;
    }
    const char* x = row_of<FP32>(a.x, row);
    const float logit = logit_of<FP32>(x, token, a.x.vocab);
    Sum s = {0.0, minus_inf()};
    Held<FP32, 64, NV> h;
    h.place(x, wave * kPart, a.x.vocab, lane);
    for (; h.first == 0 || h.first < h.words; h.first += WAVES * kPart) {
        h.load(x);
        s = join(s, h.wave_part(a.c), a.c);
    }
    s = join_waves<WAVES>(s, a.c);
    if (threadIdx.x != 0) return;
    const RowLog l = row_log(s, logit, a.inv_t);
    if (a.logprob) a.logprob[row] = (float)l.logprob;
    if (a.lse) a.lse[row] = (float)l.lse;
    if (a.wide) a.wide[row] = l.logprob;
}

// ---- few rows, or rows that do not fit: each cut into parts, a workgroup to each, which leaves its sum; whoever needs a row's joins them.
constexpr int kPartThreads = 256, kPartWords = 2;      // lanes, and words of a lane
struct PartsArgs {
    RowsArgs r;
    Sum* sums;               // [rows, parts]
    float* logits;           // [rows]: of the tokens
    uint32_t parts;
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
    Held<FP32, kPartThreads, kPartWords> h;
    h.place(x, (int32_t)part * (kPartThreads * kPartWords), a.r.x.vocab, (int)threadIdx.x);
    h.template load<false>(x);       // (the gradient reads it again)
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
    return {sum_of_wave(s.sum * (double)exp2_of(times(s.most - base_of(most), a.r.c))), most};
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
    if (a.r.wide) a.r.wide[row] = l.logprob;
}

// The gradient of a part.  Every workgroup joins its row's sums and computes the row's slope for itself; the first of a row leaves what is kept of it.
template <bool FP32>
__global__ __launch_bounds__(kPartThreads) void policy_parts_kernel(PartsArgs a) {
    const uint32_t row = blockIdx.x / a.parts, part = blockIdx.x % a.parts;
    const int64_t token = a.r.tokens[row];
    float w;
    const bool there = counts(a, row, token, &w);
    char* dx = a.r.dx ? a.r.dx + (int64_t)row * a.r.dx_stride * (FP32 ? 4 : 2) : nullptr;
    const char* x = row_of<FP32>(a.r.x, row);
    Held<FP32, kPartThreads, kPartWords> h;
    h.place(x, (int32_t)part * (kPartThreads * kPartWords), a.r.x.vocab, (int)threadIdx.x);
    if (there && dx) h.load(x);
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
    else h.store_gradient(dx, token_in(token, a.r.x.vocab), d, base_of(s.most), a.r.c.high, (float)(l.log_sum * kLog2e));
}

// ---- the gradient of the logits from the lse of an earlier call
struct GradArgs {
    Logits x;
    char* dx;
    int64_t stride;
    const int64_t* tokens;
    const float *lse, *slope;
    float scale, t, c;       // of the slopes; the temperature T, and log2(e) / T
    uint32_t parts;
};
constexpr float kMostLse = 131072.0f, kMostBase = 0x1p102f;       // (a logit of any size less kMostBase is finite)
template <bool FP32, int NV>
__global__ __launch_bounds__(kPartThreads) void gradient_kernel(GradArgs a) {
    const uint32_t row = blockIdx.x / a.parts, part = blockIdx.x % a.parts;
    char* dx = a.dx + (int64_t)row * a.stride * (FP32 ? 4 : 2);
    const char* x = row_of<FP32>(a.x, row);
    const int64_t token = a.tokens[row];
    float d = token < 0 ? 0.0f : a.slope[row] * a.scale;
    Held<FP32, kPartThreads, NV> h;
    h.place(x, (int32_t)part * (kPartThreads * NV), a.x.vocab, (int)threadIdx.x);
    if (d == 0.0f) {
        h.store_zeros(dx);
        return;
    }
    // (from kMostLse on what FP32 has lost of lse would be up to 0.8 % of the probabilities and more, at the type's lowest value all of them)
    const float lse = a.lse[row];
    if (token >= a.x.vocab || !(fabsf(lse) < kMostLse)) d = __builtin_nanf("");
    // The difference first, as in the sums: x / T - lse = (x - base) / T - rest / T with lse T = base + rest.  (x c - lse log2(e) in FP32 loses as much as lse
    // itself has lost twice more, by the constants and by the product's rounding.)
    float base = lse * a.t, shift = fmaf(lse, a.t, -base) * a.c;
    if (fabsf(base) > kMostBase) {           // (T of 2^85 or more)
        base = 0.0f;
        shift = lse * (float)kLog2e;
    }
    h.load(x);
    h.store_gradient(dx, token_in(token, a.x.vocab), d, base, a.c, shift);
}

// Three sums over a workgroup's rows, and from them the statistics.
__global__ __launch_bounds__(kPairThreads) void policy_stats_kernel(const double* terms, uint32_t rows, float kl_weight, float* stats) {
    __shared__ double part[3][kPairThreads / 64];
    double s[3] = {};
    constexpr uint32_t kAhead = 4;                                 // (loads that are on their way together)
    for (uint32_t i = threadIdx.x; i < rows; i += kAhead * kPairThreads) {
        double v[kAhead][3];
#pragma unroll
        for (uint32_t u = 0; u < kAhead; ++u)
#pragma unroll
            for (int k = 0; k < 3; ++k) v[u][k] = i + u * kPairThreads < rows ? terms[(int64_t)k * rows + i + u * kPairThreads] : 0.0;
#pragma unroll
        for (uint32_t u = 0; u < kAhead; ++u)
#pragma unroll
            for (int k = 0; k < 3; ++k) s[k] += v[u][k];
    }
#pragma unroll
    for (int k = 0; k < 3; ++k) s[k] = sum_of_wave(s[k]);
    if ((threadIdx.x & 63) < 3) part[threadIdx.x & 63][threadIdx.x >> 6] = (threadIdx.x & 63) == 0 ? s[0] : (threadIdx.x & 63) == 1 ? s[1] : s[2];
    __syncthreads();
    if (threadIdx.x != 0) return;
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        s[k] = 0.0;
#pragma unroll
        for (int j = 0; j < kPairThreads / 64; ++j) s[k] += part[k][j];
    }
    put_stats(s, kl_weight, stats);
}

struct PairArgs {
    const float* logprob;
    const double* wide;      // logprob in FP64, instead
    const float *ref, *weights;
    const int64_t* offsets;
    float *loss, *margins, *dlogprob;
    int64_t rows, pairs;
    flashoptim_preference_spec spec;
};

// What of a pair's margin the loss and its slope by the margin are.
struct PairLoss {
    double loss, slope;
};
__device__ __forceinline__ PairLoss pair_loss(const flashoptim_preference_spec& spec, double gain) {
    const double beta = spec.beta, z = beta * gain, e = spec.label_smoothing;
    if (spec.kind == FLASHOPTIM_PREFERENCE_SIGMOID) {      // (z may be infinite)
        const double t = exp(-fabs(z)), l = log1p(t), near = 1.0 / (1.0 + t), far = t * near;       // sigmoid(|z|), sigmoid(-|z|)
        const double up = z >= 0.0 ? near : far, down = z >= 0.0 ? far : near;
        const double plus = fmax(-z, 0.0) + l, minus = fmax(z, 0.0) + l;                             // -log sigmoid(z), -log sigmoid(-z)
        return {(1.0 - e) * plus + (e > 0.0 ? e * minus : 0.0), e * up - (1.0 - e) * down};
    }
    if (spec.kind == FLASHOPTIM_PREFERENCE_HINGE)        // (z may be NaN)
        return {z < 1.0 ? 1.0 - z : z >= 1.0 ? 0.0 : z, z < 1.0 ? -1.0 : z >= 1.0 ? 0.0 : z};
    const double r = gain - 0.5 / beta;
    return {r * r, 2.0 * r / beta};
}

// One workgroup for all pairs, so that the loss needs no second launch: there are a few bytes for each row of logits.  Its wavefronts are shared out over
// `groups` pairs at a time: from one wavefront each, with nothing to wait for between them, to all sixteen for a single pair.
__global__ __launch_bounds__(kPairThreads) void preference_kernel(PairArgs a, int groups) {
    constexpr int kWaves = kPairThreads / 64, kAhead = 2;
    __shared__ double gains[kWaves], losses[kWaves];
    const auto bound = [&](int64_t i) { return min(max(a.offsets[i], (int64_t)0), a.rows); };
    const bool by_turns = a.spec.order == FLASHOPTIM_PAIRS_BY_TURNS;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), waves = kWaves / groups, group = wave / waves;
    const int lane = (wave % waves) * 64 + ((int)threadIdx.x & 63), lanes = waves * 64;
    double total = 0.0;
    for (int64_t first = 0; first < a.pairs; first += groups) {
        const int64_t p = first + group;
        const bool there = p < a.pairs;
        int64_t begin[2] = {}, end[2] = {};
        double gain = 0.0;
        if (there)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int64_t of = by_turns ? 2 * p + k : p + k * a.pairs;
                begin[k] = bound(of);
                end[k] = bound(of + 1);
            }
        const int64_t longest = max(end[0] - begin[0], end[1] - begin[1]);
        for (int64_t i = lane; i < longest; i += kAhead * lanes) {      // (of both sequences, so that all loads are on their way together)
            float w[2][kAhead], r[2][kAhead];
            double v[2][kAhead];
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int u = 0; u < kAhead; ++u) {
                    const int64_t at = begin[k] + i + (int64_t)u * lanes;
                    const bool in = at < end[k];
                    w[k][u] = !in ? 0.0f : a.weights ? a.weights[at] : 1.0f;
                    v[k][u] = !in ? 0.0 : a.wide ? a.wide[at] : (double)a.logprob[at];
                    r[k][u] = in && a.ref ? a.ref[at] : 0.0f;
                }
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int u = 0; u < kAhead; ++u) {
                    const double d = w[k][u] != 0.0f ? (double)w[k][u] * (v[k][u] - (double)r[k][u]) : 0.0;
                    gain += k ? -d : d;
                }
        }
        gain = sum_of_wave(gain);
        if (waves > 1) {
            __syncthreads();
            if ((threadIdx.x & 63) == 0) gains[wave] = gain;
            __syncthreads();
            gain = 0.0;
            for (int k = 0; k < waves; ++k) gain += gains[group * waves + k];
        }
        if (!there) continue;
        const PairLoss l = pair_loss(a.spec, gain);
        total += l.loss;
        if (lane == 0 && a.margins) a.margins[p] = (float)((double)a.spec.beta * gain);
        if (!a.dlogprob) continue;
        const double d = l.slope * ((double)a.spec.beta * (double)a.spec.grad_scale / (double)a.pairs);
        for (int k = 0; k < 2; ++k)
            for (int64_t i = begin[k] + lane; i < end[k]; i += lanes) {
                const float w = a.weights ? a.weights[i] : 1.0f;
                a.dlogprob[i] = w == 0.0f ? 0.0f : (float)((k ? -d : d) * (double)w);
            }
    }
    if (a.dlogprob) {
        const int64_t first = a.pairs ? bound(0) : a.rows, last = a.pairs ? bound(2 * a.pairs) : a.rows;
        for (int64_t i = threadIdx.x; i < first; i += kPairThreads) a.dlogprob[i] = 0.0f;
        for (int64_t i = last + threadIdx.x; i < a.rows; i += kPairThreads) a.dlogprob[i] = 0.0f;
    }
    if (lane == 0) losses[group] = total;
    __syncthreads();
    if (threadIdx.x != 0) return;
    total = 0.0;
    for (int k = 0; k < groups; ++k) total += losses[k];
    *a.loss = a.pairs ? (float)(total / (double)a.pairs) : 0.0f;
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

// The most words that a row has between 16-byte borders.
int64_t words(int64_t vocab, int dtype) { return vocab * fo::elem_bytes(dtype) / 16; }

// The parts of a row, of kPartThreads lanes that hold `vecs` words each.
int64_t parts_of(int64_t vocab, int dtype, int vecs = kPartWords) {
    const int64_t n = words(vocab, dtype);
    return n > 0 ? up(n, kPartThreads * vecs) : 1;
}
// The words of a lane in the gradient's parts: two, or one where parts of that size have clearly fewer lanes without a word (8192 rows of 50257 BF16 values, 13 parts or
// 25, 279 us and 265; 16384 rows of 8192, 2 or 4, 82 and 88; 2048 rows of 128256, 32 or 63, 167 and 172) and there are not too many.  Parts that have to be joined are
// never faster with one (100 rows of 128256, policy loss, 18.6 us and 24.0).
int gradient_vecs(int64_t rows, int64_t vocab, int dtype) {
    const int64_t one = parts_of(vocab, dtype, 1);
    return one * 103 < 200 * parts_of(vocab, dtype) && rows * one <= fo::kMaxWorkItems / kPartThreads ? 1 : 2;
}
template <int N>
using Int = std::integral_constant<int, N>;
bool known(int dtype) { return dtype == FLASHOPTIM_BF16 || dtype == FLASHOPTIM_FP32; }

// Calls launch(shape) with the shape of the workgroups that hold rows of n words.
template <int LANES, int NV>
struct Shape {
    static constexpr int kLanes = LANES, kVecs = NV;
};
template <typename F>
void with_held(int64_t n, F launch) {
    if (n <= 64 * 4) launch(Shape<64, 4>{});
    else if (n <= 64 * 8) launch(Shape<64, 8>{});
    else if (n <= 256 * 8) launch(Shape<256, 8>{});
    else if (n <= 512 * 8) launch(Shape<512, 8>{});
    else if (n <= 512 * 16) launch(Shape<512, 16>{});
    else launch(Shape<1024, 16>{});
}
// Whether the policy loss holds whole rows, up to the largest shape's: short ones always (two launches against three, one row of 5000 BF16 values 7.5 us against 11.1,
// 64 of 10000 8.6 against 11.2, of 32000 11.9 against 11.6), longer ones where there are as many as fill half the chip (128256 BF16 values, 100 rows 23.8 us against
// 20.3 in parts, 128 rows 23.9 against 23.7).
constexpr unsigned kUnits = 256;      // compute units
bool holds_rows(int64_t rows, int64_t vocab, int dtype) {
    const int64_t n = words(vocab, dtype);
    return n <= 256 * 8 || (n <= 1024 * 16 && rows >= kUnits / 2);
}
// Whether log-probabilities take a row to a workgroup: short ones (one launch against two, 32000 BF16 values, one row 5.2 us against 7.2, 16 rows 5.9 against 6.3;
// 50257 values, one row 7.1 against 6.7, 64 rows 8.3 against 7.3), and as many as there are compute units (256 rows of 128256 15.3 us against 19.1, 128 rows
// 13.8 against 12.3).
bool streams_rows(int64_t rows, int64_t vocab, int dtype) { return words(vocab, dtype) <= 4096 || rows >= kUnits; }
// And by how many wavefronts: few rows by all that a workgroup may have (256 rows of 10000 BF16 values 6.1 -> 5.1 us, of 128256 17.6 -> 15.3).  Many rows by as
// many as find a part of 512 words for each, since those without one only wait (8192 rows of 4096 BF16 values by 1, 2, 4 and 8 wavefronts 16.0, 18.3, 20.9 and
// 37.1 us; of 8192 27.4, 25.8, 28.7 and 42.3; of 16384 49.7, 47.4, 45.4 and 50.9; of 24000 71.9, 69.6, 72.1 and 71.1, but 600 of these 18.0, 13.0, 11.1 and 10.5).
int stream_waves(int64_t rows, int64_t vocab, int dtype) {
    const int64_t parts = up(words(vocab, dtype), 512);
    if (rows < 2 * kUnits && parts > 1) return 16;
    return parts <= 1 ? 1 : parts <= 2 ? 2 : parts <= 4 ? 4 : 8;
}

// A call's parts in its workspace.
PartsArgs to_parts(const RowsArgs& a, int dtype, void* workspace) {
    PartsArgs p = {a, (Sum*)workspace, nullptr, (uint32_t)parts_of(a.x.vocab, dtype)};
    p.logits = (float*)(p.sums + (int64_t)a.rows * p.parts);
    return p;
}
int64_t parts_bytes(int64_t rows, int64_t vocab, int dtype) {
    return up(rows * parts_of(vocab, dtype) * (int64_t)sizeof(Sum) + rows * 4, 16) * 16;
}
int launch_parts(const PartsArgs& p, int dtype, void* stream) {
    const dim3 grid(p.r.rows * p.parts), block(kPartThreads);
    if (dtype == FLASHOPTIM_FP32) hipLaunchKernelGGL((parts_kernel<true>), grid, block, 0, (hipStream_t)stream, p);
    else hipLaunchKernelGGL((parts_kernel<false>), grid, block, 0, (hipStream_t)stream, p);
    return fo::hip_status(hipGetLastError());
}

// Rows of which a compute unit holds one, and so many that workgroups stay.
bool long_rows(int64_t rows, int64_t vocab, int dtype) { return words(vocab, dtype) > 512 * 16 && rows >= 2 * kUnits; }
template <bool FP32>
int launch_held(const RowsArgs& a, void* stream) {
    const int dtype = FP32 ? FLASHOPTIM_FP32 : FLASHOPTIM_BF16;
    const int64_t n = words(a.x.vocab, dtype);
    if (long_rows(a.rows, a.x.vocab, dtype)) {
        hipLaunchKernelGGL((policy_long_rows_kernel<FP32>), dim3(kUnits), dim3(1024), 0, (hipStream_t)stream, a);
        return fo::hip_status(hipGetLastError());
    }
    with_held(n, [&](auto shape) {
        constexpr int L = decltype(shape)::kLanes, NV = decltype(shape)::kVecs, LINES = L < 256 ? 256 / L : 1;
        hipLaunchKernelGGL((policy_rows_kernel<FP32, L, NV>), dim3((unsigned)up(a.rows, LINES)), dim3(L * LINES), 0, (hipStream_t)stream, a);
    });
    return fo::hip_status(hipGetLastError());
}

// Whether one workgroup takes all rows, a wavefront each.
bool few_rows(int64_t rows, int64_t vocab, int dtype) { return rows <= kFewRows && words(vocab, dtype) <= 64 * kFewVecs; }
template <bool FP32>
int launch_few(const RowsArgs& a, float* stats, void* stream) {
    hipLaunchKernelGGL((policy_few_rows_kernel<FP32>), dim3(1), dim3(a.rows * 64), 0, (hipStream_t)stream, a, stats);
    return fo::hip_status(hipGetLastError());
}

int check_launch(const flashoptim_matrix* logits) {
    const int64_t blocks = logits->rows * parts_of(logits->cols, logits->dtype);
    return blocks > fo::kMaxWorkItems / kPartThreads || logits->rows > fo::kMaxWorkItems / 1024 ? FLASHOPTIM_ERR_NUMEL_RANGE : FLASHOPTIM_OK;
}
int check_workspace(int64_t need, const void* workspace, int64_t bytes) {
    if (need < 0) return (int)need;
    if (need > 0 && !workspace) return FLASHOPTIM_ERR_INVALID_ARG;
    if (bytes < need) return FLASHOPTIM_ERR_WORKSPACE;
    return fo::aligned_to(workspace, 16) ? FLASHOPTIM_OK : FLASHOPTIM_ERR_MISALIGNED;
}
Factor factor_of(float temperature) {
    const double c = kLog2e / (double)temperature;
    float high = (float)c;
    if ((double)high > c) high = std::nextafter(high, 0.0f);
    const float low = (float)(c - (double)high);
    return {high, low > 0.0f ? low : std::numeric_limits<float>::denorm_min()};       // (of no weight beside high, at any temperature)
}
RowsArgs rows_args(const flashoptim_matrix* logits, const int64_t* tokens, float temperature) {
    RowsArgs a = {};
    a.x = to_dev(logits);
    a.tokens = tokens;
    a.inv_t = 1.0 / (double)temperature;
    a.c = factor_of(temperature);
    a.scale = 1.0f / temperature;
    a.rows = (uint32_t)logits->rows;
    return a;
}

}  // namespace

extern "C" {

int64_t flashoptim_token_logprob_workspace(int64_t rows, int64_t vocab, int dtype) {
    if (!known(dtype)) return FLASHOPTIM_ERR_INVALID_ARG;
    FO_TRY(check_sizes(rows, vocab));
    return rows == 0 || streams_rows(rows, vocab, dtype) ? 0 : parts_bytes(rows, vocab, dtype);
}

int flashoptim_token_logprob(const flashoptim_matrix* logits, const int64_t* tokens, float temperature, float* logprob, double* logprob64,
                             float* lse, void* workspace, int64_t workspace_bytes, void* stream) {
    FO_TRY(check_logits(logits, tokens, temperature));
    const int64_t rows = logits->rows;
    if (rows == 0) return FLASHOPTIM_OK;
    if (!logprob && !logprob64 && !lse) return FLASHOPTIM_ERR_INVALID_ARG;
    if (!fo::aligned_to(logprob, 4) || !fo::aligned_to(logprob64, 8) || !fo::aligned_to(lse, 4)) return FLASHOPTIM_ERR_MISALIGNED;
    FO_TRY(check_launch(logits));
    FO_TRY(check_workspace(flashoptim_token_logprob_workspace(rows, logits->cols, logits->dtype), workspace, workspace_bytes));
    RowsArgs a = rows_args(logits, tokens, temperature);
    a.logprob = logprob;
    a.wide = logprob64;
    a.lse = lse;
    if (streams_rows(rows, logits->cols, logits->dtype)) {
        const auto launch = [&](auto fp32, auto waves) {
            constexpr int W = decltype(waves)::value;
            hipLaunchKernelGGL((logprob_rows_kernel<decltype(fp32)::value, W>), dim3(a.rows), dim3(W * 64), 0, (hipStream_t)stream, a);
        };
        const auto with = [&](auto fp32) {
            switch (stream_waves(rows, logits->cols, logits->dtype)) {
                case 1: return launch(fp32, Int<1>{});
                case 2: return launch(fp32, Int<2>{});
                case 4: return launch(fp32, Int<4>{});
                case 8: return launch(fp32, Int<8>{});
                default: launch(fp32, Int<16>{});
            }
        };
        if (logits->dtype == FLASHOPTIM_FP32) with(std::true_type{}); else with(std::false_type{});
        return fo::hip_status(hipGetLastError());
    }
    const PartsArgs p = to_parts(a, logits->dtype, workspace);
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
    const int vecs = gradient_vecs(logits->rows, logits->cols, logits->dtype);
    const GradArgs g = {to_dev(logits), (char*)dlogits->data, dlogits->rows > 1 ? dlogits->stride : 0, tokens, lse, dlogprob, 1.0f / temperature, temperature,
                        (float)(kLog2e / (double)temperature), (uint32_t)parts_of(logits->cols, logits->dtype, vecs)};
    const dim3 grid((unsigned)(logits->rows * (int64_t)g.parts)), block(kPartThreads);
    const auto launch = [&](auto fp32, auto nv) {
        hipLaunchKernelGGL((gradient_kernel<decltype(fp32)::value, decltype(nv)::value>), grid, block, 0, (hipStream_t)stream, g);
    };
    const auto with = [&](auto fp32) {
        if (vecs == 2) launch(fp32, Int<2>{}); else launch(fp32, Int<1>{});
    };
    if (logits->dtype == FLASHOPTIM_FP32) with(std::true_type{}); else with(std::false_type{});
    return fo::hip_status(hipGetLastError());
}

int64_t flashoptim_policy_loss_workspace(int64_t rows, int64_t vocab, int dtype) {
    if (!known(dtype)) return FLASHOPTIM_ERR_INVALID_ARG;
    FO_TRY(check_sizes(rows, vocab));
    const int64_t terms = up(rows * 24, 16) * 16;
    return terms + (rows == 0 || holds_rows(rows, vocab, dtype) ? 0 : parts_bytes(rows, vocab, dtype));
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
    // (a row's inputs are read by many lanes while one writes its logprob)
    for (const float* p : {inputs->advantages, inputs->old_logprob, inputs->ref_logprob, inputs->weights})
        if (rows > 0 && p && p == logprob) return FLASHOPTIM_ERR_INVALID_ARG;
    RowsArgs a = rows_args(logits, tokens, spec->temperature);
    a.logprob = logprob;
    a.policy = {*spec, *inputs, (double*)workspace};
    if (dlogits) {
        a.dx = (char*)dlogits->data;
        a.dx_stride = rows > 1 ? dlogits->stride : 0;
    }
    if (rows > 0 && few_rows(rows, logits->cols, logits->dtype)) return logits->dtype == FLASHOPTIM_FP32 ? launch_few<true>(a, stats, stream) : launch_few<false>(a, stats, stream);
    if (rows > 0 && holds_rows(rows, logits->cols, logits->dtype)) {
        FO_TRY(logits->dtype == FLASHOPTIM_FP32 ? launch_held<true>(a, stream) : launch_held<false>(a, stream));
    } else if (rows > 0) {
        const PartsArgs p = to_parts(a, logits->dtype, (char*)workspace + up(rows * 24, 16) * 16);
        FO_TRY(launch_parts(p, logits->dtype, stream));
        const dim3 grid(p.r.rows * p.parts), block(kPartThreads);
        if (logits->dtype == FLASHOPTIM_FP32) hipLaunchKernelGGL((policy_parts_kernel<true>), grid, block, 0, (hipStream_t)stream, p);
        else hipLaunchKernelGGL((policy_parts_kernel<false>), grid, block, 0, (hipStream_t)stream, p);
        FO_TRY(fo::hip_status(hipGetLastError()));
    }
    const bool by_workgroup = holds_rows(rows, logits->cols, logits->dtype) && long_rows(rows, logits->cols, logits->dtype);
    hipLaunchKernelGGL(policy_stats_kernel, dim3(1), dim3(kPairThreads), 0, (hipStream_t)stream, a.policy.terms, by_workgroup ? kUnits : a.rows, spec->kl_weight, stats);
    return fo::hip_status(hipGetLastError());
}

int flashoptim_preference_loss(const flashoptim_preference_spec* spec, const float* logprob, const double* logprob64,
                               const float* ref_logprob, const float* weights, int64_t rows, const int64_t* offsets, int64_t pairs,
                               float* loss, float* margins, float* dlogprob, void* stream) {
    if (!spec || !loss || rows < 0 || pairs < 0 || spec->kind < 0 || spec->kind > 2 || spec->order < 0 || spec->order > 1 || (logprob && logprob64))
        return FLASHOPTIM_ERR_INVALID_ARG;
    if (!(spec->beta > 0.0f) || !std::isfinite(spec->beta) || !(spec->label_smoothing >= 0.0f && spec->label_smoothing <= 0.5f) ||
        (spec->label_smoothing != 0.0f && spec->kind != FLASHOPTIM_PREFERENCE_SIGMOID))
        return FLASHOPTIM_ERR_INVALID_ARG;
    if (rows >= ((int64_t)1 << 31) || pairs >= ((int64_t)1 << 30)) return FLASHOPTIM_ERR_NUMEL_RANGE;
    if ((rows > 0 && !logprob && !logprob64) || (pairs > 0 && !offsets)) return FLASHOPTIM_ERR_INVALID_ARG;
    for (const float* p : {logprob, ref_logprob, weights, (const float*)loss, (const float*)margins, (const float*)dlogprob})
        if (!fo::aligned_to(p, 4)) return FLASHOPTIM_ERR_MISALIGNED;
    if (!fo::aligned_to(offsets, 8) || !fo::aligned_to(logprob64, 8)) return FLASHOPTIM_ERR_MISALIGNED;
    const PairArgs a = {logprob, logprob64, ref_logprob, weights, offsets, loss, margins, dlogprob, rows, pairs, *spec};
    int groups = 1;
    while (groups < 16 && groups < pairs) groups *= 2;
    hipLaunchKernelGGL(preference_kernel, dim3(1), dim3(kPairThreads), 0, (hipStream_t)stream, a, groups);
    return fo::hip_status(hipGetLastError());
}

}  // extern "C"
