// Microscaled 4-bit matrices on gfx950: quantisation from BF16, FP32 or split weights (along rows, along columns, or both from one
// pass), the way back, and the products of a linear layer and its gradients on the matrix cores' scaled 4-bit instructions.
//
// The arithmetic of a block of 32 values: max|v| has the exponent field E, the block's scale is 2^(E - 2 - 127), so that the
// largest magnitude lies in [4, 8) on the grid {0, 0.5, 1, 1.5, 2, 3, 4, 6}.  The scaling is exact, so a code is decided by comparing
// exact numbers: v_cvt_scalef32_pk_fp4_f32 does that to nearest, ties to even, for scale bytes down to 0 and for subnormal values
// (every one of the 2^20 pairs of a check over all of these agreed); the stochastic rounding compares exactly in FP32.

#include <hip/hip_runtime.h>
#include <stdint.h>
#include <string.h>

#include <type_traits>

#include "flashoptim.h"
#include "flashoptim_host.h"
#include "flashoptim_layers.h"
#include "flashoptim_mx4.h"

namespace {

using i32x8 = int __attribute__((ext_vector_type(8)));
using bf16x4 = __bf16 __attribute__((ext_vector_type(4)));

using fo::f32x4;
using fo::i32x4;
using fo::kBlock;
using fo::kScaleBytes;
using fo::kScaleSteps;
using fo::kSegment;
using fo::kSegmentBytes;
using fo::kTileCols;
using fo::load_as;
using fo::store_as;
using fo::up;

// A 4-bit matrix as a kernel takes it.
struct Mx4 {
    uint8_t* codes;
    uint8_t* scales;
    uint32_t rows, cols;
    uint32_t segments;      // of 256 values to a row: 128 bytes of codes, 8 of scales
    uint32_t scale_pitch;   // bytes
};
Mx4 to_dev(const flashoptim_mx4& m) {
    return {m.codes, m.scales, (uint32_t)m.rows, (uint32_t)m.cols, (uint32_t)up(m.cols, kSegment), (uint32_t)(16 * up(m.cols, 2 * kSegment))};
}

enum SourceKind { kBf16, kFp32, kSplit };
struct Source {
    const void* data;
    const int8_t* rho;       // kSplit
    const uint8_t* rand;     // stochastic rounding
    int64_t stride;
    uint32_t rows, cols;
};

// load_as of data that this kernel reads once: it leaves the caches to what is read again.
template <typename T, int ALIGN>
__device__ __forceinline__ T load_once(const void* p) {
    typedef T Unaligned __attribute__((aligned(ALIGN)));
    return __builtin_nontemporal_load((const Unaligned*)p);
}

__device__ __forceinline__ float bf16_value(uint32_t bits) { return __uint_as_float(bits << 16); }

// theta' + (rho / 127) ULP(theta') / 2 (Section 3.1, Eq. 2), as the optimizer step reconstructs it.
__device__ __forceinline__ float master_weight(uint32_t bits, int rho) {
    const float base = bf16_value(bits), r = (float)rho;
    const int e = (int)(bits >> 7) & 255;
    const float q = fmaf(r, 0x1.020408p-7f, r * 0x1.020408p-35f);        // rho / 127, correctly rounded for every byte
    return e == 255 ? base : base + __builtin_amdgcn_ldexpf(q, max(e, 1) - 135);
}

// Eight consecutive values of a row as they lie in memory, with their corrections and random bytes.
struct Eight {
    i32x4 a, b;      // (b: FP32 only)
    uint64_t rho, rand;
};
template <int SRC>
__device__ __forceinline__ void load_whole(Eight& e, const Source& s, uint32_t row, uint32_t col) {
    const int64_t at = (int64_t)row * s.stride + col, packed = (int64_t)row * s.cols + col;
    if constexpr (SRC == kFp32) {
        e.a = load_once<i32x4, 4>((const float*)s.data + at);
        e.b = load_once<i32x4, 4>((const float*)s.data + at + 4);
    } else {
        e.a = load_once<i32x4, 2>((const uint16_t*)s.data + at);
    }
    if constexpr (SRC == kSplit) e.rho = load_once<uint64_t, 1>(s.rho + packed);
    if (s.rand) e.rand = load_once<uint64_t, 1>(s.rand + packed);
}
template <int SRC>
__device__ __forceinline__ void unpack(float (&v)[8], const Eight& e) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if constexpr (SRC == kFp32) {
            v[i] = __int_as_float(i < 4 ? e.a[i] : e.b[i - 4]);
        } else {
            const uint32_t bits = i % 2 ? (uint32_t)e.a[i / 2] >> 16 : (uint32_t)e.a[i / 2] & 0xffffu;
            if constexpr (SRC == kSplit) v[i] = master_weight(bits, (int)(int8_t)(e.rho >> (8 * i)));
            else v[i] = bf16_value(bits);
        }
    }
}
// The same where the row may end within the eight or before them: 0 behind its end.  What is not there is loaded from the last place that
// is: a load that is made only if it is there would wait for the one before.
template <int SRC>
__device__ __forceinline__ void load8(float (&v)[8], uint64_t& rand, const Source& s, uint32_t row, uint32_t col) {
    const uint32_t left = col < s.cols ? s.cols - col : 0;
    Eight e = {};
    if (left >= 8) {
        load_whole<SRC>(e, s, row, col);
    } else if (left > 0) {
        const int last = (int)left - 1;
        const int64_t at = (int64_t)row * s.stride + col, packed = (int64_t)row * s.cols + col;
        uint32_t w[8];
        uint8_t rho[8], r[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if constexpr (SRC == kFp32) w[i] = ((const uint32_t*)s.data)[at + min(i, last)];
            else w[i] = ((const uint16_t*)s.data)[at + min(i, last)];
            if constexpr (SRC == kSplit) rho[i] = (uint8_t)s.rho[packed + min(i, last)];
            if (s.rand) r[i] = s.rand[packed + min(i, last)];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (i > last) continue;
            if constexpr (SRC == kFp32) { if (i < 4) e.a[i] = (int)w[i]; else e.b[i - 4] = (int)w[i]; }
            else e.a[i / 2] |= (int)(w[i] << (16 * (i % 2)));
            if constexpr (SRC == kSplit) e.rho |= (uint64_t)rho[i] << (8 * i);
            if (s.rand) e.rand |= (uint64_t)r[i] << (8 * i);
        }
    }
    rand = e.rand;
    unpack<SRC>(v, e);
}

__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// The scale byte of a block whose largest magnitude has these bits.
template <bool RANDOM>
__device__ __forceinline__ uint32_t scale_byte(uint32_t largest) {
    int byte = (int)(largest >> 23) - 2;
    if (RANDOM && (largest & 0x7fffffu) > 0x400000u) ++byte;
    return largest >= 0x7f800000u ? 255u : (uint32_t)max(byte, 0);
}

// One stochastically rounded code of a value whose random byte is r.  With t = |v| 2^(127 - byte) <= 6, from 1 on the grid's codes are the upper bits of
// t's own representation (one mantissa bit), the 22 below them the share (t - a) / (b - a) in units of 2^-22: what is added carries into the
// code exactly if the share exceeds (r + 1/2) / 256.  Below 1, where the grid goes on in steps of 1/2, 2^23 t takes that place, rounded up to a whole
// number, which leaves the comparison with whole numbers as it is; of a BF16 value, 1 + t has the same bits (it is exact, or t too small to
// be rounded up).
template <bool BF16>
__device__ __forceinline__ uint32_t random_code(float v, float up_scale, uint32_t r) {
    const float t = fabsf(v) * up_scale;
    const uint32_t above = __float_as_uint(t) - (252u << 22);
    const uint32_t below = BF16 ? __float_as_uint(1.0f + t) - (254u << 22) : (uint32_t)ceilf(t * 0x1p23f);
    const uint32_t place = t < 1.0f ? below : above;
    return ((place + (0x3fffffu - 0x2000u) - (r << 14)) >> 22) | (__float_as_uint(v) >> 31) << 3;
}

// Eight codes, the first in the lowest bits.
template <bool RANDOM, bool BF16 = false>
__device__ __forceinline__ uint32_t codes8(const float* v, uint32_t byte, uint64_t r) {
    if constexpr (RANDOM) {
        const float up_scale = __uint_as_float((254u - (byte == 255u ? 0u : byte)) << 23);
        uint32_t c = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) c |= random_code<BF16>(v[i], up_scale, (uint32_t)(r >> (8 * i)) & 255u) << (4 * i);
        return byte == 255u ? 0u : c;
    } else {
        const float scale = __uint_as_float(byte << 23);
        uint32_t c = 0;
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[0], v[1], scale, 0);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[2], v[3], scale, 1);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[4], v[5], scale, 2);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[6], v[7], scale, 3);
        return byte == 255u ? 0u : c;
    }
}

// The largest of a value over the four lanes of a quad.
__device__ __forceinline__ uint32_t quad_max(uint32_t v) {
    v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0xb1, 0xf, 0xf, true));   // quad_perm [1,0,3,2]
    return max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x4e, 0xf, 0xf, true));   // quad_perm [2,3,0,1]
}

// Codes and scale of the eight values that this lane has of its quad's block.
template <bool RANDOM, bool BF16 = false>
__device__ __forceinline__ uint32_t quad_codes(const float (&v)[8], uint64_t r, uint32_t* byte) {
    uint32_t largest = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) largest = max(largest, magnitude(v[i]));
    *byte = scale_byte<RANDOM>(quad_max(largest));
    return codes8<RANDOM, BF16>(v, *byte, r);
}

// The same from eight BF16 values as they lie in memory, without unpacking them.
__device__ __forceinline__ uint32_t quad_codes_bf16(i32x4 w, uint32_t* byte) {
    using u16x2 = unsigned short __attribute__((ext_vector_type(2)));
    using bf16x2 = __bf16 __attribute__((ext_vector_type(2)));
    u16x2 largest = {};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int m = w[i] & 0x7fff7fff;
        largest = __builtin_elementwise_max(largest, __builtin_bit_cast(u16x2, m));
    }
    *byte = scale_byte<false>(quad_max((uint32_t)max(largest[0], largest[1]) << 16));
    const float scale = __uint_as_float(*byte << 23);
    bf16x2 v[4];      // (by memcpy: a bit cast of a vector's element takes its first)
    __builtin_memcpy(v, &w, 16);
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, v[0], scale, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, v[1], scale, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, v[2], scale, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, v[3], scale, 3);
    return *byte == 255u ? 0u : c;
}

// ------------------------------------------------------------------------------------------------ along rows --

// Half a wavefront handles a segment of 256 values: eight to a lane, a block to a quad.
template <int SRC, bool RANDOM>
__global__ __launch_bounds__(256) void quantize_rows(Source s, Mx4 out, uint32_t total) {
    const uint32_t unit = blockIdx.x * 8 + threadIdx.x / 32, lane = threadIdx.x % 32;
    if (unit >= total) return;
    const uint32_t row = unit / out.segments, seg = unit - row * out.segments;
    const uint32_t col = seg * kSegment + lane * 8;
    float v[8];
    uint64_t r = 0;
    load8<SRC>(v, r, s, row, col);
    uint32_t byte;
    const uint32_t c = quad_codes<RANDOM, SRC == kBf16>(v, r, &byte);
    store_as(out.codes + ((int64_t)row * out.segments + seg) * kSegmentBytes + lane * 4, c);
    uint8_t* scales = out.scales + (int64_t)row * out.scale_pitch + seg * 8;
    if (lane % 4 == 0) scales[lane / 4] = (uint8_t)byte;
    if (seg + 1 == out.segments && (out.segments & 1) && lane < 8) scales[8 + lane] = 0;
}

// ---------------------------------------------------------------------------------- along columns, or both ways --

// A workgroup handles ROWS by 128 values: the rows as above, and through LDS the columns.  The grid covers rows and columns up to whole
// segments, so that what lies behind the matrix's end is written as zeros in both layouts.  All loads of a tile are on their way together:
// where a tile reaches beyond the matrix, its lanes load from its last row, or a row's first values, and drop them.
// Bound: HBM.  An XCD goes through its tiles in bands of 1024 rows, down each column of a band: its L2 then puts the tiles' 16 or 32 bytes of a row of
// out_t together, and a band's rows of out, 64 bytes from each tile, while they are there.  In us, down whole columns / in bands / and with x read
// past the caches: 14336 x 4096 split weights from memory 63 / 57 / 54, BF16 55 / 48 / 45, along the rows 66 and 53.
template <int SRC, bool RANDOM, int ROWS>
__global__ __launch_bounds__(fo::kTileLanes) void quantize_both(Source s, Mx4 out, Mx4 out_t, bool rows_too, uint32_t row_tiles, uint32_t tiles) {
    using Cell = typename std::conditional<SRC == kBf16, uint16_t, float>::type;
    constexpr int kPasses = ROWS / 16;
    __shared__ Cell tile[ROWS][kTileCols];
    __shared__ uint8_t rands[RANDOM ? ROWS : 1][kTileCols];
    const uint32_t xcd = blockIdx.x % 8, at = xcd * (tiles / 8) + min(xcd, tiles % 8) + blockIdx.x / 8;
    constexpr uint32_t kBand = 1024 / ROWS;
    const uint32_t col_tiles = tiles / row_tiles, band = at / (kBand * col_tiles), in_band = at - band * kBand * col_tiles;
    const uint32_t height = min(kBand, row_tiles - band * kBand);
    const uint32_t row0 = (band * kBand + in_band % height) * ROWS, col0 = in_band / height * kTileCols;
    const uint32_t lane = threadIdx.x % 16, line = threadIdx.x / 16;
    const uint32_t col = col0 + lane * 8;
    const bool ragged = s.cols % 8 != 0 && col0 + kTileCols > s.cols;      // a row ends within some lane's eight values
    Eight e[kPasses];
    if (!ragged) {
#pragma unroll
        for (int i = 0; i < kPasses; ++i) load_whole<SRC>(e[i], s, min(row0 + i * 16 + line, s.rows - 1), col < s.cols ? col : 0);
    }
#pragma unroll
    for (int i = 0; i < kPasses; ++i) {
        const uint32_t row = row0 + i * 16 + line;
        float v[8];
        uint64_t r = 0;
        if (ragged) {
            if (row < s.rows) load8<SRC>(v, r, s, row, col);
        } else {
            unpack<SRC>(v, e[i]);
            r = e[i].rand;
        }
        if (row >= s.rows || col >= s.cols) {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = 0.0f;
            r = 0;
        }
        Cell* cell = &tile[i * 16 + line][lane * 8];
        if constexpr (SRC == kBf16) {
            i32x4 w;
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = (int)((__float_as_uint(v[2 * j]) >> 16) | (__float_as_uint(v[2 * j + 1]) & 0xffff0000u));
            *(i32x4*)cell = w;
        } else {
            *(f32x4*)cell = f32x4{v[0], v[1], v[2], v[3]};
            *(f32x4*)(cell + 4) = f32x4{v[4], v[5], v[6], v[7]};
        }
        if constexpr (RANDOM) *(uint64_t*)&rands[i * 16 + line][lane * 8] = r;
        if (rows_too && row < s.rows) {
            uint32_t byte;
            const uint32_t c = quad_codes<RANDOM, SRC == kBf16>(v, r, &byte);
            if (col < out.segments * kSegment) {
                store_as(out.codes + (int64_t)row * out.segments * kSegmentBytes + col / 2, c);
                if (lane % 4 == 0) out.scales[(int64_t)row * out.scale_pitch + col / kBlock] = (uint8_t)byte;
            }
        }
    }
    if (rows_too && col0 + kTileCols == out.segments * kSegment && (out.segments & 1)) {       // the row's scales behind the last segment
        const uint32_t row = row0 + threadIdx.x / 2;
        if (threadIdx.x < 2 * ROWS && row < s.rows) store_as(out.scales + (int64_t)row * out.scale_pitch + out.segments * 8 + threadIdx.x % 2 * 4, 0u);
    }
    __syncthreads();
    // a lane takes 32 rows of a column
    const uint32_t c = threadIdx.x % kTileCols, col_t = col0 + c;
#pragma unroll
    for (uint32_t block = threadIdx.x / kTileCols; block < ROWS / kBlock; block += 256 / kTileCols) {
        float v[kBlock];
        uint32_t largest = 0;
#pragma unroll
        for (int i = 0; i < kBlock; ++i) {
            if constexpr (SRC == kBf16) v[i] = bf16_value(tile[block * kBlock + i][c]);
            else v[i] = tile[block * kBlock + i][c];
            largest = max(largest, magnitude(v[i]));
        }
        const uint32_t byte = scale_byte<RANDOM>(largest);
        i32x4 codes;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            uint64_t r = 0;
            if constexpr (RANDOM) {
#pragma unroll
                for (int i = 0; i < 8; ++i) r |= (uint64_t)rands[block * kBlock + j * 8 + i][c] << (8 * i);
            }
            codes[j] = (int)codes8<RANDOM, SRC == kBf16>(v + 8 * j, byte, r);
        }
        const uint32_t at_row = row0 + block * kBlock;
        if (col_t < s.cols && at_row < out_t.segments * kSegment) {
            store_as(out_t.codes + (int64_t)col_t * out_t.segments * kSegmentBytes + at_row / 2, codes);
            uint8_t* scales = out_t.scales + (int64_t)col_t * out_t.scale_pitch;
            scales[at_row / kBlock] = (uint8_t)byte;
            if (at_row + kSegment >= out_t.segments * kSegment && (out_t.segments & 1)) scales[at_row / kBlock + 8] = 0;      // behind the last segment
        }
    }
}

// --------------------------------------------------------------------------------------------------- the way back --

__device__ __forceinline__ float code_value(uint32_t code, float scale) {
    // magnitude index 2 e + m: m / 2 for e = 0, (1 + m / 2) 2^(e - 1) else: as a float the exponent field e + 126 and the top mantissa
    // bit m, of which 0 and 1 (that is 0 and 1/2) are no such numbers
    const uint32_t i = code & 7u;
    const float v = i < 2 ? 0.5f * (float)i : __uint_as_float((i << 22) + (126u << 23));
    return __uint_as_float(__float_as_uint(v * scale) | (code & 8u) << 28);
}

template <bool FP32>
__global__ __launch_bounds__(256) void dequantize_rows(Mx4 q, void* data, int64_t stride, uint32_t total) {
    const uint32_t unit = blockIdx.x * 8 + threadIdx.x / 32, lane = threadIdx.x % 32;
    if (unit >= total) return;
    const uint32_t row = unit / q.segments, seg = unit - row * q.segments;
    const uint32_t col = seg * kSegment + lane * 8;
    if (col >= q.cols) return;
    const uint32_t c = load_as<uint32_t>(q.codes + ((int64_t)row * q.segments + seg) * kSegmentBytes + lane * 4);
    const uint32_t byte = q.scales[(int64_t)row * q.scale_pitch + seg * 8 + lane / 4];
    const float scale = __uint_as_float(byte == 0 ? 0x00400000u : byte == 255 ? 0x7fc00000u : byte << 23);
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = code_value(c >> (4 * i), scale);
    const uint32_t left = q.cols - col;
    if constexpr (FP32) {
        float* p = (float*)data + (int64_t)row * stride + col;
        if (left >= 8) {
            store_as(p, f32x4{v[0], v[1], v[2], v[3]});
            store_as(p + 4, f32x4{v[4], v[5], v[6], v[7]});
        } else {
            for (uint32_t i = 0; i < 8; ++i) if (i < left) p[i] = v[i];
        }
    } else {                     // two significant bits and an exponent of at least -128: exact in BF16
        uint16_t* p = (uint16_t*)data + (int64_t)row * stride + col;
        if (left >= 8) {
            i32x4 w;
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = (int)((__float_as_uint(v[2 * j]) >> 16) | (__float_as_uint(v[2 * j + 1]) & 0xffff0000u));
            store_as(p, w);
        } else {
#pragma unroll
            for (uint32_t i = 0; i < 8; ++i) if (i < left) p[i] = (uint16_t)(__float_as_uint(v[i]) >> 16);
        }
    }
}

// ------------------------------------------------------------------------------------------------------- products --
//
// c[i][j] = sum over k of a[i][k] b[j][k].  The matrix instruction takes 16 rows of each operand and 128 terms: lane l has row l % 16
// and, of four blocks of 32 terms, number l / 16.  Which blocks of the sum these are is ours to choose, as long as both operands agree: a
// segment of 256 terms is two instructions s = 0, 1, and quarter q of the lanes takes block 2 q + s, so that a lane's 32 bytes of
// codes and its two scale bytes are contiguous.  The instruction's rows are b's, its columns a's: a lane then holds four neighbouring
// values of a row of c.

__device__ __forceinline__ f32x4 mfma(i32x4 p, i32x4 q, f32x4 acc, int p_scale, int q_scale, int s) {
    const i32x8 pw = {p[0], p[1], p[2], p[3], 0, 0, 0, 0}, qw = {q[0], q[1], q[2], q[3], 0, 0, 0, 0};
    return s == 0 ? __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(pw, qw, acc, 4, 4, 0, p_scale, 0, q_scale)
                  : __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(pw, qw, acc, 4, 4, 1, p_scale, 1, q_scale);
}

struct Result {
    void* data;
    int64_t stride;
    uint32_t rows, cols;
};

template <bool FP32>
__device__ __forceinline__ void store_result4(const Result& c, uint32_t row, uint32_t col, f32x4 v) {
    if (row >= c.rows || col >= c.cols) return;
    const uint32_t left = c.cols - col;
    if constexpr (FP32) {
        float* p = (float*)c.data + (int64_t)row * c.stride + col;
        if (left >= 4) store_as(p, v);
        else for (uint32_t i = 0; i < 4; ++i) if (i < left) p[i] = v[i];
    } else {
        const bf16x4 w = __builtin_convertvector(v, bf16x4);
        __bf16* p = (__bf16*)c.data + (int64_t)row * c.stride + col;
        if (left >= 4) store_as(p, w);
        else for (uint32_t i = 0; i < 4; ++i) if (i < left) p[i] = w[i];
    }
}

// 16 bytes of a row of c.
template <bool FP32>
__device__ __forceinline__ void store_result16(const Result& c, uint32_t row, uint32_t col, i32x4 v) {
    if (row >= c.rows || col >= c.cols) return;
    uint8_t* p = (uint8_t*)c.data + ((int64_t)row * c.stride + col) * (FP32 ? 4 : 2);
    const uint32_t left = c.cols - col;
    if (left >= (FP32 ? 4 : 8)) {
        store_as(p, v);
    } else if constexpr (FP32) {
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) if (i < left) ((int*)p)[i] = v[i];
    } else {
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) if (i < left) ((uint16_t*)p)[i] = (uint16_t)((uint32_t)v[i / 2] >> (16 * (i % 2)));
    }
}

// A workgroup makes 16 columns by 16 rows of c; its wavefronts share out the segments of the sum and are added up through LDS.
template <bool FP32, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void product_small(Mx4 b, Mx4 a, Result c, uint32_t p_tiles) {
    __shared__ f32x4 part[WAVES][64];
    const uint32_t wave = threadIdx.x / 64, lane = threadIdx.x % 64, q = lane / 16;
    const uint32_t q_tile = blockIdx.x / p_tiles, p_tile = blockIdx.x - q_tile * p_tiles;
    const uint32_t b_row = min(p_tile * 16 + lane % 16, b.rows - 1), a_row = min(q_tile * 16 + lane % 16, a.rows - 1);
    const uint8_t* pb = b.codes + (int64_t)b_row * b.segments * kSegmentBytes + q * 32;
    const uint8_t* pa = a.codes + (int64_t)a_row * a.segments * kSegmentBytes + q * 32;
    const uint8_t* sb = b.scales + (int64_t)b_row * b.scale_pitch + q * 2;
    const uint8_t* sa = a.scales + (int64_t)a_row * a.scale_pitch + q * 2;
    f32x4 acc = {};
    for (uint32_t seg = wave; seg < b.segments; seg += WAVES) {
        i32x4 wb[2], wa[2];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            wb[s] = load_as<i32x4>(pb + (int64_t)seg * kSegmentBytes + s * 16);
            wa[s] = load_as<i32x4>(pa + (int64_t)seg * kSegmentBytes + s * 16);
        }
        const int xb = load_as<uint16_t>(sb + seg * 8), xa = load_as<uint16_t>(sa + seg * 8);
#pragma unroll
        for (int s = 0; s < 2; ++s) acc = mfma(wb[s], wa[s], acc, xb, xa, s);
    }
    part[wave][lane] = acc;
    __syncthreads();
    if (wave == 0) {
#pragma unroll
        for (int w = 1; w < WAVES; ++w) acc += part[w][lane];
        store_result4<FP32>(c, q_tile * 16 + lane % 16, p_tile * 16 + q * 4, acc);
    }
}

// Large products: a workgroup makes BP columns by BQ rows of c.  A step takes a segment of 256 terms, 128 bytes of codes of each row,
// which come to LDS straight from memory (no registers in between) while the matrix cores work on the segment before.  A wavefront makes
// BP / WP by BQ / WQ values in tiles of 32 by 32, whose instruction takes 64 terms: half h of its lanes takes blocks 4 h .. 4 h + 3 of the
// segment in four turns, so that a lane's four scales are one word.
//
// What bounds it: 8192 x 14336 x 4096 takes 430 thousand cycles, in 229 thousand of which the matrix cores are busy; between the products of two
// segments lie the meeting of all wavefronts and their first reads of LDS behind it.  And the package's power, which holds the clock at 1.82 GHz: 236 us, 4.1
// PFLOP/s; with all codes zero, in as many cycles at 2.39 GHz, 178 us, 5.4 PFLOP/s.  8192 x 8192 x 8192 246 us, 4.5 PFLOP/s, zeros 185, 5.9.
// What it took, for 8192 x 8192 x 8192 as it was before the results left through LDS:
//   * scales for 1024 terms at a time instead of 256 (a copy's rows pass the memory pipe one after the other, and 8 bytes of a row take it
//     as long as 128): 305 -> 300 us, and with 128 by 128 tiles 357 -> 296;
//   * the next segment's copies go out one by one between the products (together, all wavefronts of a workgroup queue up in front of the memory
//     pipe before their first product): 300 -> 266;
//   * steps of 128 terms, with four stages: 287 (64-byte pieces of rows).  Wavefronts of 128 by 128 values, one to a SIMD: 273.
// The tile of 256 by 256 fills the LDS (160 KB), so that one workgroup is resident on a compute unit.
using f32x16 = float __attribute__((ext_vector_type(16)));

template <int ROWS>
struct Stage {
    uint8_t codes[ROWS * kSegmentBytes];
};
template <int ROWS>
struct Scales {
    uint8_t bytes[ROWS * kScaleBytes];
};
#define FO_LDS(p) ((__attribute__((address_space(3))) void*)(p))

// `bytes` bytes from p on as a buffer; an address into it is a lane's 32-bit offset.
__device__ __forceinline__ i32x4 buffer_of(const uint8_t* p, uint32_t bytes) {
    const uint64_t at = (uint64_t)p;
    return i32x4{__builtin_amdgcn_readfirstlane((int)(uint32_t)at), __builtin_amdgcn_readfirstlane((int)(uint32_t)(at >> 32)),
                 __builtin_amdgcn_readfirstlane((int)bytes), 0x00020000};
}

// Copies 16 bytes for each lane from the buffer to LDS, consecutive lanes to consecutive places from `to` on; from an empty buffer, nothing is
// fetched.  It has no result in registers, so that written as assembly it is safe; written with the builtin, the compiler has every later read
// of LDS wait for it, whichever stage it reads.  What waits for it is wait_copies.  The compiler does not see into it, so what it would do is done here: m0
// is declared as written (it warns that it keeps nothing in m0 across a statement, as is right: it sets m0 right ahead of its own uses); s_nop
// makes the five cycles that a scalar register which a vector instruction wrote needs before a load reads it, and the one that m0 needs.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void copy_to_lds(i32x4 buffer, uint32_t lane_offset, void* to) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"((uint32_t)(uintptr_t)FO_LDS(to)), "v"(lane_offset), "s"(buffer)
                 : "memory", "m0");
}
#pragma clang diagnostic pop
// Waits until all but the last `VM` of this wavefront's copies have landed and its reads of LDS have come back.
template <int VM>
__device__ __forceinline__ void wait_copies() {
    static_assert(VM < 64, "six bits");
    __builtin_amdgcn_s_waitcnt((VM & 15) | (VM >> 4) << 14 | 0x0070);
}

// A barrier for what lies in LDS, which the waits around it have settled: the compiler, which does not know of the copies, moves no access across.
__device__ __forceinline__ void meet() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// What a wavefront copies of ROWS rows: the lane's places in them.  Behind the matrix's last row a copy takes that row again.
template <int ROWS, int WAVES>
struct Copier {
    // Copies of 1024 bytes.  All wavefronts make as many, so that they can count alike: where there are fewer of scales than wavefronts, some twice.
    static constexpr int kCodes = ROWS * kSegmentBytes / 1024 / WAVES, kAllScales = ROWS * kScaleBytes / 1024, kScales = (kAllScales + WAVES - 1) / WAVES;
    static_assert(kCodes * 1024 * WAVES == ROWS * kSegmentBytes && (kAllScales % WAVES == 0 || WAVES % kAllScales == 0), "every wavefront copies as much");
    const uint8_t *codes, *scales;      // from the tile's first row on
    uint32_t code_bytes, scale_bytes;
    uint32_t code_at[kCodes], scale_at[kScales];
    int wave;
    __device__ __forceinline__ Copier(const Mx4& m, uint32_t row0, int wave, int lane) : wave(wave) {
        const uint32_t last = min(m.rows - 1 - row0, (uint32_t)ROWS - 1), pitch = m.segments * kSegmentBytes;
        codes = m.codes + (int64_t)row0 * pitch;
        scales = m.scales + (int64_t)row0 * m.scale_pitch;
        code_bytes = (last + 1) * pitch;
        scale_bytes = (last + 1) * m.scale_pitch;
#pragma unroll
        for (int i = 0; i < kCodes; ++i) code_at[i] = fo::code_place(wave * kCodes + i, lane, last, pitch);
#pragma unroll
        for (int i = 0; i < kScales; ++i) scale_at[i] = fo::scale_place((wave * kScales + i) % kAllScales, lane, last, m.scale_pitch);
    }
    // The codes of a step; `there`: there is such a step.
    __device__ __forceinline__ i32x4 buffer(uint32_t step, bool there) const {
        const fo::CopyBuffer b = fo::copy_buffer(code_bytes, step * kSegmentBytes, there);
        return buffer_of(codes + b.begin, b.bytes);
    }
    __device__ __forceinline__ void copy_codes(i32x4 buffer, Stage<ROWS>& to, int i) const {
        copy_to_lds(buffer, code_at[i], to.codes + (wave * kCodes + i) * 1024);
    }
    __device__ __forceinline__ void copy_scales(Scales<ROWS>& to, uint32_t group, bool there) const {
        const fo::CopyBuffer b = fo::copy_buffer(scale_bytes, group * kScaleBytes, there);
        const i32x4 buffer = buffer_of(scales + b.begin, b.bytes);
#pragma unroll
        for (int i = 0; i < kScales; ++i) copy_to_lds(buffer, scale_at[i], to.bytes + (wave * kScales + i) % kAllScales * 1024);
    }
};

template <int ROWS>
__device__ __forceinline__ i32x4 piece(const Stage<ROWS>& s, int row, int c) {
    return *(const i32x4*)(s.codes + row * kSegmentBytes + (c ^ fo::code_swizzle(row)) * 16);
}
// The scales of half h of the row's blocks in the step-th segment of the 1024 terms: the lowest byte is the first one's.
template <int ROWS>
__device__ __forceinline__ int scales_of(const Scales<ROWS>& s, int row, int step, int h) {
    return *(const int*)(s.bytes + row * kScaleBytes + ((step * 8 + h * 4) ^ fo::scale_swizzle(row) * 16));
}

template <int TURN>
__device__ __forceinline__ f32x16 mfma32(i32x4 p, i32x4 q, f32x16 acc, int p_scale, int q_scale) {
    const i32x8 pw = {p[0], p[1], p[2], p[3], 0, 0, 0, 0}, qw = {q[0], q[1], q[2], q[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(pw, qw, acc, 4, 4, TURN, p_scale, TURN, q_scale);
}

template <int TURN, int BP, int BQ, int TP, int TQ>
__device__ __forceinline__ void read_turn(const Stage<BP>& p, const Stage<BQ>& q, int p0, int q0, int h, i32x4 (&pw)[TP], i32x4 (&qw)[TQ]) {
#pragma unroll
    for (int i = 0; i < TP; ++i) pw[i] = piece(p, p0 + 32 * i, 4 * h + TURN);
#pragma unroll
    for (int j = 0; j < TQ; ++j) qw[j] = piece(q, q0 + 32 * j, 4 * h + TURN);
    __builtin_amdgcn_sched_barrier(0);
}
template <int TURN, int TP, int TQ, typename F>
__device__ __forceinline__ void multiply_turn(const i32x4 (&pw)[TP], const i32x4 (&qw)[TQ], const int (&p_scale)[TP], const int (&q_scale)[TQ],
                                              f32x16 (&acc)[TP][TQ], F behind) {
#pragma unroll
    for (int i = 0; i < TP; ++i)
#pragma unroll
        for (int j = 0; j < TQ; ++j) {
            acc[i][j] = mfma32<TURN>(pw[i], qw[j], acc[i][j], p_scale[i], q_scale[j]);
            behind((TURN * TP + i) * TQ + j);
        }
    __builtin_amdgcn_sched_barrier(0);
}

// One product or two that do not depend on each other (the gradients of a linear layer): two launches would each leave compute units idle at their
// end.  With the quantisation ahead of them, 1024 x 768 x 2304 and 2304 x 768 x 1024 18.4 us, in one launch 16.8; 4096 x 14336 x 4096 and 4096 x
// 14336 x 4096 284, in one 250.
struct Product {
    Mx4 b, a;
    Result c;
    uint32_t p_tiles, tiles;
};
template <int COUNT>
struct Products {
    Product of[COUNT];
};

template <int COUNT, bool FP32, int BP, int BQ, int WP, int WQ, int STAGES, int RESIDENT>
__global__ __launch_bounds__(64 * WP * WQ, RESIDENT) void product_tiles(Products<COUNT> products) {
    constexpr int kWaves = WP * WQ, TP = BP / WP / 32, TQ = BQ / WQ / 32;
    struct Lds {
        Stage<BP> p_stage[STAGES];
        Stage<BQ> q_stage[STAGES];
        Scales<BP> p_scales[2];
        Scales<BQ> q_scales[2];
    };
    __shared__ __align__(16) Lds lds;
    auto& p_stage = lds.p_stage;
    auto& q_stage = lds.q_stage;
    auto& p_scales = lds.p_scales;
    auto& q_scales = lds.q_scales;
    // consecutive workgroups run on different XCDs: each XCD takes a stretch of the tiles, in columns of eight, whose rows it then has in its L2
    const int second = COUNT == 2 && blockIdx.x >= products.of[0].tiles;
    const Mx4 b = products.of[second].b, a = products.of[second].a;
    const Result c = products.of[second].c;
    const uint32_t p_tiles = products.of[second].p_tiles, tiles = products.of[second].tiles, q_tiles = tiles / p_tiles;
    const uint32_t index = second ? blockIdx.x - products.of[0].tiles : blockIdx.x, xcd = index % 8;
    const uint32_t tile = xcd * (tiles / 8) + min(xcd, tiles % 8) + index / 8;
    constexpr uint32_t kColumn = 8;
    const uint32_t column = tile / (kColumn * p_tiles), in_column = tile - column * kColumn * p_tiles;
    const uint32_t height = min(kColumn, q_tiles - column * kColumn);
    const uint32_t p_tile = in_column / height, q_tile = column * kColumn + in_column - p_tile * height;

    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64;
    const Copier<BP, kWaves> p_copy(b, p_tile * BP, wave, lane);
    const Copier<BQ, kWaves> q_copy(a, q_tile * BQ, wave, lane);
    const int h = lane / 32, p0 = wave / WQ * (BP / WP) + lane % 32, q0 = wave % WQ * (BQ / WQ) + lane % 32;
    const uint32_t steps = b.segments;
    f32x16 acc[TP][TQ] = {};
    auto copy = [&](i32x4 p_buffer, i32x4 q_buffer, uint32_t step, int i) {
        if (i < p_copy.kCodes) p_copy.copy_codes(p_buffer, p_stage[step % STAGES], i);
        else q_copy.copy_codes(q_buffer, q_stage[step % STAGES], i - p_copy.kCodes);
    };
    constexpr int kCopies = p_copy.kCodes + q_copy.kCodes;
    constexpr int kEvery = TP * TQ * 2 / kCopies > 0 ? TP * TQ * 2 / kCopies : 1;      // products to a copy: all in the first half of a step
    static_assert(kEvery * kCopies <= TP * TQ * 4, "every copy has its product");
    p_copy.copy_scales(p_scales[0], 0, true);
    q_copy.copy_scales(q_scales[0], 0, true);
#pragma unroll
    for (int j = 0; j < STAGES - 1; ++j)
#pragma unroll
        for (int i = 0; i < kCopies; ++i) copy(p_copy.buffer(j, j < steps), q_copy.buffer(j, j < steps), j, i);
    for (uint32_t t = 0; t < steps; ++t) {
        // this wavefront's copies for step t have landed; behind the barrier all have, and nobody reads the stage of step t - 1 any more
        wait_copies<(STAGES - 2) * kCopies>();
        meet();
        const uint32_t group = t / kScaleSteps, in_group = t % kScaleSteps, next = t + STAGES - 1;
        if (in_group == 0) {
            p_copy.copy_scales(p_scales[group % 2 ^ 1], group + 1, t + kScaleSteps < steps);
            q_copy.copy_scales(q_scales[group % 2 ^ 1], group + 1, t + kScaleSteps < steps);
        }
        const i32x4 p_buffer = p_copy.buffer(next, next < steps), q_buffer = q_copy.buffer(next, next < steps);
        auto behind = [&](int product) {
            if (product % kEvery != 0 || product / kEvery >= kCopies) return;
            __builtin_amdgcn_sched_barrier(0);
            copy(p_buffer, q_buffer, next, product / kEvery);
            __builtin_amdgcn_sched_barrier(0);
        };
        const Stage<BP>& p = p_stage[t % STAGES];
        const Stage<BQ>& q = q_stage[t % STAGES];
        int p_scale[TP], q_scale[TQ];
#pragma unroll
        for (int i = 0; i < TP; ++i) p_scale[i] = scales_of(p_scales[group % 2], p0 + 32 * i, (int)in_group, h);
#pragma unroll
        for (int j = 0; j < TQ; ++j) q_scale[j] = scales_of(q_scales[group % 2], q0 + 32 * j, (int)in_group, h);
        // the pieces of a turn are read ahead of the products of the turn before
        i32x4 pw[2][TP], qw[2][TQ];
        read_turn<0, BP, BQ, TP, TQ>(p, q, p0, q0, h, pw[0], qw[0]);
        read_turn<1, BP, BQ, TP, TQ>(p, q, p0, q0, h, pw[1], qw[1]);
        multiply_turn<0>(pw[0], qw[0], p_scale, q_scale, acc, behind);
        read_turn<2, BP, BQ, TP, TQ>(p, q, p0, q0, h, pw[0], qw[0]);
        multiply_turn<1>(pw[1], qw[1], p_scale, q_scale, acc, behind);
        read_turn<3, BP, BQ, TP, TQ>(p, q, p0, q0, h, pw[1], qw[1]);
        multiply_turn<2>(pw[0], qw[0], p_scale, q_scale, acc, behind);
        multiply_turn<3>(pw[1], qw[1], p_scale, q_scale, acc, behind);
    }
    wait_copies<0>();
    meet();
    // Out through LDS, 32 rows of c at a time, so that a wavefront's stores are whole pieces of rows: a lane has four neighbouring columns of 32 rows, and
    // stores of those, 16 bytes of each row, would take the memory pipe as long as the products (8192 x 14336 x 4096: 285 us, and 231-237 so).
    constexpr int kValue = FP32 ? 4 : 2, kRow = BP / WP * kValue, kPitch = kRow + 16, kLanes = kRow / 16, kRows = 64 / kLanes;
    static_assert(kWaves * 32 * kPitch <= (int)sizeof(Lds), "a slab for each wavefront");
    uint8_t* const slab = (uint8_t*)&lds + wave * 32 * kPitch;
    const uint32_t col = p_tile * BP + wave / WQ * (BP / WP) + lane % kLanes * (16 / kValue);
#pragma unroll
    for (int j = 0; j < TQ; ++j) {
#pragma unroll
        for (int i = 0; i < TP; ++i)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const f32x4 v = {acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]};
                uint8_t* at = slab + lane % 32 * kPitch + (32 * i + 8 * g + 4 * h) * kValue;
                if constexpr (FP32) *(f32x4*)at = v;
                else *(bf16x4*)at = __builtin_convertvector(v, bf16x4);
            }
#pragma unroll
        for (int r = 0; r < 32; r += kRows) {
            const uint32_t row = q_tile * BQ + wave % WQ * (BQ / WQ) + 32 * j + r + lane / kLanes;
            const i32x4 v = *(const i32x4*)(slab + (r + lane / kLanes) * kPitch + lane % kLanes * 16);
            store_result16<FP32>(c, row, col, v);
        }
    }
}

// ------------------------------------------------------------------------------------------- linear, for single tokens --
//
// y = Q(x) w^T for at most 16 rows of x, in one launch.  A workgroup makes 16 TILES columns.  It asks for x and its first weights, quantises x, all of
// it, into LDS (eight values to a lane, as in quantize_rows), and multiplies; its wavefronts share out the segments of the sum and are added up
// through LDS.  Every workgroup quantises x again: 8 rows of 4096 values are 240 instructions to a lane of 512, under the latency of the weights.
// (With every lane quantising the blocks that it multiplies, without LDS, the loads of x, 16 bytes from each of 32 lines, took longer than the
// weights: 8 rows on 14336 by 4096 weights 16.6 us.)
// Bound: the weights' bytes, and for few of them the latency of one pass through memory.
struct Few {
    Source x;
    Mx4 w;
    Result y;
    uint32_t code_pitch, scale_pitch;      // of x in LDS
    uint32_t units_magic;                  // item / units = the upper half of item times this, for all items there can be
};

// The last `left` of eight values in the place of the first, 0 behind them; all 0 for left <= 0.
__device__ __forceinline__ void move_down(float (&v)[8], int left) {
    const int by = left > 0 ? 8 - left : 8;
#pragma unroll
    for (int step = 8; step >= 1; step /= 2)
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = by & step ? (i + step < 8 ? v[i + step] : 0.0f) : v[i];
}
__device__ __forceinline__ i32x4 move_down(i32x4 w, int left) {
    const int by = left > 0 ? 8 - left : 8;
    if (by & 8) w = i32x4{};
    if (by & 4) w = i32x4{w[2], w[3], 0, 0};
    if (by & 2) w = i32x4{w[1], w[2], w[3], 0};
    if (by & 1) {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = (int)((uint32_t)w[i] >> 16 | (i < 3 ? (uint32_t)w[i + 1] << 16 : 0u));
    }
    return w;
}

template <int SRC, bool FP32, int WAVES, int TILES>
__global__ __launch_bounds__(64 * WAVES) void linear_small(Few a) {
    extern __shared__ __align__(16) uint8_t lds[];
    constexpr int kAhead = fo::kFewAhead;
    const uint32_t wave = threadIdx.x / 64, lane = threadIdx.x % 64, q = lane / 16, x_row = lane % 16;
    const uint32_t segments = a.w.segments;
    const uint8_t *codes[TILES], *scales[TILES];
#pragma unroll
    for (int i = 0; i < TILES; ++i) {
        const uint32_t row = min((blockIdx.x * TILES + i) * 16 + lane % 16, a.w.rows - 1);
        codes[i] = a.w.codes + (int64_t)row * segments * kSegmentBytes + q * 32;
        scales[i] = a.w.scales + (int64_t)row * a.w.scale_pitch + q * 2;
    }
    struct Weights {
        i32x4 codes[kAhead][TILES][2];
        int scales[kAhead][TILES];
    } now, next;
    auto load = [&](Weights& to, uint32_t seg) {
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            if (seg + j * WAVES >= segments) continue;
#pragma unroll
            for (int i = 0; i < TILES; ++i) {
                const uint32_t at = (seg + j * WAVES) * kSegmentBytes;
                to.codes[j][i][0] = load_as<i32x4>(codes[i] + at);
                to.codes[j][i][1] = load_as<i32x4>(codes[i] + at + 16);
                to.scales[j][i] = load_as<uint16_t>(scales[i] + (seg + j * WAVES) * 8);
            }
        }
    };
    uint8_t* const x_codes = lds;
    uint8_t* const x_scales = lds + a.x.rows * a.code_pitch;
    const uint32_t units = segments * (kSegment / 8), total = units * a.x.rows;      // of eight values: to a row, of all
    auto store = [&](uint32_t c, uint32_t byte, uint32_t row, uint32_t unit) {
        *(uint32_t*)(x_codes + row * a.code_pitch + unit * 4) = c;
        if (unit % 4 == 0) x_scales[row * a.scale_pitch + unit / 4] = (uint8_t)byte;
    };
    // The first units of x are asked for ahead of the weights: they come back in this order, and are quantised while the weights are on their way.
    // No load is made by a case distinction, which would wait for it: a unit that the row ends in, or before, loads the row's last eight values, which
    // are then moved down to where they belong.
    auto quantize = [&](auto batch) {
        constexpr int kBatch = decltype(batch)::value, kWords = SRC == kFp32 ? 2 : 1;
        i32x4 raw[kBatch][kWords];
        auto ask = [&](uint32_t at) {
#pragma unroll
            for (int j = 0; j < kBatch; ++j) {
                const uint32_t item = min(at + j * 64 * WAVES, total - 1), row = __umulhi(item, a.units_magic);
                const int64_t from = (int64_t)row * a.x.stride + min((item - row * units) * 8, a.x.cols - 8);
#pragma unroll
                for (int i = 0; i < kWords; ++i) raw[j][i] = load_as<i32x4>((const uint8_t*)a.x.data + from * (SRC == kFp32 ? 4 : 2) + 16 * i);
            }
        };
        ask(threadIdx.x);
        load(now, wave);
        for (uint32_t at = threadIdx.x; at < total; at += 64 * WAVES * kBatch) {
            if (at != threadIdx.x) ask(at);
#pragma unroll
            for (int j = 0; j < kBatch; ++j) {
                const uint32_t item = at + j * 64 * WAVES, row = __umulhi(item, a.units_magic), unit = item - row * units;
                if (item >= total) continue;
                const int left = (int)a.x.cols - (int)unit * 8;
                uint32_t byte, c;
                if constexpr (SRC == kFp32) {
                    float v[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[i] = __int_as_float(raw[j][i / 4][i % 4]);
                    if (left < 8) move_down(v, left);
                    c = quad_codes<false>(v, 0, &byte);
                } else {
                    if (left < 8) raw[j][0] = move_down(raw[j][0], left);
                    c = quad_codes_bf16(raw[j][0], &byte);
                }
                store(c, byte, row, unit);
            }
        }
    };
    if (a.x.cols >= 8) {
        if (total <= 64 * WAVES) quantize(std::integral_constant<int, 1>{});
        else quantize(std::integral_constant<int, fo::kFewBatch>{});
    } else {
        load(now, wave);
        for (uint32_t item = threadIdx.x; item < total; item += 64 * WAVES) {
            const uint32_t row = __umulhi(item, a.units_magic), unit = item - row * units;
            float v[8];
            uint64_t r = 0;
            load8<SRC>(v, r, a.x, row, unit * 8);
            uint32_t byte;
            const uint32_t c = quad_codes<false>(v, 0, &byte);
            store(c, byte, row, unit);
        }
    }
    __syncthreads();
    f32x4 acc[TILES] = {};
    for (uint32_t seg = wave; seg < segments; seg += kAhead * WAVES) {
        if (seg + kAhead * WAVES < segments) load(next, seg + kAhead * WAVES);
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            const uint32_t at = seg + j * WAVES;
            if (at >= segments) continue;
            i32x4 x[2] = {};
            int x_scale = 0;
            if (x_row < a.x.rows) {
                x[0] = *(const i32x4*)(x_codes + x_row * a.code_pitch + at * kSegmentBytes + q * 32);
                x[1] = *(const i32x4*)(x_codes + x_row * a.code_pitch + at * kSegmentBytes + q * 32 + 16);
                x_scale = *(const uint16_t*)(x_scales + x_row * a.scale_pitch + at * 8 + q * 2);
            }
#pragma unroll
            for (int i = 0; i < TILES; ++i)
#pragma unroll
                for (int s = 0; s < 2; ++s) acc[i] = mfma(now.codes[j][i][s], x[s], acc[i], now.scales[j][i], x_scale, s);
        }
        now = next;
    }
    __syncthreads();
    f32x4* const part = (f32x4*)lds;      // [wave][tile][lane], over x
#pragma unroll
    for (int i = 0; i < TILES; ++i) part[(wave * TILES + i) * 64 + lane] = acc[i];
    __syncthreads();
    if (wave < TILES) {
        f32x4 sum = part[wave * 64 + lane];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) sum += part[(w * TILES + wave) * 64 + lane];
        store_result4<FP32>(a.y, lane % 16, (blockIdx.x * TILES + wave) * 16 + q * 4, sum);
    }
}

__global__ __launch_bounds__(256) void fill_zero(Result c, int bytes) {
    const uint32_t col = blockIdx.x * 256 + threadIdx.x;
    if (col >= c.cols) return;
    for (uint32_t row = blockIdx.y; row < c.rows; row += gridDim.y) {
        if (bytes == 4) ((float*)c.data)[(int64_t)row * c.stride + col] = 0.0f;
        else ((uint16_t*)c.data)[(int64_t)row * c.stride + col] = 0;
    }
}

// ------------------------------------------------------------------------------------------------------------ host --

int check_mx4(const flashoptim_mx4* m) {
    if (!m || m->rows < 0 || m->cols < 0) return FLASHOPTIM_ERR_INVALID_ARG;
    if (m->rows >= ((int64_t)1 << 31) || m->cols >= ((int64_t)1 << 31)) return FLASHOPTIM_ERR_NUMEL_RANGE;
    // half a wavefront to a segment: a launch stays below 2^32 lanes
    if (m->rows > 0 && up(m->cols, kSegment) >= ((int64_t)1 << 27) / m->rows) return FLASHOPTIM_ERR_NUMEL_RANGE;
    if (m->rows == 0 || m->cols == 0) return FLASHOPTIM_OK;
    if (!m->codes || !m->scales) return FLASHOPTIM_ERR_INVALID_ARG;
    if (!fo::aligned_to(m->codes, 16) || !fo::aligned_to(m->scales, 16)) return FLASHOPTIM_ERR_MISALIGNED;
    return FLASHOPTIM_OK;
}

template <int SRC, bool RANDOM>
int launch_quantize(const Source& s, const flashoptim_mx4* out, const flashoptim_mx4* out_t, hipStream_t stream) {
    if (!out_t) {
        const Mx4 o = to_dev(*out);
        const uint32_t total = o.rows * o.segments;
        hipLaunchKernelGGL((quantize_rows<SRC, RANDOM>), dim3((total + 7) / 8), dim3(256), 0, stream, s, o, total);
    } else {
        // (`out`, checked as a matrix in 4 bits, keeps this small; x by itself may be a row of out_t and more than a launch of tiles)
        if (!fo::quantize_fits(s.rows, s.cols)) return FLASHOPTIM_ERR_NUMEL_RANGE;
        const Mx4 t = to_dev(*out_t), o = out ? to_dev(*out) : Mx4{};
        auto launch = [&](auto rows) {
            constexpr int R = decltype(rows)::value;
            const uint32_t row_tiles = t.segments * (kSegment / R), tiles = (uint32_t)fo::quantize_tiles(s.rows, s.cols);
            hipLaunchKernelGGL((quantize_both<SRC, RANDOM, R>), dim3(tiles), dim3(fo::kTileLanes), 0, stream, s, o, t, out != nullptr, row_tiles, tiles);
        };
        if (fo::quantize_tile_rows(s.rows, s.cols) == 32) launch(std::integral_constant<int, 32>{});
        else launch(std::integral_constant<int, 64>{});
    }
    return fo::hip_status(hipGetLastError());
}

template <int SRC>
int launch_quantize(const Source& s, const flashoptim_mx4* out, const flashoptim_mx4* out_t, hipStream_t stream) {
    return s.rand ? launch_quantize<SRC, true>(s, out, out_t, stream) : launch_quantize<SRC, false>(s, out, out_t, stream);
}

// All arguments checked.
int quantize(const flashoptim_matrix& x, const int8_t* rho, const uint8_t* rand, const flashoptim_mx4* out, const flashoptim_mx4* out_t,
             hipStream_t stream) {
    if (x.rows == 0 || x.cols == 0) return FLASHOPTIM_OK;
    const Source s = {x.data, rho, rand, x.stride, (uint32_t)x.rows, (uint32_t)x.cols};
    if (rho) return launch_quantize<kSplit>(s, out, out_t, stream);
    return x.dtype == FLASHOPTIM_FP32 ? launch_quantize<kFp32>(s, out, out_t, stream) : launch_quantize<kBf16>(s, out, out_t, stream);
}

// Calls launch with the number of wavefronts that share out a sum over this many segments.
template <typename F>
void with_waves(int64_t segments, F launch) {
    const int waves = fo::sum_waves(segments);
    if (waves == 4) launch(std::integral_constant<int, 4>{});
    else if (waves == 8) launch(std::integral_constant<int, 8>{});
    else launch(std::integral_constant<int, 16>{});
}

Result to_dev(const flashoptim_matrix& c) { return {c.data, c.stride, (uint32_t)c.rows, (uint32_t)c.cols}; }

struct Operands {
    const flashoptim_mx4 &a, &b;
    const flashoptim_matrix& c;
};

// Every c = a b^T, all of one type and shape of tiles, in one launch.
template <bool FP32, typename... T>
int launch_tiles(fo::Shape shape, hipStream_t stream, const T&... operands) {
    constexpr int kCount = sizeof...(operands);
    auto launch = [&](auto kernel, int edge, int threads) {
        auto product = [&](const Operands& o) {
            return Product{to_dev(o.b), to_dev(o.a), to_dev(o.c), (uint32_t)up(o.c.cols, edge), (uint32_t)(up(o.c.cols, edge) * up(o.c.rows, edge))};
        };
        const Products<kCount> p = {{product(operands)...}};
        hipLaunchKernelGGL(kernel, dim3(p.of[0].tiles + (kCount > 1 ? p.of[kCount - 1].tiles : 0)), dim3(threads), 0, stream, p);
    };
    if (shape == fo::kTile256) launch(product_tiles<kCount, FP32, 256, 256, 4, 2, 2, 2>, 256, 512);
    else if (shape == fo::kTile128) launch(product_tiles<kCount, FP32, 128, 128, 2, 2, 2, 2>, 128, 256);
    else launch(product_tiles<kCount, FP32, 64, 64, 2, 2, 4, 2>, 64, 256);
    return fo::hip_status(hipGetLastError());
}

int product(const flashoptim_mx4& a, const flashoptim_mx4& b, const flashoptim_matrix& c, hipStream_t stream) {
    if (c.rows == 0 || c.cols == 0) return FLASHOPTIM_OK;
    const Result r = to_dev(c);
    const bool fp32 = c.dtype == FLASHOPTIM_FP32;
    if (a.cols == 0) {
        hipLaunchKernelGGL(fill_zero, dim3((unsigned)up(c.cols, 256), (unsigned)(c.rows < 1024 ? c.rows : 1024)), dim3(256), 0, stream, r, fp32 ? 4 : 2);
        return fo::hip_status(hipGetLastError());
    }
    const fo::Shape shape = fo::product_shape(c.rows, c.cols, a.cols);
    if (shape != fo::kTiny)
        return fp32 ? launch_tiles<true>(shape, stream, Operands{a, b, c}) : launch_tiles<false>(shape, stream, Operands{a, b, c});
    const uint32_t pt = (uint32_t)up(c.cols, 16), qt = (uint32_t)up(c.rows, 16);
    auto launch = [&](auto waves) {
        constexpr int W = decltype(waves)::value;
        if (fp32) hipLaunchKernelGGL((product_small<true, W>), dim3(pt * qt), dim3(64 * W), 0, stream, to_dev(b), to_dev(a), r, pt);
        else hipLaunchKernelGGL((product_small<false, W>), dim3(pt * qt), dim3(64 * W), 0, stream, to_dev(b), to_dev(a), r, pt);
    };
    with_waves(up(a.cols, kSegment), launch);
    return fo::hip_status(hipGetLastError());
}

// Two products that do not depend on each other, in one launch where they go by the same tiles.
int two_products(const Operands& x, const Operands& y, hipStream_t stream) {
    auto empty = [](const Operands& o) { return o.c.rows == 0 || o.c.cols == 0 || o.a.cols == 0; };
    const fo::Shape shape = fo::product_shape(x.c.rows, x.c.cols, x.a.cols);
    if (empty(x) || empty(y) || x.c.dtype != y.c.dtype || shape == fo::kTiny || shape != fo::product_shape(y.c.rows, y.c.cols, y.a.cols)) {
        const int rc = product(x.a, x.b, x.c, stream);
        return rc != FLASHOPTIM_OK ? rc : product(y.a, y.b, y.c, stream);
    }
    return x.c.dtype == FLASHOPTIM_FP32 ? launch_tiles<true>(shape, stream, x, y) : launch_tiles<false>(shape, stream, x, y);
}

// What linear_small keeps of x in LDS: rows of codes begin 16 bytes apart in the banks.
int64_t few_code_pitch(int64_t k) { return up(k, kSegment) * kSegmentBytes + 16; }
int64_t few_scale_pitch(int64_t k) { return up(k, kSegment) * 8 + 8; }
// Exact for items and units below 2^16 (there are at most 12288 units of eight).
uint32_t few_units_magic(int64_t k) { return (uint32_t)(((uint64_t)1 << 32) / (uint64_t)(up(k, kSegment) * (kSegment / 8)) + 1); }

int linear_few_rows(const flashoptim_matrix& x, const flashoptim_mx4& w, const flashoptim_matrix& y, hipStream_t stream) {
    const Few a = {{x.data, nullptr, nullptr, x.stride, (uint32_t)x.rows, (uint32_t)x.cols}, to_dev(w), {y.data, y.stride, (uint32_t)y.rows, (uint32_t)y.cols},
                   (uint32_t)few_code_pitch(x.cols), (uint32_t)few_scale_pitch(x.cols), few_units_magic(x.cols)};
    const bool fp32 = y.dtype == FLASHOPTIM_FP32, x_fp32 = x.dtype == FLASHOPTIM_FP32;
    const int64_t x_bytes = x.rows * (few_code_pitch(x.cols) + few_scale_pitch(x.cols));
    const fo::FewPlan p = fo::plan_few(x.rows, y.cols, x.cols);
    auto launch = [&](auto waves, auto tiles) {
        constexpr int W = decltype(waves)::value, T = decltype(tiles)::value;
        const int64_t part_bytes = W * T * 1024;
        const unsigned bytes = (unsigned)(x_bytes > part_bytes ? x_bytes : part_bytes);
        auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)p.workgroups), dim3(64 * W), bytes, stream, a); };
        if (x_fp32) { if (fp32) go(linear_small<kFp32, true, W, T>); else go(linear_small<kFp32, false, W, T>); }
        else { if (fp32) go(linear_small<kBf16, true, W, T>); else go(linear_small<kBf16, false, W, T>); }
    };
    auto with_tiles = [&](auto waves) {
        if (p.tiles == 1) launch(waves, std::integral_constant<int, 1>{});
        else launch(waves, std::integral_constant<int, 2>{});
    };
    if (p.waves == 4) with_tiles(std::integral_constant<int, 4>{});
    else if (p.waves == 8) with_tiles(std::integral_constant<int, 8>{});
    else with_tiles(std::integral_constant<int, 16>{});
    return fo::hip_status(hipGetLastError());
}

// Codes and scales of a matrix in a workspace.
int64_t mx4_bytes(int64_t rows, int64_t cols) { return rows * (up(cols, kSegment) * kSegmentBytes + 16 * up(cols, 2 * kSegment)); }
int64_t align16(int64_t n) { return up(n, 16) * 16; }
flashoptim_mx4 carve(uint8_t*& at, int64_t rows, int64_t cols) {
    flashoptim_mx4 m = {at, at + rows * up(cols, kSegment) * kSegmentBytes, rows, cols};
    at += align16(mx4_bytes(rows, cols));
    return m;
}

int64_t check_sizes(int64_t m, int64_t n, int64_t k) {
    if (m < 0 || n < 0 || k < 0) return FLASHOPTIM_ERR_INVALID_ARG;
    const int64_t most = (int64_t)1 << 31;
    if (m >= most || n >= most || k >= most) return FLASHOPTIM_ERR_NUMEL_RANGE;
    const int64_t sizes[3] = {m, n, k};
    for (int i = 0; i < 3; ++i)
        for (int j = 0; j < 3; ++j)
            if (sizes[i] > 0 && up(sizes[j], kSegment) >= ((int64_t)1 << 27) / sizes[i]) return FLASHOPTIM_ERR_NUMEL_RANGE;
    return FLASHOPTIM_OK;
}

int check_workspace(const void* workspace, int64_t bytes, int64_t need) {
    if (need < 0) return (int)need;
    if (need == 0) return FLASHOPTIM_OK;
    if (!workspace) return FLASHOPTIM_ERR_INVALID_ARG;
    if (bytes < need) return FLASHOPTIM_ERR_WORKSPACE;
    return fo::aligned_to(workspace, 16) ? FLASHOPTIM_OK : FLASHOPTIM_ERR_MISALIGNED;
}

}  // namespace

extern "C" {

int flashoptim_mx4_quantize(const flashoptim_matrix* x, const int8_t* rho, const uint8_t* rand, const flashoptim_mx4* out,
                            const flashoptim_mx4* out_t, void* stream) {
    FO_TRY(fo::check_matrix(x));
    if (!out && !out_t) return FLASHOPTIM_ERR_INVALID_ARG;
    if (rho && x->dtype != FLASHOPTIM_BF16) return FLASHOPTIM_ERR_INVALID_ARG;
    if (out) FO_TRY(check_mx4(out));
    if (out_t) FO_TRY(check_mx4(out_t));
    if (out && (out->rows != x->rows || out->cols != x->cols)) return FLASHOPTIM_ERR_INVALID_ARG;
    if (out_t && (out_t->rows != x->cols || out_t->cols != x->rows)) return FLASHOPTIM_ERR_INVALID_ARG;
    return quantize(*x, rho, rand, out, out_t, (hipStream_t)stream);
}

int flashoptim_mx4_dequantize(const flashoptim_mx4* q, const flashoptim_matrix* x, void* stream) {
    FO_TRY(check_mx4(q));
    FO_TRY(fo::check_matrix(x));
    if (q->rows != x->rows || q->cols != x->cols) return FLASHOPTIM_ERR_INVALID_ARG;
    if (x->rows == 0 || x->cols == 0) return FLASHOPTIM_OK;
    const Mx4 m = to_dev(*q);
    const uint32_t total = m.rows * m.segments;
    if (x->dtype == FLASHOPTIM_FP32) hipLaunchKernelGGL(dequantize_rows<true>, dim3((total + 7) / 8), dim3(256), 0, (hipStream_t)stream, m, x->data, x->stride, total);
    else hipLaunchKernelGGL(dequantize_rows<false>, dim3((total + 7) / 8), dim3(256), 0, (hipStream_t)stream, m, x->data, x->stride, total);
    return fo::hip_status(hipGetLastError());
}

int64_t flashoptim_mx4_matmul_workspace(int64_t m, int64_t n, int64_t k) {
    FO_TRY(check_sizes(m, n, k));
    return 0;
}

int64_t flashoptim_mx4_linear_workspace(int64_t m, int64_t n, int64_t k) {
    FO_TRY(check_sizes(m, n, k));
    return align16(mx4_bytes(m, k));
}

int64_t flashoptim_mx4_linear_backward_workspace(int64_t m, int64_t n, int64_t k) {
    FO_TRY(check_sizes(m, n, k));
    return align16(mx4_bytes(m, n)) + align16(mx4_bytes(n, m));
}

int flashoptim_mx4_matmul(const flashoptim_mx4* a, const flashoptim_mx4* b, const flashoptim_matrix* c, void* workspace,
                          int64_t workspace_bytes, void* stream) {
    FO_TRY(check_mx4(a));
    FO_TRY(check_mx4(b));
    FO_TRY(fo::check_matrix(c));
    if (a->cols != b->cols || c->rows != a->rows || c->cols != b->rows) return FLASHOPTIM_ERR_INVALID_ARG;
    FO_TRY(check_sizes(a->rows, b->rows, a->cols));
    FO_TRY(check_workspace(workspace, workspace_bytes, 0));
    return product(*a, *b, *c, (hipStream_t)stream);
}

int flashoptim_mx4_linear(const flashoptim_matrix* x, const flashoptim_mx4* w, const flashoptim_mx4* xt, const flashoptim_matrix* y,
                          void* workspace, int64_t workspace_bytes, void* stream) {
    FO_TRY(fo::check_matrix(x));
    FO_TRY(check_mx4(w));
    FO_TRY(fo::check_matrix(y));
    if (xt) FO_TRY(check_mx4(xt));
    if (w->cols != x->cols || y->rows != x->rows || y->cols != w->rows) return FLASHOPTIM_ERR_INVALID_ARG;
    if (xt && (xt->rows != x->cols || xt->cols != x->rows)) return FLASHOPTIM_ERR_INVALID_ARG;
    FO_TRY(check_sizes(x->rows, w->rows, x->cols));
    if (!xt && fo::takes_few_rows(x->rows, y->cols, x->cols)) return linear_few_rows(*x, *w, *y, (hipStream_t)stream);
    FO_TRY(check_workspace(workspace, workspace_bytes, flashoptim_mx4_linear_workspace(x->rows, w->rows, x->cols)));
    uint8_t* at = (uint8_t*)workspace;
    const flashoptim_mx4 q = carve(at, x->rows, x->cols);
    FO_TRY(quantize(*x, nullptr, nullptr, &q, xt, (hipStream_t)stream));
    return product(q, *w, *y, (hipStream_t)stream);
}

int flashoptim_mx4_linear_backward(const flashoptim_matrix* dy, const uint8_t* rand, const flashoptim_mx4* wt, const flashoptim_mx4* xt,
                                   const flashoptim_matrix* dx, const flashoptim_matrix* dw, void* workspace, int64_t workspace_bytes,
                                   void* stream) {
    FO_TRY(fo::check_matrix(dy));
    if (!dx && !dw) return FLASHOPTIM_ERR_INVALID_ARG;
    const int64_t m = dy->rows, n = dy->cols;
    int64_t k = 0;
    if (dx) {
        FO_TRY(check_mx4(wt));
        FO_TRY(fo::check_matrix(dx));
        k = dx->cols;
        if (dx->rows != m || wt->rows != k || wt->cols != n) return FLASHOPTIM_ERR_INVALID_ARG;
    }
    if (dw) {
        FO_TRY(check_mx4(xt));
        FO_TRY(fo::check_matrix(dw));
        if (dx && dw->cols != k) return FLASHOPTIM_ERR_INVALID_ARG;
        k = dw->cols;
        if (dw->rows != n || xt->rows != k || xt->cols != m) return FLASHOPTIM_ERR_INVALID_ARG;
    }
    FO_TRY(check_workspace(workspace, workspace_bytes, flashoptim_mx4_linear_backward_workspace(m, n, k)));
    uint8_t* at = (uint8_t*)workspace;
    const flashoptim_mx4 q = carve(at, m, n), qt = carve(at, n, m);
    FO_TRY(quantize(*dy, nullptr, rand, dx ? &q : nullptr, dw ? &qt : nullptr, (hipStream_t)stream));
    if (dx && dw) return two_products({q, *wt, *dx}, {qt, *xt, *dw}, (hipStream_t)stream);
    if (dx) FO_TRY(product(q, *wt, *dx, (hipStream_t)stream));
    if (dw) FO_TRY(product(qt, *xt, *dw, (hipStream_t)stream));
    return FLASHOPTIM_OK;
}

}  // extern "C"
