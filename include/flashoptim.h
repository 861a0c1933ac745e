/*
 * flashoptim.h - C ABI of the MI355X (gfx950) FlashOptim optimizer-step library.
 *
 * The library implements the fused per-parameter optimizer step of FlashAdamW,
 * FlashSGD and FlashLion (paper Section 3.3, Algorithms 4, 5, 6) on the
 * compressed per-parameter layout of Table 1:
 *
 *     theta'  BF16   2 B   low-precision weight the model trains on
 *     rho     INT8   1 B   weight correction            (Section 3.1, Eq. 1-2, Algorithm 1)
 *     g       BF16   2 B   gradient (0 B resident with gradient release, Section 3.4)
 *     m       INT8   1 B   companded momentum code      (Section 3.2, Eq. 3, Algorithm 2)
 *     v       UINT8  1 B   companded variance code      (Section 3.2, Eq. 4, Algorithm 3; AdamW only)
 *     scales  FP16   2 B per group of G = 32 consecutive elements, per state
 *
 * General conventions
 *  - Every data pointer is a DEVICE pointer on the current HIP device, owned by the
 *    caller, and must be 16-byte aligned.  Descriptor arrays and hyper-parameter
 *    structs are HOST memory and are read before the call returns.
 *  - A tensor is its flattened, contiguous element sequence; quantisation groups are
 *    elements [32k, 32k+32) of that sequence, the last group may be short, and groups
 *    never span tensors.  A scale array holds ceil(numel/32) FP16 bit patterns.
 *  - All-zero m_q/m_scale/v_q/v_scale buffers are the initial state Q_m(0), Q_v(0)
 *    (the initialisation of Algorithm 4): a zero scale decodes to exactly zero.
 *  - Work is enqueued on `stream` (a hipStream_t passed as void*; NULL = the default
 *    stream) and the call returns without waiting.  Buffers may be reused or freed
 *    by the caller in stream order.  Calls that touch the same tensors from different
 *    streams must be ordered by the caller, as for any other kernel; calls on disjoint
 *    lists may run concurrently (the library is thread-safe).
 *  - One call covers at most 2^31 - 1 workgroups (2048 elements each for AdamW, 4096 for
 *    SGD / Lion, 256 to 2048 for the ablation variants and conversions): more returns
 *    FLASHOPTIM_ERR_NUMEL_RANGE.
 *  - Return value: FLASHOPTIM_OK (0) or a negative flashoptim_status.  Arguments are
 *    validated before anything is enqueued: when an error is returned no buffer has
 *    been modified.  Nothing throws or aborts.
 *  - Inputs are expected to be finite.  NaN/Inf values propagate into the results of
 *    their own element or group but never cause out-of-bounds accesses.  An infinite
 *    weight keeps rho = 0; the rho byte stored next to a NaN weight is unspecified.
 *  - Arithmetic: IEEE binary32, round-to-nearest-even, subnormals kept, no fused
 *    multiply-add, in the order the algorithms print it (one documented exception: the
 *    default AdamW step rounds one division faithfully, see flashoptim_adamw_step); divisions by a group scale
 *    or by a bias correction 1 - beta^t multiply by the correctly rounded FP32
 *    reciprocal of that scalar.
 *  - There is no CPU fallback: without a HIP device every compute entry point
 *    returns FLASHOPTIM_ERR_HIP.
 */
#ifndef FLASHOPTIM_H
#define FLASHOPTIM_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum flashoptim_status {
    FLASHOPTIM_OK = 0,
    FLASHOPTIM_ERR_INVALID_ARG = -1, /* null pointer, negative count, bad kind, step < 1, ... */
    FLASHOPTIM_ERR_MISALIGNED = -2,  /* a device pointer is not 16-byte aligned               */
    FLASHOPTIM_ERR_NUMEL_RANGE = -3, /* numel < 0 or >= 2^40                                  */
    FLASHOPTIM_ERR_HIP = -4,         /* a HIP runtime call failed (see flashoptim_last_hip_error) */
    FLASHOPTIM_ERR_BAD_BLOB = -5,    /* checkpoint blob too small, or header/table mismatch   */
    FLASHOPTIM_ERR_SELFTEST = -6,    /* flashoptim_selftest found a failing check             */
    FLASHOPTIM_ERR_LIST_TOO_LONG = -7, /* flashoptim_adamw_step_noalloc: more than 1024 non-empty tensors */
    FLASHOPTIM_ERR_WORKSPACE = -8    /* a workspace is smaller than the call needs */
} flashoptim_status;

/* Optimizer kinds (checkpoint entry points). */
enum { FLASHOPTIM_ADAMW = 0, FLASHOPTIM_SGD = 1, FLASHOPTIM_LION = 2 };

/* One parameter tensor in the compressed layout.  lr and weight_decay are per tensor
 * because the paper's recipes exempt biases and normalisation parameters from weight
 * decay (Appendix B) and follow a learning-rate schedule (Algorithm 4, Require). */
typedef struct flashoptim_tensor {
    void*       param;    /* [numel] BF16 theta', in/out                                    */
    int8_t*     rho;      /* [numel] INT8 weight correction, in/out                         */
    const void* grad;     /* [numel] BF16 gradient, in                                      */
    int8_t*     m_q;      /* [numel] INT8 momentum codes, in/out                            */
    uint16_t*   m_scale;  /* [ceil(numel/32)] FP16 bits, in/out                             */
    uint8_t*    v_q;      /* [numel] UINT8 variance codes, in/out; AdamW only, else NULL    */
    uint16_t*   v_scale;  /* [ceil(numel/32)] FP16 bits, in/out;   AdamW only, else NULL    */
    int64_t     numel;    /* >= 0; a tensor with numel == 0 is skipped                      */
    float       lr;       /* eta_t for this tensor                                          */
    float       weight_decay; /* lambda for this tensor (decoupled, multiplied by lr)       */
} flashoptim_tensor;

typedef struct flashoptim_adamw_hp {
    float   beta1, beta2, eps;
    int64_t step;         /* t >= 1: Algorithm 4 increments t before using it               */
} flashoptim_adamw_hp;

typedef struct flashoptim_sgd_hp { float momentum; } flashoptim_sgd_hp;

typedef struct flashoptim_lion_hp { float beta1, beta2; } flashoptim_lion_hp;

/* ---- fused steps over a list of tensors ------------------------------------------
 * One call covers the whole list: hundreds of small tensors fill the chip through a small
 * index table that the library builds once per distinct list and caches on the device; the
 * work is issued as a few back-to-back kernel launches on the given stream (one per 2^28
 * elements).  A list of length one is the gradient-release call (Section 3.4): it needs no
 * table and no device allocation.  Tables of the 256 most recently used lists are kept; a call
 * with a further distinct list frees the least recently used one after synchronising the device.  The grad pointers are not part of the
 * cached identity of a list, so gradients may live in different buffers each step.  A call whose descriptors
 * (pointers, grad pointers, numel, lr, weight_decay) equal those of the previous call on the same list enqueues
 * kernels only; changed ones are first written into the list's table by a small kernel, or, where all that has changed
 * is a rate that all tensors share, by the step itself.
 *
 * Under capture into a HIP graph: the list's tables should have been made by an earlier call (making them allocates), and
 * must be kept while the graph is in use (see the 256 lists above and release_cache).  A captured call with unchanged
 * descriptors reads gradients, rates and weight decays from the table at every replay, as the latest call on the list has
 * left them: an eager call with another rate reaches the replays.  A captured call with changed descriptors writes them
 * into the table at every replay.  A list of length one has no table: its call keeps what it was captured with.  The calls
 * that wait for completion (each says so) return FLASHOPTIM_ERR_HIP on a capturing stream, with nothing enqueued and the
 * capture intact.
 *
 * flashoptim_adamw_step: Algorithm 4, the body of the loop after the gradient (reconstruct m, v, theta; AdamW
 *   update with bias correction and decoupled weight decay; quantize m, v; split theta).
 * flashoptim_sgd_step:   Algorithm 5, loop body (m <- mu m + g; theta <- theta - eta (m + lambda theta)).
 * flashoptim_lion_step:  Algorithm 6, loop body (u = sign(b1 m + (1-b1) g); m <- b2 m + (1-b2) g;
 *   theta <- theta - eta (u + lambda theta)); sign(0) = 0.
 * tensors: host array of n_tensors descriptors (n_tensors >= 0).
 *
 * Rounding of the quotient m_hat / (sqrt(v_hat) + eps) of the AdamW update:
 *   flashoptim_adamw_step        faithful: the hardware reciprocal estimate, the quotient and one FMA residual
 *                                correction.  The result is within one ulp of the correctly rounded quotient
 *                                (flashoptim_selftest bounds this on the device) and differs from it only when
 *                                the exact quotient lies within 2^-23 ulp of the midpoint of two FP32 numbers:
 *                                about one operand pair in 10^9 (flashoptim_faithful_rounding_stats counts them).
 *                                Such a difference can move the new master weight by one FP32 ulp, hence rho by
 *                                one unit on a rare element.  Momentum codes, variance codes and all scales do
 *                                not depend on the quotient and are the exact ones in either case.  Used when
 *                                2^-60 <= eps <= 1 and the operands do not exceed 2^60; otherwise this entry point
 *                                takes the IEEE division (slower, same results as the exact entry point).
 *   flashoptim_adamw_step_exact  the quotient is correctly rounded for every input: the whole step is
 *                                bit-identical to the arithmetic stated above.  About 2 % slower on MI355X.
 * Everything else is identical between the two. */
int flashoptim_adamw_step(const flashoptim_tensor* tensors, int64_t n_tensors,
                          const flashoptim_adamw_hp* hp, void* stream);
int flashoptim_adamw_step_exact(const flashoptim_tensor* tensors, int64_t n_tensors,
                                const flashoptim_adamw_hp* hp, void* stream);
int flashoptim_sgd_step(const flashoptim_tensor* tensors, int64_t n_tensors,
                        const flashoptim_sgd_hp* hp, void* stream);
int flashoptim_lion_step(const flashoptim_tensor* tensors, int64_t n_tensors,
                         const flashoptim_lion_hp* hp, void* stream);

/* ---- the FlashAdamW step for callers that cannot allocate ---------------------------------
 * For code under HIP stream capture, tight serving loops and harnesses that forbid allocation: the same step
 * as flashoptim_adamw_step_exact, same arguments, same results bit for bit, but the call allocates nothing
 * (no hipMalloc / hipFree / hipHostMalloc, no host-to-device copy): the two device tables of a multi-tensor
 * launch are written by small kernels, from kernel arguments, into a fixed 172,036-byte device array that
 * each GPU holds from library load to process end.
 * Every table entry a call's launches read is written by that call first, so nothing left behind by an earlier
 * call (a longer list, larger tensors) is ever seen.
 * Limits: at most 1024 tensors with numel > 0 (FLASHOPTIM_ERR_LIST_TOO_LONG beyond that, nothing enqueued) and,
 * as for every step call, at most 2^31 - 1 workgroups.  Every call on a GPU shares that GPU's array: calls on
 * the same stream are ordered and safe; calls that may overlap on one GPU (different streams, several host
 * threads) race on it and must be ordered by the caller.  This entry point does not start the check of the
 * short square root (see flashoptim_short_sqrt_state): where no AdamW step call of another entry point has
 * put it on a stream of this device, or it has not finished yet, the kernels use sqrtf: same results, a few
 * percent slower. */
int flashoptim_adamw_step_noalloc(const flashoptim_tensor* tensors, int64_t n_tensors,
                                  const flashoptim_adamw_hp* hp, void* stream);

/* ---- sharding a flat tensor over ranks (Section 3.4, "Distributed training") ----------------
 * With ZeRO / FSDP-style sharding each rank owns a contiguous piece of every flattened tensor, keeps rho, the
 * state codes and their scales for that piece only, and steps it with the calls above; nothing but the BF16
 * weights is exchanged.  Quantisation groups must not straddle ranks, and every stream of a shard (the
 * 2-byte-per-group scales included) must start 16-byte aligned: this call cuts [0, numel) into `world`
 * consecutive shards on multiples of 256 elements, as evenly as that allows (sizes differ by at most 256; only
 * the last non-empty shard can be ragged; with fewer than `world` units the trailing ranks get len 0).
 * *begin, *len (HOST): the element range of `rank`.  A shard's descriptor is the tensor's descriptor with
 * param, rho, grad, m_q, v_q advanced by begin elements, m_scale and v_scale by begin / 32, numel = len;
 * stepping the shards (in one list or in `world` calls) gives the same bits as stepping the whole tensor.
 * Host arithmetic only. */
int flashoptim_shard_range(int64_t numel, int64_t world, int64_t rank, int64_t* begin, int64_t* len);

/* ---- ablation and reference variants of the steps (Section 4.3) -----------------------
 * The paper isolates its two techniques: "Weight Split" (split weights, FP32 states) and
 * "Opt. Quant." (FP32 master weights, 8-bit states); with both off the step is the plain FP32
 * optimizer (Algorithms 4-6 without their highlighted lines), here still fed BF16 gradients.
 * flags: FLASHOPTIM_SPLIT_WEIGHTS | FLASHOPTIM_QUANTIZE_STATES selects which technique is ON; both on
 * is identical to the plain entry points above.
 * With splitting off, `theta` ([numel] FP32, in/out) is the master weight and t.param / t.rho are
 * ignored; with state quantisation off, `m` (and `v` for AdamW; [numel] FP32, in/out) hold the
 * states and t.m_q / t.m_scale / t.v_q / t.v_scale are ignored.  Ignored pointers may be NULL.
 * Bytes moved per parameter (AdamW): 12.25 both on; 24 weight split only; 14.25 state quantisation
 * only; 26 both off. */
enum { FLASHOPTIM_SPLIT_WEIGHTS = 1, FLASHOPTIM_QUANTIZE_STATES = 2 };

typedef struct flashoptim_tensor_ex {
    flashoptim_tensor t;  /* compressed buffers, grad, numel, lr, weight_decay                   */
    float* theta;         /* [numel] FP32 master weight, used when weights are not split         */
    float* m;             /* [numel] FP32 momentum, used when states are not quantized           */
    float* v;             /* [numel] FP32 variance (AdamW), used when states are not quantized   */
} flashoptim_tensor_ex;

int flashoptim_adamw_step_ex(const flashoptim_tensor_ex* tensors, int64_t n_tensors,
                             const flashoptim_adamw_hp* hp, unsigned flags, void* stream);
int flashoptim_sgd_step_ex(const flashoptim_tensor_ex* tensors, int64_t n_tensors,
                           const flashoptim_sgd_hp* hp, unsigned flags, void* stream);
int flashoptim_lion_step_ex(const flashoptim_tensor_ex* tensors, int64_t n_tensors,
                            const flashoptim_lion_hp* hp, unsigned flags, void* stream);

/* ---- migration between a standard FP32 optimizer state and the compressed layout --------
 * compress_state:   theta', rho <- C(theta);  m_q, m_scale <- Q_m(m);  v_q, v_scale <- Q_v(v)
 *                   (Algorithms 1-3; the initialisation of Algorithm 4 when m = v = 0, and the way to
 *                   adopt the compressed layout from an existing 12 B/param FP32 state).
 * decompress_state: theta <- C^-1(theta', rho);  m <- Q_m^-1;  v <- Q_v^-1  (export).
 * One launch over the list.  Both layouts' buffers of every tensor are required (v, v_q, v_scale for
 * kind = FLASHOPTIM_ADAMW only); t.grad, t.lr, t.weight_decay are ignored. */
int flashoptim_compress_state(int kind, const flashoptim_tensor_ex* tensors, int64_t n_tensors, void* stream);
int flashoptim_decompress_state(int kind, const flashoptim_tensor_ex* tensors, int64_t n_tensors, void* stream);

/* ---- measurement aid (no passage of the paper: the memory ceiling of the step's traffic) ----
 * stream_probe: reads every array a step of this kind reads (gradients included) and writes every
 * array it writes back UNCHANGED, through the same launch shape and access instructions as the step,
 * with no arithmetic and, for large calls, in the order that memory serves best (not always the
 * step's).  Timing it gives the rate the memory system delivers for exactly the step's traffic
 * (12.25 B/param for AdamW, 10.125 for SGD and Lion), to set the step's own rate against.
 * Same arguments, validation, stream ordering and errors as the *_step calls; lr and weight_decay
 * are ignored; no state changes. */
int flashoptim_stream_probe(int kind, const flashoptim_tensor* tensors, int64_t n_tensors, void* stream);

/* ---- weight splitting (Section 3.1, Algorithm 1, N = 127) --------------------------
 * split:       theta (FP32) -> theta' = BF16 round-to-nearest-even, rho = Round(e / (ULP(theta')/2) * 127)
 *              Used once at the start of training (initialisation of Algorithm 4).
 * reconstruct: theta_hat = theta' + (rho/127) * ULP(theta')/2   (Eq. 2)
 * n >= 0 elements; all pointers device memory. */
int flashoptim_split_weights(const float* theta, void* param_bf16, int8_t* rho, int64_t n, void* stream);
int flashoptim_reconstruct_weights(const void* param_bf16, const int8_t* rho, float* theta, int64_t n,
                                   void* stream);

/* ---- 16-bit correction and the exhaustive reconstruction experiment (Section 4.4) ------
 * Algorithm 1 with N = 32767: rho is an INT16 (theta' + rho = 32 bits, near-lossless).  Same
 * conventions as the INT8 entry points above.  The fused steps use the INT8 form only.
 * reconstruction_sweep: pushes the FP32 bit patterns first, first + stride, ... (< 2^32; stride 1
 *   and first 0 = every FP32 value) through split then reconstruct with an 8- or 16-bit correction
 *   and returns error statistics in `stats`, a HOST array of 520 doubles:
 *   [0] values measured  [1] skipped (non-finite theta or theta')  [2] values with |theta - theta'| >
 *   ULP(theta')/2  [3] max |theta_hat - theta| / (ULP(theta')/(4N))  [4] max relative error over normal
 *   theta  [5] bit-exact reconstructions  [6] rho outside [-N, N]  [7] unused  [8 + E] sum and
 *   [264 + E] count of the relative errors of the normal values with FP32 exponent field E (their ratio
 *   is the mean relative error per exponent that Figure 3 plots).  Waits for completion. */
int flashoptim_split_weights_i16(const float* theta, void* param_bf16, int16_t* rho, int64_t n, void* stream);
int flashoptim_reconstruct_weights_i16(const void* param_bf16, const int16_t* rho, float* theta, int64_t n,
                                       void* stream);
int flashoptim_reconstruction_sweep(int correction_bits, uint64_t first, uint64_t stride, double* stats,
                                    void* stream);
/* The same experiment with a choice of how ULP(theta') is read, and per-exponent counts of bit-exact
 * reconstructions.  ulp_reading 0: Algorithm 1 as printed, one spacing per theta' (what every other entry
 * point of this library uses).  ulp_reading 1, "directional": the spacing of the BF16 grid on the side of
 * theta' on which theta lies, which is half as large when theta' is a power of two and theta lies towards
 * zero; Section 4.4 prints 99.92 % bit-exact reconstructions for the 16-bit correction, which this reading
 * reproduces over the mid-range exponents and the printed algorithm does not (99.73 %).  It exists for this
 * experiment only.  stats: HOST array of 776 doubles, the 520 above followed by [520 + E] bit-exact
 * reconstructions among the normal values with FP32 exponent field E.  [2] and [3] refer to the printed
 * ULP under both readings.  Waits for completion. */
int flashoptim_reconstruction_sweep_ex(int correction_bits, int ulp_reading, uint64_t first, uint64_t stride,
                                       double* stats, void* stream);

/* ---- companded 8-bit state codecs (Section 3.2, Algorithms 2 and 3) -----------------
 * quantize_momentum:   per group s = FP16(max|m|), code = Round(127 * 2m'/(1+|m'|)), m' = m/s
 * dequantize_momentum: m = (z / (2 - |z|)) * s, z = code/127
 * quantize_variance:   per group s = FP16(max sqrt(v)), code = Round(255 * sqrt(v)/s)
 * dequantize_variance: v = ((code/255) * s)^2
 * n >= 0 elements, scale arrays of ceil(n/32) FP16 bit patterns; all device memory. */
int flashoptim_quantize_momentum(const float* m, int8_t* q, uint16_t* scale, int64_t n, void* stream);
int flashoptim_dequantize_momentum(const int8_t* q, const uint16_t* scale, float* m, int64_t n, void* stream);
int flashoptim_quantize_variance(const float* v, uint8_t* q, uint16_t* scale, int64_t n, void* stream);
int flashoptim_dequantize_variance(const uint8_t* q, const uint16_t* scale, float* v, int64_t n, void* stream);

/* ---- linear baseline and quantisation error (Section 4.5) ------------------------------
 * The paper validates its companders against plain absmax-scaled integer quantisation: the same
 * group-wise FP16 absmax scale, no compander (momentum code = Round(127 m / s); variance code =
 * Round(255 v / s) with s the group maximum of v itself).
 * quantize_state / dequantize_state: state 0 = momentum (INT8 codes), 1 = variance (UINT8 codes);
 *   linear 0 = companded (identical to the four entry points above), 1 = the linear baseline.
 * quantization_nmse: quantizes and dequantizes x on the fly and returns in `sums` (HOST, 2 doubles)
 *   sum (x_hat - x)^2 and sum x^2, whose ratio is the normalised MSE the paper plots.  Waits for
 *   completion. */
int flashoptim_quantize_state(int state, int linear, const float* x, void* q, uint16_t* scale, int64_t n,
                              void* stream);
int flashoptim_dequantize_state(int state, int linear, const void* q, const uint16_t* scale, float* x, int64_t n,
                                void* stream);
int flashoptim_quantization_nmse(int state, int linear, const float* x, int64_t n, double* sums, void* stream);

/* ---- checkpoint (Section 3.4, "Checkpoint size": 2 + 1 + 1 + 1 bytes per parameter) --
 * The paper fixes the content, not a container.  Blob layout, little-endian:
 *   header (64 B): "FOPTCKPT" | u32 version = 1 | u32 kind | i64 step | i64 n_tensors |
 *                  i64 total_bytes | zero padding
 *   table: per tensor i64 numel | i64 offset of its first section from the blob start;
 *          padded to a multiple of 64 B
 *   per tensor, in list order, each section starting on a 64-byte boundary and zero
 *   padded: theta' (2n) | rho (n) | m codes (n) | m scales (2 ceil(n/32)) |
 *   AdamW only: v codes (n) | v scales (2 ceil(n/32))
 * checkpoint_size: total blob bytes for a list (numels: host array), or a negative status.
 * checkpoint_pack:   gathers the tensors' state into `blob` (DEVICE memory, 16-byte aligned,
 *                    blob_bytes >= checkpoint_size).  grad fields are ignored.  Does not wait; under capture
 *                    as a step call (see above), and every replay writes the step it was captured with.
 * checkpoint_unpack: scatters `blob` (DEVICE memory) back into the tensors' buffers and
 *                    returns the stored step in *step_out (host).  The header and table
 *                    are validated against (kind, list) on the device, ahead of the copy, which
 *                    writes nothing if they differ; the call waits for that verdict and the step,
 *                    and therefore for prior work on `stream`, but not for the copy (refused: until
 *                    the copy, which then does nothing, has run too). */
int64_t flashoptim_checkpoint_size(int kind, const int64_t* numels, int64_t n_tensors);
int flashoptim_checkpoint_pack(int kind, const flashoptim_tensor* tensors, int64_t n_tensors, int64_t step,
                               void* blob, int64_t blob_bytes, void* stream);
int flashoptim_checkpoint_unpack(int kind, const void* blob, int64_t blob_bytes,
                                 const flashoptim_tensor* tensors, int64_t n_tensors, int64_t* step_out,
                                 void* stream);

/* ---- microscaled 4-bit matrices: the weights' low-precision form and the products on it -------------
 * Around the step: the blocks of a model run on 4-bit copies of the weights that a step leaves, and hand back the
 * gradients that the next one takes.
 *
 * A matrix of `rows` by `cols` values in 4 bits: consecutive blocks of 32 values of a row share one power of two.
 *   codes:  [rows, 128 ceil(cols/256)] bytes, two codes to a byte, the even element in the low half.  A code is a sign
 *           bit and an index into {0, 0.5, 1, 1.5, 2, 3, 4, 6} (one mantissa bit, two exponent bits).
 *   scales: [rows, 16 ceil(cols/512)] bytes, one to a block: the block's values are its codes' times 2^(byte - 127);
 *           byte 255 makes the whole block NaN.
 * What lies behind column cols of a row is zero in both arrays (every call here writes it so, and the products count
 * on it).  Both arrays 16-byte aligned and contiguous.  rows (ceil(cols/256) + 1) <= 2^27.
 *
 * Quantisation, by block, with E the exponent field of the FP32 value max|v| of the block:
 *   to nearest:   byte = max(E - 2, 0); each v 2^(127 - byte) goes to the nearest of the eight magnitudes, ties to the
 *                 even index, what is beyond 6 to 6.
 *   stochastic (`rand` given): byte = max(E - 2, 0), one more where the mantissa of max|v| exceeds 1.5, so that
 *                 nothing lies beyond 6; with a <= |v| 2^(127 - byte) < b between neighbouring magnitudes the value goes to b
 *                 if 256 (|v| 2^(127 - byte) - a) / (b - a) > r + 1/2, r being the value's byte of `rand`.
 *   A block with an infinity or a NaN gets byte 255 and codes 0.  All of it is exact: the same bits for the same
 *   input on every path.
 *
 * flashoptim_matrix: a row-major matrix of BF16 or FP32 values whose rows begin `stride` elements apart (>= cols; any, and
 * any alignment of a value, are valid; 16-byte aligned rows are fastest).  rows, cols < 2^31. */
enum { FLASHOPTIM_BF16 = 0, FLASHOPTIM_FP32 = 1 };

typedef struct flashoptim_matrix {
    void*   data;
    int64_t rows, cols, stride;
    int32_t dtype;        /* FLASHOPTIM_BF16 or FLASHOPTIM_FP32 */
} flashoptim_matrix;

typedef struct flashoptim_mx4 {
    uint8_t* codes;
    uint8_t* scales;
    int64_t  rows, cols;
} flashoptim_mx4;

/* quantize: `out` <- x in 4 bits along its rows; `out_t` <- the transpose of x (cols by rows) in 4 bits along ITS rows, from
 *   the same pass over x.  Either may be NULL.  rho: NULL, or the [rows, cols] INT8 corrections (contiguous) of x, which is then
 *   a contiguous BF16 matrix of split weights: what is quantised is the reconstructed FP32 weight.  rand: NULL, or [rows, cols]
 *   random bytes (contiguous): stochastic rounding; out and out_t use the same byte of a value.  With out_t, ceil(rows/256) ceil(cols/256) < 2^21.
 * dequantize: x <- the values that q stands for, in BF16 (exact) or FP32 (exact). */
int flashoptim_mx4_quantize(const flashoptim_matrix* x, const int8_t* rho, const uint8_t* rand,
                            const flashoptim_mx4* out, const flashoptim_mx4* out_t, void* stream);
int flashoptim_mx4_dequantize(const flashoptim_mx4* q, const flashoptim_matrix* x, void* stream);

/* Products.  Sums are FP32, rounded once to the type of the result; the order of a sum depends on the sizes alone, so a
 * call's result is the same every time.  A product over zero terms is zero.
 * matmul: c [m, n] <- a [m, k] b [n, k]^T.
 * linear: y [m, n] <- Q(x) w^T with x [m, k] quantised to nearest along its rows and w [n, k]; if xt [k, m] is not NULL, Q(x^T) is
 *   left there for the backward pass.  Without xt a few rows are one launch, made for single tokens, through which the weights stream
 *   once: up to 16 rows, fewer with long ones (16 of 6144 values, 6 of 16384, half as many where the rows of w take a second round of workgroups).  That
 *   launch takes no workspace: NULL will do.
 * linear_backward: dx [m, k] <- Q(dy) wt^T and dw [n, k] <- Q(dy^T) xt^T, with dy [m, n] quantised along its rows and along
 *   its columns in one pass (stochastically with `rand`), wt [k, n] the transposed weights in 4 bits (quantize's out_t) and xt [k, m].
 *   dx or dw may be NULL, and with it wt or xt.  These are the gradients of the product of its quantised operands, the
 *   quantisation itself counted as the identity, each with its operands in 4 bits along its own sum.
 * workspace: DEVICE memory, 16-byte aligned, of at least the bytes that the *_workspace call returns for the same sizes (0: NULL will
 *   do; negative: a status), and the call's until its work on `stream` is done. */
int64_t flashoptim_mx4_matmul_workspace(int64_t m, int64_t n, int64_t k);
int64_t flashoptim_mx4_linear_workspace(int64_t m, int64_t n, int64_t k);
int64_t flashoptim_mx4_linear_backward_workspace(int64_t m, int64_t n, int64_t k);
int flashoptim_mx4_matmul(const flashoptim_mx4* a, const flashoptim_mx4* b, const flashoptim_matrix* c, void* workspace,
                          int64_t workspace_bytes, void* stream);
int flashoptim_mx4_linear(const flashoptim_matrix* x, const flashoptim_mx4* w, const flashoptim_mx4* xt,
                          const flashoptim_matrix* y, void* workspace, int64_t workspace_bytes, void* stream);
int flashoptim_mx4_linear_backward(const flashoptim_matrix* dy, const uint8_t* rand, const flashoptim_mx4* wt,
                                   const flashoptim_mx4* xt, const flashoptim_matrix* dx, const flashoptim_matrix* dw,
                                   void* workspace, int64_t workspace_bytes, void* stream);

/* ---- the norms before and after a block, with its gate and residual scale --------------------------------
 * Between two blocks, in one pass over each row of the residual stream x [rows, cols]:
 *   u = f, or norm(f) * post_weight + post_bias (post_norm)        f: the output of the block that ends
 *   h = residual_scale * x + branch_scale * act(gate) * u
 *   y = norm(h) * pre_weight + pre_bias                            y: the input of the block that begins
 * norm(v) = (v - mean) / sqrt(mean((v - mean)^2) + eps); kind FLASHOPTIM_RMS_NORM takes 0 for the mean.  act is the identity or the
 * sigmoid.  gate [g, cols] with g >= 1 dividing rows: row i of the result takes row i / (rows / g) of the gate (g = 1: a gate for
 * each channel; g = rows: one for each value).  Sums and everything between loads and stores are FP32; y is formed from h before
 * h is rounded.
 * Left out: weights and biases (NULL: 1, 0; biases are for layer norms only), the gate (NULL: 1), the norm in front (y NULL), the branch (f NULL: h = x, not written;
 * gate must be NULL).  x and h have one type, f, gate and y one type, which is BF16, or FP32 if x is FP32.  1 <= cols <= 16384; rows < 2^31,
 * and in the forward call less than 2^23 (2^26 for cols <= 512, 2^25 to 1024, 2^24 to 2048).
 * h may be x's own buffer, y f's.
 * stats: NULL, or [4, rows] FP32 for the backward pass: mean and 1/sqrt(...) of the norm behind, of the norm in front (0 where
 *   there is none). */
enum { FLASHOPTIM_RMS_NORM = 0, FLASHOPTIM_LAYER_NORM = 1 };
enum { FLASHOPTIM_GATE_LINEAR = 0, FLASHOPTIM_GATE_SIGMOID = 1 };

typedef struct flashoptim_block_norm_spec {
    int64_t cols;
    int32_t kind, post_norm, gate_act;
    int32_t param_dtype;                 /* of the four arrays below and of their gradients */
    float   eps, residual_scale, branch_scale;
    const void *post_weight, *post_bias, *pre_weight, *pre_bias;   /* [cols] each, or NULL */
} flashoptim_block_norm_spec;

int flashoptim_block_norm(const flashoptim_block_norm_spec* spec, const flashoptim_matrix* x, const flashoptim_matrix* f,
                          const flashoptim_matrix* gate, const flashoptim_matrix* h, const flashoptim_matrix* y, float* stats,
                          void* stream);

/* The gradients of all of that.  h (x where there is no branch), f, gate and stats as the forward call read and left them; dy: of y
 * (NULL if there was no norm in front); dh: what reaches h from elsewhere (NULL: nothing); not both NULL.
 *   dx = residual_scale (dh + the gradient through the norm in front); df, dgate (summed over the rows that share a gate), and the
 *   gradients of the four arrays, summed over all rows: of type param_dtype, [cols].
 * Every output may be NULL: it is then not wanted.  dx has the type of h, df and dgate that of f.  dx may be dh's own buffer, df f's or dy's.
 * Sums over rows have a fixed order.  workspace as above, for `gates` rows of gates (1 if there are none). */
typedef struct flashoptim_block_norm_grads {
    const flashoptim_matrix *dy, *dh;                                    /* in  */
    const flashoptim_matrix *dx, *df, *dgate;                            /* out */
    void *dpost_weight, *dpost_bias, *dpre_weight, *dpre_bias;           /* out */
} flashoptim_block_norm_grads;

int64_t flashoptim_block_norm_backward_workspace(const flashoptim_block_norm_spec* spec, int64_t rows, int64_t gates);
int flashoptim_block_norm_backward(const flashoptim_block_norm_spec* spec, const flashoptim_matrix* h, const flashoptim_matrix* f,
                                   const flashoptim_matrix* gate, const float* stats, const flashoptim_block_norm_grads* grads,
                                   void* workspace, int64_t workspace_bytes, void* stream);

/* ---- the losses on the logits, where a backward pass begins ----------------------------------------------
 * logits [rows, vocab]: BF16 or FP32, one row for each token that a model has to account for, tokens [rows] INT64 (contiguous) the
 * token itself.  With T the temperature:
 *   lse_i = log sum_j exp(logits_ij / T),    logprob_i = logits_i,t / T - lse_i   with t = tokens_i
 * A row with a negative token does not count: its logits are not read, its logprob, lse and gradients are 0.  A token of vocab or more
 * makes its row's logprob and gradients NaN, and so the loss.  So does a row that holds a NaN or +infinity, or nothing but -infinity
 * (whose lse is -infinity); a -infinity beside other values has the probability 0.  Sums over a row are FP32 by lane and FP64 where lanes
 * join, what is computed once for a row is FP64; the order of all sums depends on the sizes alone.  Vectors are contiguous FP32.
 *   1 <= vocab < 2^30 unless rows = 0; rows < 2^22, and fewer than 2^24 parts of 4096 BF16 or 2048 FP32 values; T > 0 and finite.
 * token_logprob: logprob, lse [rows] and logprob64 [rows], the same as logprob in FP64, for the difference of long sums that a preference
 *   loss is made of.  Each may be NULL (not all, unless rows = 0).
 * token_logprob_backward: dlogits_ij = dlogprob_i / T ([j = t] - exp(logits_ij / T - lse_i)), of the type of logits, from the lse that the forward
 *   call left.  That lse is rounded to FP32 goes into the exponent: the probabilities are off by |lse| 2^-24 of themselves, beside (3 |logits / T - lse| + 5) 2^-24
 *   by the exponent's own roundings and the forward call's error (T below 2^85); where |lse| is 2^17 or more (logits of the type's lowest value and no
 *   others) the gradient is NaN.  (policy_loss, which does not go by lse, has one.)
 *   The logits of a row whose dlogprob is 0 are not read; its gradient is 0.  dlogits may be logits' own buffer.
 * workspace: as in the products above, of the bytes that the *_workspace call returns for the same sizes and type.
 * Here and below, buffers that are written overlap no others of the call unless it says so. */
int64_t flashoptim_token_logprob_workspace(int64_t rows, int64_t vocab, int dtype);
int flashoptim_token_logprob(const flashoptim_matrix* logits, const int64_t* tokens, float temperature, float* logprob, double* logprob64,
                             float* lse, void* workspace, int64_t workspace_bytes, void* stream);
int flashoptim_token_logprob_backward(const flashoptim_matrix* logits, const int64_t* tokens, float temperature, const float* lse,
                                      const float* dlogprob, const flashoptim_matrix* dlogits, void* stream);

/* policy_loss: the clipped policy loss with a KL term to a reference policy, and its gradient in the same pass over the logits.  By row,
 * with A the advantage and w the weight:
 *   r = exp(logprob - old_logprob)                 (old_logprob NULL: of the policy to itself, r = 1, through which the gradient goes all the same)
 *   surrogate = -min(r A, clamp(r, 1 - clip_low, 1 + clip_high) A)               (A = 0: 0, also where r is infinite)
 *   kl = exp(d) - d - 1,  d = ref_logprob - logprob         (ref_logprob NULL: 0; kl_weight 0: in stats [2] only, whatever it is)
 *   stats [4] = { sum w (surrogate + kl_weight kl),  sum w surrogate,  sum w kl,  sum w [blocked] }     the first is the loss
 *   dlogits = grad_scale * the loss's gradient.  A row is blocked, its surrogate without gradient, where A > 0 and r > 1 + clip_high or
 *   A < 0 and r < 1 - clip_low.
 * A row whose weight is 0 does not count, as one with a negative token does not.  weights NULL: 1.  A mean is had by weights that sum to 1.
 * logprob [rows] and dlogits may be NULL (not wanted); dlogits may be logits' own buffer.  clip_low, clip_high and kl_weight are not
 * negative; clip_high may be infinite.  logprob is none of the inputs (to keep it as the next call's old_logprob, give it a buffer of its own). */
typedef struct flashoptim_policy_spec {
    float temperature, clip_low, clip_high, kl_weight, grad_scale;
} flashoptim_policy_spec;

typedef struct flashoptim_policy_inputs {
    const float *advantages, *old_logprob, *ref_logprob, *weights;       /* [rows]; all but the first may be NULL */
} flashoptim_policy_inputs;

int64_t flashoptim_policy_loss_workspace(int64_t rows, int64_t vocab, int dtype);
int flashoptim_policy_loss(const flashoptim_policy_spec* spec, const flashoptim_matrix* logits, const int64_t* tokens,
                           const flashoptim_policy_inputs* inputs, float* stats, float* logprob, const flashoptim_matrix* dlogits,
                           void* workspace, int64_t workspace_bytes, void* stream);

/* preference_loss: of pairs of sequences, one chosen and one rejected, from the log-probabilities of their tokens, in FP32 or in FP64 (the
 * other is NULL).
 *   gain(s) = sum over the rows of s of weights (logprob - ref_logprob),   z = beta (gain(chosen) - gain(rejected))
 *   loss = the mean over the pairs of, by kind:  SIGMOID  (1 - label_smoothing) log(1 + exp(-z)) + label_smoothing log(1 + exp(z))
 *                                                HINGE    max(0, 1 - z)
 *                                                SQUARED  (z / beta - 1 / (2 beta))^2
 *   margins [pairs] = z (may be NULL);  dlogprob [rows] = grad_scale * the loss's gradient (may be NULL), 0 for rows of no sequence; it may be
 *   logprob's own buffer.
 * offsets [2 pairs + 1] INT64, not descending, within [0, rows] (what lies outside is taken as the nearest bound): sequence i is the rows
 * offsets[i] .. offsets[i + 1] - 1, possibly none.  order: sequences 2p and 2p + 1 are the chosen and the rejected one of pair p
 * (FLASHOPTIM_PAIRS_BY_TURNS), or p and pairs + p (FLASHOPTIM_PAIRS_HALVES).  Rows whose weight is 0 do not count, whatever their
 * logprob; weights, ref_logprob NULL: 1, 0.  (No tokens are seen here: a row of a negative one, which token_logprob leaves a logprob of 0, is a
 * part of its sequence's gain, 0 - ref_logprob, unless its weight is 0.)  No pairs: a loss of 0.  beta > 0, 0 <= label_smoothing <= 0.5, which is for SIGMOID only.
 * Sums are FP64.  rows < 2^31, pairs < 2^30. */
enum { FLASHOPTIM_PREFERENCE_SIGMOID = 0, FLASHOPTIM_PREFERENCE_HINGE = 1, FLASHOPTIM_PREFERENCE_SQUARED = 2 };
enum { FLASHOPTIM_PAIRS_BY_TURNS = 0, FLASHOPTIM_PAIRS_HALVES = 1 };

typedef struct flashoptim_preference_spec {
    int32_t kind, order;
    float beta, label_smoothing, grad_scale;
} flashoptim_preference_spec;

int flashoptim_preference_loss(const flashoptim_preference_spec* spec, const float* logprob, const double* logprob64,
                               const float* ref_logprob, const float* weights, int64_t rows, const int64_t* offsets, int64_t pairs,
                               float* loss, float* margins, float* dlogprob, void* stream);

/* ---- the norm of all gradients and their clipping, between a backward pass and the step -----------------
 * A list of gradients, each flattened, contiguous and 16-byte aligned; src of BF16 or FP32 (src_dtype, one for the whole list).  Its
 * descriptors travel with the launches: nothing is cached, and a captured call keeps the list that it was captured with.
 * grad_norm: *factor (DEVICE memory, 16-byte aligned) <- sum_squares, the sum of the squares of all elements in FP64 (no finite gradient
 *   overflows it); norm, its root; scale = max_norm / norm where norm > max_norm, else 1, and NaN where sum_squares is not finite.  A list without
 *   elements has the norm 0.  max_norm >= 0, possibly infinite.  dst is ignored.  The order of the sum depends on the sizes alone.
 * clip_factor_from_sum: recomputes norm and scale of *factor from its sum_squares, to which other lists' or ranks' sums have been added meanwhile (shards
 *   of one model on several ranks: an all-reduce of that value).
 * clip_gradients: dst <- src * scale, rounded once, of type dst_dtype: that of src, or BF16 for FP32 src (gradients accumulated in FP32, into
 *   the ones that the step reads).  dst may be src itself if the types are the same; where scale is 1 such a buffer is not touched.  With a
 *   scale of NaN every element becomes NaN.  Other overlaps of buffers are errors of the caller.
 * 0 <= numel < 2^40 each, fewer than 2^43 together; an empty tensor's pointers are ignored.  workspace as above, for the same list. */
typedef struct flashoptim_clip_factor {
    double sum_squares;
    float  norm, scale;
} flashoptim_clip_factor;

typedef struct flashoptim_gradient {
    const void* src;
    void*       dst;
    int64_t     numel;
} flashoptim_gradient;

int64_t flashoptim_grad_norm_workspace(const flashoptim_gradient* grads, int64_t n_grads, int src_dtype);
int flashoptim_grad_norm(const flashoptim_gradient* grads, int64_t n_grads, int src_dtype, float max_norm,
                         flashoptim_clip_factor* factor, void* workspace, int64_t workspace_bytes, void* stream);
int flashoptim_clip_factor_from_sum(flashoptim_clip_factor* factor, float max_norm, void* stream);
int flashoptim_clip_gradients(const flashoptim_gradient* grads, int64_t n_grads, int src_dtype, int dst_dtype,
                              const flashoptim_clip_factor* factor, void* stream);

/* The steps above with the clipping in them: the gradients count times factor->scale (read on the device when the step runs), a product in FP32 that
 * is not rounded to BF16, and are left as they are; nothing of theirs is read or written a second time.  With a scale of 1 the results are
 * those of the step without; with a scale of NaN, that of gradients which are not finite, weights and states stay as they are (also the weight
 * decay is left out), only the rates of a list's table change.  A list's tables are the same with and without. */
int flashoptim_adamw_step_clipped(const flashoptim_tensor* tensors, int64_t n_tensors, const flashoptim_adamw_hp* hp,
                                  const flashoptim_clip_factor* factor, void* stream);
int flashoptim_adamw_step_exact_clipped(const flashoptim_tensor* tensors, int64_t n_tensors, const flashoptim_adamw_hp* hp,
                                        const flashoptim_clip_factor* factor, void* stream);
int flashoptim_sgd_step_clipped(const flashoptim_tensor* tensors, int64_t n_tensors, const flashoptim_sgd_hp* hp,
                                const flashoptim_clip_factor* factor, void* stream);
int flashoptim_lion_step_clipped(const flashoptim_tensor* tensors, int64_t n_tensors, const flashoptim_lion_hp* hp,
                                 const flashoptim_clip_factor* factor, void* stream);

/* ---- housekeeping --------------------------------------------------------------------
 * strerror: static string for a status.  last_hip_error: hipError_t value of the most recent
 * failed HIP call on this thread (0 if none).  release_cache: frees the cached device chunk
 * tables (synchronises the device first).  version: (major << 16) | minor. */
const char* flashoptim_strerror(int status);

/* ---- device self-test ------------------------------------------------------------------
 * The kernels obtain some correctly rounded results (1/s of an FP16 scale, sqrt, the
 * decision of an 8-bit code) from shorter instruction sequences that are exact provided the
 * hardware reciprocal and square root are within 1 ulp.  This call checks those provisions on
 * the current device against plain IEEE operations, exhaustively where the domain is small:
 *   [0] Newton reciprocal of every positive finite FP16 value
 *   [1] v_rcp_f32 within 1 ulp, its refinement exact, and v_sqrt_f32 within 1 ulp, for every value of [1, 4)
 *   [2] short square root (reciprocal-square-root estimate + one correction) == sqrtf for EVERY FP32 value
 *       of its range [2^-96, FLT_MAX] (1,879,048,192 values)
 *   [3] momentum codes (Algorithm 2) and [4] variance codes (Algorithm 3): the estimate equals the
 *       exact code wherever the kernel's tie test does not ask for the exact evaluation.
 *   [5] short division == IEEE division on 2^30 + 2^24 operand pairs inside its range.
 *   [6] faithful division of flashoptim_adamw_step: within 1 ulp of the IEEE quotient on the pairs of [5].
 * n_checked, n_failed: HOST arrays of 7 counters (one per section above).  Waits for completion (a
 * fraction of a second).  Returns FLASHOPTIM_OK, FLASHOPTIM_ERR_SELFTEST if any check failed, or another status. */
int flashoptim_selftest(int64_t* n_checked, int64_t* n_failed, void* stream);
/* How often the faithful division differs from the exactly rounded quotient at all, measured on this device:
 * counts (HOST, 2 entries) = {operand pairs checked (2^30 + 2^24), of these not exact}.  Waits for
 * completion.  FLASHOPTIM_ERR_SELFTEST if any quotient is off by more than one ulp. */
int flashoptim_faithful_rounding_stats(int64_t* counts, void* stream);
/* The AdamW kernels take sqrt(v_hat) as the hardware reciprocal-square-root estimate plus one correction,
 * which is the correctly rounded root only if the estimate makes it so.  They read the lower limit of that
 * sequence's use from a word of device memory that holds +inf (never used: sqrtf throughout) until the device
 * has passed a check of every FP32 value of the sequence's range, [2^-96, FLT_MAX], against sqrtf.  The first
 * AdamW step call on a device (any entry point but flashoptim_adamw_step_noalloc) puts that check on its stream
 * ahead of its own kernels, once per process and device: about 4 ms on MI355X, no allocation, no wait on the
 * host.  Kernels that run before the verdict has landed (on another stream, say) use sqrtf, with the same
 * results.  A first call made under stream capture does not start the check (it belongs in front of a graph,
 * not inside it); a later call outside capture does.  With FLASHOPTIM_FORCE_GENERAL_SQRT set to a non-zero
 * value in the environment the check is not run and the word stays at +inf.
 * Returns the state for the current device: 0 check not started, 1 verified (short sequence in use), 2 not in
 * use; negative status on a HIP error.  If the check is on its way the call waits for its verdict; in states
 * 0 and 2 it reads the word back (a blocking 4-byte copy) and returns FLASHOPTIM_ERR_SELFTEST unless it holds
 * +inf. */
int flashoptim_short_sqrt_state(void);
/* A measurement aid: samples the clock the compute units run at while other kernels execute (a step kernel
 * under the package power limit runs well below the nominal clock).  Enqueues a one-wavefront kernel on
 * `stream` (use a stream of its own, next to the work to be observed) that takes n_samples samples of
 * seconds_per_sample each and then ends; it writes 2 * n_samples uint64 values to `samples` (DEVICE memory,
 * owned by the caller, valid until the kernel has finished): for each sample the ticks of the fixed-frequency
 * counter that went by and the shader-clock cycles in the same interval.  *tick_hz (HOST) receives the tick
 * rate, so that clock = cycles / ticks * tick_hz.  1 <= n_samples <= 100000, 0 < seconds_per_sample <= 1.
 * Does not wait for completion. */
int flashoptim_clock_monitor(uint64_t* samples, int64_t n_samples, double seconds_per_sample, double* tick_hz,
                             void* stream);
/* Number of kernel launches one step call of `kind` issues for a list with these element counts
 * (host arithmetic only; for reading profiles: per-kernel durations are per launch).  Negative
 * status on invalid arguments. */
int64_t flashoptim_step_launch_count(int kind, const int64_t* numels, int64_t n_tensors);
int flashoptim_last_hip_error(void);
int flashoptim_release_cache(void);
int flashoptim_version(void);

#ifdef __cplusplus
}
#endif
#endif /* FLASHOPTIM_H */
