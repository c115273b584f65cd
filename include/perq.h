/*
 * perq.h -- C ABI of the PeRQ online path for NVIDIA B200 (sm_100a).
 *
 * PeRQ = Permute, Rotate, then Quantize.  For activation rows X[T, d] (bf16) the path is
 *
 *     (X P)  ->  (X P) R~  ->  Q((X P) R~)
 *
 * with P a channel permutation applied as a gather, R~ = I_n (x) R a block-diagonal
 * rotation whose b x b block R is the normalised Sylvester Hadamard matrix, and Q a 4-bit
 * quantiser (symmetric INT4 or MXFP4).  Citations below are to the paper's sections,
 * equations and algorithms.
 *
 * Conventions for every entry point
 *   - "device" pointers are CUDA device memory, "host" pointers ordinary host memory.
 *   - The caller owns every buffer; nothing is allocated, freed or retained by the
 *     library.
 *   - Work is enqueued on `stream` (a cudaStream_t passed as void*, NULL = default
 *     stream); no call synchronises the device unless it says so.  Outputs are valid
 *     once the caller has synchronised `stream`.
 *   - The return value is a perq_status_t.  Arguments are checked on the host before
 *     anything is launched: on an argument error nothing has been enqueued.  PERQ_ERR_CUDA
 *     (a launch or a copy that the runtime refused) can come after earlier work of the same
 *     call was enqueued: the host-buffer entry point has then already queued its copy to
 *     the device, perq_block_l1_stats its first kernel; the outputs are undefined.
 *   - Device pointers must be 16-byte aligned.  Rows are dense (row stride = d).
 *   - Inputs are assumed finite.  NaN/Inf give unspecified codes but never a fault (perq_rotate_quantize_i8 shows them).
 */
#ifndef PERQ_H
#define PERQ_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    PERQ_FMT_INT4 = 0,      /* symmetric INT4, absmax scale (fp32) per token or per group */
    PERQ_FMT_MXFP4 = 1,     /* E2M1 elements, one E8M0 scale per 32 elements */
    PERQ_FMT_F32_DEBUG = 2, /* no quantisation: the rotated row as fp32 (test hook) */
    PERQ_FMT_FP4 = 3,       /* E2M1 elements, one fp32 scale per token (Appendix B, FP4 activations) */
    PERQ_FMT_INT4_ASYM = 4, /* asymmetric INT4, (scale, zero point) per token (Appendix B, INT4 activations) */
    PERQ_FMT_INT8 = 5       /* symmetric INT8, one fp32 scale per row: perq_rotate_quantize_i8 and the products only */
} perq_fmt_t;

typedef enum { PERQ_OUT_BF16 = 0, PERQ_OUT_F16 = 1, PERQ_OUT_F32 = 2 } perq_out_t;   /* results of the products */

typedef enum {
    PERQ_OK = 0,
    PERQ_ERR_NULL = 1,   /* a required pointer is NULL */
    PERQ_ERR_SHAPE = 2,  /* T < 0, d <= 0, d % 32 != 0 or d > PERQ_MAX_D; also: a row that the general kernel cannot
                            hold in 227 KB of shared memory with its per-range tables (very small groups of very long rows) */
    PERQ_ERR_BLOCK = 3,  /* b is neither a power of two in [16, d] that divides d nor (perq_rotate_quantize) a supported b == d = 2^k * 4t */
    PERQ_ERR_GROUP = 4,  /* INT4: group not 0 and (d % group != 0, group % 8 != 0, or group neither a multiple nor a
                            divisor of b); MXFP4: group not 0/32; FP4, INT4_ASYM: not 0 */
    PERQ_ERR_FMT = 5,    /* unknown format */
    PERQ_ERR_ALIGN = 6,  /* a device pointer is not 16-byte aligned */
    PERQ_ERR_CUDA = 7,   /* the CUDA runtime reported an error (launch, copy, attribute) */
    PERQ_ERR_PERM = 8,   /* host-side permutation argument is not a permutation */
    PERQ_ERR_WORKSPACE = 9, /* workspace missing or too small */
    PERQ_ERR_UNSUPPORTED = 10 /* valid arguments that this entry point does not cover (see its description) */
} perq_status_t;

#define PERQ_MAX_D 32768
#define PERQ_MAX_N 1048576      /* channels of a product (of one expert) */
#define PERQ_MAX_EXPERTS 1024
#define PERQ_MAX_SEQUENCES 65536 /* of a call on the cache */
#define PERQ_MAX_HEADS 1024

/*
 * perq_rotate_quantize -- the online hot path, one fused pass.
 *
 * Defined by: Notation paragraph of Sec. 1 (row vector X, d = n*b, block rotation
 * R~ = I_n (x) R, permutation P e_i = e_pi(i)); the block proposition of Sec. 3 and the
 * coordinate form in the proof of the probabilistic proposition (blocks are contiguous
 * index ranges of the permuted row); Sec. 3 for the INT step size
 * s = ||X||_inf / (2^{q-1} - 1); Appendix B for the INT4 and (MX)FP4 quantisers.
 *
 * For every token row t:
 *   1. x'_i = x[t, perm[i]]                       (perm == NULL: x' = x)
 *   2. y_{j*b+i} = b^{-1/2} * sum_{k<b} (-1)^{popcount(i & k)} x'_{j*b+k}   for each block j
 *   3. INT4:  per scale range G (whole row if group == 0, else each `group` consecutive
 *             coordinates of y): a = max_G |y|, s = a / 7, code_i = clip(rne(y_i / s), -8, 7),
 *             stored scale = s as fp32.  a == 0 gives scale 0 and codes 0.
 *      MXFP4: per 32 consecutive coordinates: a = max |y|, E = floor(log2 a) - 2 clamped to
 *             [-127, 127], stored scale byte = E + 127 (0 if a == 0); element code =
 *             sign(y_i) << 3 | index of the nearest of {0, .5, 1, 1.5, 2, 3, 4, 6} to
 *             |y_i| * 2^-E, ties to the even index, saturating at 6.
 *      FP4:   per token: a = max |y|, s = a / 7 (the step the paper gives for FP4 activations), stored as
 *             fp32; element code = sign(y_i) << 3 | index of the nearest of {0, .5, 1, 1.5, 2, 3, 4, 6} to
 *             |y_i| / s, ties to the even index, saturating at 6 (so the row maximum itself saturates).
 *      INT4_ASYM: per token: s = (max y - min y) / 15, z = rne(min y / s),
 *             code_i = clip(rne(y_i / s) - z, 0, 15) (unsigned nibble); the value is s * (code_i + z).
 *             Stored: (s, z) as two fp32.  A constant row gives s = 0, z = 0, codes 0.
 *   4. byte k of the output row = code[2k] | code[2k+1] << 4  (INT4 nibbles are two's complement).
 *
 * x          device, bf16 [T, d] row-major.
 * perm       device, int32 [d], a permutation of 0..d-1, or NULL.  Out-of-range entries
 *            are clamped into range (wrong numbers, never a fault); use
 *            perq_validate_perm to check a permutation beforehand.
 * T, d       rows and channels.  T == 0 is a no-op (pointers are then not looked at).
 *            d % 32 == 0, d <= PERQ_MAX_D.
 * b          a power of two, 16 <= b <= d, with d % b == 0 (b == d is the full-vector rotation); or, for a d
 *            that is not a power of two, b == d = 2^k' * 4t with t the odd part of d and 4t one of 12, 28,
 *            36, 60, 76 (Appendix A.1, "An Optimized Non-Power-of-2 Hadamard Rotation": Llama-3-8B's
 *            14336 = 2^9 * 28, Qwen3's 3072 / 6144 / 12288 = 2^k' * 12 and 9728 = 2^7 * 76).  Step 2 is then
 *            y_i = d^{-1/2} sum_k (-1)^{popcount(floor(i/4t) & floor(k/4t))} B[i mod 4t][k mod 4t] x'_k: rotations
 *            of 4t ADJACENT inputs by a +-1 base matrix B, then k' butterfly stages over strides of 4t.  The
 *            paper does not print its base matrices; B is Paley's second construction for the prime
 *            q = 2t - 1 (symmetric, B B^T = 4t I), so codes need not equal those of another implementation's
 *            matrix.  Other non-power-of-two b, and such a b inside a longer row: PERQ_ERR_BLOCK.
 *            All of these run on tensor-core kernels when d % 128 == 0 and d <= 16384 (for 2^k' * 4t: 6 <= k' <= 10)
 *            and an INT4 group is 0 or a power of two from 32 to 1024; other widths, groups and the F32_DEBUG
 *            output run on a slower general kernel.
 * fmt        perq_fmt_t.
 * group      INT4: 0 (per token) or a multiple of 8 that divides d and is a multiple or a divisor of b.
 *            MXFP4: 0 or 32 (always 32).  FP4, INT4_ASYM: 0.
 *            Scale ranges are consecutive coordinates of the ROTATED row, independent of b.
 * out_codes  device.  INT4/MXFP4: uint8 [T, d/2].  F32_DEBUG: float [T, d] (the rotated row y).
 * out_scales device.  INT4: float [T] or [T, d/group].  MXFP4: uint8 [T, d/32].  FP4: float [T].  INT4_ASYM: float [T, 2].
 *            F32_DEBUG: unused, may be NULL.
 *
 * Codes and scales are deterministic (bit-identical from run to run).  Which kernel serves a call depends
 * on its shape; every kernel stores the fp32 rounding of the exact scale up to one more rounding of a
 * constant factor, so scales of the same row from different shapes' kernels agree to 1 ulp, not bit for bit.
 * Range limits: a token whose largest |y| lies below about 2^-120 (every input subnormal or nearly so) gets
 * the exact scale but all-zero INT4/FP4 codes from the tensor-core kernels, because the fp32 reciprocal of
 * such a scale overflows; the definition would give +-7 at the maximum.  At the other end sqrt(b) |y| has to stay
 * below 2^126 (d % 1024 == 0 with b <= 128, or unpermuted blocks of 256 to 1024: above it the codes come out 0, except in
 * large unpermuted calls, whose kernel goes up to 2^128) or below 2^128 (all other shapes).  A scale range or MX group that is part of a Hadamard block and whose outputs all
 * cancel to zero in fp32 (below about 2^-24 of the block's largest) gets scale 0.
 */
int perq_rotate_quantize(const void *x, const int32_t *perm, int64_t T, int32_t d, int32_t b,
                         int32_t fmt, int32_t group, void *out_codes, void *out_scales,
                         void *stream);

/*
 * perq_swiglu_rotate_quantize -- the same path fed by the gated activation of a feedforward block.
 *
 * Defined by: the figure on permutation equivariance (the feedforward network of a transformer block):
 * the online rotation's input is h = Swish(x W_gate) (.) (x W_up) -- an elementwise product; Swish(g) =
 * g * sigmoid(g) = g / (1 + exp(-g)) -- and the region is permutation-equivariant, so the permutation is
 * merged into the two projections and none is applied here.  With gate = x W_gate and up = x W_up given as
 * bf16, every row is
 *
 *     h_i = bf16( Swish(gate_i) * up_i )        (the real product, rounded once, to nearest even)
 *
 * followed by steps 2-4 of perq_rotate_quantize on h.  The outputs equal those of perq_rotate_quantize on a
 * materialised h; h is never written to memory (4d + d/2 bytes per token move instead of 8d + d/2).
 * The activation is evaluated in fp32 and again in fp64 wherever the fp32 value is too close to a bf16
 * rounding boundary to decide the rounding, so h is the correctly rounded value.
 *
 * gate, up   device, bf16 [T, d] row-major.      perm   must be NULL (PERQ_ERR_UNSUPPORTED otherwise).
 * Covered:   d % 1024 == 0, b <= 128, and fmt / group = MXFP4, INT4 with group 128, or INT4 per token with
 *            d <= 15360.  Anything else that perq_rotate_quantize would accept returns PERQ_ERR_UNSUPPORTED
 *            (materialise h and call perq_rotate_quantize).
 * Other arguments, outputs and errors as for perq_rotate_quantize.
 */
int perq_swiglu_rotate_quantize(const void *gate, const void *up, const int32_t *perm, int64_t T, int32_t d,
                                int32_t b, int32_t fmt, int32_t group, void *out_codes, void *out_scales,
                                void *stream);

/*
 * perq_out_sizes -- bytes of out_codes and out_scales for a call.  Host only, no CUDA.
 * Either output pointer may be NULL.
 */
int perq_out_sizes(int64_t T, int32_t d, int32_t fmt, int32_t group, size_t *codes_bytes,
                   size_t *scales_bytes);

/*
 * perq_rotate_quantize_host -- the same operation on HOST buffers.
 *
 * Copies x from host memory (pinned memory makes the copies asynchronous), runs
 * perq_rotate_quantize on the device and copies codes and scales back, all on `stream`,
 * then synchronises `stream` before returning.  `workspace` is device memory provided
 * by the caller, at least perq_host_workspace_bytes(...) long; the library allocates
 * nothing.  perm stays a DEVICE pointer (it is reused across calls) or NULL.
 *
 * Calls of 4096 rows or more are processed in four chunks of rows, and the copy back of a
 * chunk runs on an internal non-blocking stream while the next chunk is copied in; that
 * stream and five events are created once per device on first use and kept until exit.
 * Two such calls at the same time on one device (different caller streams) would share
 * those events: issue them from one thread at a time.
 */
int perq_rotate_quantize_host(const void *x_host, const int32_t *perm, int64_t T, int32_t d,
                              int32_t b, int32_t fmt, int32_t group, void *out_codes_host,
                              void *out_scales_host, void *workspace, size_t workspace_bytes,
                              void *stream);
int perq_host_workspace_bytes(int64_t T, int32_t d, int32_t fmt, int32_t group, size_t *bytes);

/*
 * perq_block_l1_stats -- the calibration statistic of the greedy mass-diffusion
 * permutation (Algorithm 1: per-coordinate mean magnitude and per-block mean l1 norm)
 * and of the block proposition's bound ||X R~||_inf <= max_j ||X_{j}||_1 / sqrt(b).
 *
 *   chan_abs_sum[c]       = sum_t |x[t, c]|                         (original channel order)
 *   block_l1_mean[j]      = (1/T) sum_t L[t, j],   L[t, j] = sum_{i<b} |x[t, perm[j*b+i]]|
 *   token_max_block_l1[t] = max_j L[t, j]
 *
 * x, perm, T, d as above (T >= 1 here unless all outputs are NULL); b a power of two
 * >= 8 dividing d.  Each output is device fp32 and may be NULL: [d], [d/b], [T].
 * workspace  device, perq_block_l1_stats_workspace_bytes(...) bytes: per-CTA partial sums
 *            that a second kernel adds in a fixed order, so results are deterministic.
 * Accumulation is fp32: sums agree with exact arithmetic to about 1e-6 relative.
 */
int perq_block_l1_stats(const void *x, const int32_t *perm, int64_t T, int32_t d, int32_t b,
                        float *chan_abs_sum, float *block_l1_mean, float *token_max_block_l1,
                        void *workspace, size_t workspace_bytes, void *stream);
int perq_block_l1_stats_workspace_bytes(int64_t T, int32_t d, int32_t b, size_t *bytes);

/*
 * perq_block_l1_stats_static -- perq_block_l1_stats for callers that cannot provide a workspace.
 *
 * (No counterpart in the paper: this is a deployment variant of the entry point above.)
 * Some hosts of this library may not allocate device memory at the point where they want
 * the statistic: code that runs inside a memory-pool-managed serving loop whose pool is
 * already fully handed out, plugins that are only given their input and output tensors,
 * or processes whose allocator must stay quiet because allocation would synchronise the
 * device.  For them the per-CTA partial sums go to a fixed array inside the library
 * instead of a caller workspace; outputs and every other argument are as above, and the
 * results are bit-identical to perq_block_l1_stats on the same inputs.
 *
 *   - The array holds PERQ_STATS_STATIC_MAX_FLOATS floats (9.25 MiB) and is part of the
 *     library image: every GPU that loads the library holds it until the process exits.
 *   - A shape is accepted when perq_block_l1_stats_workspace_bytes(T, d, b) fits in the
 *     array, i.e. min(T, 148) * (d + d/b) <= PERQ_STATS_STATIC_MAX_FLOATS; this covers
 *     every d <= 14336 with any T and b >= 8.  Larger shapes return PERQ_ERR_WORKSPACE
 *     and launch nothing.
 *   - The call allocates and frees nothing, on the device or through any library.
 *   - The first call on each device looks up the array's device address (with that
 *     device current) and remembers it; make that first call outside any stream capture.
 *   - All calls on a device share the one array.  Nothing in it has to be zero on entry
 *     (each call overwrites what it reads), but two calls whose kernels overlap on the
 *     GPU -- different streams, no ordering between them -- race on it and give wrong
 *     sums.  Calls on one stream, or ordered by events, are safe.
 */
#define PERQ_STATS_STATIC_MAX_FLOATS (148 * 16384)
int perq_block_l1_stats_static(const void *x, const int32_t *perm, int64_t T, int32_t d, int32_t b,
                               float *chan_abs_sum, float *block_l1_mean,
                               float *token_max_block_l1, void *stream);

/*
 * perq_token_diagnostics -- the per-token quantities the paper plots (the figures on the mass
 * concentration delta, on the block bound versus the block size, and on the bound versus the
 * quantization error), before their normalisation by ||X||_inf.  With x' = gather(x, perm), blocks of
 * b channels, y = x' R~ (block Hadamard rotation) and Q the symmetric 4-bit quantiser of Sec. 3 with one
 * step per token (s = ||y||_inf / 7, round to nearest even), row t of out holds
 *
 *   out[t][0] = ||x||_inf                 out[t][1] = ||x||_1
 *   out[t][2] = max_j ||x'_{j}||_1        (= b max_j delta_{j} ||x'_{j}||_inf, proposition on block rotations)
 *   out[t][3] = ||y||_inf                 out[t][4] = ||y - Q(y)||_2
 *
 * so delta = out1 / (d out0) (proposition on full-vector rotations), the normalised block bound is
 * out2 / (b out0), the outlier suppression ratio out3 / out0, the normalised error out4 / out0.
 *
 *   x, perm, T, d, b   as for perq_rotate_quantize (device pointers; perm may be NULL)
 *   out                float [T, 5], device, written in full; a zero row gives five zeros
 *   stream             cudaStream_t (0 = default); the call only enqueues work
 *
 * Arithmetic is fp32 (sums in a fixed order: outputs are deterministic); the values agree with their
 * real-arithmetic definitions to about 1e-5 relative.  The caller owns every buffer; nothing is
 * allocated.  Errors: as perq_rotate_quantize (NULL, SHAPE, BLOCK, ALIGN, CUDA).
 */
int perq_token_diagnostics(const void *x, const int32_t *perm, int64_t T, int32_t d, int32_t b,
                           float *out, void *stream);

/*
 * perq_validate_perm -- checks on the device that perm[0..d) is a permutation.
 * Writes one int32 to status_dev: 0 = valid, bit 0 = an entry out of range,
 * bit 1 = a duplicate entry.  (Algorithm 1 returns such a permutation; this guards
 * perq_rotate_quantize against a corrupted one.)
 */
int perq_validate_perm(const int32_t *perm, int32_t d, int32_t *status_dev, void *stream);

/*
 * perq_massdiff_perm -- Algorithm 1 (MassDiff), host only, no CUDA.
 *
 * Visits channels in descending chan_abs_sum (ties: lower channel first), assigns each
 * to the not-yet-full block with the smallest running sum (ties: lower block first), and
 * returns the blocks concatenated: perm[j*b + r] = r-th channel assigned to block j.  The
 * result is the `perm` argument of perq_rotate_quantize / perq_block_l1_stats.
 * chan_abs_sum_host: float [d] (e.g. copied back from perq_block_l1_stats; the mean is a
 * positive multiple of the sum, so sums give the same permutation).  perm_host: int32 [d].
 * Running sums are kept in double.  b >= 1, d % b == 0.
 */
int perq_massdiff_perm(const float *chan_abs_sum_host, int32_t d, int32_t b, int32_t *perm_host);

/*
 * perq_chan_abs_max, perq_absmax_perm, perq_zigzag_perm -- the permutations the paper compares MassDiff with
 * (Appendix C, paragraph "Permutations", Table "permute_fn_ablations"; Sec. 4.2 on the zigzag assignment).
 *
 *   perq_chan_abs_max   device: chan_abs_max[c] = max_t |x[t, c]| (float [d], written in full; x bf16 [T, d]
 *                       device, 16-byte aligned; d % 32 == 0).  Enqueues a memset and one kernel on `stream`.
 *   perq_absmax_perm    host only: the channels in descending order of that maximum (equal values: lower
 *                       channel first).
 *   perq_zigzag_perm    host only: the same visiting order dealt to the n = d / b blocks back and forth
 *                       (ranks 0..n-1 to blocks 0..n-1, ranks n..2n-1 to blocks n-1..0, ...); slot r of
 *                       block j holds the channel that round r gave it: perm[j*b + r].
 * The paper prints neither procedure; these are the readings this library takes.  Host arrays: float [d] in,
 * int32 [d] out; the result is a `perm` argument of perq_rotate_quantize / perq_block_l1_stats.
 * Errors: NULL, SHAPE, BLOCK (b < 1 or d % b != 0), ALIGN, CUDA.
 */
int perq_chan_abs_max(const void *x, int64_t T, int32_t d, float *chan_abs_max, void *stream);
int perq_absmax_perm(const float *chan_abs_max_host, int32_t d, int32_t *perm_host);
int perq_zigzag_perm(const float *chan_abs_max_host, int32_t d, int32_t b, int32_t *perm_host);

/*
 * perq_massdiff_perm_device -- Algorithm 1 (MassDiff) on the device: the same permutation as
 * perq_massdiff_perm, entry for entry, from a device array, so that a calibration pass (statistic ->
 * permutation -> permuted rotate+quantize) needs no copy to the host.
 *
 *   chan_abs_sum     float [d], device (e.g. the output of perq_block_l1_stats); finite, non-negative
 *   perm             int32 [d], device, written in full
 *   workspace        device, at least d * 4 bytes (the channels in visiting order); caller-owned
 *   stream           cudaStream_t (0 = default); two kernels are enqueued, nothing is synchronised
 *
 * b >= 1, d % b == 0, d <= PERQ_MAX_D and at most 4096 blocks (d / b).  One CTA serves the channels in batches,
 * about 0.11 ms for a statistic of d = 8192, b = 32; masses that fall steeply are served one by one (about 1.2 ms
 * there).  NaN and negative masses count as 0, infinity as the largest float.
 * Errors: NULL, SHAPE, BLOCK (also: too many blocks), WORKSPACE, ALIGN, CUDA.
 */
int perq_massdiff_perm_device(const float *chan_abs_sum, int32_t d, int32_t b, int32_t *perm,
                              void *workspace, size_t workspace_bytes, void *stream);

/*
 * perq_rotate_quantize_i8 -- the path with 8-bit codes: rows of tokens, or of weight channels, for the products below.
 *
 * Defined by: steps 1 and 2 of perq_rotate_quantize and the symmetric quantiser of Sec. 3 with q = 8, one step per row:
 *     a = max_i |y_i|,  s = a / 127,  code_i = rne(y_i / s)   (ties to even; a == 0 gives scale 0 and codes 0)
 * with codes decided in exact arithmetic and s stored as fp32.  y = x' (no rotation) for b == 1.
 *
 * x, perm, T, d as for perq_rotate_quantize.  b: 1, or a power of two from 16 to 512 that divides d (larger powers of two that
 * divide d: PERQ_ERR_UNSUPPORTED).  out_codes int8 [T, d], out_scales float [T].
 * Deterministic.  Every finite row is served, down to subnormals and up to the largest numbers of bf16.  A row with an infinity or a NaN
 * has codes 0 and the scale that the formula gives, infinite or NaN, so that its results in the products are not finite either.
 * Errors: NULL, SHAPE, BLOCK, UNSUPPORTED, ALIGN, CUDA.
 */
int perq_rotate_quantize_i8(const void *x, const int32_t *perm, int64_t T, int32_t d, int32_t b, void *out_codes,
                            float *out_scales, void *stream);

/*
 * perq_code_sums -- sums[r] = sum_k code[r][k] of rows of INT8 or INT4 codes (device int32 [rows]): what the products want of the
 * weights for asymmetric tokens, made once with them.  fmt: PERQ_FMT_INT8, PERQ_FMT_INT4.  rows == 0 is a no-op; d as above.
 * Errors: NULL, SHAPE, FMT, ALIGN, CUDA.
 */
int perq_code_sums(const void *codes, int32_t fmt, int64_t rows, int32_t d, int32_t *sums, void *stream);

/*
 * perq_matmul_i8 -- the linear layer that reads the path's codes: the product of codes in 8-bit integers with a scale for
 * each token and each weight channel.
 *
 * Defined by: Sec. 4.3 and the figure on permutation equivariance (the rotated, quantised activations enter the down
 * projection, whose rows carry the same rotation: (X R~)(W R~)^T = X W^T) and the quantisers of Sec. 3 and Appendix B, whose
 * values are s * code and, asymmetric, s * (code + z).  For token t and weight channel n
 *
 *     y[t][n] = s_t * s_n * ( sum_k a[t][k] w[n][k]  +  z_t * c_n ),      c_n = sum_k w[n][k]
 *
 * with z_t = 0 unless a_fmt is PERQ_FMT_INT4_ASYM.  The first sum is exact (32-bit integers; |sum| < 2^31 for every d
 * allowed); it, the corrected sum, the two products and the result are each rounded once to fp32, the result then to
 * out_type, to nearest even.  Results are the same from run to run and do not depend on which kernel serves the call.
 *
 *   a_codes, a_scales   device: codes and scales of T rows as perq_rotate_quantize writes them for INT4 per token (uint8
 *                       [T, d/2], float [T]) and INT4_ASYM (uint8 [T, d/2], float [T, 2]: step, zero point), or as
 *                       perq_rotate_quantize_i8 does (int8 [T, d], float [T])
 *   a_fmt               PERQ_FMT_INT8, PERQ_FMT_INT4 or PERQ_FMT_INT4_ASYM
 *   w_codes, w_scales   device: the same of N weight channels (rows [N, d]); w_fmt PERQ_FMT_INT8 or PERQ_FMT_INT4
 *   w_sums              device int32 [N]: c_n, from perq_code_sums; read for INT4_ASYM only (else it may be NULL)
 *   T, N, d             T == 0 is a no-op; T <= 2^30; 1 <= N <= PERQ_MAX_N; d % 32 == 0, d <= PERQ_MAX_D
 *   out                 device [T, N] of out_type (perq_out_t), row stride N, written in full
 *   workspace           device, at least perq_matmul_i8_workspace_bytes(...) bytes (NULL where that is 0).  What is enough for T
 *                       tokens is enough for fewer with the same N, d and formats (and E).  Calls of many tokens spread packed
 *                       operands to bytes there, in each call: T d bytes of tokens, N d of weights (E N d).  Its contents need
 *                       not be kept; calls that may overlap need one each.
 *
 * Scales that are infinite or NaN give what fp32 arithmetic makes of the formula.  All device pointers 16-byte aligned.
 * Errors: NULL, SHAPE, FMT (formats and out_type), ALIGN, WORKSPACE, CUDA.
 */
int perq_matmul_i8(const void *a_codes, const float *a_scales, int32_t a_fmt, const void *w_codes, const float *w_scales,
                   int32_t w_fmt, const int32_t *w_sums, int64_t T, int32_t N, int32_t d, void *out, int32_t out_type,
                   void *workspace, size_t workspace_bytes, void *stream);
int perq_matmul_i8_workspace_bytes(int64_t T, int32_t N, int32_t d, int32_t a_fmt, int32_t w_fmt, size_t *bytes);

/*
 * perq_grouped_matmul_i8 -- the same product grouped by expert, with ragged sizes (no counterpart in the paper, whose
 * models are dense: a feedforward block of several experts has one down projection each).
 *
 * Rows offsets[e] .. offsets[e + 1] of the tokens are expert e's, whose weights are w_codes[e]; an expert may have none.
 *
 *   w_codes             codes of [E, N, d]; w_scales float [E, N]; w_sums int32 [E, N]
 *   offsets             device int32 [E + 1], not decreasing, in 0 .. T.  The host does not look at it, so the call can be
 *                       captured and replayed with other offsets.  Entries outside 0 .. T are taken into it, and an entry
 *                       below an earlier one counts as that one: wrong numbers, never a fault.
 *   T                   rows of a_codes and out.  Rows before offsets[0] and from offsets[E] on are neither computed nor written.
 *   E                   1 .. PERQ_MAX_EXPERTS, E * N <= 2^30
 * Everything else as for perq_matmul_i8.
 */
int perq_grouped_matmul_i8(const void *a_codes, const float *a_scales, int32_t a_fmt, const void *w_codes, const float *w_scales,
                           int32_t w_fmt, const int32_t *w_sums, const int32_t *offsets, int64_t T, int32_t E, int32_t N,
                           int32_t d, void *out, int32_t out_type, void *workspace, size_t workspace_bytes, void *stream);
int perq_grouped_matmul_i8_workspace_bytes(int64_t T, int32_t E, int32_t N, int32_t d, int32_t a_fmt, int32_t w_fmt,
                                           size_t *bytes);

/*
 * The 8-bit cache of keys and values: one token's keys and values are what the path's quantiser makes of rows of D channels, but with
 * one step for a page's tokens of a head, so that attention reads a byte for a channel and next to nothing for its steps.
 *
 *   k_codes, v_codes    device int8 [n_pages, heads, page, D]: pages of a pool
 *   k_steps, v_steps    device float [n_pages, heads]: value = step * code
 *   page                tokens of a page: 16, 32, 64 or 128;  D: 64 or 128;  heads <= PERQ_MAX_HEADS, n_pages * heads * page < 2^31
 *   pages               device int32 [S, width]: position j of sequence i lies in page pages[i, j / page], at place j % page
 *   offsets             device int32 [S + 1], not decreasing, in 0 .. T: rows offsets[i] .. offsets[i + 1] of a call are sequence i's, n_i of them
 *   lengths             device int32 [S]: tokens of sequence i, its rows of the call included.  They are its last ones: row r of it has the
 *                       position lengths[i] - n_i + r.  The same array serves the call that writes a step's tokens and the one that attends.
 *   b                   block of the keys' rotation (queries' too): 1 (none), or a power of two from 16 to D.  It cancels in the product of a
 *                       query with a key; values are kept as they come (a rotation of theirs can be merged into the weights around them).
 *   T, S, width         rows of the call (T <= 2^30; T == 0 or S == 0 is a no-op), S <= PERQ_MAX_SEQUENCES, width * page <= 2^30
 *
 * The host looks at none of the device arrays, so calls can be captured and replayed with other sequences.  Offsets and lengths outside their range
 * (0 .. T; 0 .. width * page) are taken into it, pages outside 0 .. n_pages - 1 are not written and, read, are zeros (perq_cache_read_i8) or any page
 * (perq_attention_i8): wrong numbers, never a fault.  Rows of the call that are no sequence's are neither read nor written, and rows at positions below 0 (lengths[i] <
 * n_i) are in no page.  All device pointers 16-byte aligned.
 *
 * perq_cache_write_i8 -- rotates, quantises and writes new tokens.
 *
 * For each page and head that rows of the call fall into, with y the new keys times I (x) H_b / sqrt(b), or the new values, and a = max |y| over them:
 *
 *     step = fp32(a / 127), or, where earlier tokens of the sequence lie in the page, the larger of that and the step there
 *     new tokens: code = clip(rne(y / step), -127, 127);  earlier ones, where the step has grown: code = clip(rne(code * old step / step), -127, 127)
 *
 * decided in exact arithmetic (a step of 0 gives codes 0).  What is in a page behind a sequence's last token stays.  A page whose first token is written starts anew,
 * whatever its step was.  Values in the cache depend on how its tokens were split over calls, and on nothing else: results are bit-equal from run to run.
 * A page and head that an infinity or a NaN is written to has codes 0 and a step that is not finite, and so has what attends to it, until its first token is written again.
 *
 *   k, v                device, bf16 or f16 (in_type, a perq_out_t) [T, heads, D], tokens k_stride and v_stride elements apart (multiples of 8, at least heads * D)
 *   No two sequences of a call may have rows in the same page (pages that are only read may be shared).
 * Errors: NULL, SHAPE, BLOCK, FMT, ALIGN, CUDA.
 */
int perq_cache_write_i8(const void *k, const void *v, int32_t in_type, int64_t k_stride, int64_t v_stride, const int32_t *offsets, const int32_t *lengths,
                        const int32_t *pages, int64_t T, int32_t S, int32_t heads, int32_t D, int32_t b, int32_t page, int64_t n_pages, int32_t width,
                        void *k_codes, float *k_steps, void *v_codes, float *v_steps, void *stream);

/*
 * perq_cache_read_i8 -- the tokens lengths[i] - n_i .. lengths[i] - 1 of every sequence: step * code, keys times I (x) H_b / sqrt(b) again, which is its own
 * inverse; dense [T, heads, D] of out_type each, fp32 until the last rounding.  Rows at positions below 0 are zeros.  Errors: as for writing.
 */
int perq_cache_read_i8(const void *k_codes, const float *k_steps, const void *v_codes, const float *v_steps, const int32_t *offsets, const int32_t *lengths,
                       const int32_t *pages, int64_t T, int32_t S, int32_t heads, int32_t D, int32_t b, int32_t page, int64_t n_pages, int32_t width, void *k,
                       void *v, int32_t out_type, void *stream);

/*
 * perq_attention_i8 -- attention of the call's rows over the cache, their own tokens (written before) included:
 *
 *     out[t, h] = sum_j p_j v_j,   p = softmax over the visible j of scale * <q[t, h], k_j>
 *
 * with k and v the cache's values of head h / group, q rotated as the keys are.  A row at position i sees j <= i; with a window W > 0 of those only j > i - W and
 * the first tokens j < sinks.  A row that sees nothing is 0.
 *
 *   q                   device, bf16 or f16 (in_type) [T, heads * group, D], tokens q_stride elements apart (a multiple of 8, at least heads * group * D)
 *   heads, group        heads of the cache, and heads of queries to each; heads * group <= PERQ_MAX_HEADS
 *   most                at least the rows of the longest sequence of the call (T will do; the least is the fastest).  Of a longer one, rows from
 *                       `most` on are left as they are.
 *   out                 device, dense [T, heads * group, D] of out_type
 *   workspace           device, at least perq_attention_i8_workspace_bytes(...) bytes.  What is enough for T, S and most is enough for less of each
 *                       with the same heads, group and D; 80 MB are the most (a B200, D = 128, `most` * group above 32), 2.5 MB up to there, as for decode steps.  Its contents need not be
 *                       kept; calls that may overlap need one each.
 *   scale               of the logits: finite (SHAPE)
 *
 * Rotated queries are rounded.  Where min(T, most) * group is at most 32: to whole multiples of 1/16256 of the row's largest, so by 2^-15 of that.  Else it may be so, or to fp16 with the row's largest,
 * before its rotation, between 1 and 2, so by 2^-11 of a channel (bf16 and fp16 without a rotation are kept, but for 2^-25 of the largest): which of the two a sequence has depends on its rows and on those
 * of the others in the call.  Exponentials are off by up to 2^-18 of themselves.  Probabilities times their values' step are rounded to fp16: off by 2^-11 of each, or by 2^-32 of the row's largest
 * such product where that is more (so those below 2^-32 of it may be left out of the sum over values; the sum of probabilities has them in fp32).  Sums are fp32 or wider, and added in an order that does not change from run to run.  A query that is not finite gives a row of NaN.
 * A row's largest channel times |scale| lies between 2^-110 and 2^110, or logits lose bits.  Steps are not negative.  Values' below 2^-64 count as 2^-64 (codes of such pages are 0 where
 * perq_cache_write_i8 writes a step of 0), and keys' or values' above 2^126 may count as not finite.  Values' steps of one sequence and head should lie within 2^80 of each other (0 counts as 2^-64): probabilities below 2^-45 may be left out beyond.
 * Errors: NULL, SHAPE, BLOCK, FMT, ALIGN, WORKSPACE, CUDA.
 */
int perq_attention_i8(const void *q, int32_t in_type, int64_t q_stride, const void *k_codes, const float *k_steps, const void *v_codes, const float *v_steps,
                      const int32_t *offsets, const int32_t *lengths, const int32_t *pages, int64_t T, int32_t S, int32_t heads, int32_t group, int32_t D,
                      int32_t b, int32_t page, int64_t n_pages, int32_t width, int32_t most, float scale, int32_t window, int32_t sinks, void *out,
                      int32_t out_type, void *workspace, size_t workspace_bytes, void *stream);
int perq_attention_i8_workspace_bytes(int64_t T, int32_t S, int32_t heads, int32_t group, int32_t D, int32_t most, size_t *bytes);

/*
 * perq_device_error -- reads (synchronously, cudaMemcpyFromSymbol) the library's device-side
 * error word on the current device into *flags_host.  0 = no error.  Bit 0 is set when a
 * bounded wait inside a kernel ran out (an asynchronous copy that never completed); the
 * kernel then stops early and its outputs are incomplete.  Bits 1 and 2: such a wait inside the
 * permuted and grouped kernels, for an exact maximum (1) or a free buffer (2); bit 3: in the
 * statistic; bits 4 to 6: in the products and the
 * kernel of 8-bit codes; bit 7: in the attention over the 8-bit cache.  Kernels only ever set bits; the word keeps them until perq_device_error_clear.
 *
 * perq_device_error_clear -- writes 0 to that word on the current device (synchronously,
 * cudaMemcpyToSymbol), so that a later read reports only what happened since.  Call it with no
 * kernel of the library in flight on the device, or a bit set concurrently may be lost.
 */
int perq_device_error(uint32_t *flags_host);
int perq_device_error_clear(void);

/* Text for a status code (static storage).  Library version = major*10000 + minor*100 + patch. */
const char *perq_status_string(int status);
int perq_version(void);

#ifdef __cplusplus
}
#endif
#endif /* PERQ_H */
