/*
 * convfwd.h -- C ABI of the MI355X (gfx950) forward-convolution library.
 *
 * The operation is the convolution layer the paper defines in Section 2
 * ("Background": output = conv(input, filters); each output value is the dot
 * product of one filter with a window of the input slid with a spatial stride)
 * with the activation fused into the output write as in Section 3
 * ("Graph-level Optimizations"), plus a per-output-channel bias:
 *
 *   out[n,k,oy,ox] = act( bias[k] + sum_{c,r,s} in[n,c,oy*stride-pad+r,ox*stride-pad+s]
 *                                                * filt[k,c,r,s] )
 *
 * zero padding, no filter flip, OH = floor((H+2*pad-R)/stride)+1 (OW likewise;
 * floor reproduces the in->out sizes of Appendix A), groups = 1, dilation = 1.
 *
 * Conventions shared by every entry point
 *   - Tensors are dense, C order: in [N][C][H][W], filt [K][C][R][S],
 *     out [N][K][OH][OW], element type `dtype` (fp32, or fp16/bf16 storage with
 *     fp32 accumulation and one round-to-nearest-even on the store).
 *   - `bias` is [K] fp32 or NULL (= no bias); it is added in fp32 before `act`.
 *   - All tensor pointers are DEVICE pointers owned by the caller.  The library
 *     reads in/filt/bias, writes out (which must not alias them), keeps no pointer
 *     after returning, never allocates or frees device memory and never
 *     synchronises, except conv_autotune() which times kernels and therefore
 *     synchronises `stream`.
 *   - `stream` is a hipStream_t passed as void* (NULL = the default stream).
 *     Kernels are enqueued on it and the call returns immediately.
 *   - Return value: 0 on success, a negative conv_status otherwise.  Descriptor
 *     and pointer validation happens before the first HIP call, so the error
 *     paths work on a host without a GPU.
 *   - Thread safety: the variant cache is guarded by a mutex; kernels hold no state.
 */
#ifndef CONVFWD_H
#define CONVFWD_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { CONV_F32 = 0, CONV_F16 = 1, CONV_BF16 = 2 } conv_dtype; /* storage type of in/filt/out */

enum {
    CONV_FLAG_RELU = 1u,      /* act = max(x,0); without it act is the identity */
    /* Optional channel-innermost formats (the paper's explicit data-format conversions, Section 3 "Graph-level
     * Optimizations"): the same operation on tensors stored as in [N][H][W][C], filt [K][R][S][C], out [N][OH][OW][K].
     * Kernels exist for fp16/bf16 with IN_NHWC and FILT_KRSC both set, C % 8 == 0 (and K % 8 == 0 with OUT_NHWC) and
     * an input and a filter tensor below 1 GiB each,
     * and, with OUT_NHWC alone (planar input and filters, channel-innermost output), for the fp16/bf16 first layers the
     * strided window kernels serve (3 channels, 11x11 stride 4 or 7x7 stride 2; K % 4 == 0): the conversion then costs
     * nothing.  Any other combination of these bits gives CONV_ENOVARIANT.  conv_convert_layout() converts tensors. */
    CONV_FLAG_IN_NHWC = 2u,
    CONV_FLAG_OUT_NHWC = 4u,
    CONV_FLAG_FILT_KRSC = 8u,
    /* Filters handed over in the Winograd F(2x2,3x3) domain, as written by conv_transform_filters() for the same
     * descriptor (without this bit): at inference the weights are constants, so the filter transform is one of the
     * conversions the paper does ahead of time (Section 3, "Graph-level Optimizations").  Only the Winograd variants
     * serve such a descriptor (fp32, 3x3, stride 1, pad <= 1, C % 8 == 0; otherwise CONV_ENOVARIANT), and they then
     * need no workspace.  Not combinable with the channel-innermost bits. */
    CONV_FLAG_FILT_WINOGRAD = 16u,
    /* A 3x3 stride-2 max-pool (no padding, the pooling layers of the paper's networks) fused behind the activation:
     * out holds [N][K][PH][PW] (or [N][PH][PW][K] with OUT_NHWC), PH = (OH-3)/2 + 1, PW = (OW-3)/2 + 1, each element
     * the maximum of act(conv + bias) over its window -- the convolution's own output is never written (the paper's
     * rule for fusing an operation into the write of the convolution result, Section 3 "Graph-level Optimizations").
     * Needs OH, OW >= 3.  Served by the window kernels whose workgroup holds a whole output image (stride 1; fp16/bf16:
     * OH*OW <= 192 for 3x3 and 5x5 windows, <= 768 for 5x5 channel-innermost; fp32: 3x3 windows, OH*OW <= 208, planar
     * tensors), and for fp16/bf16 first layers (C = 3; 11x11 stride 4 or 7x7 stride 2; any image size; planar input,
     * pooled output in either format, K % 8 == 0 for the channel-innermost one) by a kernel whose workgroups compute tiles
     * of pooled outputs; other descriptors give CONV_ENOVARIANT and the caller
     * runs maxpool_fwd() behind the convolution.  The result is bit-identical to that sequence run with the same
     * variant (for the first-layer kernel: with a kernel that sums in the same order), NaN sums included (with the activation they become 0 before the pool, as in the sequence; without it a
     * NaN in the window is the result); only the sign of a zero result can differ when the activation is the identity.
     * Not combinable with CONV_FLAG_FILT_WINOGRAD. */
    CONV_FLAG_MAXPOOL_3X3S2 = 32u,
    /* Filters handed over in the order the 16-bit matrix instructions consume them, as written by
     * conv_transform_filters() for the same descriptor with this bit set: the other ahead-of-time filter conversion
     * (Section 3, "Graph-level Optimizations"; the filter operand then goes from memory straight into the multiplying
     * wave's registers).  fp16/bf16, stride 1, C % 16 == 0, windows the packed-filter kernels are built for (3x3,
     * 5x5) with pad < window, input channel-innermost (CONV_FLAG_IN_NHWC), output in either format; otherwise
     * CONV_ENOVARIANT.  Not combinable with CONV_FLAG_FILT_KRSC, CONV_FLAG_FILT_WINOGRAD or CONV_FLAG_MAXPOOL_3X3S2. */
    CONV_FLAG_FILT_PACKED = 64u
};

typedef enum {
    CONV_OK = 0,
    CONV_EINVAL = -1,     /* NULL descriptor/pointer; N,C,H,W,K,R,S < 1; stride < 1; pad < 0; window larger than
                             the padded input; a tensor with 2^31 or more elements or 4 GiB or more; a tensor pointer
                             that is not 16-byte aligned; unknown flag bits */
    CONV_EDTYPE = -2,     /* dtype is not one of conv_dtype */
    CONV_EWORKSPACE = -3, /* workspace NULL/too small for what was asked (forced split variant, autotune) */
    CONV_EHIP = -4,       /* a HIP call failed; conv_strerror(CONV_EHIP) carries the HIP message */
    CONV_ENOVARIANT = -5, /* variant index out of range, or no kernel accepts this descriptor */
    CONV_EIO = -6         /* autotune-cache file could not be read or written, or is malformed */
} conv_status;

typedef struct {
    int32_t N, C, H, W;   /* input batch, channels, height, width            */
    int32_t K, R, S;      /* output channels, window height, window width    */
    int32_t stride, pad;  /* same stride and symmetric zero pad on both axes */
    int32_t dtype;        /* conv_dtype                                      */
    uint32_t flags;       /* CONV_FLAG_*                                     */
} conv_desc;

/* Extent of the tensor the call writes: (OH, OW) by the formula above, or (PH, PW) with CONV_FLAG_MAXPOOL_3X3S2.
 * Pure host code.  CONV_EINVAL if the descriptor is not valid. */
int conv_out_shape(const conv_desc* desc, int32_t* OH, int32_t* OW);

/* FLOPs of the layer in the convention of Appendix A: 2*N*K*OH*OW*C*R*S.  0 if the descriptor is invalid. */
double conv_flops(const conv_desc* desc);

/*
 * Bytes of device workspace with which every variant valid for `desc` can run
 * (split-reduction variants keep fp32 partial sums there, the Winograd variants
 * the transformed filters, 16-bit window variants a copy of the input and the
 * filters in the order their kernel reads).  conv_fwd() needs none.  Returns 0 for an invalid
 * descriptor.
 */
size_t conv_workspace_bytes(const conv_desc* desc);

/*
 * Enqueue the fused convolution on `stream` using the variant selected for
 * `desc` (forced > autotuned/cached > heuristic), restricted to variants that
 * need no workspace.  Asynchronous; see the conventions above.
 */
int conv_fwd(const conv_desc* desc, const void* in, const void* filt, const float* bias, void* out,
             void* stream);

/*
 * As conv_fwd, but may also pick a variant that needs scratch memory (paper,
 * Section 3 "Variant Selection and Autotuning": several variants per
 * operation): a split-reduction variant, whose partial sums go to `workspace`
 * (device memory, 256-byte aligned, contents undefined afterwards) and are then
 * reduced in a fixed order, or, for fp32 3x3 stride-1 layers, a Winograd
 * F(2x2,3x3) variant (the algorithm the paper names as its main open topic,
 * Section 4 "Experimental Results"), which first writes the transformed filters
 * there.  One of those (winos_*), and one for fp32 first layers (swins_*), multiply on the 16-bit matrix units, each fp32 operand split into three parts that
 * together hold all of it; results that are infinite, NaN or beyond about 2^79 they sum once more the direct way, so that a
 * call with such data can take several times as long (up to about 20 times where every result is beyond that size).
 * Results are bit-reproducible either way.  If `workspace_bytes` is too small for the selected variant
 * the best variant that fits is used instead; CONV_EWORKSPACE only if a forced
 * variant does not fit.
 */
int conv_fwd_ws(const conv_desc* desc, const void* in, const void* filt, const float* bias, void* out,
                void* workspace, size_t workspace_bytes, void* stream);

/*
 * For callers that cannot allocate device memory or be handed a workspace (code under HIP graph capture, serving
 * loops, harnesses that forbid hipMalloc): conv_fwd_ws with the scratch memory taken from an array the library holds
 * itself, CONV_STATIC_SCRATCH_BYTES per GPU, resident from library load to process end.  The call allocates and frees
 * nothing.  The variant is selected as conv_fwd_ws selects it with unlimited workspace (forced > autotuned/cached >
 * cost model); when that variant needs more than CONV_STATIC_SCRATCH_BYTES the call is rejected with CONV_EWORKSPACE
 * (conv_strerror names the variant and both sizes) and nothing is enqueued -- use conv_fwd or conv_fwd_ws then.  (The
 * kernels that keep a copy of the input or split filters in scratch, bwin_*, pwin_*_prep, winos_* and swins_*, give way to the pick
 * that fits.)
 * Results are bit-identical to conv_fwd_ws running the same variant.  Nothing in the array has to start at zero
 * (every partial sum and every transformed filter is written before it is read), and its contents are undefined
 * afterwards.  Every call on one GPU shares that GPU's array: calls that overlap in time on one GPU (different
 * streams, or threads) race on it and must be serialised by the caller; calls on one stream are ordered.
 */
#define CONV_STATIC_SCRATCH_BYTES (32u << 20)
int conv_fwd_static(const conv_desc* desc, const void* in, const void* filt, const float* bias, void* out,
                    void* stream);

/*
 * Brute-force autotuning (paper, Section 3 "Variant Selection and Autotuning":
 * exhaustive search over a fixed set of configurations, by measured run time):
 * runs every variant valid for `desc` that fits `workspace_bytes` on the given
 * buffers, times it with device events on `stream`, and records the fastest in
 * the in-process cache used by conv_fwd/conv_fwd_ws (two entries: best overall,
 * best without workspace).  `out` is overwritten.  Synchronises `stream`.
 * `workspace` may be NULL (then only variants without workspace are tried).
 * Every candidate's output is cross-checked before it may win (the paper's tuning flow verifies outputs numerically,
 * Section 4 "Experimental Setup"): the output of a reference candidate (the first unsplit direct variant that fits)
 * is kept, and a candidate whose output differs from it by more than 2e-5 (fp32), 5e-3 (fp16) or 1e-2 (bf16: one
 * rounding step of an 8-bit significand) in the max-normalised sense of conv_compare_outputs() is neither timed nor
 * selected; conv_variant_time_us() then reports -2 for it.  For this check -- and only here -- the call allocates and
 * frees a temporary device buffer of the size of `out`.  Test hook: when the environment variable
 * CONVFWD_AUTOTUNE_CORRUPT names a variant, the first bytes of that candidate's output are overwritten from the host
 * before the check, so that the rejection path can be exercised without a wrong kernel.
 */
int conv_autotune(const conv_desc* desc, const void* in, const void* filt, const float* bias, void* out,
                  void* workspace, size_t workspace_bytes, void* stream);

/* Number of variants valid for `desc` (negative conv_status on error).  Pure host code. */
int conv_variant_count(const conv_desc* desc);

/*
 * Name of variant `idx` in [0, conv_variant_count) -- or, with idx = -1, of the
 * variant conv_fwd_ws would pick now given unlimited workspace; idx = -2, of the
 * one conv_fwd would pick -- copied NUL-terminated into buf[0..n).  Names read
 * like the paper's tuning strings, e.g. "igemm_f32_M128N128K16_w2x2" or "..._sk4".
 */
int conv_variant_name(const conv_desc* desc, int idx, char* buf, size_t n);

/* Workspace bytes variant `idx` of `desc` needs (0 for unsplit direct variants); negative conv_status on error. */
long long conv_variant_workspace(const conv_desc* desc, int idx);

/* Force variant `idx` for this exact descriptor in later conv_fwd/conv_fwd_ws calls (tests run every variant this
 * way); idx = -1 removes the override. */
int conv_force_variant(const conv_desc* desc, int idx);

/* Last measured time (microseconds per launch) of variant `idx` from conv_autotune in this process; -1 if it was not
 * tried (no autotune yet, or it did not fit the workspace), -2 if the cross-check rejected its output. */
double conv_variant_time_us(const conv_desc* desc, int idx);

/*
 * Device-side time of the currently selected variant (the one conv_fwd_ws would run with this workspace): `launches`
 * back-to-back launches on `stream`, bracketed by two events; *us_per_launch = elapsed / launches.  This is the paper's
 * measurement rule (Section 4, "Experimental Results": device timers around the calls, host overheads excluded), used
 * by the benchmark for layers whose run time is of the order of a host-side launch.  Synchronises the stream.
 * Pointers, alignment and errors as conv_fwd_ws; launches >= 1 and us_per_launch != NULL, else CONV_EINVAL.
 */
int conv_time_us(const conv_desc* desc, const void* in, const void* filt, const float* bias, void* out, void* workspace,
                 size_t workspace_bytes, void* stream, int launches, double* us_per_launch);

/*
 * The error metric of the parity tests and of the autotuner's cross-check on two device tensors of `elements`
 * elements of `dtype`: max_i |got_i - ref_i| / max(max_j |ref_j|, 1e-30); infinity if `got` holds a NaN, or an
 * infinity where `ref` is finite (the paper compares outputs with relative tolerances, Section 4 "Experimental
 * Setup").  Synchronises `stream`; allocates 256 bytes of device scratch for the duration of the call.
 */
int conv_compare_outputs(int32_t dtype, const void* got, const void* ref, size_t elements, void* stream,
                         double* max_norm_err);

/*
 * Autotune cache persistence: a text file, one line per descriptor
 * ("N C H W K R S stride pad dtype flags | best-name | best-no-workspace-name").
 * A saved file starts with an identity line ("#! convfwd-cache device=<arch/name/CUs> registry=<hash of the
 * library's variant list>"): measurements are only valid for the device model and the set of kernels they were
 * taken with, so load refuses (CONV_EIO) a file whose identity line names another registry, or another device
 * when both sides know theirs ("none" = written or read on a host without a GPU); a file without an identity line
 * (hand-written) is accepted.  Load merges into the in-process cache and ignores lines naming unknown
 * variants; a missing, unreadable or malformed file gives CONV_EIO and leaves
 * the cache as it was.  conv_cache_clear drops every cached and forced choice.
 */
int conv_cache_load(const char* path);
int conv_cache_save(const char* path);
void conv_cache_clear(void);

/*
 * Cooperative tile load plan (paper, Section 3 "Metaprogramming for NN
 * Convolutions": `threads` threads loading `words` words need ceil(words/threads)
 * loads each, and only the last one needs a bounds guard, and only when `words`
 * is not a multiple of `threads`).  The tile loaders of the kernels are unrolled
 * from the same rule at compile time; this host entry point exposes it for
 * checking.  CONV_EINVAL if either count is < 1.
 */
int conv_coop_load_plan(int threads, int words, int* loads_per_thread, int* last_load_guarded);

/*
 * Per-channel spatial max-pool, window win x win, stride `stride`, no padding,
 * OH = floor((H-win)/stride)+1 (the glue between layers of a convolution stack;
 * paper, Section 2).  in [N][C][H][W] -> out [N][C][OH][OW], element type
 * `dtype`, device pointers, asynchronous on `stream`.  On every path (either layout, and the pool fused into a
 * convolution without activation) the window is scanned row by row, the first of equal values is kept (so the sign
 * of a zero is that of the first zero) and a NaN anywhere in the window is the result.
 */
int maxpool_fwd(int32_t N, int32_t C, int32_t H, int32_t W, int32_t win, int32_t stride, int32_t dtype,
                const void* in, void* out, void* stream);

/* The same pooling on either tensor layout: in_nhwc / out_nhwc != 0 means channel-innermost ([N][H][W][C]) for that
 * side, 0 means [N][C][H][W].  With different layouts on the two sides it is also the format conversion between two
 * layers.  Errors as maxpool_fwd. */
int maxpool_fwd_layout(int32_t N, int32_t C, int32_t H, int32_t W, int32_t win, int32_t stride, int32_t dtype,
                       int32_t in_nhwc, int32_t out_nhwc, const void* in, void* out, void* stream);

/*
 * A straight-line schedule of operations issued with ONE call (paper, Section 3 "Code Generation, Scheduling, and
 * Execution": every ND-Array is allocated up front and the operations are issued in a topological order): each
 * element is a conv_fwd_ws, maxpool_fwd_layout or conv_convert_layout call with its arguments, and conv_run_ops
 * enqueues them in array order on `stream` exactly as those calls would -- same validation, same variant selection,
 * same kernels -- without returning to the caller in between, so that a chain of microsecond kernels is not paced by
 * the caller's own per-call cost.  Stops at the first element that fails and returns its status (*failed_index, if not
 * NULL, receives its index; earlier elements stay enqueued); CONV_EINVAL for a NULL array, count < 0 or an unknown kind.
 *   kind CONV_OP_CONV:    desc, in, filt, bias, out, workspace, workspace_bytes as conv_fwd_ws
 *   kind CONV_OP_MAXPOOL: in, out; p[0..8] = N, C, H, W, win, stride, dtype, in_nhwc, out_nhwc as maxpool_fwd_layout
 *   kind CONV_OP_CONVERT: in, out; p[0..3] = A, B, S, dtype as conv_convert_layout
 */
typedef enum { CONV_OP_CONV = 0, CONV_OP_MAXPOOL = 1, CONV_OP_CONVERT = 2 } conv_op_kind;
typedef struct {
    int32_t kind;           /* conv_op_kind */
    conv_desc desc;         /* CONV_OP_CONV only */
    const void* in;
    const void* filt;       /* CONV_OP_CONV only */
    const float* bias;      /* CONV_OP_CONV only; may be NULL */
    void* out;
    void* workspace;        /* CONV_OP_CONV only; may be NULL */
    size_t workspace_bytes;
    int32_t p[9];           /* CONV_OP_MAXPOOL / CONV_OP_CONVERT parameters */
} conv_op;
int conv_run_ops(const conv_op* ops, int32_t count, void* stream, int32_t* failed_index);

/*
 * Explicit data-format conversion (paper, Section 3, "Graph-level Optimizations"): out[a][s][b] = in[a][b][s] for
 * dense tensors of `dtype` elements.  (A,B,S) = (N,C,H*W) turns [N][C][H][W] into [N][H][W][C]; (N,H*W,C) turns it
 * back; (K,C,R*S) turns filters [K][C][R][S] into [K][R][S][C].  Device pointers, out must not alias in; enqueued on
 * `stream`.  CONV_EINVAL for NULL/aliased pointers, extents < 1, A > 65535 or 2^31 or more elements.
 */
int conv_convert_layout(int32_t A, int32_t B, int32_t S, int32_t dtype, const void* in, void* out, void* stream);

/*
 * Ahead-of-time filter conversions as explicit, separately timed calls (paper, Section 3 "Graph-level
 * Optimizations": data-format conversions are operations of their own).  `filt` is the KCRS filter tensor (device,
 * 16-byte aligned); the result goes to `out` (device, 256-byte aligned, conv_transformed_filter_bytes(desc) bytes,
 * layout private to the library), which is then passed as `filt` of the layer's descriptor with the format's bit set.
 * The target format is the one whose bit `desc` carries:
 *   CONV_FLAG_FILT_WINOGRAD  U = G g G^T of the Winograd F(2x2,3x3) variants (fp32);
 *   CONV_FLAG_FILT_PACKED    the matrix-instruction operand order of the packed-filter kernels (fp16/bf16);
 * with neither bit it is the Winograd domain for fp32 and the packed order for fp16/bf16.  Other bits of `desc`
 * describe the layer as usual.  conv_transformed_filter_bytes returns 0, conv_transform_filters CONV_ENOVARIANT, when
 * no kernel of that format serves the layer; CONV_EINVAL for NULL or misaligned pointers.  Enqueued on `stream`.
 */
size_t conv_transformed_filter_bytes(const conv_desc* desc);
int conv_transform_filters(const conv_desc* desc, const void* filt, void* out, void* stream);

/*
 * Measured ceilings of the device, for reporting next to the published peaks (the paper's own practice of timing on
 * the device with device-level timers, Section 4 "Experimental Setup").  All synchronise `stream`.
 *  - conv_probe_mfma_peak: TFLOP/s of a register-only MFMA issue loop for `dtype` with 16x16 or 32x32 blocks
 *    (`block` = 16 or 32); `scratch` is any 4-byte device location (never written in practice).
 *  - conv_probe_stream_bandwidth: GB/s (bytes read + bytes written) of a plain copy of `bytes` from `src` to `dst`,
 *    both device pointers, 16-byte aligned, not overlapping.
 *  - conv_probe_mfma_mix: the same issue loop with exactly `waves_per_simd` (1..4) waves on every SIMD and
 *    `valu_per_mfma` (0, 2, 4 or 8) vector-ALU instructions between consecutive MFMAs: how much of the issue rate a
 *    given occupancy reaches, and whether vector-ALU work hides behind matrix work.  With `distinct_operands` != 0
 *    (16-bit types, valu_per_mfma = 0) every MFMA of a round reads operand registers of its own, as a real kernel
 *    does, instead of one shared pair.  Writes TFLOP/s and the nanoseconds one SIMD spends per MFMA.
 */
int conv_probe_mfma_peak(int32_t dtype, int32_t block, void* scratch, void* stream, double* tflops);
int conv_probe_mfma_mix(int32_t dtype, int32_t block, int32_t waves_per_simd, int32_t valu_per_mfma,
                        int32_t distinct_operands, void* scratch, void* stream, double* tflops, double* ns_per_mfma);
int conv_probe_stream_bandwidth(const void* src, void* dst, size_t bytes, void* stream, double* gbytes_per_s);

/*
 * Operators at the end of a network: from the trunk's features (or the pixels of a channel-innermost tensor) to what the
 * network answers with, and the gradients a head is trained with.  All of them work on `rows` rows (images, tokens,
 * pixels); element (t, j) of a tensor is at t * ld + j, with the row stride `ld` in elements.
 *
 * Conventions, next to those at the top of this file:
 *   - `dtype` is the storage type of the float tensors; per-row and per-column vectors (gamma, beta, bias, scales,
 *     statistics, log probabilities and their gradients) are fp32, dense.  Sums and statistics are fp32 or int32.
 *   - Float tensors have to be aligned to their element only and row strides are free (>= the row's length), so a slice
 *     of a larger tensor can be passed; 8-bit tensors start on 16 bytes and have row strides divisible by 16.
 *   - rows = 0 is valid and enqueues nothing (layernorm_bwd still writes its zero sums).  rows < 2^31; a tensor spans at most 2^62
 *     bytes (row stride times rows), CONV_EINVAL beyond.
 *   - Outputs alias no input, except where said.
 *   - Results do not depend on scheduling (no floating-point atomics): the same call gives the same bits.
 */

/*
 * Layer norm over the columns: y[t][j] = (x[t][j] - mean_t) * rstd_t * gamma[j] + beta[j], mean_t the row's mean,
 * rstd_t = 1 / sqrt(var_t + eps) with the variance taken around that mean (in a second pass over the held row).
 * gamma NULL = ones, beta NULL = zeros; mean and rstd (fp32 [rows], what layernorm_bwd needs) may be NULL.
 * ldx is the row stride of x and dx, ldy that of y and dy.  CONV_EINVAL for rows < 0, cols < 1 or >= 2^30, a stride
 * below cols, eps < 0, infinite or NaN, NULL or misaligned pointers.
 */
typedef struct {
    int64_t rows;
    int64_t ldx, ldy; /* row strides in elements */
    int32_t cols;
    int32_t dtype;    /* conv_dtype of x, y, dx, dy */
    float eps;
} norm_desc;
int layernorm_fwd(const norm_desc* desc, const void* x, const float* gamma, const float* beta, void* y, float* mean,
                  float* rstd, void* stream);

/*
 * Its gradients: with xh = (x - mean) * rstd and g = dy * gamma,
 *   dx = rstd * (g - avg_j(g) - xh * avg_j(g * xh)),   dgamma[j] = sum_t dy * xh,   dbeta[j] = sum_t dy.
 * Any of dx, dgamma and dbeta may be NULL, not all; gamma NULL = ones.  dx may be dy itself where ldx == ldy.  The sums over the
 * rows are formed in fp32, per workgroup first and then over the workgroups' partial sums in `workspace`
 * (layernorm_bwd_workspace_bytes(desc) bytes, 16-byte aligned; CONV_EWORKSPACE if it is smaller; not needed, and may be NULL,
 * when neither dgamma nor dbeta is asked for).
 */
size_t layernorm_bwd_workspace_bytes(const norm_desc* desc);
int layernorm_bwd(const norm_desc* desc, const void* x, const void* dy, const float* gamma, const float* mean,
                  const float* rstd, void* dx, float* dgamma, float* dbeta, void* workspace, size_t workspace_bytes,
                  void* stream);

/*
 * Rows to 8 bits with a scale each: scale[t] = max(max_j |x[t][j]| * fl(1/127), 2^-126), q[t][j] = x[t][j] * fl(1/scale[t])
 * rounded to the nearest whole number (ties to even), so that q * scale stands for x and |q| <= 127.  A row that holds a
 * NaN or an infinity gets the scale NaN and zeros: what is computed from it is NaN.  q has the row stride ldq
 * (divisible by 16, >= cols); the bytes from cols up to the next multiple of 16 are written as zeros, those beyond are left.
 * 1 <= cols < 2^30.  Weights [N][K] are quantised by the same call, a scale for each output channel.
 */
typedef struct {
    int64_t rows;
    int64_t ldx, ldq; /* row strides in elements */
    int32_t cols;
    int32_t dtype;    /* conv_dtype of x */
} quant_desc;
int quantize_rows(const quant_desc* desc, const void* x, int8_t* q, float* scale, void* stream);

/* layernorm_fwd whose result, rounded to `dtype`, is quantised as by quantize_rows without being written: q has the row
 * stride desc->ldy (divisible by 16).  Codes and scales are bit for bit those of the two calls. */
int layernorm_quant_fwd(const norm_desc* desc, const void* x, const float* gamma, const float* beta, int8_t* q,
                        float* scale, void* stream);

/*
 * Matrix product in 8-bit integers: out[t][n] = act(float(sum_k a[t][k] * w[n][k]) * (a_scale[t] * w_scale[n]) + bias[n])
 * for a [rows][K] and w [N][K]; the sum is exact (int32; K < 2^17).  a_scale is [rows], w_scale [N], bias [N] or NULL.
 * CONV_FLAG_RELU: act(x) = max(x, 0), a NaN stays NaN.  Rows of a and w are read in pieces of 16 bytes: the bytes from K
 * up to the next multiple of 16 have to be readable; their values do not matter.  `workspace`
 * (int_linear_workspace_bytes(desc) bytes, which may be 0; 16-byte aligned) holds partial sums of few-row products; NULL or a smaller one gives
 * CONV_EWORKSPACE when bytes are needed.  1 <= N < 2^24, K >= 1; lda, ldw >= K and divisible by 16; ldo >= N.
 */
typedef struct {
    int64_t rows;
    int64_t lda, ldw, ldo; /* row strides in elements */
    int32_t N, K;
    int32_t dtype;         /* conv_dtype of out */
    uint32_t flags;        /* CONV_FLAG_RELU or 0 */
} int_linear_desc;
size_t int_linear_workspace_bytes(const int_linear_desc* desc);
int int_linear_fwd(const int_linear_desc* desc, const int8_t* a, const float* a_scale, const int8_t* w,
                   const float* w_scale, const float* bias, void* out, void* workspace, size_t workspace_bytes,
                   void* stream);
/* Name of the form that int_linear_fwd takes for this descriptor and these operands' addresses (which count modulo 128; NULL counts
 * as a multiple), NUL-terminated in buf[0..n), e.g. "rows32_split3" or "tile64x128_lines"; empty for no rows.  Pure host code. */
int int_linear_form(const int_linear_desc* desc, const int8_t* a, const int8_t* w, char* buf, size_t n);

/*
 * Log probabilities of given tokens under softmax over the columns (classes, a vocabulary), with lse_t = log sum_j exp(x_tj):
 *   logp[t] = x[t][target[t]] - lse_t,   entropy[t] = -sum_j p_tj log p_tj (nats; p log p = 0 where p = 0),
 *   top_id[t][0..top), top_logp[t][0..top): the `top` likeliest columns, by value and, where values are equal, by the lower
 *   index (+0 and -0 are equal; a NaN counts as the largest), and their log probabilities.
 * Log probabilities are taken from the distance to the row's largest logit, so they do not lose bits where lse is large.
 * target is int64 [rows]: a negative one stands for "no token" (logp 0, no gradient), one >= cols gives NaN.
 * Any output may be NULL, not all; target may be NULL if logp is; top_id and top_logp are dense [rows][top] and go together;
 * 0 <= top <= min(64, cols), ignored if both are NULL.  Masked columns are -inf; a row of -inf only has lse, logp and top_logp -inf, entropy 0 and the columns
 * 0, 1, ... as top_id.  A row with a NaN or +inf has NaN for all values.
 * `workspace` (logprob_workspace_bytes(desc), may be 0; 16-byte aligned) joins rows that are split over several workgroups.
 * CONV_EINVAL for rows < 0, cols < 1 or >= 2^31 - 2^20, strides below cols, top outside its range, NULL or misaligned pointers.
 */
typedef struct {
    int64_t rows;
    int64_t ldx, ldg; /* row strides of the logits and of their gradient, in elements */
    int32_t cols;
    int32_t dtype;    /* conv_dtype of the logits and of their gradient */
    int32_t top;
} logprob_desc;
size_t logprob_workspace_bytes(const logprob_desc* desc);
int logprob_fwd(const logprob_desc* desc, const void* logits, const int64_t* target, float* logp, float* lse,
                float* entropy, int64_t* top_id, float* top_logp, void* workspace, size_t workspace_bytes, void* stream);

/*
 * The gradient in the logits of sum_t g_logp[t] * logp[t] + g_entropy[t] * entropy[t]:
 *   dlogits[t][j] = g_logp[t] * ([j == target[t]] - p_tj) - g_entropy[t] * p_tj * (log p_tj + entropy[t]),
 * p from lse and entropy of the forward pass (so it is off by |lse| units of 2^-24, as lse is).  g_logp or g_entropy may be NULL (zeros), not both; target goes with g_logp, entropy with
 * g_entropy.  Rows whose lse is -inf get zeros.  dlogits may be the logits themselves where ldx == ldg.  desc->top is not read.
 */
int logprob_bwd(const logprob_desc* desc, const void* logits, const int64_t* target, const float* lse,
                const float* entropy, const float* g_logp, const float* g_entropy, void* dlogits, void* stream);

/*
 * Linear layers in float types: out[t][n] = act(z[t][n]) + residual[t][n],  z[t][n] = sum_k x[t][k] * w[n][k] + bias[n],
 * for x [rows][K] and w [N][K].  act is nothing, CONV_FLAG_RELU (max(z, 0), a NaN stays NaN), LINEAR_FLAG_GELU (z Phi(z), Phi the
 * normal distribution) or LINEAR_FLAG_SILU (z / (1 + exp(-z))).  bias (fp32 [N]) and residual may be NULL; pre, where it is not NULL, receives z
 * (what linear_bwd needs where there is an activation).  ldr is the row stride of the residual, ldo that of out, pre and dout; the
 * residual may be out itself where ldr == ldo.  All sums are fp32; out and pre are each rounded once.
 * fp32 products of more than a few rows are formed from three bf16 parts of each operand, six products of them: what is left out is below 2^-25 of each
 * term.  There an operand's infinity, NaN or magnitude above 0x1.FEp127 makes NaN of the outputs it reaches, and parts below 2^-126 count as zero.
 * `workspace` (linear_workspace_bytes(desc), may be 0; 16-byte aligned) holds partial sums of shared reductions; NULL or a smaller one gives
 * CONV_EWORKSPACE when bytes are needed.  Operands whose rows start on 16 bytes are loaded faster.
 * CONV_EINVAL for rows < 0, N or K outside [1, 2^24), strides below the row's length, unknown flags or more than one activation, NULL or misaligned
 * pointers, outputs that are inputs.
 */
#define LINEAR_FLAG_GELU 0x100u
#define LINEAR_FLAG_SILU 0x200u
typedef struct {
    int64_t rows;
    int64_t ldx, ldw, ldr, ldo; /* row strides in elements */
    int32_t N, K;
    int32_t dtype;              /* conv_dtype of all but bias and dbias */
    uint32_t flags;
} linear_desc;
size_t linear_workspace_bytes(const linear_desc* desc);
int linear_fwd(const linear_desc* desc, const void* x, const void* w, const float* bias, const void* residual, void* out,
               void* pre, void* workspace, size_t workspace_bytes, void* stream);

/*
 * Its gradients: with dz = dout * act'(pre) (the slope of ReLU at 0 is 0),
 *   dx[t][k] = sum_n dz[t][n] * w[n][k],   dw[n][k] = sum_t dz[t][n] * x[t][k],   dbias[n] = sum_t dz[t][n];
 * the residual's gradient is dout.  Any of dx (row stride ldx), dw (ldw) and dbias (fp32 [N]) may be NULL, not all; x is read for dw, w for dx, pre
 * where there is an activation: each may be NULL otherwise.  dz is kept in as many bits as the results need: in 16-bit types as two values of the type (16 bits in bf16,
 * 22 in fp16, none lost to fp16's range) behind GELU and SiLU, where no infinity in x or w passes to a result but as NaN.  rows = 0 gives zero dw and dbias.  `workspace`: linear_bwd_workspace_bytes(desc), as above.
 */
size_t linear_bwd_workspace_bytes(const linear_desc* desc);
int linear_bwd(const linear_desc* desc, const void* x, const void* w, const void* pre, const void* dout, void* dx, void* dw,
               float* dbias, void* workspace, size_t workspace_bytes, void* stream);

/* Name of the form that a product takes for this descriptor and these operands' addresses (which count modulo 16), NUL-terminated in
 * buf[0..n), e.g. "rows16", "rows32x64" (rows x outputs), "tile256x256", "split_tile64x64_split4" or "parts_tile128x128" (of dz in two parts); `which`: 0 the product of linear_fwd, 1 and 2 those of linear_bwd for dx and
 * dw.  Empty for no rows.  Pure host code. */
int linear_form(const linear_desc* desc, const void* x, const void* w, int which, char* buf, size_t n);

/*
 * What stands between two blocks of rows, in one call: the norm behind a block, its gate and scale, the residual sum, and the norm before the
 * next block.
 *   u = norm(h) * gamma_h + beta_h  with RESIDUAL_NORM_POST, else h
 *   sum[t][j] = r[t][j] + scale[j] * gate[t / gate_rows][j] * u[t][j],   r_out = sum rounded,   y = norm(sum) * gamma + beta
 * norm is layer norm's (x - mean) * rstd, or with RESIDUAL_NORM_RMS x * rstd with rstd = 1 / sqrt(mean of x^2 + eps); y is formed from the sum before it
 * is rounded.  gate has a row of `cols` for every gate_rows rows (1: each row its own; the last may stand for fewer; 0: no gate,
 * and the pointer is NULL); with RESIDUAL_NORM_SIGMOID it multiplies as 1 / (1 + exp(-gate)).  gamma_h, beta_h (NULL without RESIDUAL_NORM_POST), scale,
 * gamma, beta: fp32 [cols], NULL = ones, zeros, ones, ones, zeros.  y may be NULL (no norm behind).  stats: fp32 [rows][4], 16-byte aligned,
 * receives mean and rstd of h and mean and rstd of the sum (0 and 1 where there is no norm, 0 for means under RMS); may be NULL.
 * r_out may be r.  Row strides: ldr of r, r_out, dr, dr_out; ldh of h, dh; ldg of gate, dgate; ldy of y, dy.
 * CONV_EINVAL for rows or gate_rows < 0, cols < 1 or >= 2^27, strides below cols (ldg only with a gate), eps < 0, infinite or NaN, unknown flags, a gate without gate_rows
 * or the reverse, NULL or misaligned pointers, other outputs that are inputs.
 */
#define RESIDUAL_NORM_RMS 1u
#define RESIDUAL_NORM_POST 2u
#define RESIDUAL_NORM_SIGMOID 4u
typedef struct {
    int64_t rows;
    int64_t ldr, ldh, ldg, ldy; /* row strides in elements */
    int32_t gate_rows;
    int32_t cols;
    int32_t dtype;              /* conv_dtype of r, r_out, h, gate, y and their gradients */
    float eps;
    uint32_t flags;
} residual_norm_desc;
int residual_norm_fwd(const residual_norm_desc* desc, const void* r, const void* h, const void* gate, const float* gamma_h,
                      const float* beta_h, const float* scale, const float* gamma, const float* beta, void* r_out, void* y,
                      float* stats, void* stream);

/*
 * Its gradients from dr_out and dy (either may be NULL: zeros) with r_out and stats as the forward pass left them: with xh and hh the normed rows,
 *   dr = dr_out + rstd * (dy gamma - avg(dy gamma) - xh avg(dy gamma xh)),   p = dr * gate,
 *   dh = rstd_h * (g - avg(g) - hh avg(g hh)) with g = p * scale * gamma_h  (p * scale without RESIDUAL_NORM_POST; no avg(.) of its own under RMS),
 *   dgate = sum over the rows that share it of dr * scale * u (times s (1 - s) for a sigmoid s),
 *   dgamma_h = sum_t p scale hh,  dbeta_h = sum_t p scale,  dscale = sum_t p u,  dgamma = sum_t dy xh,  dbeta = sum_t dy.
 * Any output may be NULL, not all; no output is an input.  r_out is read where dy is given, stats there and with RESIDUAL_NORM_POST.  Sums over rows are
 * fp32, in `workspace` (residual_norm_bwd_workspace_bytes(desc), 16-byte aligned; CONV_EWORKSPACE if it is smaller).  rows = 0 gives zero sums.
 * Gradients of the vectors go with what they belong to: dgamma_h and dbeta_h with RESIDUAL_NORM_POST, dgate with a gate.
 */
size_t residual_norm_bwd_workspace_bytes(const residual_norm_desc* desc);
int residual_norm_bwd(const residual_norm_desc* desc, const void* r_out, const void* h, const void* gate, const float* gamma_h,
                      const float* beta_h, const float* scale, const float* gamma, const float* stats, const void* dr_out,
                      const void* dy, void* dr, void* dh, void* dgate, float* dgamma_h, float* dbeta_h, float* dscale,
                      float* dgamma, float* dbeta, void* workspace, size_t workspace_bytes, void* stream);

/*
 * The direction of an update made orthogonal by Newton-Schulz steps, for each of `batch` matrices x [rows][cols]:
 *   X = x / (|x| + eps), |x| the root of the sum of the squares;  `steps` times  X <- a X + (b X X^T + c (X X^T)^2) X;  out = X.
 * The polynomial a s + b s^3 + c s^5 moves every singular value s of X towards one; e.g. 3.4445, -4.7750, 2.0315 and five steps.  Coefficients have to keep
 * the elements of X and of b X X^T + c (X X^T)^2 below 15 (any that keep the singular values below 1.5 with |b|, |c| <= 5 do); beyond, results may be infinite or NaN.
 * X is held in 22 bits or more and multiplied in two fp16 parts of 11 bits each with fp32 sums: results are off by some 2e-6 of their norm before the rounding to the type.  A
 * matrix with a NaN or an infinity gives NaN; one of zeros stays zero where eps > 0.
 * Matrix i starts stride_x (stride_o) elements behind matrix i - 1, its rows ldx (ldo) apart; out may be x where the strides are the same.  `workspace`:
 * orthogonalize_workspace_bytes(desc), 16-byte aligned, CONV_EWORKSPACE if it is smaller.  batch = 0 enqueues nothing.
 * CONV_EINVAL for batch < 0 or >= 2^31, rows or cols outside [1, 2^20] or both above 2^17, steps outside [1, 100], strides below a row's length, matrices that overlap in out (stride_o below
 * rows * ldo for batch > 1), coefficients that are not finite, eps < 0, infinite or NaN, NULL or misaligned pointers.
 */
typedef struct {
    int64_t batch;
    int64_t ldx, ldo;           /* row strides in elements */
    int64_t stride_x, stride_o; /* from a matrix to the next, in elements */
    int32_t rows, cols;
    int32_t dtype;              /* conv_dtype of x and out */
    int32_t steps;
    float a, b, c, eps;
} orthogonal_desc;
size_t orthogonalize_workspace_bytes(const orthogonal_desc* desc);
int orthogonalize(const orthogonal_desc* desc, const void* x, void* out, void* workspace, size_t workspace_bytes, void* stream);

/* Text for a conv_status; for CONV_EHIP it includes the message of the last failed HIP call of this thread. */
const char* conv_strerror(int status);

#ifdef __cplusplus
}
#endif
#endif /* CONVFWD_H */
