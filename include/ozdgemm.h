/*
 * ozdgemm.h -- C ABI of the MI355X (gfx950) emulated-DGEMM library.
 *
 * C = alpha * op(A) * op(B) + beta * C in FP64, computed with Ozaki scheme I on the INT8
 * matrix units: FP64 operands are aligned per row of op(A) / per column of op(B), cut into
 * 8-bit two's-complement digits ("slices") with the unsigned-slice encoding, the kept slice
 * pairs are multiplied with exact int32 accumulation, and the integer products are recombined
 * in FP64.  A device-resident guard (Inf/NaN scan, Exponent Span Capacity estimate, verdict)
 * chooses the slice count or routes the call to a native FP64 GEMM, with no host-device
 * synchronisation (paper: sections "Unsigned Slice Encoding", "ESC: Exponent Span Capacity
 * Estimation", "ADP: Automatic Dynamic Precision", flowchart of the GEMM decision process).
 *
 * Conventions
 *   - BLAS dgemm semantics, column-major.  op(X) = X for trans 'N'/'n', X^T for 'T'/'t'.
 *     op(A) is m x k, op(B) is k x n, C is m x n.  lda >= max(1, rows of stored A), etc.
 *   - A, B, C, workspace and result are DEVICE pointers owned by the caller.  A and B are only
 *     read.  C is overwritten; it is not read when beta == 0.  The library never allocates or
 *     frees device memory and never synchronises: a call only enqueues kernels on `stream`
 *     (a hipStream_t passed as void*) and returns.
 *   - m == 0 or n == 0: nothing is done.  k == 0 or alpha == 0: C = beta * C.
 *     Limits: m, n <= 2^22, k <= 2^21, m*n*k <= 2^52 (larger sizes are an argument error).
 *   - Return values report host-side argument errors only.  Numerical conditions (Inf/NaN in
 *     the inputs, exponent span too wide, emulation predicted slower) are never errors: they
 *     select the native FP64 path and are recorded in *result.
 *   - Negative zeros in A and B are treated as zero.
 */
#ifndef OZDGEMM_H
#define OZDGEMM_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct oz_handle* oz_handle_t;

typedef enum {
    OZ_OK = 0,
    OZ_ERR_ARG = 1,        /* bad trans, negative or too large size, leading dimension too small, bad option */
    OZ_ERR_WORKSPACE = 2,  /* workspace NULL, misaligned (256 B) or smaller than required */
    OZ_ERR_DEVICE = 3,     /* device is not gfx950, or the current device is not the handle's */
    OZ_ERR_HIP = 4         /* a HIP runtime call (launch, event) failed */
} oz_status_t;

/* How the slice count is chosen (section "Performance Evaluation": "no ADP", "ADP forced to
 * 55 bits", "ADP in dynamic mode"; section "Numerical Accuracy": with/without fallback). */
typedef enum {
    OZ_DYNAMIC = 0,         /* scan + ESC; S = ceil((target_bits + ESC + 2) / 8); native FP64 on
                               Inf/NaN, when target_bits + ESC > max_bits, or when the heuristic
                               predicts emulation to be slower */
    OZ_FORCED_GUARDED = 1,  /* scan + ESC run (their cost is paid), S forced from max_bits; only
                               Inf/NaN selects the native path */
    OZ_FIXED_GUARDED = 2,   /* S from max_bits; native path on Inf/NaN, on target_bits + ESC > max_bits, or
                               when the S slices cannot carry target_bits + ESC (S slices carry 8S - 2
                               magnitude bits: ceil((target_bits + ESC + 2) / 8) > S) */
    OZ_FIXED_UNGUARDED = 3, /* S from max_bits; no Inf/NaN test, no ESC, never falls back */
    OZ_NATIVE = 4           /* always the FP64-MFMA GEMM */
} oz_mode_t;

typedef struct {
    int32_t mode;         /* oz_mode_t */
    int32_t target_bits;  /* mantissa bits to preserve for the dominant products (default 53) */
    int32_t max_bits;     /* fixed modes: bits that set S = ceil((max_bits+1)/8) (55 -> 7 slices);
                             guarded/dynamic modes: cap on target_bits + ESC.  1..200 */
    int32_t slices;       /* > 0 overrides the slice count of the fixed/forced modes (1..26) */
    int32_t esc_block;    /* block length b of the coarsened ESC; 0 = 64.  Multiple of 16, <= 1024 */
    int32_t heuristic;    /* OZ_DYNAMIC only: 1 = apply the run-time cost model, 0 = do not.  The model is
                             first evaluated on the host for the smallest slice count any input can
                             get (ESC = 1); if that already loses against FP64 the call runs the
                             native GEMM without scanning A and B: reason 3, esc -1, infnan 0 */
    int32_t tile_slices;  /* OZ_DYNAMIC only: 1 = every 256 x 256 block of C takes the slice count of its
                             own ESC, S_T = ceil((target_bits + ESC_T + 2) / 8): the ESC is a property of
                             a dot product (section "ESC"), and a tighter estimate is what section
                             "Limitations and Future Directions" asks for.  Operands are still sliced
                             once, into max S_T planes; a block multiplies the pairs s + t <= S_T - 1.
                             Fallback decisions stay global (largest ESC); the cost model is fed the
                             mean pair count per block, rounded up.  0 = one slice count for all of C */
} oz_opts_t;

/* Decision record, written to DEVICE memory by the verdict kernel. */
typedef struct {
    int32_t fallback;       /* 0 = emulated, 1 = native FP64 */
    int32_t reason;         /* 0 none, 1 Inf/NaN in A or B, 2 bits > max_bits, 3 heuristic, 4 OZ_NATIVE */
    int32_t slices_used;    /* S of the emulated path, 0 when fallback */
    int32_t esc;            /* coarsened ESC (clamped to 4096), -1 when not computed */
    int32_t required_bits;  /* target_bits + ESC, 0 when not computed */
    int32_t infnan;         /* 1 when the scan saw an all-ones exponent field */
    int32_t slices_min;     /* smallest slice count of any 256 x 256 block of C (== slices_used unless
                               tile_slices); 0 when fallback */
    int32_t reserved_;      /* 0 */
    int64_t pair_tiles;     /* slice-pair products of 256 x 256 blocks of C that the call multiplies:
                               sum over blocks of S_T (S_T + 1) / 2; 0 when fallback */
} oz_result_t;

/* Cost model of the run-time heuristic (section "Heuristic run time Selection"); integer
 * arithmetic so that host, device and any checker agree bit for bit:
 *   t_emu = fixed_ns + (2mnk / int8_ops_per_ns) * S(S+1)/2
 *           + ((16+S)(mk+kn) + (2S+22)mn) / bytes_per_ns,     t_f64 = 2mnk / fp64_flops_per_ns,
 * emulation is "slower" when t_emu > t_f64.  With tile_slices the factor S(S+1)/2 is replaced by the
 * mean pair count per 256 x 256 block of C, rounded up; S in the streaming term is the largest S_T. */
typedef struct {
    int64_t int8_ops_per_ns;
    int64_t fp64_flops_per_ns;
    int64_t bytes_per_ns;
    int64_t fixed_ns;
} oz_heuristic_t;

/* Section "GPU-Resident Integration": the whole decision process lives on the device, so the
 * host-side state is small.  Creates a handle bound to HIP device `device` (must be gfx950): the
 * device's compute-unit count, the cost-model constants of the run-time heuristic, the event
 * pool of the stage timer, the side streams (default priority) and events of the batched call, and
 * the device address of the static workspace of oz_dgemm_static on that device.  Allocates host
 * memory, streams and events, no device memory; *handle is NULL on failure.
 * Errors: OZ_ERR_ARG (handle NULL), OZ_ERR_DEVICE (no such device / not gfx950), OZ_ERR_HIP (the
 * static workspace's address could not be resolved). */
oz_status_t oz_create(oz_handle_t* handle, int device);

/* Releases what oz_create made (host memory, streams, events).  Work already enqueued with the handle is
 * not waited for: it only references caller-owned device memory.  OZ_ERR_ARG on NULL. */
oz_status_t oz_destroy(oz_handle_t handle);

/* Fills *opts with the defaults: OZ_DYNAMIC, target 53, max 200, slices 0, esc_block 0, heuristic 1,
 * tile_slices 1. */
void oz_default_opts(oz_opts_t* opts);

/* Replaces the heuristic's constants (defaults are calibrated for MI355X). */
oz_status_t oz_set_heuristic(oz_handle_t handle, const oz_heuristic_t* model);

/* Sections "Unsigned Slice Encoding" and "ADP" fix what a call stores between its steps: the
 * row/column exponents, the per-block Max/Min exponent tables of the coarsened ESC, the S slice
 * planes of each operand and the S anti-diagonal sums per k-block.  Returns the bytes of device
 * workspace oz_dgemm needs for this problem and these options, sized for the largest slice count
 * the options allow (fixed modes: the S of max_bits/slices; OZ_DYNAMIC: the S of max_bits, or the
 * largest S the cost model still calls faster when heuristic = 1).  Host-only, no device access.
 * Returns 0 on invalid arguments. */
size_t oz_dgemm_workspace_bytes(oz_handle_t handle, char transa, char transb,
                                int64_t m, int64_t n, int64_t k, const oz_opts_t* opts);

/* The emulated DGEMM with guardrails: the flowchart of the GEMM decision process, steps in the
 * order of sections "Pre-processing and Safety Checks" (Inf/NaN scan), "Exponent Span
 * Estimation" (block Max/Min tables, coarsened ESC), "Heuristic run time Selection" (verdict),
 * "Unsigned Slice Encoding" (slicing), "FP64 Emulation on Low-Precision Units" (slice-pair INT8
 * GEMMs, FP64 recomposition), with the native FP64 GEMM as the other branch.  All kernels are
 * enqueued on `stream`; the ones after the verdict read the device-resident record.
 *   A, B, C: device, column-major, leading dimensions in elements (see Conventions above).
 *   workspace: device, 256-byte aligned, >= oz_dgemm_workspace_bytes(...); contents are scratch
 *     on entry and hold the intermediates afterwards (oz_dgemm_layout).  Calls sharing a
 *     workspace must be ordered on one stream.
 *   result: device oz_result_t written by the verdict kernel, may be NULL.
 * Errors (nothing is enqueued): OZ_ERR_ARG, OZ_ERR_WORKSPACE, OZ_ERR_DEVICE; OZ_ERR_HIP if a
 * launch failed. */
oz_status_t oz_dgemm(oz_handle_t handle, void* stream, char transa, char transb,
                     int64_t m, int64_t n, int64_t k, double alpha,
                     const double* A, int64_t lda, const double* B, int64_t ldb,
                     double beta, double* C, int64_t ldc,
                     const oz_opts_t* opts, void* workspace, size_t workspace_bytes,
                     oz_result_t* result);

/* oz_dgemm for callers that cannot allocate device memory or pass a workspace: code under HIP
 * graph capture, tight serving loops, harnesses that forbid hipMalloc.  The workspace is a
 * static device array inside the library, OZ_STATIC_SCRATCH_BYTES per GPU (each GPU the library
 * runs on holds its own copy until the process ends; its address is resolved once per handle in
 * oz_create).  The call allocates nothing and frees nothing: it only enqueues the same kernels as
 * oz_dgemm on `stream`.  All other arguments, conventions and the record are those of oz_dgemm.
 *   - A problem whose oz_dgemm_workspace_bytes(...) exceeds OZ_STATIC_SCRATCH_BYTES is refused
 *     with OZ_ERR_WORKSPACE before anything is enqueued (256 MiB holds e.g. 2048^3 with 7 slices,
 *     or 1024^3 in OZ_DYNAMIC with max_bits = 200).
 *   - The array keeps the previous call's contents; every stage rewrites what it reads, nothing
 *     is assumed to start at zero.
 *   - All calls on one GPU, from any handle or thread, share the one array: calls that overlap in
 *     time on a GPU race.  Order them on one stream (or with events). */
#define OZ_STATIC_SCRATCH_BYTES (256u << 20)
oz_status_t oz_dgemm_static(oz_handle_t handle, void* stream, char transa, char transb,
                            int64_t m, int64_t n, int64_t k, double alpha,
                            const double* A, int64_t lda, const double* B, int64_t ldb,
                            double beta, double* C, int64_t ldc,
                            const oz_opts_t* opts, oz_result_t* result);

/* batch_count independent problems of one shape: problem b uses A + b*stride_a, B + b*stride_b,
 * C + b*stride_c (strides in elements; 0 repeats an operand; the C blocks must not overlap) and
 * writes its own record to results[b] (device array of batch_count records, may be NULL).  Every
 * problem goes through the whole decision process on its own, so slice counts and fallbacks may
 * differ inside a batch (the paper's application runs show a distribution of slice counts over
 * the GEMMs of one factorisation: section "Application-Level Integration").
 * Concurrency follows the workspace: with room for q >= 2 times oz_dgemm_workspace_bytes(...)
 * (each rounded up to 256 bytes) the problems run q at a time, q <= OZ_BATCH_LANES: problems that leave much of
 * the GPU idle share their launches on `stream` (native products of a whole batch where nothing is decided on the
 * device, unless q at a time with k split are faster), larger ones run on streams the handle owns, forked from and joined to `stream` with events (so the call
 * still only enqueues, and everything it enqueued is ordered before later work on `stream`); with room for one they
 * run one after the other on `stream`.  Stage timing (oz_profile_*) records serial batches only.
 * Two batched calls on one handle must not overlap in time (they share the handle's streams).
 * batch_count == 0 is a no-op; errors are those of oz_dgemm, checked before anything is enqueued. */
#define OZ_BATCH_LANES 4
oz_status_t oz_dgemm_strided_batched(oz_handle_t handle, void* stream, char transa, char transb,
                                     int64_t m, int64_t n, int64_t k, double alpha,
                                     const double* A, int64_t lda, int64_t stride_a,
                                     const double* B, int64_t ldb, int64_t stride_b,
                                     double beta, double* C, int64_t ldc, int64_t stride_c,
                                     int64_t batch_count, const oz_opts_t* opts,
                                     void* workspace, size_t workspace_bytes, oz_result_t* results);

/* Complex product by the 4M method (section "Conclusion": the emulated DGEMM and its guardrails
 * extend to ZGEMM via 4M): C = alpha * op(A) * op(B) + beta * C with complex matrices stored
 * interleaved (re, im), column-major, leading dimensions in complex elements; op is 'N', 'T' or
 * 'C' (conjugate transpose).  A and B are split into real and imaginary parts, the four real
 * products  Pr = Ar Br - Ai Bi,  Pi = Ar Bi + Ai Br  run through the emulated DGEMM on `stream` (each with its
 * own scan, ESC and verdict; the second of each pair is added to the first), together where one alone would leave
 * much of the GPU idle, else one after the other, and C = alpha (Pr + i Pi) + beta C is formed with every real product and sum
 * rounded separately.  alpha, beta: host pointers to (re, im).  C is not read when beta == 0.
 * results: device array of four records (Ar Br, Ai Bi, Ar Bi, Ai Br) or NULL.  workspace as for
 * oz_dgemm: oz_zgemm_workspace_bytes(...) has room for what the chosen way needs (planar copies of A and B, the planar
 * products, the real calls' workspaces); with less, down to one planar product and one real call's workspace
 * (oz_dgemm_workspace_bytes), they run one after the other.  Stage timing records those only.  k == 0 gives C = beta C.  Errors as oz_dgemm. */
size_t oz_zgemm_workspace_bytes(oz_handle_t handle, char transa, char transb,
                                int64_t m, int64_t n, int64_t k, const oz_opts_t* opts);
oz_status_t oz_zgemm(oz_handle_t handle, void* stream, char transa, char transb,
                     int64_t m, int64_t n, int64_t k, const double* alpha,
                     const void* A, int64_t lda, const void* B, int64_t ldb,
                     const double* beta, void* C, int64_t ldc,
                     const oz_opts_t* opts, void* workspace, size_t workspace_bytes,
                     oz_result_t* results);

/* Layout of the intermediate buffers inside the workspace after an oz_dgemm call, for
 * inspection by tests (all offsets in bytes from `workspace`):
 *   eA   int32[mp]              row exponents of op(A); -12288 marks an all-zero row
 *   eB   int32[np]              column exponents of op(B)
 *   As   int8 [S_cap][kp/16][mp][16]   slice s of op(A): element (i,l) at
 *                               ((s*(kp/16) + l/16)*mp + i)*16 + l%16; padding is zero
 *   Bs   int8 [S_cap][kp/16][np][16]   slice t of op(B): element (l,j) likewise with j for i
 *   T    int32[nkb][np][mp]     leading word of the aggregated anti-diagonal sums of k-block kb: with
 *                               P_d = sum_{s+t=d} As_s Bs_t^T the exact integer Z = sum_d P_d 256^(S-1-d)
 *                               is T * 256^(S-1) + sum_{d>=1} L_d 256^(S-1-d); element (i,j) at
 *                               (kb*np + j)*mp + i
 *   L    int8 [nkb][S_cap-1][np/4][mp][4]   balanced digit L_d in [-128,127], d >= 1, of element (i,j) at
 *                               (((kb*(S_cap-1) + d-1)*(np/4) + j/4)*mp + i)*4 + j%4
 *   tileS int32[np/256][mp/256]  slice count of block (ti, tj) of C at tj*(mp/256) + ti (written only
 *                               with tile_slices in OZ_DYNAMIC mode); the same number of int32 follows it: the
 *                               order in which the slice GEMM dealt the blocks to its workgroups
 * mp, np = m, n rounded up to 256; kp = k rounded up to 128; kblk = k-block length for S_cap. */
typedef struct {
    int64_t mp, np, kp, s_cap, nkb, kblk;
    size_t off_eA, off_eB, off_As, off_Bs, off_T, off_L, off_record, off_tileS;
    size_t total_bytes;
} oz_layout_t;

oz_status_t oz_dgemm_layout(oz_handle_t handle, char transa, char transb,
                            int64_t m, int64_t n, int64_t k, const oz_opts_t* opts,
                            oz_layout_t* layout);

/* Stage timing with HIP events on the call's own stream.  oz_profile_enable(h, n) makes the
 * next n oz_dgemm calls record an event after every stage; oz_profile_read(h, call, ms)
 * (after the stream has been synchronised by the caller) writes OZ_NUM_STAGES durations in
 * milliseconds.  Stages: 0 scan (Inf/NaN + exponent min/max), 1 ESC, 2 verdict (about 0: the ESC
 * kernel's last workgroup gives it), 3 slicing, 4 slice-pair INT8 GEMMs, 5 FP64 recomposition, 6 native FP64 GEMM. */
#define OZ_NUM_STAGES 7
oz_status_t oz_profile_enable(oz_handle_t handle, int32_t max_calls);
oz_status_t oz_profile_read(oz_handle_t handle, int32_t call, float* stage_ms);

/* The fallback branch of the decision process on its own (sections "Pre-processing and Safety
 * Checks" and "Heuristic run time Selection": the native FP64 GEMM that Inf/NaN inputs, too wide
 * an exponent span or an inefficient slice count route to), and the baseline the paper's speed-ups
 * are quoted against.  Same conventions as oz_dgemm; no workspace, no record; only enqueues.
 * Errors: OZ_ERR_ARG, OZ_ERR_DEVICE, OZ_ERR_HIP. */
oz_status_t oz_native_dgemm(oz_handle_t handle, void* stream, char transa, char transb,
                            int64_t m, int64_t n, int64_t k, double alpha,
                            const double* A, int64_t lda, const double* B, int64_t ldb,
                            double beta, double* C, int64_t ldc);

/* ---- 8-bit block-scaled operands, their products, and rows sorted by group ------------------------
 *
 * The same matrix units, used once per product: operands in 8-bit floating point with a scale for each block of
 * 128 along the contraction, as language models are trained and served with.  Conventions of this part:
 *   - Matrices are row-major with the contraction contiguous: a product is C = A * B^T with A m x k, B n x k, C m x n.
 *   - Device pointers owned by the caller, work enqueued on `stream`, nothing allocated, nothing synchronised, as above.
 *   - Sizes of zero are no errors.  Limits, beyond which calls return OZ_ERR_ARG: rows and columns <= 2^24; of 8-bit matrices bytes per row
 *     < 2^23 and scales per row < 2^17; leading dimensions of the others <= 2^32 elements; groups <= 1024, choices < 2^30.  Some
 *     calls name more.
 *   - offsets: device int32[groups + 1], ascending from 0 to at most the number of rows: rows offsets[g] .. offsets[g+1] - 1
 *     are group g's.  Groups may be empty. */
typedef enum { OZ_F32 = 0, OZ_BF16 = 1, OZ_F16 = 2, OZ_E4M3 = 3, OZ_E5M2 = 4, OZ_E8M0 = 5 } oz_type_t;

/* A matrix of 8-bit floats with its scales: element (r, c) stands for data * scale of block (r / block_rows, c / 128).
 * OZ_E8M0 scales are bytes b for 2^(b-127), 255 for NaN: the matrix unit applies them itself.  OZ_F32 scales may have any value; a block's
 * sum is multiplied by B's, then by A's, in 32 bits. */
typedef struct {
    void* data;           /* (r, c) at r*ld + c; 16-byte aligned */
    void* scale;          /* (i, b) at i*scale_ld + b; 4-byte aligned */
    int64_t ld;           /* bytes per row, multiple of 16, >= columns */
    int64_t scale_ld;     /* elements per row of blocks, >= ceil(columns / 128); OZ_E8M0: multiple of 4 */
    int64_t stride;       /* bytes from one matrix of a batch, or one group's, to the next; multiple of 16 */
    int64_t scale_stride; /* the same for the scales, in elements; OZ_E8M0: multiple of 4 */
    int32_t type;         /* OZ_E4M3 or OZ_E5M2 */
    int32_t scale_type;   /* OZ_E8M0 or OZ_F32 */
    int32_t block_rows;   /* 1 or 128 */
    int32_t reserved_;    /* 0 */
} oz_scaled_t;

/* X (rows x cols, row-major, OZ_F32 / OZ_BF16 / OZ_F16, batch matrices stride_x elements apart) in 8-bit floats: `by_rows` as it is,
 * `by_columns` transposed (cols x rows), either may be NULL; both have the same block_rows.  The scale of a block is 2^e with the
 * least e >= -126 that keeps its largest |x| within the type's range (448, 57344), 1 for a block of zeros; values are x 2^-e
 * rounded to nearest even, the only rounding there is.  A block that holds an infinity or a NaN becomes NaN, with scale NaN.
 * Columns up to the next multiple of 16 are written, as zeros.
 *   order (may be NULL; batch 1, block_rows 1): row r is row order[r] / order_div of X (x_rows of them), zeros where order[r] is negative
 *     or the row is not there.
 *   offsets (may be NULL; batch 1, block_rows 1): the columns of by_columns are cut into groups: group g's rows of X become columns from
 *     128 * sum_{g' < g} ceil(count_g' / 128) on, zeros up to the next multiple of 128; rows behind the last group are left out.
 *     by_columns needs ld >= 128 * w and scale_ld >= w with w = floor((rows + 127 * min(groups, rows)) / 128).
 * Limits: cols < 2^22, rows * ceil(cols / 128) <= 2^27, batch <= 65535. */
oz_status_t oz_quantize(oz_handle_t handle, void* stream, int64_t rows, int64_t cols, const void* X, int64_t ldx, int32_t x_type,
                        int64_t batch, int64_t stride_x, const int32_t* order, int64_t order_div, int64_t x_rows,
                        const int32_t* offsets, int64_t groups, const oz_scaled_t* by_rows, const oz_scaled_t* by_columns);

/* C = A B^T (+ C if accumulate), C row-major m x n in OZ_F32, OZ_BF16 or OZ_F16, ldc in elements.  A in OZ_E4M3 or OZ_E5M2, B in OZ_E4M3;
 * both with scales of one type.  k == 0: C = 0, or C as it is.
 * Sums are held in 32 bits and rounded once to C's type.  For OZ_F32 that is all; for OZ_BF16 and OZ_F16 the 8-bit matrix instruction first adds
 * products by eights (k = 8i .. 8i + 7) and cuts each off, towards zero, at 2^-13 of the largest of the eight.  On data of one order of
 * magnitude that is 1.4e-5 of the result, far below its rounding; where large products cancel within an eight, ask for OZ_F32.
 * Limits: ceil(m / 64) * ceil(n / 64) < 2^24, with up to 64 rows (per group on average) ceil(m / 16) * ceil(n / 16) < 2^22; with groups of
 * rows, groups + 1 more in the first factor.
 * workspace: 256-byte aligned, oz_scaled_gemm_workspace_bytes(...) bytes (0: may be NULL): parts of a k that is cut where the output alone
 * leaves the GPU idle, added in their order. */
size_t oz_scaled_gemm_workspace_bytes(oz_handle_t handle, int64_t m, int64_t n, int64_t k);
oz_status_t oz_scaled_gemm(oz_handle_t handle, void* stream, int64_t m, int64_t n, int64_t k, const oz_scaled_t* A, const oz_scaled_t* B,
                           void* C, int64_t ldc, int32_t c_type, int32_t accumulate, void* workspace, size_t workspace_bytes);

/* Rows in groups: rows offsets[g] .. of C = the same rows of A times B_g^T, B_g at B->data + g * B->stride.  Rows of C behind the last
 * group are set to zero.  m: rows of A and of C. */
oz_status_t oz_scaled_gemm_grouped(oz_handle_t handle, void* stream, int64_t groups, const int32_t* offsets, int64_t m, int64_t n, int64_t k,
                                   const oz_scaled_t* A, const oz_scaled_t* B, void* C, int64_t ldc, int32_t c_type);

/* Contraction in groups: C_g = A_g B_g^T (+ C_g), A_g and B_g the columns that oz_quantize gives group g in by_columns with the
 * same offsets; C_g at C + g * stride_c elements.  An empty group's C_g is zero, or as it is.  k: columns of A and B, a multiple of 128. */
oz_status_t oz_scaled_gemm_grouped_k(oz_handle_t handle, void* stream, int64_t groups, const int32_t* offsets, int64_t m, int64_t n, int64_t k,
                                     const oz_scaled_t* A, const oz_scaled_t* B, void* C, int64_t ldc, int64_t stride_c, int32_t c_type,
                                     int32_t accumulate);

/* tokens * topk choices, chosen[t * topk + j] the expert that token t takes as its j-th (int32 or int64: id_bytes 4 or 8; a value outside
 * 0 .. experts-1, such as -1, is a choice that is dropped), sorted by expert, each expert's in their own order:
 *   offsets int32[experts + 1]   slots offsets[e] .. offsets[e+1] - 1 are expert e's
 *   order   int32[tokens * topk] slot -> choice, -1 behind the last
 *   place   int32[tokens * topk] choice -> slot, -1 if dropped
 * workspace: 256-byte aligned, oz_sort_tokens_workspace_bytes(...) bytes (0: may be NULL). */
size_t oz_sort_tokens_workspace_bytes(oz_handle_t handle, int64_t tokens, int64_t topk, int64_t experts);
oz_status_t oz_sort_tokens(oz_handle_t handle, void* stream, int64_t tokens, int64_t topk, int64_t experts, const void* chosen,
                           int32_t id_bytes, int32_t* offsets, int32_t* order, int32_t* place, void* workspace, size_t workspace_bytes);

/* Y[place[t * topk + j]] = X[t] for every choice that has a place: rows of `cols` values sorted by expert; rows s of Y (tokens * topk of
 * them) with order[s] negative become zero.  type of X and Y: OZ_F32, OZ_BF16 or OZ_F16.  topk <= 64.
 * Limits: tokens * ceil(cols * bytes / 4096) <= 2^26 - 4. */
oz_status_t oz_gather_rows(oz_handle_t handle, void* stream, int64_t tokens, int64_t topk, int64_t cols, int32_t type, const void* X,
                           int64_t ldx, const int32_t* order, const int32_t* place, void* Y, int64_t ldy);

/* Y[t] = sum_j weights[t * topk + j] * X[place[t * topk + j]], j ascending, in 32 bits, rounded once; choices without a row in X (slots rows)
 * are left out.  weights NULL: all 1 (the gradient of oz_gather_rows).  topk <= 64.  Limits: tokens * ceil(cols / 512) <= 2^26 - 4. */
oz_status_t oz_combine_rows(oz_handle_t handle, void* stream, int64_t tokens, int64_t topk, int64_t cols, int32_t type, const void* X,
                            int64_t ldx, int64_t slots, const int32_t* place, const float* weights, void* Y, int64_t ldy);

/* Gradients of oz_combine_rows: dX[place] = weight * dY[t], rows of slots that no choice has (order[s] negative) zero; dweights = <dY[t],
 * X[place]>, 0 for dropped choices.  dweights NULL, or weights NULL: not computed, or 1.  Limits: slots <= 2^26 - 4. */
oz_status_t oz_combine_rows_grad(oz_handle_t handle, void* stream, int64_t tokens, int64_t topk, int64_t cols, int32_t type, const void* dY,
                                 int64_t lddy, const void* X, int64_t ldx, int64_t slots, const int32_t* order, const int32_t* place,
                                 const float* weights, void* dX, int64_t lddx, float* dweights);

/* ---- the router's choice, weights in 4 bits, orthogonal updates --------------------------------------
 * Conventions as in the part above. */

/* A router's choice: each token's topk experts by falling score (ties: the lowest expert), and their weights.  With p = softmax(scores of the token):
 *   ids     int32[tokens * topk]   the token's j-th expert; -1 where it has none
 *   weights float[tokens * topk]   p of that expert (normalize 0), or its share of the chosen ones' sum (1); 0 where there is none
 * and, unless all four are NULL, of the whole batch:
 *   counts  int32[experts]         how often each was chosen
 *   counted int32[1]               tokens that have an expert
 *   shares  float[experts]         P_e, the mean of p_e over those tokens
 *   loss    float[1]               experts * sum_e f_e P_e, f_e = counts_e / sum of counts: 1 where choices are even, up to experts where they are not
 * scores: tokens x experts, rows ld elements apart, OZ_F32, OZ_BF16 or OZ_F16; a score of -infinity is an expert that is not to be had.
 * live: uint8[tokens] or NULL; tokens with 0, and those that no expert is to be had for, are padding: they have no ids, weights of 0, and do not
 * count; what stands in the scores of a token that is not live may be anything.  A NaN is above every other score, and makes its token's
 * probabilities NaN, as +infinity does (and with them P and the loss).
 * experts <= 1024, topk <= 64 and <= experts.  Sums are in a fixed order: two runs give the same bits.
 * workspace (only with counts): 256-byte aligned, oz_choose_experts_workspace_bytes(...) bytes. */
size_t oz_choose_experts_workspace_bytes(oz_handle_t handle, int64_t tokens, int64_t experts);
oz_status_t oz_choose_experts(oz_handle_t handle, void* stream, int64_t tokens, int64_t experts, int64_t topk, const void* scores, int64_t ld,
                              int32_t type, const uint8_t* live, int32_t normalize, int32_t* ids, float* weights, int32_t* counts, int32_t* counted,
                              float* shares, float* loss, void* workspace, size_t workspace_bytes);

/* The scores' gradient from that of the weights (dweights, tokens x topk, or NULL: none) and, unless counts and counted are NULL, from factor * *dloss
 * (dloss a device pointer; NULL: 1) for the loss.  ids, weights, counts, counted: as oz_choose_experts left them with the same scores, live and
 * normalize; counts may have been added up over several GPUs since: f_e then is theirs.  dscores: type and columns of scores; zero for padding
 * and for experts that are not to be had (NaN for all of a token where its probabilities are).  Which experts are chosen has no gradient, so f_e is a
 * constant here. */
oz_status_t oz_choose_experts_grad(oz_handle_t handle, void* stream, int64_t tokens, int64_t experts, int64_t topk, const void* scores, int64_t ld,
                                   int32_t type, const uint8_t* live, int32_t normalize, const int32_t* ids, const float* weights,
                                   const float* dweights, const int32_t* counts, const int32_t* counted, const float* dloss, float factor,
                                   void* dscores, int64_t ldd);

/* A matrix in 4 bits: element (r, c) stands for scale * (code - zero), with the scale and the zero point of row r and group c / group. */
typedef struct {
    void* data;           /* codes 0 .. 15 of columns 2i (low half) and 2i + 1 of row r at r*ld + i; 16-byte aligned */
    void* scale;          /* (g, r) at g*scale_ld + r */
    void* zero;           /* as scale, of its type, any value; NULL: 8 */
    int64_t ld;           /* bytes per row, multiple of 16, >= 16 * ceil(columns / 32) */
    int64_t scale_ld;     /* elements per group, >= rows */
    int64_t stride;       /* bytes from one matrix of a batch, or one group's, to the next; multiple of 16 */
    int64_t scale_stride; /* the same for scale and zero, in elements */
    int32_t scale_type;   /* OZ_F32, OZ_BF16 or OZ_F16 */
    int32_t group;        /* columns that share a scale: 32, 64 or 128 */
    int32_t reserved_;    /* 0 */
} oz_packed_t;

/* X (rows x cols, batch matrices stride_x elements apart) in 4 bits.  Without W->zero: scale = max|x| / 7 of the group, rounded to its type,
 * code = min(max(rint(x / scale), -8), 7) + 8.  With: scale = (max(x, 0) - min(x, 0)) / 15, zero = rint(-min(x, 0) / scale),
 * code = min(max(rint(x / scale) + zero, 0), 15).  Quotients are float32, rint is to nearest even.  A group of zeros has scale 0; one with an
 * infinity or a NaN, or whose scale is beyond its type's range, has scale NaN.  Codes up to the next multiple of 32 columns are written, as 0.
 * Limits: rows * ceil(cols / 512) <= 2^26 - 4, batch <= 65535. */
oz_status_t oz_pack4(oz_handle_t handle, void* stream, int64_t rows, int64_t cols, const void* X, int64_t ldx, int32_t x_type, int64_t batch,
                     int64_t stride_x, const oz_packed_t* W);

/* The other way: X = the values that W stands for, rounded once to x_type. */
oz_status_t oz_unpack4(oz_handle_t handle, void* stream, int64_t rows, int64_t cols, void* X, int64_t ldx, int32_t x_type, int64_t batch,
                       int64_t stride_x, const oz_packed_t* W);

/* Y = X W^T, X m x k in OZ_F32, OZ_BF16 or OZ_F16, W n x k in 4 bits, Y m x n.  Made for few rows (a token, a few in flight): W is read once for every 16 or 32
 * rows of X.  offsets NULL, groups 0: one matrix.  Otherwise rows offsets[g] .. of Y = the same rows of X times W_g^T, and rows of Y behind the last
 * group are set to zero.  Sums are held in 32 bits, each group's of code - 8 before it is scaled (X and Y in OZ_BF16: of 128 + code, less 136 times the
 * sum of x, some 10^-5 of the largest terms, which the rounding of Y hides); the one rounding to fewer bits is the result's.  A result that is not finite
 * this way is computed once more as the sum of x * (scale * (code - zero)) in 64 bits: an infinity in X keeps its product's sign, NaN comes of a NaN, of
 * infinities of both signs or of one times a value of zero alone, and no sum leaves the range on the way.
 * k == 0: Y = 0.  Limits: (ceil(m / 16) + groups + 1) * ceil(n / 16) < 2^22. */
oz_status_t oz_packed_gemm(oz_handle_t handle, void* stream, int64_t groups, const int32_t* offsets, int64_t m, int64_t n, int64_t k, const void* X,
                           int64_t ldx, int32_t x_type, const oz_packed_t* W, void* Y, int64_t ldy, int32_t y_type);

/* Y = X made orthogonal, batch matrices of rows x cols, by `steps` Newton-Schulz steps Z <- a Z + (b A + c A^2) Z, A = Z Z^T, from Z = X / (|X| + eps) with
 * |X| the square root of the sum of squares (Z is taken transposed where rows > cols).  With a = 3.4445, b = -4.775, c = 2.0315 five steps bring singular
 * values above 0.003 |X| into 0.68 .. 1.13 or so: the direction of a weight update that keeps X's singular vectors.
 * Z is held as 4096 Z, elements of A off its diagonal as 16384 A and those of b A + c A^2 as 4096 of them, in 16-bit floating point (up to 65504): the
 * coefficients have to keep singular values below 2 and the last below 16, or elements become infinite (these do: 1.3 and 4).  X in OZ_BF16: operands
 * of the products have 11 bits, among them the off-diagonals of A, which have no more in b A either, and Z itself has 22: an error of about 0.002 of the
 * result with its rounding.  OZ_F32, OZ_F16 (and values of OZ_BF16 given as OZ_F32): operands of 22 bits, Z of 32, about 10^-6, in some three times as long.
 * Diagonals and sums are in 32 bits, |X| in 64.  A matrix of zeros stays one if eps > 0; an infinity or a NaN makes NaN of its matrix.
 * Y may be X, with the same strides.  Sums are in a fixed order.  Limits: rows, cols <= 32768, batch <= 65535, 1 <= steps <= 64.
 * workspace: 256-byte aligned, oz_orthogonalize_workspace_bytes(...) bytes (up to 24 per element of a few matrices, of which more are done in turn). */
size_t oz_orthogonalize_workspace_bytes(oz_handle_t handle, int64_t batch, int64_t rows, int64_t cols, int32_t type);
oz_status_t oz_orthogonalize(oz_handle_t handle, void* stream, int64_t batch, int64_t rows, int64_t cols, int32_t type, const void* X, int64_t ldx,
                             int64_t stride_x, void* Y, int64_t ldy, int64_t stride_y, int32_t steps, float a, float b, float c, float eps,
                             void* workspace, size_t workspace_bytes);

const char* oz_status_string(oz_status_t status);

#ifdef __cplusplus
}
#endif
#endif /* OZDGEMM_H */
