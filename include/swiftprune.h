/*
 * swiftprune.h -- C ABI of the B200 (sm_100a) SwiftPrune pruning pass.
 *
 * The library implements the per-layer pruning pass of SwiftPrune
 * (arXiv 2501.16376): calibration statistics (Algorithm 1, step 1), the
 * Hessian-free contribution metric (Eq. 8), the EWMA running-threshold
 * selection that replaces sorting (Algorithm 1; state rules in Table 2; the
 * parameter la per pruning ratio in Table 3), the N:M group selection
 * (Section 3.3) and the write-back of the pruned weights (Algorithm 1,
 * "w_i = 0" / "c_i = w_i").
 *
 * General conventions
 *   - Unless a parameter says "host", every data pointer is a DEVICE pointer to
 *     memory owned by the caller, on the device the context was created for.
 *     The library owns only the context (O(d_in) device memory).
 *   - Calls enqueue work on the caller's stream (sp_stream = cudaStream_t passed
 *     as void*; NULL = the default stream) and return without synchronising,
 *     except sp_create, sp_destroy, sp_get_stats, sp_set_stats and sp_search_la, which say so.
 *   - Arguments are validated on the host before anything is launched; a
 *     non-SP_OK status means nothing was enqueued by that call.  No call
 *     throws, traps or aborts.
 *   - A weight matrix W is [n_rows, d_in] row-major 16-bit floats with leading
 *     dimension ldw (elements, >= d_in): one row per output neuron, one column
 *     per input channel.  Rows are pruned independently (Section 2; the row loop of
 *     Algorithm 1 runs in parallel).
 *   - A mask is [n_rows, ceil(d_in/32)] uint32, row-major, no padding between
 *     rows; bit j of word k of a row is the keep flag of column 32k+j
 *     (1 = kept, 0 = pruned; bits past d_in are 0).
 *   - Pruned weights are written as +0 (bit pattern 0x0000); kept weights are
 *     copied bit for bit.
 *   - Fast paths need 16-byte aligned base pointers and leading dimensions
 *     that are multiples of 8 elements; anything else is handled by slower
 *     element-wise paths with identical results.
 *   - One context belongs to one layer input of width d_in; layers that read
 *     the same input (q/k/v; gate/up) share it.  A context must not be used
 *     from two streams at once.
 */
#ifndef SWIFTPRUNE_H_
#define SWIFTPRUNE_H_

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct sp_ctx sp_ctx; /* opaque, library-owned */
typedef void *sp_stream;      /* a cudaStream_t */

typedef enum {
    SP_OK = 0,
    SP_ERR_INVALID_ARG = 1, /* null pointer, negative size, unknown enum value */
    SP_ERR_SHAPE = 2,       /* ld < d_in, d_in % M != 0, size over a stated maximum */
    SP_ERR_DTYPE = 3,
    SP_ERR_STATE = 4,       /* selection or scoring before any calibration data */
    SP_ERR_DEGENERATE = 5,  /* S == 0 or non-finite statistics (sp_get_stats reports it) */
    SP_ERR_CUDA = 6,        /* a CUDA runtime call failed; see sp_last_cuda_error */
    SP_ERR_NOMEM = 7
} sp_status;

typedef enum { SP_F16 = 0, SP_BF16 = 1 } sp_dtype;

/* How the EWMA selection treats Algorithm 1's step "S = S - w_i^2" (Table 2, row S).
 * In binary32 the subtraction changes S only if w_i^2 reaches a quarter of the spacing of
 * floats at S, which calibration-scale statistics (S ~ tokens * d_in) never allow. */
typedef enum {
    SP_S_GATED = 0,      /* Algorithm 1 as printed, at scan speed: rows are scanned in parallel with
                            S at its initial value; a row holding a weight that could change S is
                            detected before that weight's tile is stored and finished
                            sequentially from there in the same kernel, so the result is the
                            printed algorithm for every row (the default) */
    SP_S_LITERAL_W2 = 1, /* the printed update, evaluated sequentially along every row */
    SP_S_FROZEN = 2,     /* S keeps its initial value whatever is pruned */
    SP_S_READING_X2 = 3, /* the other conceivable reading of that row of Table 2: S is a sum of
                            x^2, and a pruned weight takes its channel's x_i^2 out of it
                            ("S = S - x_i^2"); evaluated sequentially along every row.  This
                            changes S by tens of percent and is not what the paper prints:
                            offered for comparison */
    SP_S_LITERAL_SCAN = 4 /* the printed update again, but rows scanned by whole warps: every
                            256-column tile is decided by fix-point sweeps (decide with the S the
                            previous sweep's decisions imply, prefix-sum the pruned w^2, repeat
                            until nothing changes; a tile that does not settle in 8 sweeps hands
                            the row to the sequential walk and counts in SP_COUNTER_S_HAZARD).
                            Same decisions as SP_S_LITERAL_W2 up to re-association (the tolerance
                            of the scans); several times faster when rows are few and long */
} sp_s_update;

/* Parameters of Algorithm 1 (alpha, beta: Table 2; la: Table 3). */
typedef struct {
    float alpha;
    float beta;
    float la;
    int s_update; /* an sp_s_update */
} sp_ewma_params;

/* Entries of the optional device counter block passed to the selection calls. */
enum { SP_COUNTER_KEPT = 0, SP_COUNTER_S_HAZARD = 1, SP_NUM_COUNTERS = 2 };

/* ------------------------------------------------------------------ context */

/*
 * Creates the context for one layer input of d_in channels on CUDA device
 * `device` (1 <= d_in <= 2^20).  Allocates its device memory (statistics,
 * per-channel factors, partial sums) and synchronises with that device once.
 * The statistics start empty.
 */
sp_status sp_create(sp_ctx **out, int64_t d_in, int device);

/* Frees the context (synchronises with its device first).  NULL is allowed. */
sp_status sp_destroy(sp_ctx *ctx);

/* ------------------------------------------------------------------ calibration (Algorithm 1, step 1) */

/* Forgets all accumulated statistics. */
sp_status sp_calib_reset(sp_ctx *ctx, sp_stream stream);

/*
 * Adds one batch of calibration activations: for every channel q,
 *     colsq[q] += sum_t X[t, q]^2.
 * colsq[q] is the "x_q^2" of Eq. 8, i.e. the q-th diagonal entry of X X^T
 * (Section 2: H = 2 X X^T), and S = sum_q colsq[q] is Algorithm 1's step 1.
 * X is [n_tokens, d_in] row-major of `dtype` with leading dimension ldx
 * (elements).  n_tokens == 0 is a no-op.  Squares are exact in fp32; sums of
 * at most 8 squares are formed in fp32 and then accumulated in fp64.  The
 * result does not depend on run-to-run scheduling (no floating-point atomics).
 */
sp_status sp_calib_accumulate(sp_ctx *ctx, const void *X, sp_dtype dtype, int64_t n_tokens,
                              int64_t ldx, sp_stream stream);

/*
 * The same with flags.  The library's kernels are launched so that a kernel may be scheduled
 * while its predecessor on the stream drains; sp_calib_accumulate still reads X only after
 * everything queued earlier on the stream has completed (ordinary stream semantics: the
 * preceding kernel may be the one that writes X).  SP_CALIB_X_COMPLETE is the caller's promise
 * that X was complete before the operation that precedes this call on the stream began (e.g.
 * calibration data prepared long before, with library calls in between): the kernel then
 * streams X while that predecessor is still finishing and orders only its update of the
 * statistics after it.  With the flag set wrongly the statistics are silently wrong.
 */
enum { SP_CALIB_X_COMPLETE = 1 };
sp_status sp_calib_accumulate_ex(sp_ctx *ctx, const void *X, sp_dtype dtype, int64_t n_tokens,
                                 int64_t ldx, unsigned flags, sp_stream stream);

/*
 * One batch for each of several layer inputs (the inputs of one transformer block, say) in one
 * launch: the effect of sp_calib_accumulate_ex(ctxs[i], batches[i].X, dtype,
 * batches[i].n_tokens, batches[i].ldx, flags, stream) for every i - Algorithm 1's step 1 is a
 * sum per channel, and the channels of different inputs have nothing to do with each other.
 * The sums agree with those of the single calls to rounding (the tokens of a batch may be cut
 * into slabs differently, which moves the last bits of a sum) and are, like theirs,
 * reproducible bit for bit for a given sequence of calls.  For inputs so narrow or batches so
 * short that a launch of their own would be mostly ramp-up.  ctxs and batches are HOST arrays of n_items entries (1 <= n_items <=
 * SP_MAX_MULTI); the contexts must all be different (two batches of one launch cannot update
 * the same sums: SP_ERR_INVALID_ARG) and on one device; a batch with n_tokens == 0 is skipped;
 * batches that do not allow 16-byte access get launches of their own.
 */
typedef struct {
    const void *X;    /* device, [n_tokens, d_in of its context] of the call's dtype */
    int64_t n_tokens;
    int64_t ldx;      /* elements */
} sp_batch;
sp_status sp_calib_accumulate_multi(sp_ctx *const *ctxs /* host */,
                                    const sp_batch *batches /* host */, int n_items,
                                    sp_dtype dtype, unsigned flags, sp_stream stream);

/*
 * Finalisation of several contexts at once: S and the per-channel factors of Eq. 8 for every
 * listed context that has batches pending, by one launch (what sp_score(ctx, NULL, ...) does for
 * one context; the selection calls do it implicitly).  A context without calibration data gives
 * SP_ERR_STATE; a context may appear more than once.
 */
sp_status sp_finalize_multi(sp_ctx *const *ctxs /* host */, int n_items, sp_stream stream);

/*
 * Reads the statistics back to HOST buffers (any may be NULL) and synchronises
 * the stream: colsq_host[d_in] (fp64), *S_host, factor_host[d_in] (the fp32
 * per-channel factor c_q = 1/(2(1 - colsq[q]/S)) of Eq. 8), *n_tokens_host.
 * Returns SP_ERR_DEGENERATE if S is zero or not finite, SP_ERR_STATE if no
 * token has been accumulated.
 */
sp_status sp_get_stats(sp_ctx *ctx, double *colsq_host, double *S_host, float *factor_host,
                       int64_t *n_tokens_host, sp_stream stream);

/*
 * Replaces the statistics by colsq_host[d_in] (HOST, fp64) and a token count
 * (> 0), e.g. to resume from saved statistics.  Synchronises the stream.
 */
sp_status sp_set_stats(sp_ctx *ctx, const double *colsq_host, int64_t n_tokens, sp_stream stream);

/*
 * One-shot statistics without any allocation (the paper has no counterpart: this exists for
 * callers, not for the method).  Some programs must not allocate device memory while they
 * run: code executing inside a framework that owns the whole memory pool, a service that has
 * handed all remaining memory to its caches, a real-time loop that cannot afford the implicit
 * device-wide synchronisation of cudaMalloc/cudaFree.  sp_create allocates, so such callers
 * cannot use a context.  This call computes, for ONE batch X [n_tokens, d_in] (n_tokens >= 1),
 * what sp_calib_accumulate + finalisation compute, on the CURRENT device, and copies the
 * results into the caller's DEVICE buffers (each may be NULL): colsq_out[d_in] (fp64),
 * factor_out[d_in] (fp32 c_q of Eq. 8), S_out[1] (fp64).  Its working memory is a fixed array
 * inside the library image (about 4.4 MB per GPU, held until the process exits), hence:
 *   - d_in must be <= 16384, else SP_ERR_SHAPE and nothing is enqueued;
 *   - it calls no cudaMalloc/cudaFree and no allocating library routine;
 *   - all calls on one device share that array: calls whose GPU work may overlap (different
 *     streams, different threads) race and give wrong results - keep them on one stream or
 *     order them with events.  Nothing is kept between calls;
 *   - the first call on each device looks up the array's device address (a host-side,
 *     synchronous runtime query) and may make the CUDA runtime load the library's kernels,
 *     which can allocate; make that first call before starting any stream capture and before
 *     the phase in which nothing may be allocated.
 * Results agree with the context path to rounding (the token slabs may be cut differently).
 */
sp_status sp_calib_stats_noalloc(const void *X, sp_dtype dtype, int64_t n_tokens, int64_t d_in,
                                 int64_t ldx, double *colsq_out, float *factor_out, double *S_out,
                                 sp_stream stream);

/* ------------------------------------------------------------------ metric (Eq. 8) */

/*
 * Finalises the statistics (S and the per-channel factor c_q) if new batches
 * arrived since the last finalisation, and, if scores_out is not NULL, writes
 *     L[r, q] = (w[r,q] * w[r,q]) * c_q ,   c_q = 0.5 / (1 - colsq[q] / S)
 * as fp32 [n_rows, d_in] (dense, leading dimension d_in), which is Eq. 8 with S
 * at its initial value.  All operations are IEEE binary32 with one rounding
 * each, in exactly this order: u = colsq32/S32, den = 1-u, c = 0.5/den,
 * w2 = w*w (exact), L = w2*c.  W may be NULL when scores_out is NULL
 * (finalise only).  The selection calls finalise implicitly.
 */
sp_status sp_score(sp_ctx *ctx, const void *W, sp_dtype dtype, int64_t n_rows, int64_t ldw,
                   float *scores_out, sp_stream stream);

/* ------------------------------------------------------------------ selection */

/* Table 3: la for a pruning ratio in (0, 1).  The five listed ratios (0.5 .. 0.9)
 * return the printed values; other ratios are interpolated linearly between, or
 * extrapolated from, the nearest two (the paper gives no values there). */
sp_status sp_la_for_sparsity(float sparsity, float *la_out);

/*
 * Algorithm 1 (EWMA running threshold) on every row of W, fused with the
 * write-back.  Along each row, for i = 0 .. d_in-1:
 *     L_i as in sp_score;  est starts at L_0, dev at 0 (Table 2);
 *     prune w_i  iff  L_i < est - la * dev      (state before the update);
 *     est <- (1-alpha) est + alpha L_i;  dev <- (1-beta) dev + beta |est - L_i|
 *     (dev uses the updated est, as Algorithm 1 orders the two steps).
 * Column 0 of every row is therefore never pruned.
 *   sparsity   nominal pruning ratio; la = sp_la_for_sparsity(sparsity),
 *              alpha = beta = 0.125 (Section 4.2), SP_S_GATED.  The achieved ratio
 *              is only approximately the nominal one.
 *   mask_out   nullable; mask as described above.
 *   W_out      nullable; pruned copy of W with leading dimension ldo; may alias W
 *              exactly (same pointer, same ld) for in-place pruning.
 *   counters   nullable; SP_NUM_COUNTERS device uint64 the call ADDS to:
 *              [SP_COUNTER_KEPT] kept weights, [SP_COUNTER_S_HAZARD] rows that held a weight
 *              able to change S in binary32 and were therefore finished sequentially
 *              (SP_S_GATED only; 0 at calibration scale).
 * The scan evaluates the two recurrences as warp-level affine scans in fp32; results differ
 * from a sequential fp32 evaluation by re-association only.  A row that SP_S_GATED finishes
 * sequentially costs about as much as a thousand scanned rows: when the statistics are so
 * small that most rows need it, SP_S_LITERAL_W2 is the faster way to the same result.
 */
sp_status sp_select_unstructured(sp_ctx *ctx, const void *W, sp_dtype dtype, int64_t n_rows,
                                 int64_t ldw, float sparsity, uint32_t *mask_out, void *W_out,
                                 int64_t ldo, unsigned long long *counters, sp_stream stream);

/* Same with explicit parameters (0 < alpha, beta <= 1; la finite). */
sp_status sp_select_unstructured_ex(sp_ctx *ctx, const void *W, sp_dtype dtype, int64_t n_rows,
                                    int64_t ldw, const sp_ewma_params *params /* host */,
                                    uint32_t *mask_out, void *W_out, int64_t ldo,
                                    unsigned long long *counters, sp_stream stream);

/*
 * Diagnostic behind the paper's Fig. 2 (est and dev tracking the mean and the L1 deviation of L
 * along a row): writes, for every weight of every row, the state Algorithm 1 tests it against -
 * est_out[r, i] and dev_out[r, i] are est and dev BEFORE the update of element i (so
 * est_out[r, 0] = L_0, dev_out[r, 0] = 0) - and scores_out[r, i] = L_i; each fp32
 * [n_rows, d_in], dense, nullable.  Evaluated sequentially along each row in binary32 with one
 * rounding per operation (one thread per row: meant for a handful of rows, not for speed);
 * params->s_update selects whether "S = S - w_i^2" is applied to pruned weights.
 */
sp_status sp_ewma_trace(sp_ctx *ctx, const void *W, sp_dtype dtype, int64_t n_rows, int64_t ldw,
                        const sp_ewma_params *params /* host */, float *est_out, float *dev_out,
                        float *scores_out, sp_stream stream);

/*
 * Searches la for a requested pruning ratio (the paper tunes la per ratio by hand, Table 3, and
 * names "finding the optimal sparsity" and frequent re-pruning as the use, Sections 1 and 4.2).
 * With S frozen the pruned fraction is a non-increasing function of la, so the call bisects
 * la on [-8, 8]: each of the `iterations` (1..64) steps runs Algorithm 1 over W at the midpoint
 * in count-only mode (W is read, nothing is written).  For rows that allow 16-byte access
 * (W 16-byte aligned, ldw and d_in multiples of 8) the bisection state stays on the device and
 * the call SYNCHRONISES the stream once, at the end; otherwise the kept count is read back after
 * every step (one synchronisation per step).  *la_out (host) receives the visited la whose
 * pruned fraction is closest to target_sparsity, *achieved_out (host, nullable) that fraction.
 * Follow with sp_select_unstructured_ex(la) to prune.
 */
sp_status sp_search_la(sp_ctx *ctx, const void *W, sp_dtype dtype, int64_t n_rows, int64_t ldw,
                       float target_sparsity, float alpha, float beta, int iterations,
                       float *la_out /* host */, double *achieved_out /* host */,
                       sp_stream stream);

/*
 * Section 3.3: N:M selection fused with the write-back.  Every row is cut into
 * contiguous groups of M columns starting at column 0; in each group the N
 * weights with the largest L (as in sp_score) are kept and the M-N smallest are
 * pruned; among equal scores the lower column is pruned first; a NaN score
 * ranks above every number.  M is 4 or 8, 0 < N < M, d_in % M == 0
 * (else SP_ERR_SHAPE).  2:4 keeps two of every four.
 */
sp_status sp_select_nm(sp_ctx *ctx, const void *W, sp_dtype dtype, int64_t n_rows, int64_t ldw,
                       int N, int M, uint32_t *mask_out, void *W_out, int64_t ldo,
                       sp_stream stream);

/*
 * Grouped selection.  Layers that read the same input (q/k/v; gate/up) share a context and the
 * per-channel factors, and Algorithm 1 treats every row on its own (its row loop is
 * parallel), so their rows can be pruned by one launch: small layers then no longer pay a
 * launch and a ramp-up each.  mats (HOST array, 1 <= n_mats <= SP_MAX_GROUP) lists the
 * matrices, all of `dtype`; every entry follows the rules of the single-matrix call (mask_out
 * and W_out nullable, W_out may alias W exactly).  The result for each matrix is identical to
 * that of its own sp_select_unstructured[_ex] / sp_select_nm call.  Matrices that do not allow
 * 16-byte access, or (N:M) ask for different outputs than their neighbours, get launches of
 * their own.
 */
enum { SP_MAX_GROUP = 8 };
typedef struct {
    const void *W;
    int64_t n_rows;
    int64_t ldw;
    uint32_t *mask_out;
    void *W_out;
    int64_t ldo;
} sp_matrix;
sp_status sp_select_unstructured_group(sp_ctx *ctx, const sp_matrix *mats /* host */, int n_mats,
                                       sp_dtype dtype, float sparsity,
                                       unsigned long long *counters, sp_stream stream);
sp_status sp_select_unstructured_group_ex(sp_ctx *ctx, const sp_matrix *mats /* host */, int n_mats,
                                          sp_dtype dtype, const sp_ewma_params *params /* host */,
                                          unsigned long long *counters, sp_stream stream);
sp_status sp_select_nm_group(sp_ctx *ctx, const sp_matrix *mats /* host */, int n_mats,
                             sp_dtype dtype, int N, int M, sp_stream stream);

/*
 * Algorithm 1 on matrices that read DIFFERENT layer inputs (all layers of a transformer block,
 * say), in one launch where their layouts allow: item i is mats[i] pruned with the statistics of
 * ctxs[i] (HOST arrays of n_items entries, 1 <= n_items <= SP_MAX_MULTI; a context may appear
 * more than once; all contexts on one device, each with calibration data, else
 * SP_ERR_INVALID_ARG / SP_ERR_STATE; mats[i] must be at least ctxs[i]'s d_in wide).  The rows
 * of Algorithm 1 are independent problems whatever matrix they belong to, so the result for
 * each matrix is identical to that of its own sp_select_unstructured[_ex] call on its context;
 * what changes is the cost: one launch, whose tail the short rows fill, instead of one launch
 * and one ramp-up per layer input.  Every context with batches pending is finalised on `stream`
 * first (all of them by one launch).  counters (nullable, device) are totals over all items.  sp_select_nm_multi is the
 * same for the N:M rule of Section 3.3 (every ctxs[i]'s d_in a multiple of M, else
 * SP_ERR_SHAPE; matrices that ask for different outputs than their neighbours, or do not allow
 * 16-byte access, get launches of their own).
 */
enum { SP_MAX_MULTI = 16 };
sp_status sp_select_unstructured_multi(sp_ctx *const *ctxs /* host */,
                                       const sp_matrix *mats /* host */, int n_items,
                                       sp_dtype dtype, float sparsity,
                                       unsigned long long *counters, sp_stream stream);
sp_status sp_select_nm_multi(sp_ctx *const *ctxs /* host */, const sp_matrix *mats /* host */,
                             int n_items, sp_dtype dtype, int N, int M, sp_stream stream);
sp_status sp_select_unstructured_multi_ex(sp_ctx *const *ctxs /* host */,
                                          const sp_matrix *mats /* host */, int n_items,
                                          sp_dtype dtype, const sp_ewma_params *params /* host */,
                                          unsigned long long *counters, sp_stream stream);

/*
 * Section 3.3, compressed output: 2:4 selection (exactly as sp_select_nm with N = 2, M = 4)
 * written as the kept values plus per-group indices in the same pass, so that a consumer of
 * 2:4 sparsity needs no dense pruned matrix and no separate conversion step (Section 3.3 makes
 * the same point about the 2:4 pattern and sparse hardware).  The layout is this library's own:
 *   values_out  [n_rows, d_in/2] of `dtype`, leading dimension ldv (elements, >= d_in/2): the
 *               two kept weights of group g of a row at columns 2g, 2g+1, in column order,
 *               copied bit for bit;
 *   meta_out    [n_rows, ceil(d_in/32)] uint32, no padding between rows: bits 4g..4g+3 of
 *               word k describe group 8k+g as  idx0 | idx1 << 2,  idx0 < idx1 being the
 *               positions (0..3) of the kept weights inside the group; bits past d_in/4 groups
 *               are 0.
 * d_in % 4 == 0 (else SP_ERR_SHAPE).  The fast path needs values_out 8-byte aligned and
 * ldv % 4 == 0 in addition to the usual conditions on W.
 */
sp_status sp_select_24_compressed(sp_ctx *ctx, const void *W, sp_dtype dtype, int64_t n_rows,
                                  int64_t ldw, void *values_out, int64_t ldv, uint32_t *meta_out,
                                  sp_stream stream);

/*
 * Algorithm 1's write-back on its own: W_out = W where the mask bit is 1, +0
 * elsewhere.  W_out may alias W exactly.  Needs no context.
 */
sp_status sp_apply_mask(const void *W, sp_dtype dtype, int64_t n_rows, int64_t n_cols, int64_t ldw,
                        const uint32_t *mask, void *W_out, int64_t ldo, sp_stream stream);

/* ------------------------------------------------------------------ microscaled 4-bit weights */

/*
 * A pruned matrix held in 4 bits per weight plus a scale byte for every 32 (17/32 byte per
 * weight), and its product with activations.  The format is microscaled 4-bit floating point: in
 * every block of 32 consecutive columns of a row (the last block of a row may be short)
 *     value = code * 2^(byte - 127),   code in {0, .5, 1, 1.5, 2, 3, 4, 6} with a sign,
 *     byte  = floor(log2 max|w|) - 2 + 127, at least 0;
 * codes are nearest to w / 2^(byte - 127), ties to the even code, magnitudes above 6 become 6.  A
 * weight of 0 keeps the value 0, so pruning survives.  A block that holds a NaN or an infinity
 * gets byte 255 and all its values are NaN.  Layout (the library's own):
 *   codes   [n_rows, ldc bytes]: two codes per byte, the even column in the low half (bit 3 of a
 *           code: sign, bits 2..0: index into the list above); block b of a row takes the bytes
 *           16b .. 16b+15; columns past n_cols hold code 0.  16-byte aligned, ldc a multiple of
 *           16 and >= 16 * ceil(n_cols / 32);
 *   scales  sp_mx4_scale_bytes(n_rows, n_cols) bytes, 16-byte aligned: tiles of 512 bytes for 128
 *           rows x 4 blocks (n_cols / 128 tiles, rounded up, for the first 128 rows, and so on);
 *           byte (r % 32) * 16 + (r / 32 % 4) * 4 + b % 4 of a tile belongs to row r, block b; the
 *           bytes of rows and blocks that do not exist are 0.
 * These calls need no context and work on the CURRENT device.
 */

/* Size of the scale array of an n_rows x n_cols matrix; 0 for an empty one or negative sizes. */
int64_t sp_mx4_scale_bytes(int64_t n_rows, int64_t n_cols);

/*
 * Quantises W [n_rows, n_cols] (leading dimension ldw).  mask (nullable, the layout of the
 * selection calls) prunes on the way: weights whose keep bit is 0 count as 0.
 */
sp_status sp_mx4_quantize(const void *W, sp_dtype dtype, int64_t n_rows, int64_t n_cols,
                          int64_t ldw, const uint32_t *mask, uint8_t *codes, int64_t ldc,
                          uint8_t *scales, sp_stream stream);

/* The way back: W_out [n_rows, n_cols] = the values, rounded to dtype (exact where the codes
 * came from a matrix of that dtype). */
sp_status sp_mx4_dequantize(const uint8_t *codes, int64_t ldc, const uint8_t *scales,
                            int64_t n_rows, int64_t n_cols, sp_dtype dtype, void *W_out,
                            int64_t ldo, sp_stream stream);

/*
 * Y [n_tokens, n_rows] = X [n_tokens, n_cols] V^T, V the values of (codes, scales), sums in
 * binary32, rounded once to dtype (that of X and Y).  mode:
 *   SP_MX4_A16   X as it is (what decoding steps use);
 *   SP_MX4_A4    X quantised like the weights first, 32 channels at a time (what long prompts
 *                use: both operands then go to the 4-bit tensor cores as they are).
 * workspace: sp_mx4_linear_workspace bytes of device memory, 16-byte aligned, contents arbitrary
 * before and after (NULL where that is 0, and with SP_MX4_A16 where X is 16-byte aligned and ldx a
 * multiple of 8: only other rows are copied there).  n_cols >= 1.  Y must not overlap X or the workspace.
 */
typedef enum { SP_MX4_A16 = 0, SP_MX4_A4 = 1 } sp_mx4_mode;
sp_status sp_mx4_linear_workspace(int64_t n_tokens, int64_t n_rows, int64_t n_cols, int mode,
                                  int64_t *bytes /* host */);
sp_status sp_mx4_linear(const void *X, sp_dtype dtype, int64_t n_tokens, int64_t ldx,
                        const uint8_t *codes, int64_t ldc, const uint8_t *scales, int64_t n_rows,
                        int64_t n_cols, int mode, void *Y, int64_t ldy, void *workspace,
                        int64_t workspace_bytes, sp_stream stream);

/* ------------------------------------------------------------------ 8-bit key/value cache */

/*
 * Keys and values held as 8-bit floats (e4m3: sign, 4 exponent bits, 3 mantissa bits, no
 * infinities) with one power-of-two scale for each block of tokens and head, K and V apart:
 *     value = code * scale,  scale = 2^e,  e the least whole number >= -126 with
 *     max|v| <= 448 * 2^e over the block's finite values (a floating code loses no precision to
 *     a power-of-two scale); codes are nearest to v / scale, ties to even; a NaN or an infinity
 *     is stored as NaN.
 * A block holds block_tokens consecutive tokens of one sequence for every head; token j of
 * sequence b lies in block table[b, j / block_tokens] at place j % block_tokens.  A table entry
 * outside [0, n_blocks) names no block: its tokens are not written and take no part.
 * All pointers are device pointers; k and v 16-byte aligned.  Requirements: head_dim 64 or 128,
 * block_tokens 16, 32 or 64, n_kv_heads <= 65535, n_seqs <= 32767 (else SP_ERR_SHAPE).  The calls
 * work on the CURRENT device.
 */
typedef struct {
    void *k, *v;               /* codes [n_blocks, n_kv_heads, block_tokens, head_dim] */
    float *k_scale, *v_scale;  /* [n_blocks, n_kv_heads] */
    const int32_t *table;      /* [n_seqs, ld_table]; the first table_cols of a row are used */
    int64_t n_blocks, n_seqs, table_cols, ld_table;
    int n_kv_heads, head_dim, block_tokens;
} sp_cache;

/* Strides in elements of a [sequence, token, head, head_dim] tensor of 16-bit floats; a head's
 * values are consecutive. */
typedef struct {
    int64_t seq, token, head;
} sp_strides;

/*
 * Writes the tokens K, V [n_seqs, n_new, n_kv_heads, head_dim] at the places start[b] ..
 * start[b] + count[b] - 1 of every sequence (start, count: device int32; count nullable: n_new
 * everywhere; larger counts and places past the table are cut off, negative ones write nothing).
 * A block that already holds tokens before start[b] keeps its scale, or, where the new tokens
 * need a larger one, has its codes brought to that; a block whose first token is new starts
 * afresh.  Places after the written ones are left as they are.
 */
sp_status sp_cache_append(const sp_cache *cache /* host struct */, const void *K,
                          const sp_strides *k_strides, const void *V, const sp_strides *v_strides,
                          sp_dtype dtype, int64_t n_new, const int32_t *start,
                          const int32_t *count, sp_stream stream);

/*
 * Attention of n_q query tokens per sequence over the cache:
 *     O[b, i, h] = sum_j p[j] v[j],  p = softmax over j of scale * q[b, i, h] . k[j]
 * with lens[b] (device int32) tokens in the cache, the call's own n_q included: query i sits at
 * place lens[b] - n_q + i and sees the tokens up to it.  n_heads is a multiple of n_kv_heads;
 * consecutive heads share a kv head.  A query that sees no token gives 0 and lse -inf.  What lies
 * in the cache past a query's place takes no part, whatever it is.  max_len >= every lens[b]
 * (tokens past it are ignored).  lse (nullable): [n_seqs, n_q, n_heads], log of the sum of
 * exp(scale * q . k).  Scores and sums are binary32; the weights enter their product to 2^-22 of
 * themselves and 2^-44 of the row's largest.
 * acc_out (nullable) [n_seqs, n_kv_heads, ld_acc], ld_acc >= max_len, accumulates the attention
 * that every token received, for sp_cache_evict:
 *     acc_out[b, g, j] = acc_in[b, g, j] + sum of p[j] over the queries and the heads of group g
 * for j < lens[b], 0 up to max_len; acc_in (nullable: zeros; may be acc_out) counts as 0 for the
 * call's own n_q tokens.  workspace as in sp_mx4_linear.  The pool may have at most 2^31 - 1
 * rows n_blocks * n_kv_heads * block_tokens here (else SP_ERR_SHAPE).
 */
sp_status sp_cache_attention_workspace(const sp_cache *cache, int64_t n_q, int n_heads,
                                       int64_t max_len, int want_acc, int64_t *bytes /* host */);
sp_status sp_cache_attention(const sp_cache *cache, const void *Q, const sp_strides *q_strides,
                             sp_dtype dtype, int64_t n_q, int n_heads, const int32_t *lens,
                             int64_t max_len, float scale, void *O, const sp_strides *o_strides,
                             float *lse, const float *acc_in, float *acc_out, int64_t ld_acc,
                             void *workspace, int64_t workspace_bytes, sp_stream stream);

/*
 * Keeps, for every sequence and kv head on its own, m = min(lens[b], budget) of the tokens: the
 * last min(recent, m), and of those before them the ones with the largest acc[b, g, j]
 * (accumulated attention; NaN above every number, among equals the lower j first, -0 equal to 0).
 * They are laid, in their order, into the first ceil(budget / block_tokens) blocks of dst's
 * table, with new scales; slots past m hold zeros.  dst has the head count, head size and block
 * size of src (else SP_ERR_SHAPE) and none of src's blocks (the pools may be the same).
 *   kept_out  [n_seqs, n_kv_heads, budget]: the kept places j, ascending, -1 past m;
 *   acc_out   nullable [n_seqs, n_kv_heads, ld_acc_out], ld_acc_out >= budget: acc of the kept
 *             tokens, 0 past m; must not overlap acc;
 *   lens_out  nullable [n_seqs]: m; must not overlap lens.
 */
sp_status sp_cache_evict(const sp_cache *src, const int32_t *lens, int64_t max_len,
                         const float *acc, int64_t ld_acc, int64_t budget, int64_t recent,
                         const sp_cache *dst, int32_t *kept_out, float *acc_out,
                         int64_t ld_acc_out, int32_t *lens_out, sp_stream stream);

/*
 * Waits of the kernels above on their own copies and tensor-core work are bounded; *expired
 * receives how many ran out on the current device since the last clear (0 unless the device or
 * the library is at fault; results of such a call are wrong).  Synchronises the device.
 */
sp_status sp_wait_status(int *expired /* host */, int clear);

/* ------------------------------------------------------------------ host-buffer variants */

/*
 * The same operations (Algorithm 1 step 1; Section 3.3; Algorithm 1) for data that lives in
 * HOST memory: X_host, W_host, mask_host and W_out_host are host pointers (pinned memory lets
 * the transfers overlap the kernels; pageable memory works but copies synchronously).  The
 * matrix is streamed through two device staging slots of 64 MiB owned by the context (created,
 * together with two internal streams, by the first such call on a context - that call
 * allocates): host->device copy, kernel and device->host copy of successive row chunks overlap.
 * Work is ordered after everything already queued on `stream`, and `stream` completes only
 * after the last result has reached the host; the calls themselves do not wait.  mask_host and
 * W_out_host may each be NULL; W_out_host may equal W_host (same ld) for in-place pruning.
 * Results are identical to the device-pointer calls.
 */
sp_status sp_calib_accumulate_host(sp_ctx *ctx, const void *X_host, sp_dtype dtype,
                                   int64_t n_tokens, int64_t ldx, sp_stream stream);
sp_status sp_select_nm_host(sp_ctx *ctx, const void *W_host, sp_dtype dtype, int64_t n_rows,
                            int64_t ldw, int N, int M, uint32_t *mask_host, void *W_out_host,
                            int64_t ldo, sp_stream stream);
sp_status sp_select_unstructured_host(sp_ctx *ctx, const void *W_host, sp_dtype dtype,
                                      int64_t n_rows, int64_t ldw, float sparsity,
                                      uint32_t *mask_host, void *W_out_host, int64_t ldo,
                                      sp_stream stream);

/* ------------------------------------------------------------------ diagnostics */

/*
 * Index checks of the debug build (python -m paper_2501_16376_b200.build --debug ->
 * libswiftprune_debug.so, same ABI).  In that build the kernels check the indices of their
 * stores; an out-of-range access is skipped and recorded instead of faulting (nothing traps).
 * *violations receives the number of skipped accesses on the current device since the last
 * clear (-1 in the release build, which compiles no checks); first_code / first_index /
 * first_limit (nullable) describe the first one (codes in csrc/sp_debug.cuh); clear != 0 resets
 * the records.  Synchronises the device.
 */
sp_status sp_debug_status(int *violations /* host */, int *first_code /* host */,
                          int64_t *first_index /* host */, int64_t *first_limit /* host */,
                          int clear);

const char *sp_status_string(sp_status status);
/* Text of the last CUDA error this thread saw inside the library ("" if none). */
const char *sp_last_cuda_error(void);
/* Kernels launched by the library since it was loaded (all threads). */
uint64_t sp_launch_count(void);

#ifdef __cplusplus
}
#endif
#endif /* SWIFTPRUNE_H_ */
