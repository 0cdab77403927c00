/*
 * ptq.h -- C ABI of the B200 (sm_100a) per-layer quantizer: sensitivity-ordered, row-parallel
 * quantization with one shared inverse Hessian (Sec. 4 of the paper).
 *
 * Data model (Sec. 3): W is [rows x cols] = d_row x d_col, X is [cols x n] = d_col x N, the layer
 * computes W X and the objective is ||W X - What X||^2 (Eq. 2).
 *
 * Rules common to every entry point
 *   - Every data pointer is a DEVICE pointer owned by the caller (unless a parameter says "host").
 *     The library allocates no device memory: scratch comes from the caller's workspace `ws`, whose
 *     minimum size is given by ptq_workspace_bytes().  Base pointers must be 16-byte aligned.
 *   - Matrices are row-major.  H, Hinv: float64 [cols x cols], full symmetric storage.
 *   - Calls are asynchronous on `stream` (a cudaStream_t passed as void*).  The return value reports
 *     argument errors found on the host (nothing is launched then).  Conditions found on the device
 *     (not positive definite, non-finite input, bounded wait expired) are recorded in the caller's
 *     `status` word, int32[4] = {code, index, aux, 0}; the first error sticks, so the caller zeroes it
 *     before a sequence of calls and reads it after synchronising the stream.
 *   - Inputs are never modified; outputs are fully overwritten (H of ptq_hessian_accumulate is updated).
 *   - Results are deterministic: fixed reduction orders, no floating-point atomics.
 *   - Host-side state (SM count, kernel attributes) is kept per device and looked up with the caller's current
 *     device, so one process may drive several devices; calls may come from several host threads as long as calls
 *     that share a stream, a workspace or output buffers are ordered by the caller.
 *   - Size limits: ptq_quantize_layer (and its dynamic variant) takes rows <= 65535 and cols <= 65535, ptq_prepare_hinv
 *     cols <= 65535 (PTQ_ERR_UNSUPPORTED beyond).
 *   - No exceptions, no exit(), no stdout, no device trap, no unbounded device-side wait.
 */
#ifndef PTQ_H_
#define PTQ_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    PTQ_OK = 0,
    PTQ_ERR_INVALID_ARG = 1,
    PTQ_ERR_ALIGNMENT = 2,
    PTQ_ERR_WORKSPACE = 3,
    PTQ_ERR_NOT_SPD = 4,     /* status[1] = failing pivot index (not positive, not finite, or too small to be inverted) */
    PTQ_ERR_NONFINITE = 5,
    PTQ_ERR_TIMEOUT = 6,     /* a bounded device-side wait expired */
    PTQ_ERR_CUDA = 7,        /* a CUDA runtime call failed on the host */
    PTQ_ERR_UNSUPPORTED = 8,
    PTQ_ERR_STATIC_SCRATCH = 9 /* ptq_sensitivity_order_static: rows x cols beyond the built-in scratch array */
} ptq_status;

/* Damping (Implementation Details: a constant is added to the diagonal of H). */
typedef enum {
    PTQ_DAMP_REL_MEAN_DIAG = 0, /* lambda = damp * mean(diag H) */
    PTQ_DAMP_ABS = 1            /* lambda = damp (the paper's 0.1) */
} ptq_damp_mode;

/* Column score (Sec. 4.1 names the keys err / w / sensi; Sec. 4.2 step 2 sums them per column). */
typedef enum {
    PTQ_SCORE_QERR = 0,  /* Eq. 10: (w - quant(w))^2 / (2 [Hinv]_jj)   (default) */
    PTQ_SCORE_PRUNE = 1, /* Eq. 8 :  w^2 / (2 [Hinv]_jj) */
    PTQ_SCORE_ERR = 2,   /* (w - quant(w))^2 */
    PTQ_SCORE_W = 3,     /* w^2 */
    PTQ_SCORE_NONE = 4,  /* no sorting: identity order */
    /* Sec. 4.1 names each key in a descending ("des") and an ascending ("asc") variant.  Descending is the default
     * (and the method's); adding this flag to a mode sorts by S ascending.  Equal scores keep the lower column
     * index first in both directions. */
    PTQ_SCORE_ASCENDING = 16
} ptq_score_mode;

typedef enum {
    PTQ_CALL_HESSIAN_ACCUMULATE = 0,
    PTQ_CALL_PREPARE_HINV = 1,
    PTQ_CALL_SENSITIVITY_ORDER = 2,
    PTQ_CALL_QUANTIZE_LAYER = 3,
    PTQ_CALL_HESSIAN_ACCUMULATE_F64 = 4,
    PTQ_CALL_QUANTIZE_LAYER_DYNAMIC = 5,
    PTQ_CALL_QUANTIZE_LAYER_PER_ROW = 6
} ptq_call_id;

/* Minimum workspace, in bytes, for one call with these sizes (host function, no CUDA calls). */
size_t ptq_workspace_bytes(int call_id, int rows, int cols, int n);

/*
 * H += 2 * X X^T  (Sec. 3: the second derivative of Eq. 2 with respect to one row of W).
 *   H    [cols x cols] float64, in/out; the caller zeroes it before the first chunk of calibration columns
 *   X    [cols x n]    float32, row stride ldx >= n elements (vector loads are used when X is 16-byte aligned
 *                      and ldx is a multiple of 4)
 * The product is formed on the tensor cores from error-free integer slices of X, so H carries
 * float64-level accuracy (relative error about 1e-12 or better).
 */
int ptq_hessian_accumulate(double *H, const float *X, int cols, int n, int64_t ldx, void *ws, size_t ws_bytes,
                           int32_t *status, void *stream);

/*
 * The same accumulation for a convolutional layer, straight from the layer's input (Sec. 3: for a convolution d_col
 * is the number of weights of one filter, channels * kh * kw, and the columns of X are the input patches those
 * weights see).  With out_h = (height + 2 pad - kh) / stride + 1 (out_w alike), cols = channels * kh * kw and
 * n = batch * out_h * out_w:
 *     X[(c * kh + ki) * kw + kj][(b * out_h + oy) * out_w + ox] = act[b][c][oy * stride + ki - pad][ox * stride + kj - pad]
 * (zero outside the image), H += 2 X X^T.  The patches are never written out: the slicing pass reads act in place.
 *   H    [cols x cols] float64, in/out (row and column order: channel-major, then ki, then kj, the layout of a
 *        convolution weight [out_channels][channels][kh][kw] flattened per filter)
 *   act  [batch][channels][height][width] float32, contiguous
 * Workspace: ptq_workspace_bytes(PTQ_CALL_HESSIAN_ACCUMULATE, 0, cols, n).  Calling it once per calibration batch
 * accumulates over batches.  Sizes beyond cols = 2^20 or n = 2^30 return PTQ_ERR_UNSUPPORTED.
 */
int ptq_hessian_accumulate_conv(double *H, const float *act, int batch, int channels, int height, int width, int kh,
                                int kw, int stride, int pad, void *ws, size_t ws_bytes, int32_t *status, void *stream);

/* Same contract, computed with float64 FMAs (cross-check of the tensor-core path). */
int ptq_hessian_accumulate_f64(double *H, const float *X, int cols, int n, int64_t ldx, void *ws, size_t ws_bytes,
                               int32_t *status, void *stream);

/*
 * Hinv = (H + lambda I)^-1 by Cholesky factorisation and inversion of the factor (Sec. 5 item 1).
 *   H          [cols x cols] float64, const
 *   Hinv       [cols x cols] float64, out
 *   Hinv_diag  [cols] float64, out (the diagonal of Hinv, what the sensitivities need)
 *   lambda_out [1] float64, out (device)
 * A non-positive pivot sets status = {PTQ_ERR_NOT_SPD, pivot index}.
 */
int ptq_prepare_hinv(const double *H, int cols, int damp_mode, double damp, double *Hinv, double *Hinv_diag,
                     double *lambda_out, void *ws, size_t ws_bytes, int32_t *status, void *stream);

/*
 * Helper: per-row asymmetric min-max grid whose range always contains 0, from the original W
 * (Sec. 3, OBQ paragraph: a fixed grid of width Delta).  scale, zero: [rows] float32, out.
 * quant_i(w) = scale_i * (clamp(rint(w / scale_i) + zero_i, 0, 2^bits - 1) - zero_i), rint = ties to even.
 */
int ptq_minmax_grid(const float *W, int rows, int cols, int64_t ldw, int bits, float *scale, float *zero,
                    int32_t *status, void *stream);

/*
 * Sec. 4.2 steps 1-3: S_j = sum_i score(w_ij) from the original W and diag(Hinv); perm = columns by S descending
 * (ascending with PTQ_SCORE_ASCENDING added to score_mode), equal scores keep the lower column index first.
 * S [cols] float64 out, perm [cols] int32 out.
 */
int ptq_sensitivity_order(const float *W, int rows, int cols, int64_t ldw, const double *Hinv_diag, const float *scale,
                          const float *zero, int bits, int score_mode, double *S, int32_t *perm, void *ws,
                          size_t ws_bytes, int32_t *status, void *stream);

/*
 * ptq_sensitivity_order for callers that cannot hand the library any scratch memory.  (The paper has no
 * counterpart: this is a packaging variant of the call above, with the same inputs, outputs and arithmetic.)
 *
 * Who needs it: code that runs where device allocation is off limits -- inside a region that must not call
 * cudaMalloc (a latency-critical serving loop, a process whose memory pool is owned and fully handed out by
 * another component, a plug-in that is given device pointers but no allocator) -- and that therefore cannot size
 * and provide the `ws` buffer the ordinary call asks for.  This entry point takes no workspace: the per-row-chunk
 * partial sums live in an array compiled into the library, PTQ_STATIC_SCRATCH_BYTES large.  Every device that loads
 * the library carries that array until the process exits, whether or not this function is ever called.
 *
 * Limits and rules
 *   - ceil(rows / 64) * cols * 8 bytes must not exceed PTQ_STATIC_SCRATCH_BYTES (e.g. 4096 x 11008 fits);
 *     larger problems return PTQ_ERR_STATIC_SCRATCH and launch nothing.
 *   - It never calls cudaMalloc, cudaFree or any allocating routine.  Every call looks up the array's device address
 *     (cudaGetSymbolAddress, with the caller's device current; nothing is remembered between calls, so the address
 *     is right after a cudaDeviceReset too).  The first such lookup on a device initialises the library's module
 *     there: make the first call on each device outside any stream capture.
 *   - All calls on one device share the one array, and it keeps whatever the previous call left there.  The
 *     kernels overwrite every element they later read, so no clearing is needed; but two calls that may run at
 *     the same time on the GPU (different streams, or different host threads) race on it: keep calls to this
 *     entry point ordered on one stream, or serialise them yourself.
 */
#define PTQ_STATIC_SCRATCH_BYTES (6u << 20)
int ptq_sensitivity_order_static(const float *W, int rows, int cols, int64_t ldw, const double *Hinv_diag,
                                 const float *scale, const float *zero, int bits, int score_mode, double *S,
                                 int32_t *perm, int32_t *status, void *stream);

/*
 * Sec. 4.2 steps 3-5: permute W and Hinv by perm, then quantize one column at a time, all rows in parallel;
 * after each column the remaining columns absorb the error (Eq. 11) and the shared inverse Hessian is
 * updated (Eq. 12).  The updates are applied in blocked form through the upper Cholesky factor of the
 * permuted inverse Hessian, whose row p equals row p of the Eq.-12-updated matrix divided by the square
 * root of its pivot.
 *   codes      [rows x cols] uint8, out, one code per byte, ORIGINAL column order
 *   What       [rows x cols] float32, out (may be NULL): scale_i * (code - zero_i)
 *   H_undamped [cols x cols] float64 and loss_out [1] float64 (device): loss = ||W X - What X||^2
 *              = 1/2 tr(dW H dW^T); pass NULL for either to skip
 */
int ptq_quantize_layer(const float *W, int rows, int cols, int64_t ldw, const double *Hinv, const int32_t *perm,
                       const float *scale, const float *zero, int bits, uint8_t *codes, float *What,
                       const double *H_undamped, double *loss_out, void *ws, size_t ws_bytes, int32_t *status,
                       void *stream);

/*
 * The column loop with dynamic re-ranking.  Sec. 5 writes the sort inside the per-column loop; read literally, the
 * columns still to be quantized are ranked again while the loop runs.  Every `block` columns the scores of the
 * REMAINING columns are recomputed from the current (compensated) weights and the diagonal of the current
 * (Eq.-12-updated) inverse Hessian, the remaining columns are sorted by them (keys, direction and tie rule of
 * ptq_sensitivity_order; ties by ORIGINAL column index) and the next `block` columns are quantized in that order
 * with Eq. 11 / Eq. 12.  block >= cols is ptq_sensitivity_order followed by ptq_quantize_layer.
 *   block      a multiple of 64, or >= cols (PTQ_ERR_UNSUPPORTED otherwise)
 *   order_out  [cols] int32, out: the sequence in which the columns were quantized
 *   other arguments as for ptq_quantize_layer (outputs in original column order); Hinv_diag is not needed
 * Workspace: ptq_workspace_bytes(PTQ_CALL_QUANTIZE_LAYER_DYNAMIC, rows, cols, 0).
 */
int ptq_quantize_layer_dynamic(const float *W, int rows, int cols, int64_t ldw, const double *Hinv, const float *scale,
                               const float *zero, int bits, int score_mode, int block, uint8_t *codes, float *What,
                               int32_t *order_out, const double *H_undamped, double *loss_out, void *ws,
                               size_t ws_bytes, int32_t *status, void *stream);

/*
 * The non-parallel arm of the paper's ablation (Sec. 4.2, the paragraph on the per-row inverse Hessians; Table 3's rows
 * without the parallel tick): every row ranks its own weights by their sensitivities (the keys of
 * ptq_sensitivity_order applied to that single row, Sec. 4.1) and is quantized in that order against its own copy of
 * the inverse Hessian -- what the shared-inverse-Hessian method avoids.  Cost rows * cols^3 / 3 and one cols x cols
 * matrix per row in flight, so only narrow layers are taken: cols <= 128 (PTQ_ERR_UNSUPPORTED beyond).
 *   perm_rows [rows x cols] int32, out: the order each row used
 *   other arguments as for ptq_quantize_layer; the diagonal of Hinv is read from Hinv itself
 * Workspace: ptq_workspace_bytes(PTQ_CALL_QUANTIZE_LAYER_PER_ROW, rows, cols, 0).
 */
int ptq_quantize_layer_per_row(const float *W, int rows, int cols, int64_t ldw, const double *Hinv, const float *scale,
                               const float *zero, int bits, int score_mode, uint8_t *codes, float *What,
                               int32_t *perm_rows, const double *H_undamped, double *loss_out, void *ws,
                               size_t ws_bytes, int32_t *status, void *stream);

/*
 * Sec. 4.2 step 3 alone: perm = the indices 0 .. cols-1 sorted by S descending (ascending != 0: ascending), equal
 * scores keep the lower index first.  For callers that form S themselves, e.g. by summing the per-shard scores of a
 * layer whose rows are spread over several GPUs (Sec. 4.2 step 2 is a sum over rows, so it splits over row shards).
 *   S [cols] float64, perm [cols] int32 out.  No workspace.
 */
int ptq_sort_scores(const double *S, int cols, int ascending, int32_t *perm, void *stream);

/*
 * C += alpha * A B^T for float64 operands, formed on the tensor cores from error-free int8 slices of the operands (the
 * way ptq_hessian_accumulate forms H), to float64 accuracy: the product behind the deferred part of Eq. 11,
 * W[:, later] -= E[:, block] U[block, later], exposed for cross-checks and for callers who want it on its own.
 *   C [m x n] float64, row stride ldc, in/out
 *   A [m x k] float64, row stride lda
 *   B: b_is_kn = 0: [n x k], row stride ldb;  b_is_kn = 1: the matrix is stored as [k x n] (so C += alpha A B), stride ldb
 *   k <= 16384 (PTQ_ERR_UNSUPPORTED beyond).  Rows of A / of B with wildly different magnitudes are fine (each has its
 *   own power-of-two scale); within a row, entries below 2^-54 of the row's largest magnitude are rounded away.
 *   A NaN, an infinity or a magnitude of 2^900 and more is recorded in `status` (PTQ_ERR_NONFINITE, index = the row of A
 *   or of B^T) and makes every entry of C that its row enters NaN.
 * Workspace: ptq_gemm_nt_sliced_workspace_bytes(m, n, k).
 */
size_t ptq_gemm_nt_sliced_workspace_bytes(int m, int n, int k);
int ptq_gemm_nt_sliced(double *C, int64_t ldc, const double *A, int64_t lda, const double *B, int64_t ldb, int b_is_kn,
                       int m, int n, int k, double alpha, void *ws, size_t ws_bytes, int32_t *status, void *stream);

/*
 * ------------------------------------------------------------------------------------------------------------------
 * Serving a quantized network: products in 8-bit floating point, and a key-value cache held in 4 bits.  The rules at the top of
 * this file hold here too; what these calls add to them:
 *   - `type` parameters name the element type of the caller's activations (ptq_type).
 *   - Calls with nothing to do (no rows, no tokens) return PTQ_OK and launch nothing.
 *   - A request's table holds at most 2^30 tokens (max_pages * page_size; PTQ_ERR_UNSUPPORTED beyond).
 *   - An output that shares memory with an input, with the workspace or with another output is refused (PTQ_ERR_INVALID_ARG), and so
 *     is one whose own rows overlap.  What counts are all bytes from an array's first to its last; only rows of heads with the same
 *     strides (q and out of ptq_cache_attention, k and v of ptq_cache_read) may alternate in one buffer.
 *   - Sizes that live on the device (lengths, offsets, page and slot numbers) are checked there: an entry that is out of range is
 *     recorded in `status` (PTQ_ERR_INVALID_ARG, index = request or token) and is never used as an address.
 * ------------------------------------------------------------------------------------------------------------------
 */
typedef enum { PTQ_F32 = 0, PTQ_F16 = 1, PTQ_BF16 = 2 } ptq_type;

/*
 * Casts a matrix to 8-bit floating point (e4m3: 3 fraction bits, largest magnitude 448) with one scale for each block of
 * block_rows x 128 values (the last block of a row or column may be narrower):
 *     scale = 2^e, e the least integer >= -126 with max |x| <= 448 2^e;    q = x / scale, rounded to nearest even.
 * A power of two makes the quotient exact, so that a code is one rounding of x.
 *   x       [rows x cols] of x_type, row stride ldx (16-byte loads are used where base and stride allow)
 *   block_rows  1 (activations: a scale per row and 128 columns) or 128 (weights: a scale per 128 x 128)
 *   q       [rows x cols] bytes, out, row stride ldq, a multiple of 16 (that of a single row may be any); bytes behind a row's last
 *           column are left as they are
 *   scale   [ceil(rows / block_rows) x ceil(cols / 128)] float32, out, row stride ld_scale
 * A NaN or an infinity is recorded in `status` (PTQ_ERR_NONFINITE, index = row, or first row of the block); its block's codes and
 * scale become NaN, and with them what a product makes of that row (or of those columns).
 */
int ptq_fp8_quantize(const void *x, int x_type, int rows, int cols, int64_t ldx, int block_rows, uint8_t *q, int64_t ldq,
                     float *scale, int64_t ld_scale, int32_t *status, void *stream);

/*
 * C = A B^T of operands in 8-bit floating point with block scales, as ptq_fp8_quantize makes them (any float32 scales are taken;
 * the product of a scale_a and a scale_b has to lie within float32 too):
 *     C[i][j] = sum_b scale_a[i][b] scale_b[j / 128][b] sum_{k in block b} A[i][k] B[j][k],    blocks of 128 along k
 * Within a block the products are summed on the tensor cores, the blocks are joined in float32, and the result is rounded once to
 * c_type.
 *   C       [m x n] of c_type, out, row stride ldc (beyond 64 rows, rows that are multiples of 16 bytes are written up to five times
 *           as fast)
 *   A       [m x k] bytes, row stride lda;  scale_a [m x ceil(k / 128)], row stride ld_scale_a
 *   B       [n x k] bytes (a weight matrix as the layer stores it), row stride ldb;  scale_b [ceil(n / 128) x ceil(k / 128)]
 *   lda, ldb: multiples of 16 (PTQ_ERR_ALIGNMENT otherwise; that of a single row may be any); what lies behind a row's last column
 *           is not read
 * Few rows (a decoded token) are bound by the one read of B; no workspace.  Beyond m = 2^20 or n = 2^22: PTQ_ERR_UNSUPPORTED.
 */
int ptq_fp8_matmul(void *C, int c_type, int64_t ldc, const uint8_t *A, int64_t lda, const float *scale_a, int64_t ld_scale_a,
                   const uint8_t *B, int64_t ldb, const float *scale_b, int64_t ld_scale_b, int m, int n, int k, int32_t *status,
                   void *stream);

/*
 * The cache: pages[num_pages][kv_heads][page_size / 16] tiles of 16 tokens.  A tile holds, for one key-value head,
 *     K codes [16][head_dim / 2], K grids [16][head_dim / 32] uint16, V codes, V grids
 * with two 4-bit codes a byte (the even value in the low half).  Every 32 values share a min-max grid whose range contains 0, as
 * the rows of ptq_minmax_grid do: with lo = min(0, min), hi = max(0, max),
 *     s = the least fp16 number of 6 significant bits >= (hi - lo) / 15, within [2^-19, 2112];   z = clamp(rint(-lo / s), 0, 15)
 *     code = clamp(rint(x / s) + z, 0, 15), held value = s (code - z)
 * and the grid's 16 bits are the fp16 pattern of s (whose low five bits are 0) with z in the lowest four.  A held value has at
 * most ten significant bits, so it is an fp16 number and nothing is rounded when it is used; magnitudes beyond 15 x 2112 saturate.
 * 4.5 bits a value: 144 bytes for a token's key and value in a head of 128.
 *   page_size  16, 32, 64, 128, 256, 512 or 1024 tokens;  head_dim  64 or 128 (PTQ_ERR_UNSUPPORTED otherwise)
 * ptq_cache_page_bytes: the size of one page, 0 for what is not supported (host function, no CUDA calls).  A token's slot is
 * page * page_size + its place in the page; num_pages * page_size <= 2^31 - 1.
 */
size_t ptq_cache_page_bytes(int page_size, int kv_heads, int head_dim);

/*
 * Where the new tokens of a batch of requests go: extends the requests' block tables by pages of the free list and lists slot and
 * position of every new token, in one launch.
 *   kv_lens     [batch] int32: tokens cached of each request;  new_tokens [batch] int32: how many are added (0 is fine)
 *   block_table [batch x max_pages] int32, in/out, row stride ld_table: the pages of each request in order.  The entry of a page
 *               that new tokens fill up is read, those of pages that begin with a new token are written, others stay.
 *   free_pages  [num_free] int32: pages are taken from its front, in the order of the requests and of their pages
 *   slots       [max_tokens] int32, out;  positions [max_tokens] int32, out: of the new tokens of request 0, then 1, ...; -1 in both
 *               behind the last token, which ptq_cache_append skips (a batch padded to a fixed size, as a captured graph needs it)
 *   cu_q        [batch + 1] int32, out: first new token of each request, and their number
 *   kv_lens_out [batch] int32, out: kv_lens + new_tokens; a buffer of its own, not kv_lens
 *   taken       [1] int32, out: pages taken from the free list
 * If a request does not fit (its table row, max_tokens, num_free, a negative length), status gets PTQ_ERR_INVALID_ARG with the
 * first such request, and nothing is done for any: slots and positions are all -1, cu_q all 0, kv_lens_out = kv_lens, taken 0 and
 * the table as it was.
 */
int ptq_cache_plan(const int32_t *kv_lens, const int32_t *new_tokens, int batch, int page_size, int32_t *block_table,
                   int64_t ld_table, int max_pages, const int32_t *free_pages, int num_free, int32_t *slots, int32_t *positions,
                   int max_tokens, int32_t *cu_q, int32_t *kv_lens_out, int32_t *taken, int32_t *status, void *stream);

/*
 * Writes keys and values of tokens into the cache.
 *   k, v   [tokens][kv_heads][head_dim] of `type`; strides between tokens and between heads in elements, a head's values contiguous
 *   slots  [tokens] int32; a negative slot is skipped.  The slots of one call differ from one another.
 * A NaN is held as 0, an infinity as the end of its group's grid; both are recorded (PTQ_ERR_NONFINITE, index = token), and the
 * cache itself stays finite.
 */
int ptq_cache_append(void *pages, int num_pages, int page_size, int kv_heads, int head_dim, const void *k, int64_t k_token,
                     int64_t k_head, const void *v, int64_t v_token, int64_t v_head, int type, const int32_t *slots, int tokens,
                     int32_t *status, void *stream);

/* The values that the cache holds at `slots`, to k and v (as above, written); rows of negative slots are left as they are. */
int ptq_cache_read(const void *pages, int num_pages, int page_size, int kv_heads, int head_dim, void *k, int64_t k_token,
                   int64_t k_head, void *v, int64_t v_token, int64_t v_head, int type, const int32_t *slots, int tokens,
                   int32_t *status, void *stream);

/*
 * Attention of the newest tokens of a batch of requests over what is cached of them, themselves included.  Request r has the rows
 * cu_q[r] .. cu_q[r + 1] - 1 of q, the last of its kv_lens[r] tokens; with n of them, row i stands at position p = kv_lens[r] - n + i
 * and sees the keys j < kv_lens[r] with j <= p (causal) and j > p - window (window > 0):
 *     out = sum_j softmax_j(scale q . k_j) v_j,     lse = log sum_j exp(scale q . k_j)
 * A row that sees no key gets out = 0 and lse = -infinity.  Query head h reads key-value head h / (q_heads / kv_heads).
 *   q, out  [total_q][q_heads][head_dim] of `type` (PTQ_F16 or PTQ_BF16), strides between tokens and heads in elements; the cache is
 *           read as fp16 either way, and bf16 queries are brought to fp16 by a power of two for each row: values down to 2^-31 of a
 *           row's largest stay as they are, smaller ones are off by at most 2^-39 of it
 *   lse     [total_q][q_heads] float32, or NULL
 *   block_table, kv_lens, cu_q: as ptq_cache_plan leaves them (kv_lens_out).  Rows behind cu_q[batch] are left as they are.
 *           With a window, the entries of pages whose tokens all lie below the first row's window may be anything.
 *   scale   any number up to 2e38 in magnitude; scores, and scale times the largest |q| of a row, have to lie within float32
 *   max_q   the most rows that any request has (it chooses kernels and the workspace; any bound is right, a tight one is fast)
 * Scores, their maximum and sum, and the output are held in float32; the probabilities enter the second product as fp16: rounded to
 * 11 bits, and small ones to within 2^-40 of the row's largest in calls with max_q x q_heads / kv_heads up to 16, to within 2^-33 of it
 * in others.
 * Workspace: ptq_cache_attention_workspace_bytes(q_heads, kv_heads, head_dim, batch, total_q, max_q) (host function, no CUDA
 * calls; 0 for what is not supported); it does not depend on lengths.
 */
size_t ptq_cache_attention_workspace_bytes(int q_heads, int kv_heads, int head_dim, int batch, int total_q, int max_q);
int ptq_cache_attention(void *out, int64_t o_token, int64_t o_head, float *lse, const void *q, int64_t q_token, int64_t q_head,
                        int type, int q_heads, const void *pages, int num_pages, int page_size, int kv_heads, int head_dim,
                        const int32_t *block_table, int64_t ld_table, int max_pages, const int32_t *kv_lens, const int32_t *cu_q,
                        int batch, int total_q, int max_q, float scale, int causal, int window, void *ws, size_t ws_bytes,
                        int32_t *status, void *stream);

const char *ptq_status_string(int code);
int ptq_version(void);

/*
 * Self-test of the bounded device-side waits (instrumentation; the paper has no counterpart).  Launches a kernel that
 * calls the library's own wait routine on a target nothing will ever reach, with the given limit in SM clock cycles:
 *   which = 0 : the grid-wide barrier of the factorisation kernel (one CTA per SM), asked for one arrival too many
 *   which = 1 : the counter wait of the column sweep, on a counter that nobody raises
 * The wait must run out, the kernel records {PTQ_ERR_TIMEOUT, CTA index, 1 + which} in `status` and returns; the
 * context stays usable.  ws: at least 16 bytes of device scratch.  limit_cycles in [1, 4e9].
 */
int ptq_selftest_wait_timeout(int which, long long limit_cycles, void *ws, size_t ws_bytes, int32_t *status,
                              void *stream);

/*
 * Self-test of what the sweep does when the factorisation it runs behind gives up (instrumentation; the paper has no
 * counterpart).  Runs both on a unit layer of 64 x 64 in one launch, with the sweep waiting, for limit_cycles SM clock cycles,
 * for one arrival more than the factorisation makes.  The CTAs of the sweep must record {PTQ_ERR_TIMEOUT, CTA index, 6} in
 * `status`, raise the abort word that the rest of the sweep polls, and return.  abort_word: int32 (device), receives that word.
 * ws: PTQ_ABANDONED_SWEEP_BYTES of device scratch.  limit_cycles in [1, 4e9].
 */
#define PTQ_ABANDONED_SWEEP_BYTES 262144
int ptq_selftest_abandoned_sweep(long long limit_cycles, void *ws, size_t ws_bytes, int32_t *abort_word, int32_t *status,
                                 void *stream);

/*
 * Self-test of the arithmetic on pivots (instrumentation; the paper has no counterpart): rcp[i] = 1 / x[i] and
 * rsq[i] = 1 / sqrt(x[i]) as the factorisations form them, for x[i] from the smallest normal number up to 1e300.
 *   x, rcp, rsq [n] float64 (device)
 */
int ptq_selftest_reciprocal(const double *x, int n, double *rcp, double *rsq, void *stream);

/*
 * Float64 throughput probe (instrumentation; the paper has no counterpart): launches one kernel of 4 CTAs x 256 threads
 * per SM in which every thread runs `iters` rounds of eight independent chains of float64 FMAs (kind 0) or of float64
 * tensor-core MMAs m8n8k4 (kind 1), and nothing else.  *flops_out (host) receives the floating-point operations of
 * that launch (FMA = 2); the caller times the launch on its stream.  sink: one device double (never written).
 */
int ptq_fp64_probe(int kind, int iters, double *sink, double *flops_out, void *stream);

/*
 * Launch accounting (instrumentation; the paper has no counterpart).  Host-side state of the calling process.
 *   ptq_kernel_count / ptq_kernel_name : the library's kernels, by id.
 *   ptq_launch_count(id)   : launches of kernel `id` since the library was loaded; id < 0 gives the total.
 *   ptq_profile_enable(on) : while on, every launch is bracketed by CUDA events on its stream (this perturbs
 *                            timing, so profile on passes that are not themselves being timed); each call clears
 *                            the records taken so far.
 *   ptq_profile_read(id, total_ms, launches) : host pointers; waits for the recorded events and sums the device
 *                            time of kernel `id` over the recorded launches.
 */
/* The persistent cooperative kernels (factorisation, column sweep, both in one launch) take one CTA per SM and occupy an SM
 * each, so two of them never share the GPU.  ptq_set_cta_limit(limit) makes the calls issued afterwards ON THE CURRENT DEVICE
 * launch at most `limit` CTAs (0: no limit, the default): a caller that runs independent layers on several streams sets
 * about sm_count / streams, so that their factorisations and sweeps run side by side (those of layers up to a few thousand
 * columns are bound by a dependency chain, not by the number of SMs).  Results do not depend on the limit.
 * Returns PTQ_ERR_INVALID_ARG for a negative limit. */
int ptq_set_cta_limit(int limit);

int ptq_kernel_count(void);
const char *ptq_kernel_name(int kernel_id);
long long ptq_launch_count(int kernel_id);
int ptq_profile_enable(int on);
int ptq_profile_read(int kernel_id, double *total_ms, long long *launches);

#ifdef __cplusplus
}
#endif
#endif /* PTQ_H_ */
