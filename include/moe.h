/* moe.h -- C ABI of the per-GPU Mixture-of-Experts expert layer for AMD MI355X (gfx950).
 *
 * The layer is the one GEM (GPU-variability-aware expert-to-GPU mapping) profiles and balances:
 * a router selects the top-k of E experts for every token (paper Sec. 2.1), the token is sent to
 * the GPU holding those experts, each expert is a feed-forward network, and the results return
 * to the token (Sec. 7).  The latency of this layer as a function of the number of tokens a GPU
 * receives is the per-GPU curve C_g(n) of the paper's score (Sec. 3.3.3, Eq. 1); the per-expert
 * token counts are one row of its expert-utilisation trace (Sec. 3.3.1).  The paper gives no
 * formulas for the layer itself; the ones used here are the standard ones: softmax over the k
 * selected router logits, SwiGLU experts  y = W2^T( silu(W1^T x) * (W3^T x) ).
 *
 * Conventions
 *   - Every tensor pointer is DEVICE memory owned by the caller, unless marked "host".
 *     The library allocates no device memory: its scratch is the workspace given to moe_create.
 *   - `stream` is a hipStream_t passed as void* (NULL = the default stream).  All calls enqueue
 *     work on it and return; none synchronises with the host.
 *   - bf16 tensors are passed as void*; they are row-major and 16-byte aligned.
 *   - Shapes: T tokens, d model width, f expert width, E experts seen by the router, k experts
 *     per token, experts [e_lo, e_lo+E_local) resident on this GPU.  d and f must be multiples
 *     of 64; 1 <= k <= min(E, 16); E <= 256; 1 <= E_local <= E.
 *   - Errors are return codes.  Arguments are validated on the host before any launch: a call that
 *     returns MOE_ERR_INVALID_ARG, MOE_ERR_UNSUPPORTED_SHAPE or MOE_ERR_WORKSPACE_TOO_SMALL has launched
 *     nothing.  MOE_ERR_DEVICE reports a HIP call that failed part-way; in a call of several stages
 *     (moe_permute, moe_grouped_ffn, moe_layer_forward) the stages enqueued before it still run, and the
 *     outputs are then undefined.  T == 0 is MOE_OK and a no-op.
 *   - Calls on one moe_ctx must not overlap in time (they share its workspace).  Counters of the router live in it
 *     from call to call: after calls that did overlap, later ones may count wrongly until the context is created anew.
 *   - The calls that take a stream only launch kernels on it (no memsets, no allocation, no host
 *     synchronisation), so they may be recorded under stream capture and replayed as a HIP graph; the
 *     exceptions are contexts created with MOE_FLAG_STAGE_EVENTS (they record events), moe_profile_ffn,
 *     moe_measure_mfma_rate(_of) and moe_measure_hbm_read_rate (they time and wait).
 */
#ifndef MOE_H_
#define MOE_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct moe_ctx moe_ctx; /* opaque, host memory */

typedef enum {
    MOE_OK = 0,
    MOE_ERR_INVALID_ARG = 1,        /* null / misaligned pointer, T out of range, ...          */
    MOE_ERR_UNSUPPORTED_SHAPE = 2,  /* shape outside the limits listed above                   */
    MOE_ERR_WORKSPACE_TOO_SMALL = 3,
    MOE_ERR_DEVICE = 4              /* a HIP call failed (launch error, wrong architecture)    */
} moe_status;

typedef struct {
    int32_t T_max;    /* largest T any call will pass                                          */
    int32_t d, f;     /* model width, expert FFN width                                         */
    int32_t E, k;     /* experts seen by the router, experts per token                         */
    int32_t e_lo;     /* first resident expert                                                 */
    int32_t E_local;  /* number of resident experts (== E: all of them)                        */
    uint32_t flags;   /* MOE_FLAG_*                                                            */
} moe_shape;

#define MOE_FLAG_STAGE_EVENTS 1u /* moe_layer_forward records HIP events around every stage   */

enum { MOE_STAGE_ROUTE = 0, MOE_STAGE_PERMUTE = 1, MOE_STAGE_GEMM1 = 2, MOE_STAGE_GEMM2 = 3,
       MOE_STAGE_COMBINE = 4, MOE_NUM_STAGES = 5 };

const char* moe_status_string(moe_status s);

/* Text of the most recent failing HIP call behind a MOE_ERR_DEVICE on this thread, or of a size limit that
 * a call without a context exceeded ("" if none).
 * The pointer stays valid; the text changes with the next device error. */
const char* moe_last_device_error(void);

/* Bytes of device workspace a context of this shape needs (0 if the shape is unsupported). */
size_t moe_workspace_bytes(const moe_shape* shape /* host */);

/* Creates a context over a caller-owned device workspace of at least moe_workspace_bytes().
 * The workspace must stay valid until moe_destroy.  Must be called with the target device
 * current; clears a few KB of the workspace with a blocking memset.  *ctx is NULL on error. */
moe_status moe_create(moe_ctx** ctx, const moe_shape* shape /* host */, void* workspace,
                      size_t workspace_bytes);
void moe_destroy(moe_ctx* ctx);

/* Number of rows the staged buffers (xp, y, tok_of) must hold for T tokens:
 * T * min(k, E_local), the largest possible number of local (token, expert) assignments. */
int64_t moe_rows_capacity(const moe_shape* shape /* host */, int32_t T);

/* ---- one-off, at model-load time (the analogue of loading each expert's weights onto its
 * assigned GPU, paper Sec. 3.3.4); not part of the layer latency ------------------------------ */

/* Router matrix Wg [d, E] fp32 row-major -> opaque packed form (two bf16 terms per weight, laid
 * out in the order the matrix-core operand fragments are loaded). */
size_t moe_packed_router_bytes(const moe_shape* shape /* host */);
moe_status moe_pack_router(moe_ctx* ctx, const float* Wg, void* router_packed, void* stream);

/* Expert weights W1, W3 [E_local, d, f] and W2 [E_local, f, d], bf16 row-major -> opaque packed
 * form (3 * E_local * d * f bf16 values: every 32-column x 16-reduction-element block stored as the
 * 1 KB matrix-core operand fragment one wavefront loads; W1 and W3 interleaved in blocks of 32
 * output columns so one accumulator tile holds both branches of the SwiGLU). */
size_t moe_packed_weight_bytes(const moe_shape* shape /* host */);
moe_status moe_pack_weights(moe_ctx* ctx, const void* W1, const void* W3, const void* W2,
                            void* packed, void* stream);

/* ---- the hot path ---------------------------------------------------------------------------- */

/* Router (paper Sec. 2.1: per-token choice of the k experts; Sec. 3.3.1: its output is the trace):
 *   logit[t,e] = sum_i x[t,i] * Wg[i,e] (+ bias[e]);  topk_idx[t,0..k) = the k largest, slot 0
 *   the largest, equal logits resolved to the lower expert index;  topk_w[t,j] = softmax over
 *   the k selected logits;  counts[e] = number of (t, j) with topk_idx[t,j] == e, over all E.
 * x [T, d] bf16; bias [E] fp32 or NULL; topk_idx [T, k] int32; topk_w [T, k] fp32;
 * counts [E] int32 (overwritten). */
moe_status moe_route(moe_ctx* ctx, const void* x, const void* router_packed, const float* bias,
                     int32_t T, int32_t* topk_idx, float* topk_w, int32_t* counts, void* stream);

/* Dispatch by expert (paper Sec. 2.1: each token goes to where its experts are hosted):
 *   offsets[e'] = number of assignments to resident experts before e_lo + e' (exclusive prefix
 *   sum, offsets[E_local] = number of local assignments);  the destination row of (t, j) with
 *   e = topk_idx[t,j] resident is row_of[t,j] = offsets[e-e_lo] + #{t' < t : t' selected e}
 *   (expert-contiguous, ascending token order inside an expert); row_of = -1 for non-resident
 *   experts;  tok_of[row] = t;  xp[row, :] = x[t, :].
 * xp [rows_capacity, d] bf16 or NULL (skip the row copy); offsets [E_local+1]; row_of [T, k];
 * tok_of [rows_capacity]. */
moe_status moe_permute(moe_ctx* ctx, const void* x, const int32_t* topk_idx, int32_t T, void* xp,
                       int32_t* offsets, int32_t* row_of, int32_t* tok_of, void* stream);

/* moe_permute for callers that can neither allocate device memory nor bring a workspace: code under HIP
 * graph capture, tight serving loops, harnesses that forbid hipMalloc.  No context: the shape comes as
 * arguments (d is only used for the row copy), the outputs are those of moe_permute, bit for bit.  The call
 * allocates nothing and frees nothing; its only scratch, the per-256-token-block expert histograms, is a
 * static device array of 1 MiB that every GPU the library runs on holds until the process ends.  Limit:
 * ceil(T / 256) * E_local <= 262144 entries (e.g. T = 2^20 with up to 64 resident experts, T = 262144 with
 * 256), otherwise MOE_ERR_WORKSPACE_TOO_SMALL with the sizes in moe_last_device_error(); T <= 2^20.  The array
 * keeps the previous call's contents (every entry a call reads it has written itself first), and calls that
 * overlap in time on one GPU share it and race: run them on one stream, or otherwise one after the other.
 * The first call on a device looks up the array's device address (no allocation, but do it outside a
 * stream capture). */
moe_status moe_permute_noalloc(const void* x, const int32_t* topk_idx, int32_t T, int32_t d, int32_t E,
                               int32_t k, int32_t e_lo, int32_t E_local, void* xp, int32_t* offsets,
                               int32_t* row_of, int32_t* tok_of, void* stream);

/* Expert FFN over expert-contiguous rows (the expert kernel the paper profiles in isolation, Sec. 3.3.2):
 *   for offsets[e'] <= r < offsets[e'+1]:
 *       y[r, :] = W2[e']^T ( silu(W1[e']^T xp[r]) * (W3[e']^T xp[r]) )
 *   bf16 operands, fp32 accumulation; the intermediate [rows, f] is stored as bf16 in the
 *   workspace.  Experts with no rows cost nothing and their weights are not read.
 * xp, y [n_rows_cap, d] bf16; offsets [E_local+1] (device; values are not read by the host);
 * n_rows_cap: host upper bound on offsets[E_local], at most moe_rows_capacity(shape, T_max).  The launches
 * are sized from it (the per-expert counts stay on the device), so a tight bound is cheaper than a loose
 * one; at low loads (up to 192 rows per expert on average) the second GEMM runs as several reduction
 * ranges whose fp32 partial sums are added in a fixed order.  The bound is checked on the device: if
 * offsets[E_local] exceeds n_rows_cap the call computes nothing (no row of y is written) and sets the flag
 * moe_ffn_refused_flag points to; the host cannot see that without reading the flag, the return code stays
 * MOE_OK. */
moe_status moe_grouped_ffn(moe_ctx* ctx, const void* xp, const int32_t* offsets,
                           int32_t n_rows_cap, const void* packed, void* y, void* stream);

/* Weighted return to token order (paper Sec. 7: tokens return to their origin):
 *   out[t, :] = sum_j topk_w[t,j] * y[row_of[t,j], :]   (slots with row_of < 0 contribute 0),
 *   summed in slot order in fp32, one write per output element, no atomics.
 * y [rows_capacity, d] bf16; out [T, d] bf16. */
moe_status moe_combine(moe_ctx* ctx, const void* y, const int32_t* row_of, const float* topk_w,
                       int32_t T, void* out, void* stream);

/* The whole layer on one stream with no host synchronisation: route, dispatch, experts, combine.
 * Intermediates live in the workspace; the row copy is folded into the first GEMM's operand load.
 * With E_local < E, `out` is this GPU's partial sum (tokens with no resident expert give 0).
 * counts_out [E] int32 or NULL. */
moe_status moe_layer_forward(moe_ctx* ctx, const void* x, const void* router_packed,
                             const float* bias, const void* packed, int32_t T, void* out,
                             int32_t* counts_out, void* stream);

/* ---- operators around the experts' weights: training them, and serving them in 4 bits --------------------------
 *
 * These calls need no context.  Pointers are device memory unless marked "host"; matrices are row-major with rows
 * `ld*` values apart (a multiple of 8 bf16 or 4 fp32 values, at most 2^21), every base pointer 16-byte aligned.
 * Widths (K, N, f) are multiples of 8 (K of 32 for 4-bit values), at most 2^17; E <= 256.  A call only launches
 * kernels on `stream`.  Tensors without rows may be NULL.  Outputs share no byte with inputs or with each other but where a call
 * says so (MOE_ERR_INVALID_ARG); views into the same wider rows, side by side, are no such case.  Workspaces share none with anything.
 *
 * Rows grouped by expert lie as moe_permute leaves them: expert e has rows [offsets[e], offsets[e+1]), offsets [E+1] is
 * read on the device, n_rows_cap (<= 2^24) is the host's bound on offsets[E] and sizes the launch.  Rows from offsets[E] on are
 * neither read nor written.  Offsets that do not ascend or pass the bound never lead out of [0, n_rows_cap). */

typedef enum { MOE_BF16 = 0, MOE_F32 = 1 } moe_type;

/* The grouped products take a workspace of at least the bytes that their *_workspace_bytes functions give for the same sizes (0: it may be
 * NULL; 64 MiB at the most): partial sums where a long reduction of few tiles, or of the last ones, is cut into ranges.  16-byte
 * aligned, used until the call's work is done; calls that may overlap need one each. */

/* y[r, :] = x[r, :] . W[e] for the rows r of every expert e: bf16 operands, fp32 sums, bf16 results rounded once.
 * W is [E, K, N] (transpose_w == 0; the layout of W1, W3 and W2) or [E, N, K] (transpose_w != 0: x times W[e]^T).  The
 * gradient of x is this call on the gradient of y with transpose_w the other way round.
 * x [n_rows_cap, K], y [n_rows_cap, N]. */
size_t moe_grouped_gemm_workspace_bytes(int32_t n_rows_cap, int32_t E, int32_t K, int32_t N, int32_t transpose_w);
moe_status moe_grouped_gemm(const void* x, int64_t ldx, const void* w, int32_t transpose_w, const int32_t* offsets,
                            int32_t n_rows_cap, int32_t E, int32_t K, int32_t N, void* y, int64_t ldy, void* workspace,
                            size_t workspace_bytes, void* stream);

/* Gradient of the weights: dw[e] = sum over the rows r of expert e of x[r, :]^T dy[r, :]  (fp32 sums in a fixed order).
 * dw [E, K, N] of `type` (moe_type); experts without rows get zeros.  accumulate != 0 (fp32 only): added to what dw
 * holds, experts without rows are left alone. */
size_t moe_grouped_gemm_wgrad_workspace_bytes(int32_t n_rows_cap, int32_t E, int32_t K, int32_t N);
moe_status moe_grouped_gemm_wgrad(const void* x, int64_t ldx, const void* dy, int64_t lddy, const int32_t* offsets,
                                  int32_t n_rows_cap, int32_t E, int32_t K, int32_t N, void* dw, int32_t type,
                                  int32_t accumulate, void* workspace, size_t workspace_bytes, void* stream);

/* h = silu(g) * u with g = gu[:, :f], u = gu[:, f:2f] (bf16).  n_rows: NULL, or the number of rows there are on the device
 * (e.g. offsets + E), at most n_rows_cap; later rows are left alone.  gu [n_rows_cap, 2f], h [n_rows_cap, f].  h may lie in the place of
 * g or of u. */
moe_status moe_swiglu(const void* gu, int64_t ldgu, const int32_t* n_rows, int32_t n_rows_cap, int32_t f, void* h,
                      int64_t ldh, void* stream);

/* Gradient of moe_swiglu: dgu[:, :f] = dh u s(g) (1 + g (1 - s(g))), dgu[:, f:] = dh g s(g), s the logistic function.
 * h NULL, or the rows of moe_swiglu formed again (a program then need not keep them).  dgu may be gu itself; each half of it, and h, may lie
 * in the place of dh, g or u. */
moe_status moe_swiglu_backward(const void* dh, int64_t lddh, const void* gu, int64_t ldgu, const int32_t* n_rows,
                               int32_t n_rows_cap, int32_t f, void* dgu, int64_t lddgu, void* h, int64_t ldh, void* stream);

/* Global norm of n gradients: norm[0] = sqrt(sum over tensors and values of g^2), squares added in 64 bits in a fixed order.
 * grads, counts, types: host arrays [n] of device pointers (aligned to their values), numbers of values and moe_type;
 * norm [1] fp32.  workspace: moe_grad_norm_workspace_bytes(n) bytes, 8-byte aligned, used until the call's work is done.
 * The host arrays are read before the call returns. */
size_t moe_grad_norm_workspace_bytes(int32_t n);
moe_status moe_grad_norm(const void* const* grads /* host */, const int64_t* counts /* host */, const int32_t* types /* host */,
                         int32_t n, void* workspace, size_t workspace_bytes, float* norm, void* stream);

/* The same norm, and outs[i] = scale * grads[i] with scale = min(1, max_norm / (norm + 1e-6)), of grads[i]'s type.  outs[i] is
 * grads[i] itself (in place: nothing is written where the scale is 1) or memory of its own.  A norm that is not a number
 * makes every value one; an infinite one gives 0 * g. */
moe_status moe_clip_grad_norm(const void* const* grads /* host */, void* const* outs /* host */, const int64_t* counts /* host */,
                              const int32_t* types /* host */, int32_t n, float max_norm, void* workspace, size_t workspace_bytes,
                              float* norm, void* stream);

/* Microscaled 4-bit floating point: blocks of 32 neighbouring values of a row share a scale 2^e,
 *   e = max(floor(log2(largest magnitude)) - 2, -127);  a value is 2^e times one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 with a sign,
 *   the nearest one, ties to the even code, at most 6.
 * values [rows, K/2]: two codes a byte, the lower index in the lower half (sign bit, then the magnitude's number 0..7);
 * scales [rows, moe_mxfp4_scale_cols(K)]: e + 127; 0 in blocks of zeros and behind the last block (the products rely on it),
 * 255 in a block that holds an infinity or a NaN: the whole block then stands for NaN. */
int32_t moe_mxfp4_scale_cols(int32_t K); /* K / 32 up to the next multiple of 16; 0: K is not supported */
moe_status moe_mxfp4_quantize(const void* x, int32_t type, int64_t ldx, const int32_t* n_rows, int32_t n_rows_cap, int32_t K,
                              void* values, void* scales, void* stream); /* n_rows as in moe_swiglu */

/* Weights W [E, K, N] bf16, once at load time: values [E, N, K/2], scales [E, N, scale_cols(K)], blocks along K. */
moe_status moe_mxfp4_quantize_weights(const void* w, int32_t E, int32_t K, int32_t N, void* values, void* scales, void* stream);

/* The values that rows of codes and scales stand for, in bf16 (exact). */
moe_status moe_mxfp4_dequantize(const void* values, const void* scales, int64_t rows, int32_t K, void* x, int64_t ldx,
                                void* stream);

/* y[r, :] = x[r, :] . W[e]^T on such operands: exact products, fp32 sums, bf16 results rounded once.
 * x_values [n_rows_cap, K/2], x_scales [n_rows_cap, scale_cols(K)], w_values [E, N, K/2], w_scales [E, N, scale_cols(K)]. */
size_t moe_mxfp4_grouped_gemm_workspace_bytes(int32_t n_rows_cap, int32_t E, int32_t K, int32_t N);
moe_status moe_mxfp4_grouped_gemm(const void* x_values, const void* x_scales, const void* w_values, const void* w_scales,
                                  const int32_t* offsets, int32_t n_rows_cap, int32_t E, int32_t K, int32_t N, void* y,
                                  int64_t ldy, void* workspace, size_t workspace_bytes, void* stream);

/* ---- norms around a block ------------------------------------------------------------------------------------------
 *
 * What stands before a layer and behind it on the residual stream.  Rows as above, at most 2^24 of them, d values wide: a multiple of
 * 8, at most 16384.  x_type: moe_type of the stream (x, out, their gradients); y_type: of what goes into a block and comes out of it (y, h,
 * gates of every value, their gradients), the same as x_type or bf16 beside an fp32 stream.  Weights [d] of w_type, all of a call
 * alike, 16-byte aligned; NULL: ones.  Gradients of weights [d] are fp32 sums in a fixed order.  n_rows as in moe_swiglu: later rows are left
 * alone and add nothing.  Sums over a row are in 32 bits (as in any such norm a row whose squares pass their range has the factor 0);
 * each result is rounded once.  A row that holds a NaN spoils that row and the weights' gradients, no other one.
 * Row-shaped outputs may each lie exactly in the place of a row-shaped input. */

/* h = x r w with r = 1 / sqrt(mean over the row of x^2 + eps).  eps >= 0.  h is of h_type (as y_type above). */
moe_status moe_rms_norm(const void* x, int32_t x_type, int64_t ldx, const void* w, int32_t w_type, float eps, const int32_t* n_rows,
                        int32_t n_rows_cap, int32_t d, void* h, int32_t h_type, int64_t ldh, void* stream);

/* Its gradient: dx = dres + r (p - x r^2 mean(p x)) with p = dh w, dw = sum over the rows of dh x r.  dres (of x_type): NULL, or the
 * gradient that x has by another way.  dw: NULL: not wanted.  workspace: moe_norm_backward_workspace_bytes bytes (the same for both
 * gradients below), 16-byte aligned, used until the call's work is done; NULL where no gradient of weights is wanted. */
size_t moe_norm_backward_workspace_bytes(int32_t n_rows_cap, int32_t d);
moe_status moe_rms_norm_backward(const void* dh, int32_t h_type, int64_t lddh, const void* x, int32_t x_type, int64_t ldx, const void* w,
                                 int32_t w_type, float eps, const void* dres, int64_t lddres, const int32_t* n_rows, int32_t n_rows_cap,
                                 int32_t d, void* dx, int64_t lddx, float* dw, void* workspace, size_t workspace_bytes, void* stream);

/* A block's end: n = y w, or y r_y w where norm != 0 (r_y of y's rows as above);  out = scale x + gate n;  h = out r_out w_next, the norm
 * of the block behind, taken before out is rounded.  gate: NULL (1); [n_rows_cap] fp32, a number for each row (ldgate 0); or
 * [n_rows_cap, d] of y_type (ldgate > 0).  h NULL: out alone. */
moe_status moe_residual_norm(const void* x, int32_t x_type, int64_t ldx, const void* y, int32_t y_type, int64_t ldy, const void* w,
                             int32_t w_type, int32_t norm, const void* gate, int64_t ldgate, float scale, const void* w_next, float eps,
                             const int32_t* n_rows, int32_t n_rows_cap, int32_t d, void* out, int64_t ldout, void* h, int64_t ldh,
                             void* stream);

/* Its gradients, of out (dout, x_type; NULL: zeros) and of h (dh, y_type; NULL: h was not asked for, out is then not read):
 *   D = dout + r (p - out r^2 mean(p out)) with p = dh w_next and r of out's rows;  dx = scale D;
 *   dn = gate D;  dy = r_y (q - y r_y^2 mean(q y)) with q = dn w (without a norm: dy = q);  dgate = D n, summed over the row where the gate
 *   is the row's;  dw = sum over the rows of dn y r_y;  dw_next = sum of dh out r.
 * dgate (as gate, fp32 [n_rows_cap] or y_type with rows lddgate apart), dw, dw_next: NULL: not wanted. */
moe_status moe_residual_norm_backward(const void* dout, int64_t lddout, const void* dh, int64_t lddh, const void* out, int32_t x_type,
                                      int64_t ldout, const void* y, int32_t y_type, int64_t ldy, const void* w, int32_t w_type, int32_t norm,
                                      const void* gate, int64_t ldgate, float scale, const void* w_next, float eps, const int32_t* n_rows,
                                      int32_t n_rows_cap, int32_t d, void* dx, int64_t lddx, void* dy, int64_t lddy, void* dgate,
                                      int64_t lddgate, float* dw, float* dw_next, void* workspace, size_t workspace_bytes, void* stream);

/* ---- orthogonalised updates ------------------------------------------------------------------------------------------
 *
 * Each matrix of a stack g [E, rows, cols] brought near the orthogonal matrix next to it (the same singular vectors, singular values near 1):
 *   X = g / (|g| + eps), |g| the root of the sum of its squares;  for (a, b, c) of each step:  S = X X^T,  X = a X + (b S + c S S) X;
 *   out = scale X
 * (where rows > cols: the same on the transpose).  coefficients: host, [steps][3], read before the call returns; steps from 1 to 64.
 * Operands of the products are kept in one or two 16-bit parts (22 bits), sums in 32 bits, |g| in 64.  With a not far below b and c an fp32 result is about as
 * far from the exact one as with products in 32 bits (where |g| is far below eps, and the steps next to a mere factor, 6 10^-7 of its norm at most), a bf16 result
 * 1 to 1.4 times as far as its own rounding (up to 2.5 after steps whose slope is large where singular values come to lie: such schedules are better damped).
 * |a| is at most 4000, |b| and |c| 10^6.  The parts' scales follow from bounds that hold for any matrix: |X| begins at 1, and a s + b s^3 + c s^5 bounds what a
 * step makes of it.  Steps whose bounds of the singular values before each step stay below 16, and of a + b s^2 + c s^4 below 4000, never leave their range
 * (the usual schedules: 2 and 9); with others a matrix whose own singular values do gives NaN or infinities.  One that holds a NaN or an infinity gives NaN.
 * Neither spoils another.  A matrix of zeros gives zeros (eps > 0).
 * g and out: rows ldg / ldout values apart (at least cols), matrices stride_g / stride_out values apart, pointers aligned to their values; any
 * sizes from 1 to 2^17, rows * cols <= 2^29, E <= 256.  out may be exactly g (of the same type); otherwise they share no byte.
 * workspace: moe_orthogonalize_workspace_bytes bytes, 256-byte aligned, used until the call's work is done.  Matrices are kept padded: the smaller side to
 * 32, 64 or 128, from 129 on to a multiple of 256 at most; the larger to a multiple of 64, from 129 of the smaller on of 256 at most, and 32 more.  It takes 8 bytes for every
 * value of these, 12 for those of a square of the smaller side (by itself and 32 more), 8 for each row and 4112 a matrix, and up to 64 MiB for sums: of a
 * row of 131072 256 bytes a value, of 4096 x 14336 12.  At most 8 GiB (or what one matrix needs): larger stacks are gone through in turns.  0: sizes that are
 * refused. */
size_t moe_orthogonalize_workspace_bytes(int32_t E, int32_t rows, int32_t cols);
moe_status moe_orthogonalize(const void* g, int32_t type, int64_t stride_g, int64_t ldg, int32_t E, int32_t rows, int32_t cols,
                             const float* coefficients /* host */, int32_t steps, float eps, float scale, void* out, int32_t out_type,
                             int64_t stride_out, int64_t ldout, void* workspace, size_t workspace_bytes, void* stream);

/* ---- introspection --------------------------------------------------------------------------- */

/* Mean milliseconds of each stage over the moe_layer_forward calls made since the previous
 * read-out (at most the 64 most recent) on a context created with MOE_FLAG_STAGE_EVENTS.
 * Blocks until the last of those calls has completed.  ms: host, MOE_NUM_STAGES floats. */
moe_status moe_stage_times(moe_ctx* ctx, float* ms /* host */);

/* Largest token-tile height of the expert GEMMs for this shape.  An expert's rows are cut into
 * ceil(n / height) tiles of nearly equal height (multiples of 32 rows); the work per tile grows in
 * steps of 32 rows, which sets the staircase of the latency-vs-load curve (the
 * paper's tile boundaries, Sec. 3.3.2). */
int32_t moe_tile_rows(const moe_ctx* ctx);

/* Variability-profiling microbenchmark (paper Sec. 3.3.2, "Step-2"): launches the isolated expert
 * kernels (moe_grouped_ffn: GEMM1 + SwiGLU + GEMM2) on synthetic rows at each target token count
 * and records the average latency -- one sample of this GPU's token-vs-latency curve C_g(n) per
 * count.  For point i, token_counts[i] rows of xp are spread evenly over the E_local resident
 * experts (the first token_counts[i] % E_local experts get one more), the kernels are launched
 * warmup + iters times on `stream`, and ms[i] = mean milliseconds per launch over the timed ones
 * (HIP events on `stream`).  xp and y: device, at least max(token_counts) rows of d bf16 values each;
 * token_counts and ms: host, n_points entries; every count <= moe_rows_capacity(shape, T_max).
 * Unlike the hot-path calls this one BLOCKS until the measurements are done, and it overwrites the
 * context's offsets scratch. */
moe_status moe_profile_ffn(moe_ctx* ctx, const void* xp, const void* packed, void* y,
                           const int32_t* token_counts /* host */, int32_t n_points, int32_t warmup,
                           int32_t iters, float* ms /* host */, void* stream);

/* ---- host-side steps (everything below up to moe_gem_place takes HOST pointers and runs on the CPU, as in
 * the paper; the inputs are what the GPU path produces) ------------------------------------------------- */

/* Sampling plan of the variability profiler (paper Sec. 3.3.2, Step-2: latency jumps at tile boundaries,
 * so sample there; sample sparsely at high counts).  Token counts to measure, ascending, no duplicates:
 * 1; every multiple m*boundary up to min(dense_max, n_max) together with m*boundary + after (the first
 * count at which the jump is complete) where that is <= n_max; then every sparse_step tokens from the last
 * dense boundary on, below n_max; and n_max.  Requires boundary, sparse_step, n_max >= 1,
 * 1 <= after <= boundary, dense_max >= 0.  *n_out = number of counts; with cap == 0 nothing is written (size
 * query); cap < *n_out gives MOE_ERR_WORKSPACE_TOO_SMALL. */
moe_status moe_curve_sample_counts(int32_t boundary, int32_t dense_max, int32_t n_max, int32_t sparse_step,
                                   int32_t after, int32_t* counts_out /* [cap] */, int32_t cap, int32_t* n_out);

/* The curve C_g(n) rebuilt from n_samples measured points (counts strictly ascending, ms their latencies;
 * Sec. 3.3.2: linear interpolation between samples): ms_out[i] = latency at tokens[i] tokens = the straight
 * line between the neighbouring samples, the first sample's value below it, the last one's above it, 0 for
 * tokens <= 0.  The mapping search (moe_gem_*) reads its curves the same way. */
moe_status moe_curve_eval(const int32_t* counts, const double* ms, int32_t n_samples, const int32_t* tokens,
                          int32_t n_tokens, double* ms_out /* [n_tokens] */);

/* Sum of C_g(n) over n_lo <= n <= n_hi: the kernel time a sweep of every token count would cost, for the
 * comparison with the sampled profile (Sec. 4.6 of the paper reports that ratio). */
moe_status moe_curve_sum(const int32_t* counts, const double* ms, int32_t n_samples, int32_t n_lo, int32_t n_hi,
                         double* sum_out);

/* Statistics of the expert-utilisation trace (paper Sec. 3.3.1, Step-1; Sec. 3.2): trace[t*E + e] = tokens
 * routed to expert e at step t.  u_out[e] = mean over the S steps.  r_out[a*E + b] = Pearson correlation
 * coefficient of the loads of experts a and b across the steps (NaN if either load is constant). */
moe_status moe_trace_mean_utilisation(const int32_t* trace, int32_t S, int32_t E, double* u_out /* [E] */);
moe_status moe_trace_correlation(const int32_t* trace, int32_t S, int32_t E, double* r_out /* [E*E] */);

/* Mapping search (paper Sec. 3.3.3 "Step-3", Eq. 1; appendix algorithms for the initial mapping, the
 * refinement and the restarts).  trace as above (the counts_out rows of S consecutive calls); one
 * token-vs-latency curve per GPU (moe_profile_ffn samples): GPU g's samples are curve_counts / curve_ms
 * [curve_offsets[g], curve_offsets[g+1]), token counts strictly ascending, read as in moe_curve_eval.
 * E must be a multiple of G: every GPU hosts E / G experts.  mapping[e] = GPU of expert e. */

/* S(M) = sum over steps of max over GPUs of C_g(tokens routed to GPU g at that step)  (Eq. 1). */
moe_status moe_gem_score(const int32_t* trace, int32_t S, int32_t E, int32_t G, const int32_t* curve_counts,
                         const float* curve_ms, const int32_t* curve_offsets /* [G+1] */,
                         const int32_t* mapping /* [E] */, double* score_out);

/* K restarts of: greedy initial mapping (experts by mean utilisation, heaviest first, each on the
 * GPU with a free slot that gives the lowest score of the partial mapping; restart i > 0 sorts by
 * u_e * (1 + 0.2 * noise[i*E + e]), noise in [-1, 1) drawn by the caller), then repeated best
 * cross-GPU swap until the best swap lowers the score by less than 0.1 %.  Returns the
 * lowest-scoring mapping, its score and (optionally) the number of swaps its refinement took.
 * noise may be NULL when K == 1.  Ties go to the lower expert / GPU index and the first pair. */
moe_status moe_gem_place(const int32_t* trace, int32_t S, int32_t E, int32_t G, const int32_t* curve_counts,
                         const float* curve_ms, const int32_t* curve_offsets /* [G+1] */,
                         const float* noise /* [K][E] */, int32_t K, int32_t* mapping_out /* [E] */,
                         double* score_out, int32_t* swaps_out /* or NULL */);

/* Tuning hook: force the token-tile class of the expert GEMMs (1: row tiles of up to 288 rows, the main
 * class; 5: the class of decode-sized loads -- two wavefronts per workgroup, 128 weight rows and up to 64
 * token rows per work item, four workgroups to a compute unit; 0: up to 128 rows; 2, 3, 4: row tiles of up to
 * 64, 32, 256 rows, kept for tuning runs (4 on the kernel of class 1); -1: choose from the expected rows per
 * expert and the work items of the launches, the default: class 0 below 12 rows per expert, class 5 up to 24,
 * class 1 above; up to 4 rows class 5 where the first GEMM has few work items; from 12 to 24 rows class 0 or 1
 * where both GEMMs fill the device). */
moe_status moe_set_tile_class(moe_ctx* ctx, int32_t tile_class);

/* Measurement aid for roofline reports: the bf16 matrix-core rate this device SUSTAINS under a load of
 * nothing but v_mfma_f32_16x16x32_bf16 (the instruction the grouped GEMM issues) on changing pseudo-random
 * operands (no memory traffic, every SIMD of every compute unit busy, independent accumulators), in
 * TFLOP/s.  The published peak assumes the maximum clock; under a dense MFMA load the chip runs at the clock
 * its power limit allows.  Runs `launches` >= 1 launches of iters_per_wave * 128 MFMAs per wavefront on
 * `stream`, times them with events and waits for them.
 * tflops: host pointer.  Errors: MOE_ERR_INVALID_ARG, MOE_ERR_DEVICE. */
moe_status moe_measure_mfma_rate(int32_t iters_per_wave, int32_t launches, float* tflops /* host */, void* stream);
/* The same measurement on a chosen instruction shape: 0 = v_mfma_f32_32x32x16_bf16 (half as many instructions
 * for the same flop), 1 = v_mfma_f32_16x16x32_bf16 (identical to moe_measure_mfma_rate).  Under the power limit
 * the sustained rate depends on the shape.  Errors as above. */
moe_status moe_measure_mfma_rate_of(int32_t shape, int32_t iters_per_wave, int32_t launches,
                                    float* tflops /* host */, void* stream);

/* Measurement aid for roofline reports: the rate at which this device streams `bytes` bytes (>= 16; the tail
 * below a multiple of 16 is not read) of the device buffer `buf` (16-byte aligned, only read) through a
 * read-only kernel whose threads keep eight 16-byte loads in flight, with plain loads (nontemporal == 0) or
 * with the non-temporal hint the weight-streaming kernels use, in GB/s.  What a memory-bound kernel can
 * reach lies below the published 8 TB/s; this is the reference the weight-streaming launches are held
 * against.  Runs one warm-up launch and `launches` >= 1 timed ones on `stream` and waits for them.
 * gb_per_s: host pointer.  Errors: MOE_ERR_INVALID_ARG, MOE_ERR_DEVICE. */
moe_status moe_measure_hbm_read_rate(const void* buf /* device */, size_t bytes, int32_t nontemporal,
                                     int32_t launches, float* gb_per_s /* host */, void* stream);

/* Device pointer (into the workspace) to an int32 that the most recent moe_grouped_ffn / moe_layer_forward /
 * moe_profile_ffn call on this context set to 1 if it refused its offsets (offsets[E_local] above the host's
 * row bound; nothing was computed) and to 0 otherwise. */
moe_status moe_ffn_refused_flag(moe_ctx* ctx, const int32_t** flag);

/* Device pointers into the workspace holding the intermediates of the most recent
 * moe_layer_forward: topk_idx [T,k], topk_w [T,k], offsets [E_local+1], row_of [T,k]. */
moe_status moe_layer_intermediates(moe_ctx* ctx, const int32_t** topk_idx, const float** topk_w,
                                   const int32_t** offsets, const int32_t** row_of);

#ifdef __cplusplus
}
#endif
#endif /* MOE_H_ */
