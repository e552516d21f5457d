/*
 * entmax_attn.h - C ABI of the MI355X (gfx950) alpha-entmax attention library.
 *
 * The library computes, per (batch, head) and per query row r (AdaSplash-2 paper):
 *     S = Q K^T / sqrt(d)                                              (Eq. 2)
 *     P = [(alpha-1) S - tau]_+^{1/(alpha-1)},  sum_j P_rj = 1          (Eq. 3, Eq. 4)
 *     O = P V                                                          (Eq. 2)
 * with tau solved per row from an on-chip histogram of the scores within one unit of the row
 * maximum (Eq. 6-9, Prop. 1) followed by a safeguarded Halley/Newton refinement (Sec. 3.1-3.3,
 * Alg. 1) whose evaluations of f run over the row's candidate scores, listed during the one dense
 * sweep of Q K^T, and the gradient of
 * sum(O * dO) with respect to Q, K, V (Sec. 3.3 "Backward pass", Alg. 2-3).  Key tiles
 * whose probabilities are all zero are recorded in a bit-packed block mask (App. C.4) and
 * skipped in the output phase and in both backward kernels.
 *
 * Conventions common to every entry point
 *   - All tensor arguments are DEVICE pointers owned by the caller.  Tensors are
 *     contiguous [B, H, N, d] with d fastest.  Inputs Q, K, V, dO have the element type
 *     named by `dtype`; O, dQ, dK, dV, tau are always float32.
 *   - N must be a positive multiple of 64 and at most 131072; d must be 64 or 128;
 *     1 < alpha <= EA_ALPHA_MAX.  With bf16 inputs, values of magnitude above 65504 are outside the
 *     library's domain (second-stage products run on fp16 copies): they enter those copies as
 *     +-65504 and are counted in EA_STAT_F16_CLAMPED.
 *   - Causal masking: key j is visible to query r iff j <= r.
 *   - The library allocates nothing and never synchronises: all work is enqueued on
 *     `hip_stream` (a hipStream_t passed as void*; NULL = the default stream).  Scratch
 *     space is the caller's `workspace` (device memory, 256-byte aligned), of at least
 *     entmax_attn_workspace_bytes(...) bytes.
 *   - Return value: EA_OK (0) on success.  On any negative code nothing has been
 *     enqueued, except EA_ERR_HIP where earlier launches of the same call may have been.
 *   - Calls that share a workspace must be ordered on one stream.
 */
#ifndef ENTMAX_ATTN_H
#define ENTMAX_ATTN_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* Element type of Q, K, V, dO.  Entry points take it as a plain int (any other value is answered
 * with EA_ERR_DTYPE, or a size of 0). */
typedef enum { EA_F32 = 0, EA_BF16 = 1 } ea_dtype;

/* Largest alpha accepted.  Sec. 3.2 covers every alpha > 1 (secant steps above 2); the bound keeps
 * the backward's U = P^(2-alpha) = y^(1/(alpha-1) - 1), which grows without limit as a probability
 * approaches zero once alpha > 2, inside the range of the fp16 operands of the second-stage
 * products: with alpha <= 3 the exponent is at least -1/2. */
#define EA_ALPHA_MAX 3.0f

enum {
    EA_OK = 0,
    EA_ERR_NULL = -1,       /* a required pointer is NULL */
    EA_ERR_ALPHA = -2,      /* alpha not finite or outside (1, EA_ALPHA_MAX] */
    EA_ERR_SHAPE = -3,      /* B, H <= 0, N not a positive multiple of 64 or > 131072, d not in {64, 128} */
    EA_ERR_DTYPE = -4,      /* unknown ea_dtype */
    EA_ERR_WORKSPACE = -5,  /* workspace NULL, misaligned or too small */
    EA_ERR_HIP = -6,        /* a HIP call failed; see entmax_attn_last_hip_error() */
    EA_ERR_TOO_LARGE = -7,  /* the problem needs more scratch than an allocation-free entry point holds */
    EA_ERR_LAYOUT = -8      /* a pointer or stride is not a multiple of 16 bytes, a stride is negative, or rows that are written overlap */
};

/* The workspace starts with EA_STATS_COPIES copies of EA_STATS_WORDS 64-bit counters
 * ([copy][counter]); the value of a counter is the sum over the copies (see entmax_attn_fwd). */
#define EA_STATS_WORDS 16
#define EA_STATS_COPIES 64
enum {
    /* units: 64x32 score sub-tiles (64 streamed rows x 32 register-resident rows), the piece one
     * wavefront computes per MFMA block pair; one matmul on a sub-tile is 2*64*32*d flops */
    EA_STAT_TAU_TILES = 0,   /* sub-tiles scored by the dense threshold sweep and by any sweep-based refinement (1 matmul each) */
    EA_STAT_OUT_TILES = 1,   /* sub-tiles scored by the output phase (2 matmuls each where P != 0) */
    EA_STAT_DELTA_TILES = 2, /* unused (delta is found inside the dQ sweep) */
    EA_STAT_DQ_TILES = 3,    /* sub-tiles visited by the dQ kernel (4 matmuls each) */
    EA_STAT_DKDV_TILES = 4,  /* sub-tiles visited by the dK/dV kernel (4 matmuls each) */
    EA_STAT_SWEEPS = 5,      /* work-groups that ran the sweep-based threshold kernel (each runs one refinement sweep) */
    EA_STAT_MASK_TILES = 6,  /* sub-tiles scored when the backward rebuilds the mask (1 matmul each) */
    EA_STAT_OUT_PV_TILES = 7, /* sub-tiles of the output phase whose P V product was issued */
    EA_STAT_LIST_OVERFLOW = 8, /* 64-row blocks whose candidate lists overflowed (redone by the sweep-based kernel) */
    EA_STAT_GATHER_ROWS = 9,  /* rows whose output was gathered from their listed support (no output-phase matmuls) */
    EA_STAT_BWD_LIST_TILES = 10, /* sub-tiles scored when the backward lists the supports of sparse row groups (1 matmul each) */
    EA_STAT_BWD_GATHER_ROWS = 11, /* rows whose gradients were formed entry by entry from their listed support */
    EA_STAT_F16_CLAMPED = 12  /* bf16 input values of magnitude above 65504 that were copied as +-65504 into the fp16 operands of the matrix kernels: non-zero means the inputs were outside the library's domain */
};

/* Edge of the square score tiles that one bit of the block mask stands for (64). */
int entmax_attn_mask_tile(void);

/* Bytes of workspace needed by entmax_attn_fwd (is_bwd == 0) or entmax_attn_bwd
 * (is_bwd != 0) for this problem; 0 if the shape or dtype is invalid. */
size_t entmax_attn_workspace_bytes(int B, int H, int N, int d, int dtype, int causal, int is_bwd);

/*
 * Forward (Alg. 1): row maximum, histogram and candidate lists (one dense sweep) -> histogram
 * solve and refinement on the lists (+ working mask) -> output, whose row sums check f once more.
 * A 64-row block with a row that has more candidates than its two lists hold (256 each, one per
 * half of the lanes that computed its scores) is redone by the sweep-based threshold kernel.
 *   Q, K, V     in   [B,H,N,d] of `dtype`
 *   O           out  [B,H,N,d] float32
 *   tau         out  [B,H,N]   float32, raw convention: P = [(alpha-1) S - tau]_+^{1/(alpha-1)}
 *   block_mask  out  [B,H,N/64,ceil(N/64/32)] int32; bit k of word m of row i is set iff some
 *                    P > 0 (at the returned tau) in the 64x64 tile (i, 32m+k) (App. C.4);
 *                    bits of tiles above the causal diagonal and padding bits are 0
 *   iters       out  [B,H,N] int32, may be NULL: number of refinement iterations the row
 *                    needed; one iteration = one evaluation of f over the true scores followed
 *                    by one update (Sec. 3.3 Phase 3); the check that the output phase gets
 *                    from its row sums counts only where it moved tau
 * The first EA_STATS_COPIES * EA_STATS_WORDS uint64 of `workspace` are zeroed by the call and
 * then hold the executed-tile counters of this call (EA_STAT_*, summed over the copies),
 * readable after the stream has drained.
 */
int entmax_attn_fwd(const void* Q, const void* K, const void* V,
                    float* O, float* tau, int32_t* block_mask, int32_t* iters,
                    int B, int H, int N, int d, int dtype, float alpha, int causal,
                    void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * Backward (Alg. 2-3): dQ kernel (which also finds delta) over mask rows, dK/dV kernel over mask columns.
 *   Q, K, V, dO in   [B,H,N,d] of `dtype`
 *   O           in   [B,H,N,d] float32, the forward's output; used only to centre the dQ sums
 *                    (<dO_r, O_r> is subtracted from dP before rounding); may be NULL, at the price
 *                    of extra rounding error in dQ when dP is large and nearly constant on a row's support
 *   tau         in   [B,H,N] float32 as returned by the forward
 *   block_mask  in   as returned by the forward, or NULL: then it is rebuilt from tau with one
 *                    dense score sweep
 *   dQ, dK, dV  out  [B,H,N,d] float32, overwritten
 * Counters as for the forward.
 */
int entmax_attn_bwd(const void* Q, const void* K, const void* V, const void* O, const void* dO,
                    const float* tau, const int32_t* block_mask,
                    float* dQ, float* dK, float* dV,
                    int B, int H, int N, int d, int dtype, float alpha, int causal,
                    void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * entmax_attn_bwd for a caller that still holds the forward call's workspace.  The forward leaves,
 * for every row group whose output it formed from listed supports, each row's support (raw score
 * and key index) at the front of its candidate lists; with them the backward need not find the
 * supports again (one score sweep over the marked tiles less).  Results as entmax_attn_bwd.
 *   fwd_workspace  in  the workspace of the entmax_attn_fwd call (same Q, K, V, shape, dtype, alpha,
 *                      causal) that produced O, tau and block_mask, not written to since; at least
 *                      entmax_attn_workspace_bytes(..., is_bwd = 0) bytes, 256-byte aligned.  The
 *                      backward reads it and leaves it as it found it.
 *   block_mask     in  required here (the forward's).
 * EA_ERR_NULL if fwd_workspace is NULL, EA_ERR_WORKSPACE if it is misaligned or too small or the mask
 * is missing.  Handing over a workspace that does not belong to these tensors gives wrong gradients
 * (or reads of rows that do not exist): the library cannot tell.
 */
int entmax_attn_bwd_with_lists(const void* Q, const void* K, const void* V, const void* O, const void* dO,
                               const float* tau, const int32_t* block_mask,
                               void* fwd_workspace, size_t fwd_workspace_bytes,
                               float* dQ, float* dK, float* dV,
                               int B, int H, int N, int d, int dtype, float alpha, int causal,
                               void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * Right-edge binning (Sec. 3.2, the paragraph after Prop. 1): an approximate forward.  Rounding
 * every score up to its bin's right edge instead of down to the left one moves the histogram's root
 * up by one bin width h = 1/63, to tau_h + h >= tau*.  With the switch on, entmax_attn_fwd (and the
 * per-head variant) takes that root as the threshold and does no refinement: `tau` holds it
 * (tau* <= tau < tau* + h + 2e-6 (1 + |tau|)), P = [(alpha-1) S - tau]_+^{1/(alpha-1)} has a support
 * inside the exact one and rows that sum to at most 1, O = P V, `block_mask` is P's.  Sparser and
 * cheaper than the exact result, not equal to it.  entmax_attn_bwd on these outputs evaluates the
 * formulas of Sec. 3.3 at that tau; they are the gradient only for the exact threshold.
 * The switch belongs to the calling host thread (off at its start) and applies to the forward calls
 * that thread makes after it; entmax_attn_decode is not affected.  Returns EA_OK.
 */
int entmax_attn_right_edge_enable(int on);

/*
 * The same two operations with one alpha per head (Sec. 3.2 gives the solver for every alpha
 * above 1; heads of one layer may use different values).  `alpha_per_head` is a HOST pointer to H
 * floats, each in (1, 2]; it is read before the call returns.  Head h of every batch entry uses
 * alpha_per_head[h].  When the values differ, all heads run the general-alpha code (power functions
 * through exp2/log2) and a table of per-head constants is written into the workspace first; when
 * they are all equal the call is the single-alpha one.  Everything else as in entmax_attn_fwd /
 * entmax_attn_bwd; EA_ERR_ALPHA if any value is outside (1, EA_ALPHA_MAX].
 */
int entmax_attn_fwd_alpha_per_head(const void* Q, const void* K, const void* V,
                                   float* O, float* tau, int32_t* block_mask, int32_t* iters,
                                   int B, int H, int N, int d, int dtype, const float* alpha_per_head, int causal,
                                   void* workspace, size_t workspace_bytes, void* hip_stream);
int entmax_attn_bwd_alpha_per_head(const void* Q, const void* K, const void* V, const void* O, const void* dO,
                                   const float* tau, const int32_t* block_mask,
                                   float* dQ, float* dK, float* dV,
                                   int B, int H, int N, int d, int dtype, const float* alpha_per_head, int causal,
                                   void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * Inference variant on materialised logits (the paper's appendix on language modelling; Sec. 5
 * names an optimised inference kernel as future work): one query row per head against all N
 * cached keys, no causal mask.
 *     z = K q / sqrt(d),  p = [(alpha-1) z - tau]_+^{1/(alpha-1)} with sum p = 1,  o = p V
 *   q           in   [B,H,d] of `dtype`
 *   K, V        in   [B,H,N,d] of `dtype`; any N in 1 .. 4194304, d 64 or 128
 *   O           out  [B,H,d] float32
 *   tau         out  [B,H]   float32, raw convention as in entmax_attn_fwd
 *   support     out  [B,H]   int32, may be NULL: number of keys with p > 0
 *   iters       out  [B,H]   int32, may be NULL: evaluations of f the refinement took
 * A first kernel reads K once and keeps, per work-group, only the logits within the window of Eq. 5
 * below the largest logit it has met so far (value and key index, in per-group lists in the workspace)
 * and its own maximum; a second kernel solves tau per head from the kept logits (histogram of the
 * scores within one unit of the maximum, Eq. 5-9, then the hybrid refinement of Sec. 3.2) and gathers
 * the rows of V in the support.  Conventions, error
 * codes and workspace rules as above; entmax_attn_decode_workspace_bytes returns 0 for a bad shape.
 */
size_t entmax_attn_decode_workspace_bytes(int B, int H, int N, int d, int dtype);
int entmax_attn_decode(const void* q, const void* K, const void* V,
                       float* O, float* tau, int32_t* support, int32_t* iters,
                       int B, int H, int N, int d, int dtype, float alpha,
                       void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * entmax_attn_decode for callers that cannot allocate device memory or pass a workspace: code under
 * HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.  Same inputs, outputs,
 * kernels and results as entmax_attn_decode; the scratch (per-group maxima and counts, kept logits)
 * is an array inside the library's code object, entmax_attn_decode_static_max_bytes() bytes
 * (33 MiB) per GPU, held until the process ends; its device address is looked up on the first call
 * on each device.  The call allocates and frees nothing and clears nothing (the kernels write every
 * scratch word before they read it).
 *   - EA_ERR_TOO_LARGE, nothing enqueued, when entmax_attn_decode_workspace_bytes(B, H, N, d, dtype)
 *     exceeds entmax_attn_decode_static_max_bytes() (about B*H*N <= 4 Mi keys, e.g. 32 heads x 128k).
 *   - All calls on one GPU share that GPU's array: calls that overlap on one GPU (different streams
 *     without ordering, or several host threads) race.  Order them on one stream.
 */
size_t entmax_attn_decode_static_max_bytes(void);
int entmax_attn_decode_static(const void* q, const void* K, const void* V,
                              float* O, float* tau, int32_t* support, int32_t* iters,
                              int B, int H, int N, int d, int dtype, float alpha, void* hip_stream);

/*
 * Queries and keys in the attention's layout, from what a layer's projections give: the RMS norm
 * of each head's row and its rotation by the token's position, in one pass.  With Hq = Hk and N a multiple of 64 they are what
 * entmax_attn_fwd takes; with other N and fewer key heads than query heads, what the 4-bit cache and the decode from it take (below).
 *     y = w x / sqrt(mean(x^2) + eps)                               (norm != 0; else y = x)
 *     (a, b) -> (a cos t - b sin t, a sin t + b cos t),   t = position[axis(i)] * inv_freq[i]
 * for the pairs i = 0 .. rot/2 - 1 of the row's first `rot` elements: (i, i + rot/2), or the neighbours
 * (2i, 2i + 1) if `interleaved`; elements from `rot` on are not rotated.  Pairs are dealt to n_axes position
 * axes in order: the first sections[0] pairs turn with the first axis, the next sections[1] with the
 * second, and so on (text: one axis; images and video: height and width, or time, height and width).
 *   q, k        in   [B,N,Hq,d], [B,N,Hk,d] of `dtype`, elements of a row contiguous; q_strides, k_strides: HOST
 *                    pointers to three strides each (batch, token, head), in elements, not negative; 0
 *                    repeats a row.  Views of one projection's rows are what they are for.
 *   q_out, k_out out [B,Hq,N,d], [B,Hk,N,d] of `dtype`, contiguous (N = 1: what entmax_attn_decode takes as q)
 *   q_weight, k_weight in [d] float32, may be NULL (ones); they go with norm != 0
 *   positions   in   [n_axes,B,N] int32, any value;  inv_freq in [rot/2] float32 (both unused if rot = 0)
 *   sections    in   HOST pointer to n_axes pair counts that sum to rot/2; may be NULL for one axis
 * Angles are formed in 64 bits from the int32 position and the float32 frequency; everything else is in float32
 * (a row whose squares add up to 2^128 or more is normed to zeros), rounded once to `dtype`.  B N <= 2^27, d 64 or 128, rot a multiple of 8 (0 .. d), at most 4 axes, eps > 0.
 * EA_ERR_LAYOUT if q, k, an output, a weight or a stride is not a multiple of 16 bytes.
 *
 * entmax_attn_qk_norm_rope_bwd: the gradient.  It takes dQ, dK as entmax_attn_bwd returns them, where the shape is one of
 * entmax_attn_fwd's; from any other attention, dQ and dK summed over the query heads that share a key head.
 *   dq_out, dk_out in [B,Hq,N,d], [B,Hk,N,d] float32, contiguous
 *   dq, dk      out  like q, k, of `dtype`, with strides of their own (rows must not overlap); for an input whose rows
 *                    repeat (stride 0) they hold the gradient of each use
 *   dq_weight, dk_weight out [d] float32, overwritten; NULL where not wanted
 *   workspace        entmax_attn_qk_norm_rope_workspace_bytes(d) bytes, 256-byte aligned; may be NULL if no
 *                    weight gradient is wanted
 * Results repeat bit for bit.  No output may overlap an input.
 */
int entmax_attn_qk_norm_rope_fwd(const void* q, const void* k, void* q_out, void* k_out,
                                 const int64_t* q_strides, const int64_t* k_strides,
                                 const float* q_weight, const float* k_weight, const int32_t* positions, const float* inv_freq,
                                 int B, int Hq, int Hk, int N, int d, int dtype,
                                 int rot, int n_axes, const int* sections, int interleaved, int norm, float eps, void* hip_stream);
size_t entmax_attn_qk_norm_rope_workspace_bytes(int d);
int entmax_attn_qk_norm_rope_bwd(const void* q, const void* k, const float* dq_out, const float* dk_out, void* dq, void* dk,
                                 const int64_t* q_strides, const int64_t* k_strides, const int64_t* dq_strides, const int64_t* dk_strides,
                                 const float* q_weight, const float* k_weight, const int32_t* positions, const float* inv_freq,
                                 float* dq_weight, float* dk_weight,
                                 int B, int Hq, int Hk, int N, int d, int dtype,
                                 int rot, int n_axes, const int* sections, int interleaved, int norm, float eps,
                                 void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * A paged key/value cache in 4 bits, for serving: requests of different lengths, each a list of pages.
 *
 * Format.  `cache` is [n_pages][entmax_attn_cache4_page_bytes(Hk, d, page_size)] bytes, 16-byte aligned.  A page holds
 * page_size (16, 32, 64, 128 or 256) tokens of all Hk key/value heads; head h's part starts at h times
 * page_size * 17 d / 16 bytes and is
 *     key codes [page_size][d/2], key scales [page_size][d/32], value codes [page_size][d/2], value scales [page_size][d/32].
 * 32 neighbouring values share the scale 2^(byte - 127); a code is a sign bit above three bits that stand for
 * 0, 0.5, 1, 1.5, 2, 3, 4, 6; the value with the lower index is in the lower half of its byte.  A slot is
 * page * page_size + (token within the page); n_pages * page_size < 2^31.
 *
 * entmax_attn_cache_tables: one step of a scheduler, on the GPU.  Request r goes from lens[r] cached tokens to
 * new_lens[r]: more (a prompt, a chunk of one, a token), fewer (an ended request: 0; a draft that was not accepted),
 * or as many.
 *   lens, new_lens in  [R] int32
 *   block_table in/out [R][max_blocks] int32: the pages of each request in the order of its tokens; entries behind them are
 *                      left as they were
 *   free_pages, free_count in/out [n_pages], [1] int32: a stack of the free pages.  First the pages that shrinking requests
 *                      leave go on top, the last request's last page first; then the growing requests, in order, take
 *                      theirs from the top.  (A step and the step back leave the stack as it was.)
 *   lens_out    out    [R] int32: the length the request has now; may be `lens` itself, not new_lens
 *   token_start out    [R+1] int32: the new tokens of request r are the rows token_start[r] .. token_start[r+1] - 1 of a batch
 *                      of new tokens, whether they were granted or not
 *   slots, positions out [max_tokens] int32: each row's slot and position in its request; slot -1 in the rows of a
 *                      request that was refused, and slot -1, position 0 in the rows behind the last
 *   status      out    [4] int32: rows in use (at most max_tokens), requests refused, requests with a length that is negative or
 *                      above max_blocks * page_size (nothing is done for them), page ids outside 0 .. n_pages - 1 met, and pages
 *                      given back to a stack that held n_pages already (free_count was wrong; such pages are lost)
 * A request that wants more pages than are left after the requests before it, or whose rows end behind max_tokens, is
 * refused whole: its length and pages stay, and so it is for the later ones that want any (pages; rows).  R <= 4096,
 * max_blocks * page_size <= 2^22.  The pages of a request must be its own: the call cannot tell.
 *
 * entmax_attn_cache4_write: keys and values of T tokens to their slots.
 *   K, V        in   rows [T][Hk][d] of `dtype`; k_strides, v_strides: HOST pointers to two strides each (token, head), in elements
 *   slots       in   [T] int32; a row whose slot is negative or past the cache is skipped.  The slots of a call must
 *                    differ: of two rows with one slot, either's codes and scales may stand there.
 * A block's scale is 2^s, s = floor(log2 max|x|) - 2, or one more where max|x| > 7 * 2^s, within 2^-126 .. 2^125; x / 2^s
 * is rounded to the nearest code, ties to the even one, above 6 to 6.  A block that holds an infinity or a NaN gets
 * scale byte 255 and reads as NaN.
 *
 * entmax_attn_cache4_read: the rows of T slots as the cache holds them (exact in either type), for attention over cached keys with
 * entmax_attn_fwd, or to move requests.  Rows of K, V whose slot is negative or past the cache are left as they were.
 * T = 0 is allowed in both and does nothing.
 *
 * entmax_attn_decode_cache4: entmax_attn_decode against the cache: one query per head and request.
 *   q           in   [R,Hq,d] of `dtype`; Hq is a multiple of Hk, query head h attends to head h / (Hq / Hk)
 *   block_table in   [R][max_blocks], lens in [R] int32: request r has the first lens[r] tokens of its pages.
 *   O           out  [R,Hq,d] float32;  tau out [R,Hq] float32, raw convention as in entmax_attn_fwd
 *   support     out  [R,Hq] int32, may be NULL: number of keys with p > 0
 *   max_len          at least the largest length, at most 2^22 and max_blocks * page_size: the launch and the workspace go by it
 *                    (about 4 R Hq max_len bytes, whatever the lengths: 1.1 GB for 64 requests of 32 heads with max_len 131072)
 * A request of length 0 gets O = 0, tau = 0, support 0.  One whose length is negative or above max_len, or that has a
 * page id outside 0 .. n_pages - 1 among the pages it attends to, gets NaN and support -1, and so does a head whose query or
 * keys hold an infinity or a NaN, or where 2^floor(log2 max|q|) of the head's query times the scale of a block of its keys
 * reaches 2^109 (a score might then pass 2^120).  What other heads hold, and the cache behind a request's last token, has no
 * effect.
 * Scores are formed on the matrix cores from the 4-bit keys and q in four (bf16) or five (float32) 8-bit terms: a bf16
 * element is exact down to 2^-17 of the largest of its row and known to 2^-25 of that below, a float32 element is exact down to
 * 2^-6 and known to 2^-30 (rows whose largest element is below 2^-100 lose more); the rest is in float32.
 * A probability is the power r = 1 / (alpha - 1) of a float32 difference: with alpha next to 1 it is known to about r 2^-21 of it.
 * Results repeat bit for bit.  Two calls at once need two workspaces.
 */
size_t entmax_attn_cache4_page_bytes(int Hk, int d, int page_size);      /* 0 for a bad shape */
int entmax_attn_cache_tables(const int32_t* lens, const int32_t* new_lens, int32_t* block_table, int32_t* free_pages,
                             int32_t* free_count, int32_t* lens_out, int32_t* token_start, int32_t* slots, int32_t* positions,
                             int32_t* status, int R, int max_blocks, int page_size, int n_pages, int max_tokens, void* hip_stream);
int entmax_attn_cache4_write(const void* K, const void* V, const int64_t* k_strides, const int64_t* v_strides, const int32_t* slots,
                             void* cache, int T, int Hk, int d, int dtype, int n_pages, int page_size, void* hip_stream);
int entmax_attn_cache4_read(const void* cache, const int32_t* slots, void* K, void* V, const int64_t* k_strides, const int64_t* v_strides,
                            int T, int Hk, int d, int dtype, int n_pages, int page_size, void* hip_stream);
size_t entmax_attn_decode_cache4_workspace_bytes(int R, int Hq, int Hk, int d, int max_len);     /* 0 for a bad shape */
int entmax_attn_decode_cache4(const void* q, const void* cache, const int32_t* block_table, const int32_t* lens,
                              float* O, float* tau, int32_t* support,
                              int R, int Hq, int Hk, int d, int dtype, int max_len, int max_blocks, int n_pages, int page_size,
                              float alpha, void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * The same in 8 bits, for keys and values that 4 bits do not hold well enough: about twice the bytes.
 *
 * Format.  `cache` is [n_pages][entmax_attn_cache8_page_bytes(Hk, d, page_size)] bytes, 16-byte aligned.  Head h's part of a page starts at
 * h times 2 page_size d + max(16, page_size / 2) bytes and is
 *     key codes [page_size][d], value codes [page_size][d], key scales [page_size/16], value scales [page_size/16] (float32).
 * The d values of 16 neighbouring tokens share a scale; a value is its code (a signed byte, -127 .. 127) times the scale's
 * magnitude.  Code -128 is not a number, and a scale whose sign bit is clear has none in its block.  Tables and slots as above.
 *
 * entmax_attn_cache8_write: keys and values of T tokens to their slots, arguments as entmax_attn_cache4_write.  Rows of one block
 * have to stand next to each other in the call, as the rows of a request do that entmax_attn_cache_tables makes slots for; they are
 * appended: with s_new = max|x| / 127 over them and one head (rounded to float32, at least 2^-126 unless they are all zero; infinities and NaN
 * left out), the block's scale becomes the larger of s_new and what it was.  If it grows, the codes c of the rows in front of the
 * lowest one written become c s_old / s rounded to the nearest integer (ties to the even one, here and below).  If row 0 of the block is
 * written, the block starts anew with s_new.  A code is x / s rounded to the nearest integer, an infinity or a NaN code -128.  What rows
 * behind the lowest one written held, and are not written themselves, is lost.  Where the slots of a call are not different, or rows of one block
 * stand apart, the codes and scales of that block are undefined.
 * A value is off by at most half the scale that its row was written with and half of each larger scale that its block took on since: s / 2, 1/254 of
 * the largest value (2^-119 or above), in a block that one call wrote; up to 8 s where sixteen calls wrote it and each brought a larger value than the
 * ones before.  How the same tokens are cut into calls thus changes codes.
 *
 * entmax_attn_cache8_read: as entmax_attn_cache4_read; a value is code times scale in float32, rounded to `dtype`.
 *
 * entmax_attn_decode_cache8: as entmax_attn_decode_cache4, against this cache, and with a sliding window:
 *   window, sinks    with window > 0 the query of a request of length n sees the keys j with j >= n - window and those with j < sinks; with
 *                    window = 0 all.  Pages without a key that is seen are not read, nor are their entries of block_table
 *                    (they stay the request's: the calls that give pages back take them from its end).
 * The workspace is 4.125 R Hq n to 4.125 R Hq (n + 445) + 510 bytes, n = max_len or, with a window, the smaller of max_len and window + sinks: the keys are taken in
 * whole blocks of 64, and a head has room for three blocks more.  A head gets NaN and support -1 where its query, or a key that it sees, holds an
 * infinity or a NaN, where a page id that it needs is out of range, or where 2^floor(log2 max|q|) of its query times the scale of
 * sixteen keys that it sees reaches 2^104.  Scores: integer products of the codes with q in three (bf16) or four (float32) 8-bit terms, summed
 * exactly; q is known to 2^-21 (bf16; exact down to 2^-13) or 2^-28 (float32) of the power of two at or below the largest of its row (rows
 * below 2^-90 lose more).  All else as there.
 */
size_t entmax_attn_cache8_page_bytes(int Hk, int d, int page_size);      /* 0 for a bad shape */
int entmax_attn_cache8_write(const void* K, const void* V, const int64_t* k_strides, const int64_t* v_strides, const int32_t* slots,
                             void* cache, int T, int Hk, int d, int dtype, int n_pages, int page_size, void* hip_stream);
int entmax_attn_cache8_read(const void* cache, const int32_t* slots, void* K, void* V, const int64_t* k_strides, const int64_t* v_strides,
                            int T, int Hk, int d, int dtype, int n_pages, int page_size, void* hip_stream);
size_t entmax_attn_decode_cache8_workspace_bytes(int R, int Hq, int Hk, int d, int max_len, int window, int sinks);   /* 0 for a bad shape */
int entmax_attn_decode_cache8(const void* q, const void* cache, const int32_t* block_table, const int32_t* lens,
                              float* O, float* tau, int32_t* support,
                              int R, int Hq, int Hk, int d, int dtype, int max_len, int max_blocks, int n_pages, int page_size,
                              int window, int sinks, float alpha, void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * Pages that several requests hold, in either cache: several answers to one prompt, beams, a prefix that many requests begin with.
 *   shares      in/out [n_pages] int32: holders of a page beyond the first, 0 at the start.  entmax_attn_cache_tables knows nothing of
 *               them: it may grow any request, but a request whose pages others hold is shortened and ended by entmax_attn_cache_fork.
 *
 * entmax_attn_cache_fork: request r becomes the first new_lens[r] tokens of what request parents[r] held before the call, all
 * requests at once: itself shortened (parents[r] = r), ended (0), left as it is (its own length), or a fork of another.
 *   lens, parents, new_lens in [R] int32; a request with a parent that is none, a new length that is negative or above its parent's, or a length of its own
 *               that is negative or above max_blocks * page_size stays as it is, to its last token and page (others that end in that page get copies)
 *   block_table, free_pages, free_count in/out as in entmax_attn_cache_tables.  First the pages that nobody holds any more go on top of the
 *               stack, the last request's last page first (a page that several requests leave counts as the last one's).  Then each
 *               request that ends inside a page that others hold too gets a page of its own from the top, in order; one of those that end in a page
 *               keeps it, if none holds it whole: the first that is its own parent, else the first.  (New tokens may then be
 *               written to every request but one that stays because of its arguments and ends in a page that others hold.)
 *   lens_out    out    [R] int32: the lengths now; may be `lens` itself, not parents or new_lens.  Where no page is left for a copy, the request
 *               ends before the page that was to be copied
 *   moves       out    [R][2] int32, 8-byte aligned: pages to be copied, from and to, before either is written to; -1 behind the last
 *   status      out    [4] int32: moves, requests for whose copy no page was left, requests that stay as they are because of
 *               their arguments, page ids outside 0 .. n_pages - 1 met, and pages that the stack had no room for (as there)
 *   workspace   entmax_attn_cache_fork_workspace_bytes bytes, 256-byte aligned
 *
 * entmax_attn_cache_compact: the pages in use move to the front: with `used` pages not on the stack, the i-th free page below `used` takes the
 * i-th page in use from `used` on.  Every output may be its input itself.
 *   table_out   out    [R][max_blocks]: block_table with the pages' new ids, all other entries as they were
 *   free_out    out    [n_pages]: the stack of the free pages, the lowest on top, and -1 at its bottom for each of its entries that was out of range or
 *               on it already (free_count stays, and no page in use is on the stack); entries behind it as they were
 *   shares_out  out    [n_pages] (0 for a free page); NULL if shares is
 *   moves       out    [n_pages / 2][2] int32, 8-byte aligned: from and to, -1 behind the last; no page that is moved from is moved to
 *   status      out    [4] int32: moves, pages in use, lengths out of range (their tables stay), page ids that are out of range, twice on the
 *               stack, or free but in a table (a table's entries of this kind stay)
 *
 * entmax_attn_cache_copy: pages moves[i] = (from, to), i < count[0] and i < max_moves, of page_bytes (a multiple of 16) bytes each, from `src` to `dst`, which may
 * be one cache if no page is both, nor the target of two.  Pairs with an id out of range are skipped.
 *
 * Results of all three repeat bit for bit.  R <= 4096, max_blocks * page_size <= 2^22, n_pages * page_size < 2^31.
 */
size_t entmax_attn_cache_fork_workspace_bytes(int R, int max_blocks);    /* 0 for a bad shape */
int entmax_attn_cache_fork(const int32_t* lens, const int32_t* parents, const int32_t* new_lens, int32_t* block_table, int32_t* free_pages,
                           int32_t* free_count, int32_t* shares, int32_t* lens_out, int32_t* moves, int32_t* status,
                           int R, int max_blocks, int page_size, int n_pages, void* workspace, size_t workspace_bytes, void* hip_stream);
size_t entmax_attn_cache_compact_workspace_bytes(int n_pages);           /* 0 for a bad number */
int entmax_attn_cache_compact(const int32_t* lens, const int32_t* block_table, const int32_t* free_pages, const int32_t* free_count,
                              const int32_t* shares, int32_t* table_out, int32_t* free_out, int32_t* shares_out, int32_t* moves, int32_t* status,
                              int R, int max_blocks, int page_size, int n_pages, void* workspace, size_t workspace_bytes, void* hip_stream);
int entmax_attn_cache_copy(const void* src, void* dst, const int32_t* moves, const int32_t* count, int max_moves, size_t page_bytes,
                           int src_pages, int dst_pages, void* hip_stream);

/* Static, human-readable text for a return code. */
const char* entmax_attn_strerror(int code);

/* hipError_t (as int) of the most recent failing HIP call made by this library on the calling
 * thread, 0 if none. */
int entmax_attn_last_hip_error(void);

/* Measurement and test aids (per-kernel timers, the gather switch, the matrix-core rate probe, the
 * histogram stage's read-out) are declared in entmax_attn_aids.h: none of them is needed to use the
 * library. */

#ifdef __cplusplus
}
#endif
#endif /* ENTMAX_ATTN_H */
