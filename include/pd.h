/*
 * pd.h -- C ABI of the MI355X (gfx950) block-sparse attention path of
 * Prefilling-dLLM: chunked prefill, per-step chunk/token selection, and
 * sparse decode attention.
 *
 * Conventions shared by every entry point
 * ---------------------------------------
 * - Plain C.  No HIP or torch types: device buffers are `void *` (or typed
 *   pointers to device memory), the stream is a `hipStream_t` passed as
 *   `void *` (NULL = the default stream).
 * - Ownership: every pointer is caller-owned DEVICE memory, contiguous in the
 *   layout stated next to it, 16-byte aligned.  The library allocates nothing,
 *   frees nothing and never synchronises; every call only enqueues kernels on
 *   `stream` and returns.  Scratch space is the caller's `workspace`, sized by
 *   pd_workspace_bytes().  Calls on different streams must not share outputs
 *   or workspace.
 * - Errors: arguments are checked on the host before anything is launched; on
 *   error nothing is launched, no output is touched, a status is returned and
 *   a thread-local message is kept for pd_last_error_message().  A failed
 *   launch returns PD_ERR_HIP.  Faults inside a kernel surface at the caller's
 *   next synchronisation on `stream`.
 * - Size limits besides those of each entry point: element offsets inside one
 *   sequence's cache, chunk sequence, decode block or decode KV rows stay
 *   below 2^31, and every launch grid (prefill, selection, decode, Split-S
 *   merge) below 2^31 workgroups; larger calls return PD_ERR_BAD_DIMS, and
 *   the size queries return 0 for them.
 * - Element type: all Q/K/V/O/cache tensors of one call have the type
 *   `dims->dtype` (bf16 or fp32).  Scores, key means and LSEs are fp32;
 *   indices are int32.  Arithmetic is fp32 (bf16 inputs feed bf16 matrix
 *   cores with fp32 accumulation; the attention probabilities are rounded to
 *   bf16 before the P*V product on the bf16 path and stay fp32 on the fp32
 *   path).
 *
 * Symbols (the paper's problem statement, Section 5): B sequences, N chunks of
 * C content tokens each with a BOS token prepended, L_q query rows, L_m (= |m|)
 * pseudo-label rows, L_d decode rows, H_q query heads, H_kv key/value heads
 * (query head h reads KV head h / (H_q/H_kv)), head dimension d, top-K chunks
 * and a budget of B_tok tokens per kept chunk.  S_c = 1 + C + L_q + L_m is the
 * length of one chunk sequence [BOS; c; q; m].
 */
#ifndef PD_H
#define PD_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  PD_OK = 0,
  PD_ERR_NULL_PTR = 1,    /* a required pointer is NULL                          */
  PD_ERR_BAD_DIMS = 2,    /* a size is out of range (see each entry point)       */
  PD_ERR_UNSUPPORTED = 3, /* H_q % H_kv != 0, d not in {64,128}, unknown dtype    */
  PD_ERR_MISALIGNED = 4,  /* a pointer is not 16-byte aligned                     */
  PD_ERR_WORKSPACE = 5,   /* workspace NULL or smaller than pd_workspace_bytes()  */
  PD_ERR_HIP = 6          /* a kernel launch failed                               */
} pd_status;

/* PD_FP8_E4M3, PD_FP4_E2M1: the elements of a paged cache only (see pd_paged_dims). */
typedef enum { PD_BF16 = 0, PD_FP32 = 1, PD_FP8_E4M3 = 2, PD_FP4_E2M1 = 3 } pd_dtype;

typedef struct {
  int32_t batch;        /* B >= 1                                                   */
  int32_t n_chunks;     /* N, 1..1024                                               */
  int32_t chunk_len;    /* C, 1..4096 content tokens; the cache holds 1+C rows      */
  int32_t q_len;        /* L_q >= 1 query rows                                      */
  int32_t m_len;        /* L_m >= 0 pseudo-label rows                               */
  int32_t dec_len;      /* L_d >= 1 decode rows                                     */
  int32_t n_heads_q;    /* H_q >= 1                                                 */
  int32_t n_heads_kv;   /* H_kv >= 1, divides H_q                                   */
  int32_t head_dim;     /* d, 64 or 128                                             */
  int32_t dtype;        /* pd_dtype                                                 */
  float sm_scale;       /* softmax scale; <= 0 selects 1/sqrt(d)                    */
  int32_t qm_per_chunk; /* 0: the q/m rows are one tensor shared by all chunks,
                           [B][L_q+L_m][H][d];  1: one copy per chunk,
                           [B][N][L_q+L_m][H][d]                                    */
  int32_t out_fp32;     /* 0: o and o_dec have element type dtype; 1: they are fp32
                           (bf16 inputs, fp32 outputs: no output rounding)          */
  int32_t tok_score_dir; /* token score of pd_prefill_chunks: 0 = both sums of
                           Eq. 5 (default); 1 = its first sum only, the mass the
                           query rows put on the token (the query-to-chunk score
                           of the paper's retention-score ablation)                 */
} pd_dims;

/*
 * Stage (a), one layer: chunk prefill (Section 5.1, Eq. 2), the chunk KV
 * cache, the chunk key summary, and the eviction score of Eq. 5 (Section 5.2).
 *
 * For every sequence b, chunk n and query head h, the S_c rows
 * [BOS; c_1..c_C; q_1..q_Lq; m_1..m_Lm] of chunk n attend to each other with
 * full bidirectional softmax(scale * Q K^T) V and to nothing outside the chunk.
 *
 * Inputs (element type dims->dtype):
 *   q_pre  [B][N][1+C][H_q][d]   chunk rows, slot 0 = the BOS token
 *   k_pre, v_pre [B][N][1+C][H_kv][d]
 *   q_qm   query + pseudo-label rows, [B][L_q+L_m][H_q][d] (shared) or
 *          [B][N][L_q+L_m][H_q][d] (qm_per_chunk = 1); rows 0..L_q-1 are the
 *          query rows
 *   k_qm, v_qm  likewise with H_kv heads
 * Outputs:
 *   o         [B][N][S_c][H_q][d]   attention output, rows ordered BOS, c, q, m
 *             (element type dtype, or fp32 when out_fp32 = 1)
 *   k_cache, v_cache [B][N][H_kv][1+C][d]  exact copies of the chunk rows
 *             (BOS at slot 0), chunk-contiguous per KV head
 *   tok_score fp32 [B][N][C]  e(c_j) of Eq. 5: for content token j, the
 *             softmax mass the L_q query rows put on it plus the mass it puts
 *             on the L_q query columns, summed over all H_q heads (the first
 *             term alone when dims->tok_score_dir = 1)
 *   tok_rank  int32 [B][N][C]  rank of token j among the C tokens of its chunk
 *             by tok_score: 0 = highest, ties to the lower index (Section 5.2:
 *             tokens are ranked by eviction score)
 *   key_mean  fp32 [B][N][H_kv][d]  mean of the C content keys (BOS excluded)
 *   chunk_score fp32 [B][N] or NULL  prefill-time chunk score, lower = more
 *             relevant: an attention-space reading of the length-normalised
 *             NLLs s_I + s_P of Section 5.1 (Eqs. 3-4).  With a(r) the mass
 *             q/m row r puts on the chunk's C content columns, averaged over
 *             the H_q heads: s = -(1/L_q) sum_{query rows} ln a(r)
 *             - (1/L_m) sum_{pseudo-label rows} ln a(r) (second term only when
 *             L_m >= 1).  Select with pd_select_ranked(lowest = 1).
 * workspace: >= pd_workspace_bytes(dims, 0, 0, 0, 0) bytes.
 * Errors: PD_ERR_BAD_DIMS for a size out of range; see the status list.
 */
pd_status pd_prefill_chunks(const pd_dims *dims,
                            const void *q_pre, const void *k_pre, const void *v_pre,
                            const void *q_qm, const void *k_qm, const void *v_qm,
                            void *o, void *k_cache, void *v_cache,
                            float *tok_score, int32_t *tok_rank, float *key_mean, float *chunk_score,
                            void *workspace, size_t ws_bytes, void *stream);

/*
 * Stage (b) from given chunk scores (Section 5.2, inter-chunk sparsity: keep
 * the K chunks with the lowest combined score), e.g. the chunk_score of
 * pd_prefill_chunks, selected once before the denoising loop.
 * Keeps the top_k lowest (lowest = 1) or highest (lowest = 0) of
 * chunk_score fp32 [B][N] (ties to the lower index; -0 equals +0), and the
 * tokens of each kept chunk with rank < tok_budget in tok_rank int32
 * [B][N][C].  Outputs as pd_score_select: chunk_idx int32 [B][top_k]
 * ascending; tok_slot int32 [B][top_k][tok_budget] ascending slots in 1..C.
 * Sizes: 1 <= top_k <= N, 1 <= tok_budget <= C.  No workspace.
 */
pd_status pd_select_ranked(const pd_dims *dims, int32_t top_k, int32_t tok_budget, const float *chunk_score,
                           int32_t lowest, const int32_t *tok_rank, int32_t *chunk_idx, int32_t *tok_slot,
                           void *stream);

/*
 * Stage (b), one layer, one denoising step: chunk scores, top-K chunks
 * (Section 5.2, inter-chunk sparsity) and the top-B_tok tokens of each kept
 * chunk by the Eq. 5 score (intra-chunk sparsity), read from the token ranks
 * that pd_prefill_chunks wrote (a token is kept iff its rank < B_tok).
 *
 * The chunk score is an attention-space stand-in for the paper's NLL score:
 *   s[b][n] = sum_h scale * < mean_r q_dec[b][r][h], key_mean[b][n][h/G] >,
 * higher = kept.  Ties rank the lower chunk (token) index first.
 * Inputs:  q_dec [B][L_d][H_q][d] (dims->dtype), key_mean fp32 [B][N][H_kv][d],
 *          tok_rank int32 [B][N][C] (a permutation of 0..C-1 per chunk).
 * Outputs: chunk_idx int32 [B][top_k], ascending chunk indices;
 *          tok_slot  int32 [B][top_k][tok_budget], ascending cache slots in
 *          1..C of the kept tokens of chunk chunk_idx[b][k] (slot = token+1);
 *          chunk_score fp32 [B][N] or NULL.
 * Sizes: 1 <= top_k <= N, 1 <= tok_budget <= C.
 * workspace: >= pd_workspace_bytes(dims, top_k, tok_budget, 0, 1) bytes.
 */
pd_status pd_score_select(const pd_dims *dims, int32_t top_k, int32_t tok_budget,
                          const void *q_dec, const float *key_mean, const int32_t *tok_rank,
                          int32_t *chunk_idx, int32_t *tok_slot, float *chunk_score,
                          void *workspace, size_t ws_bytes, void *stream);

/*
 * pd_score_select without a workspace, for callers that cannot allocate
 * device memory (code under HIP graph capture, tight serving loops, harnesses
 * that forbid hipMalloc).  Same arguments, outputs and errors as
 * pd_score_select minus the workspace: its scratch (the B*N*H_q*ceil(L_d/128)
 * fp32 chunk-score terms, rounded up to 256 bytes) lives in a static array of
 * 4 MiB per GPU, held by the library from the first call on that GPU until the
 * process ends; a call that needs more returns PD_ERR_BAD_DIMS.  The current device's array is used (call
 * with the stream's device current).  Every call on one GPU shares that
 * array: calls that overlap in time on one GPU (other streams, other threads)
 * race and must be serialised by the caller.  Nothing is allocated and nothing
 * needs clearing: every call rewrites the terms before it reads them.
 */
pd_status pd_score_select_noalloc(const pd_dims *dims, int32_t top_k, int32_t tok_budget,
                                  const void *q_dec, const float *key_mean, const int32_t *tok_rank,
                                  int32_t *chunk_idx, int32_t *tok_slot, float *chunk_score, void *stream);

/*
 * Stage (c), one layer, one denoising step: the L_d decode rows attend
 * (bidirectionally) over, in order, for each kept chunk chunk_idx[b][k]: its
 * BOS row (cache slot 0) and the rows at slots tok_slot[b][k][*]; then rows
 * 0..n_static-1 of the static query KV; then their own L_d rows (Section 5.3,
 * prefix reuse).  L_kv = top_k*(1+tok_budget) + n_static + L_d rows.
 *
 * Inputs (dims->dtype): q_dec [B][L_d][H_q][d]; k_dec, v_dec [B][L_d][H_kv][d];
 *   k_cache, v_cache as written by pd_prefill_chunks; k_static, v_static
 *   [B][L_q+L_m][H_kv][d] (rows 0..n_static-1 used; may be NULL when
 *   n_static = 0); chunk_idx, tok_slot as written by pd_score_select (entries
 *   must lie in 0..N-1 and 1..C).
 * Outputs: o_dec [B][L_d][H_q][d] (dtype, or fp32 when out_fp32 = 1);
 *   lse_dec fp32 [B][H_q][L_d] natural-log
 *   row LSE, or NULL (bf16 path: the log of the sum of
 *   the bf16-rounded softmax weights that multiply V, within log(1 + 2^-8)).
 * num_splits: the KV rows are cut into that many shards processed in
 *   parallel and merged by log-sum-exp (the paper's Split-S); 0 = chosen by the
 *   library from the sizes; otherwise 1..64.
 * Sizes: 1 <= top_k <= N, 1 <= tok_budget <= C, 0 <= n_static <= L_q + L_m.
 * workspace: >= pd_workspace_bytes(dims, top_k, tok_budget, num_splits, 2)
 *   bytes (may be 0, then workspace may be NULL).
 */
pd_status pd_sparse_decode_attn(const pd_dims *dims, int32_t top_k, int32_t tok_budget,
                                const void *q_dec, const void *k_dec, const void *v_dec,
                                const void *k_cache, const void *v_cache,
                                const int32_t *chunk_idx, const int32_t *tok_slot,
                                const void *k_static, const void *v_static, int32_t n_static,
                                void *o_dec, float *lse_dec, int32_t num_splits,
                                void *workspace, size_t ws_bytes, void *stream);

/*
 * Static-selection mode (the paper selects once, before the denoising loop:
 * Section 5.2 selection from the pseudo-label rows, reused for every step of
 * Section 5.3).  Three calls per layer replace the per-step pd_score_select +
 * gathered decode:
 *
 * pd_score_select_static: as pd_score_select, but the mean query is taken
 *   over the L_m pseudo-label rows of q_qm (rows L_q..L_q+L_m-1 of each
 *   sequence's q/m block, in the layout dims->qm_per_chunk gives; chunk 0's
 *   copy when per chunk) instead of the decode rows.  Needs m_len >= 1.
 *   workspace: >= pd_workspace_bytes(dims, top_k, tok_budget, 0, 1) bytes.
 *
 * pd_gather_selected: copies, once, the prefix rows a decode step reads into
 *   contiguous buffers k_sel, v_sel [B][H_kv][top_k*(1+tok_budget)][d]
 *   (dims->dtype): for each kept chunk chunk_idx[b][k] in order, its BOS row
 *   (slot 0) and then the rows at slots tok_slot[b][k][*].  Bit-exact copies;
 *   no workspace.
 *
 * pd_sparse_decode_attn_compact: pd_sparse_decode_attn whose prefix rows are
 *   rows 0..n_sel-1 of k_sel, v_sel [B][H_kv][n_sel][d] instead of rows
 *   gathered from the chunk cache (0 <= n_sel <= 2^20; k_sel/v_sel may be
 *   NULL when n_sel = 0).  With the buffers of pd_gather_selected and
 *   n_sel = top_k*(1+tok_budget) the result is that of pd_sparse_decode_attn
 *   with the same selection.  workspace: >= pd_compact_workspace_bytes bytes.
 * Errors as for the per-step calls.
 */
pd_status pd_score_select_static(const pd_dims *dims, int32_t top_k, int32_t tok_budget,
                                 const void *q_qm, const float *key_mean, const int32_t *tok_rank,
                                 int32_t *chunk_idx, int32_t *tok_slot, float *chunk_score,
                                 void *workspace, size_t ws_bytes, void *stream);
pd_status pd_gather_selected(const pd_dims *dims, int32_t top_k, int32_t tok_budget,
                             const void *k_cache, const void *v_cache,
                             const int32_t *chunk_idx, const int32_t *tok_slot,
                             void *k_sel, void *v_sel, void *stream);
pd_status pd_sparse_decode_attn_compact(const pd_dims *dims, int32_t n_sel,
                                        const void *q_dec, const void *k_dec, const void *v_dec,
                                        const void *k_sel, const void *v_sel,
                                        const void *k_static, const void *v_static, int32_t n_static,
                                        void *o_dec, float *lse_dec, int32_t num_splits,
                                        void *workspace, size_t ws_bytes, void *stream);
size_t pd_compact_workspace_bytes(const pd_dims *dims, int32_t n_sel, int32_t num_splits);

/*
 * Full-mask cache construction (Section 6, the ablation of the KV cache
 * construction strategy): once the chunks are selected, the kept rows and the
 * query are re-encoded jointly, with the decoding mask, at continuous
 * positions.  pd_gather_joint builds the joint rows of every sequence; one
 * pd_sparse_decode_attn_compact call over them (dims->dec_len = L_j,
 * n_sel = 0, n_static = 0, k_sel / v_sel / k_static / v_static NULL, q_dec,
 * k_dec, v_dec = q_joint, k_joint, v_joint) is the dense joint attention, and
 * k_pref, v_pref (the same K, V rows in the compact prefix layout) then serve
 * as the prefix (n_sel = L_j) of the decoding steps'
 * pd_sparse_decode_attn_compact calls.
 *
 * Joint rows, L_j = top_k*(1+tok_budget) + L_q per sequence: for each kept
 * chunk k = 0..top_k-1 (chunk_idx[b][k]) its BOS row (slot 0) and the rows at
 * slots tok_slot[b][k][*]; then query rows 0..L_q-1 of the q/m block (layout
 * per dims->qm_per_chunk, chunk 0's copy when per chunk).  Q rows come from
 * q_pre, K and V rows from k_cache / v_cache (kept rows) or q_qm / k_qm / v_qm
 * (query rows).
 * Positions: the chunk forward placed slot s of every chunk at s and query row
 * j at C+1+j; jointly, kept chunk k starts at k*(C+1), so its rows move by
 * k*(C+1), and the query rows move by (top_k-1)*(C+1).  Q and K are rotated
 * by the rotate-half rotary embedding with frequencies
 * rope_base^(-2i/d), i = 0..d/2-1 (element i pairs with element i + d/2);
 * the angle and the rotation are evaluated in double precision and rounded
 * once to dims->dtype.  V is copied.  rope_base = 0: no rotation (bit-exact
 * copies).
 *
 * Inputs (dims->dtype): q_pre [B][N][1+C][H_q][d] (as given to
 *   pd_prefill_chunks); k_cache, v_cache as written by pd_prefill_chunks;
 *   q_qm, k_qm, v_qm as given to pd_prefill_chunks; chunk_idx [B][top_k],
 *   tok_slot [B][top_k][tok_budget] as written by the selection calls
 *   (entries must lie in 0..N-1 and 1..C).
 * Outputs (dims->dtype, caller-owned): q_joint [B][L_j][H_q][d], k_joint and
 *   v_joint [B][L_j][H_kv][d]; k_pref and v_pref [B][H_kv][L_j][d], the same
 *   K and V values (both NULL: not written; one NULL: PD_ERR_NULL_PTR).  No
 *   workspace; asynchronous on stream.
 * Sizes: 1 <= top_k <= N, 1 <= tok_budget <= C, rope_base finite and >= 0.
 * Errors: PD_ERR_NULL_PTR, PD_ERR_MISALIGNED, PD_ERR_BAD_DIMS,
 *   PD_ERR_UNSUPPORTED, PD_ERR_HIP.
 */
pd_status pd_gather_joint(const pd_dims *dims, int32_t top_k, int32_t tok_budget,
                          const int32_t *chunk_idx, const int32_t *tok_slot,
                          const void *q_pre, const void *k_cache, const void *v_cache,
                          const void *q_qm, const void *k_qm, const void *v_qm, double rope_base,
                          void *q_joint, void *k_joint, void *v_joint, void *k_pref, void *v_pref,
                          void *stream);

/*
 * Head norms and rotary positions: what turns the projected query and key rows
 * of n_rows tokens into the rows that the attention entry points take.  For
 * every head row x (d elements) of q and k
 *   y_i = x_i * w_i / sqrt(mean_j x_j^2 + eps)        (w_q for q, w_k for k)
 * and then, for i = 0..d/2-1 with the angle a = pos[t] * rope_base^(-2i/d),
 *   out_i = y_i cos a - y_{i+d/2} sin a,  out_{i+d/2} = y_{i+d/2} cos a + y_i sin a.
 * w_q (w_k) NULL: the query (key) heads are not normalised.  rope_base = 0: no
 * rotation, pos may be NULL.  Norms in fp32 (a head whose squares sum to more
 * than fp32 holds gives zeros; with eps = 0 the mean square has to be at least 2^-126,
 * one that vanishes in fp32 gives infinities, and NaN for elements of zero); the
 * angle in double precision,
 * reduced to one turn before its sine and cosine are taken in fp32; one
 * rounding to the element type at the end.
 *
 * Inputs (element type dtype, PD_BF16 or PD_FP32): q, k: row t of q holds its
 *   n_heads_q heads of d = head_dim contiguous elements one after another at
 *   element t * q_stride (likewise k, n_heads_kv, k_stride), so that both may
 *   point into the rows of a fused projection.  w_q, w_k [d].  pos int32
 *   [n_rows], any values.
 * Outputs: q_out, k_out, laid out the same with q_out_stride, k_out_stride.
 *   q_out may be q itself with the same stride (k_out likewise); other overlaps
 *   of inputs and outputs, and of q_out and k_out, are not allowed.
 * Sizes: n_rows >= 0 (0: nothing is done), n_heads_q >= 0 and n_heads_kv >= 0
 *   with at least one head in all (the pointers of a tensor without heads may
 *   be NULL), d in {64, 128}, strides >= heads * d and multiples of 16 bytes,
 *   eps >= 0 finite, rope_base >= 0 finite.  No workspace.
 */
pd_status pd_qk_norm_rope(int32_t n_rows, int32_t n_heads_q, int32_t n_heads_kv, int32_t head_dim, int32_t dtype,
                          const void *q, int64_t q_stride, const void *k, int64_t k_stride,
                          const void *w_q, const void *w_k, float eps, const int32_t *pos, double rope_base,
                          void *q_out, int64_t q_out_stride, void *k_out, int64_t k_out_stride, void *stream);

/*
 * Paged key/value cache: sequences of different and growing lengths over one
 * pool of pages.  A page holds R = page_rows consecutive rows of one sequence,
 * for every KV head.  Position p of sequence b is row p % R of page
 * page_table[b][p / R].
 *
 * With cache_dtype = PD_FP8_E4M3 a head's row is held as E4M3 values (the OCP
 * format with NaN and no infinities, largest value 448) times a power of two:
 * e is the least exponent with max|x| <= 448 * 2^e over the row's finite
 * elements, within -100..120 (-100 for a row of zeros), the values are
 * x * 2^-e rounded to nearest even, and the byte e + 127 is kept beside them.
 * NaN and infinities become NaN.  Scaling by a power of two is exact, so that
 * the rounding to E4M3 is the only one.
 *
 * With cache_dtype = PD_FP4_E2M1 a head's row is held as E2M1 values (0, 0.5, 1,
 * 1.5, 2, 3, 4, 6 and their negatives, codes 0..7 and 8..15 in this order), two a
 * byte with the even channel in the low four bits, times a power of two for each
 * 32 neighbouring channels: e is the least exponent with max|x| <= 6 * 2^e over
 * them, within -100..126 (-100 for zeros), the values are x * 2^-e rounded to
 * nearest even, and the byte e + 127 is kept.  Where one of the 32 is NaN or an
 * infinity the byte is 255, and all of them read as NaN.
 */
typedef struct {
  int32_t batch;        /* B, 1..65536 sequences                                    */
  int32_t new_len;      /* L_n >= 1: places for the new rows of a sequence           */
  int32_t n_heads_q;    /* H_q >= 1                                                  */
  int32_t n_heads_kv;   /* H_kv >= 1, divides H_q                                    */
  int32_t head_dim;     /* d, 64 or 128                                              */
  int32_t dtype;        /* of queries, new rows and outputs: PD_BF16 or PD_FP32      */
  int32_t cache_dtype;  /* of the pages: dtype, or PD_FP8_E4M3 or PD_FP4_E2M1 when
                           dtype = PD_BF16                                           */
  int32_t page_rows;    /* R: 16, 32, 64, 128 or 256                                 */
  int32_t n_pages;      /* pages in the pool, >= 1                                   */
  int32_t max_pages;    /* entries of a sequence in page_table, >= 1                 */
  float sm_scale;       /* softmax scale; <= 0 selects 1/sqrt(d)                     */
  int32_t causal;       /* 1: a new row sees the positions up to its own; 0: all
                           kv_len positions                                          */
} pd_paged_dims;

/* Device memory of the cache.  kv_len and new_rows are read on the device:
 * values outside 0..max_pages*R and 0..L_n are taken as the nearer bound. */
typedef struct {
  void *k_pages, *v_pages;    /* [n_pages][H_kv][R][d], cache_dtype (PD_FP4_E2M1:
                                 [n_pages][H_kv][R][d/2] bytes)                      */
  uint8_t *k_exp, *v_exp;     /* exponent bytes: PD_FP8_E4M3 [n_pages][H_kv][R],
                                 PD_FP4_E2M1 [n_pages][H_kv][d/32][R], else NULL     */
  void *k_bounds;             /* [n_pages][H_kv][2][d], dtype: per channel the least
                                 and the largest key of a page, as given to
                                 pd_paged_append (before quantisation); NULL: not
                                 kept (pd_paged_select needs it)                     */
  const int32_t *page_table;  /* [B][max_pages]; only entries of pages that hold rows
                                 are read                                            */
  const int32_t *kv_len;      /* [B] rows of each sequence, the new ones included    */
  const int32_t *new_rows;    /* [B] new rows of each sequence, or NULL: L_n each    */
} pd_paged_cache;

/*
 * Writes new rows into the pages: row r < new_rows[b] of sequence b is its
 * position kv_len[b] - new_rows[b] + r (positions below 0 are not written).
 * k_new, v_new (dtype): row (b, r) holds its H_kv heads of d contiguous
 * elements at element (b * L_n + r) * stride.  k_bounds, where kept: a page
 * whose row 0 is written begins with the new rows of this call, any other page's
 * bounds are widened by them; NaNs do not count.  Everything else in the pool is left as it
 * is.  A page may be written through one sequence only in a call.  A page id
 * outside 0..n_pages-1 is not written to.
 * Strides: >= H_kv * d, multiples of 16 bytes.  No workspace.
 */
pd_status pd_paged_append(const pd_paged_dims *dims, const pd_paged_cache *cache, const void *k_new,
                          int64_t k_stride, const void *v_new, int64_t v_stride, void *stream);

/*
 * pd_paged_append of rows as a projection gives them, with what pd_qk_norm_rope does
 * to query and key rows on the way: new row r < new_rows[b] of sequence b is normed
 * (w_q, w_k; NULL: not) and turned by its position, pos[b][r] or, with pos NULL, its
 * position in the sequence kv_len[b] - new_rows[b] + r; the query row is written to
 * q_out, the key row and the value row as it is into the pages.  Formulas, pairs and
 * frequencies are pd_qk_norm_rope's; rope_base = 0: no rotation.  Norm and rotation are
 * evaluated in double precision, the result is rounded to fp32 and then to dtype, and from
 * there the pages and k_bounds hold what pd_paged_append makes of the rows, to the bit.
 * (pd_qk_norm_rope works in fp32: an element of its results may differ by one
 * rounding.)  With eps = 0 a head of zeros gives NaN; one with an infinity gives NaN in
 * its place, and zeros elsewhere before the rotation.
 * q, k_new, v_new (dtype): row (b, r) holds its heads of d contiguous elements at element
 *   (b * L_n + r) * stride (each its own: all may point into the rows of a fused
 *   projection).  w_q, w_k [d].  pos int32 [B][L_n], any values, or NULL.
 * q_out [B][L_n][H_q][d] (dtype), as pd_paged_attn takes it: every row r < new_rows[b] is
 *   written, those whose position in the sequence lies below 0 too, and others are left as they
 *   were.  It may be q itself where q_stride = H_q * d; other overlaps of inputs and outputs are
 *   not allowed.  q and q_out both NULL: keys and values alone.
 * Strides: >= heads * d, multiples of 16 bytes.  eps >= 0 and rope_base >= 0 finite.  No workspace.
 */
pd_status pd_paged_append_rope(const pd_paged_dims *dims, const pd_paged_cache *cache, const void *q,
                               int64_t q_stride, const void *k_new, int64_t k_stride, const void *v_new,
                               int64_t v_stride, const void *w_q, const void *w_k, float eps, const int32_t *pos,
                               double rope_base, void *q_out, void *stream);

/*
 * Reads rows back: k_out, v_out [B][H_kv][n_rows][d] (dtype) receive positions
 * first..first+n_rows-1 of every sequence, dequantised; this is the prefix
 * layout of pd_sparse_decode_attn_compact.  Rows of positions >= kv_len[b] are
 * left as they were.  A page id outside 0..n_pages-1 gives NaN rows.  What an
 * E4M3 or E2M1 value times its power of two stands for is exact in bf16, except that
 * 2^128, which magnitudes from 1.9375 * 2^127 (E2M1: 1.75 * 2^127) round to, reads as
 * infinity.
 * Sizes: first >= 0, n_rows >= 1, first + n_rows <= max_pages * R.  No workspace.
 */
pd_status pd_paged_read(const pd_paged_dims *dims, const pd_paged_cache *cache, int32_t first, int32_t n_rows,
                        void *k_out, void *v_out, void *stream);

/*
 * Chooses pages for each query: for sequence b and KV head g, a page's score is
 * the largest, over the G * new_rows[b] query rows of the group (G = H_q/H_kv),
 * of  sum_i q_i * (q_i >= 0 ? hi_i : lo_i)  with the page's bounds lo, hi: no
 * key of the page, as it was given to pd_paged_append, has a larger product with the
 * row.  The keys that an E4M3 cache holds of them are rounded, by at most 2^-4 of an
 * element, 2^-17 of the row's largest or 2^-110 (E2M1: 1/5 of an element, 1/12 of the
 * largest of its 32 or 2^-102), so their products may exceed the score by as much.  Products and sums are in double precision.  The top_k best of
 * the sequence's ceil(kv_len/R) pages are kept; its first n_first and last n_last
 * pages rank above all others, a NaN score above every number, and ties go to the
 * lower page.
 * q [B][L_n][H_q][d] (dtype).  page_idx int32 [B][H_kv][top_k]: the kept pages'
 * indices in the sequence (p / R), ascending; -1 behind the last where the
 * sequence has fewer pages.
 * Sizes: 1 <= top_k <= max_pages <= 65536, n_first, n_last >= 0.
 * workspace: >= pd_paged_workspace_bytes(dims, top_k, 0) bytes.
 */
pd_status pd_paged_select(const pd_paged_dims *dims, const pd_paged_cache *cache, const void *q, int32_t top_k,
                          int32_t n_first, int32_t n_last, int32_t *page_idx, void *workspace, size_t ws_bytes,
                          void *stream);

/*
 * Attention of the new rows over the pages: row r < new_rows[b] of sequence b
 * attends to the positions p of its cache with p <= kv_len[b] - new_rows[b] + r
 * (causal = 1) or p < kv_len[b] (causal = 0), its own rows included (append
 * first).  page_idx NULL (top_k = 0): all pages; otherwise [B][H_kv][top_k]
 * page indices as written by pd_paged_select: KV head g attends to the visible
 * positions of those pages alone (an entry outside 0..max_pages-1 is skipped, a
 * page named twice counts twice).
 * q, o [B][L_n][H_q][d] (dtype); lse fp32 [B][H_q][L_n] natural-log row LSE, or
 * NULL.  Rows r >= new_rows[b] of o and lse are left as they were.  A row that
 * sees no position, or only scores of -inf, gets o = 0 and lse = -inf.  What
 * the pages hold behind kv_len is never used, whatever its bits.  A page id
 * outside 0..n_pages-1 makes the rows of o and lse that see one of its positions NaN,
 * and no others.
 * With dtype = PD_BF16 the weights multiply V as two bf16 terms (15 bits) where a
 * KV head has at most 16 query rows, G * L_n <= 16, and rounded to bf16 where it has
 * more or the pages are PD_FP4_E2M1 (their sum, and so lse, is taken before); sums are fp32 and divided at the
 * end, so they overflow where 256 * sum |v| over the visible keys passes 2^128.
 * A visible value that is infinite gives the infinity, or NaN where its weight
 * has underflowed (about 2^-126 of the row's largest); NaN gives NaN.
 * The lengths are known on the device alone: the split of long sequences over
 * workgroups, and their join, are planned there.
 * Exponent bytes are those that pd_paged_append writes.
 * workspace: >= pd_paged_workspace_bytes(dims, top_k, 1) bytes (may be 0, then
 * workspace may be NULL).
 */
pd_status pd_paged_attn(const pd_paged_dims *dims, const pd_paged_cache *cache, const void *q,
                        const int32_t *page_idx, int32_t top_k, void *o, float *lse, void *workspace,
                        size_t ws_bytes, void *stream);

/*
 * pd_paged_attn within a sliding window, with the first positions visible
 * throughout: row r < new_rows[b], which is position p = kv_len[b] - new_rows[b] + r,
 * attends to the positions j that pd_paged_attn lets it see (j <= p, or all with
 * causal = 0) and that lie in its window, j > p - window, or among the first,
 * j < n_sinks.  With causal = 0 a window bounds what lies before a row; the positions
 * behind it, which are new rows, are all seen.  Pages none of whose positions a row
 * of the call sees are not read, and neither are their entries in page_table, so that they may be
 * given to other sequences.  Everything else is as for pd_paged_attn over all
 * pages: o, lse, rows that see nothing, page ids outside the pool, values that are
 * not finite, rounding.
 * Sizes: window >= 1, n_sinks >= 0 (those beyond all positions count as all).
 * Which kernel runs, and whether long windows are cut over workgroups, goes by the sizes
 * in dims: give L_n the most new rows of the call, not more.  Where few sequences of a batch have
 * many new rows and the others one or a few, and the window is long, two calls, one for either
 * kind, take less than one (H_q = 32, H_kv = 8, window 8192, one sequence of 512 new rows and three of one: 314 us
 * in one call, 119 and 24 in two).
 * workspace: >= pd_paged_window_workspace_bytes(dims, window, n_sinks) bytes (may be
 * 0, then workspace may be NULL), which grow with the window and not with max_pages.
 */
pd_status pd_paged_window_attn(const pd_paged_dims *dims, const pd_paged_cache *cache, const void *q,
                               int32_t window, int32_t n_sinks, void *o, float *lse, void *workspace,
                               size_t ws_bytes, void *stream);

/* Workspace bytes of pd_paged_window_attn.  Returns 0 for invalid arguments. */
size_t pd_paged_window_workspace_bytes(const pd_paged_dims *dims, int32_t window, int32_t n_sinks);

/* Workspace bytes for `which` = 0 pd_paged_select, 1 pd_paged_attn (top_k = 0:
 * over all pages).  Returns 0 for invalid arguments. */
size_t pd_paged_workspace_bytes(const pd_paged_dims *dims, int32_t top_k, int32_t which);

/* Bytes of ONE of k_cache / v_cache for one layer: B*N*H_kv*(1+C)*d*elem. */
size_t pd_cache_bytes(const pd_dims *dims);

/* Workspace bytes for `which` = 0 prefill, 1 select, 2 decode (num_splits as
 * passed to pd_sparse_decode_attn; 0 = automatic).  Returns 0 for invalid
 * dims (the matching entry point then reports the error). */
size_t pd_workspace_bytes(const pd_dims *dims, int32_t top_k, int32_t tok_budget,
                          int32_t num_splits, int32_t which);

/* The number of KV shards pd_sparse_decode_attn uses for these arguments. */
int32_t pd_decode_splits(const pd_dims *dims, int32_t top_k, int32_t tok_budget,
                         int32_t n_static, int32_t num_splits);

/* Diagnostic: the device's achievable dense bf16 MFMA rate, the yardstick the
 * attention kernels are compared with besides the published peak.
 * Launches n_workgroups (1..2^20) workgroups of 4 waves; each wave runs iters
 * iterations of 8 v_mfma_f32_32x32x16_bf16 (32768 FLOP each) on register
 * operands, so one call performs n_workgroups * 4 * iters * 8 * 32768 FLOP.
 * sink: caller-owned device buffer of n_workgroups * 256 floats (16-B aligned)
 * that receives one value per thread.  Asynchronous on stream; time it with
 * events.  Errors: PD_ERR_NULL_PTR, PD_ERR_BAD_DIMS, PD_ERR_MISALIGNED,
 * PD_ERR_HIP. */
pd_status pd_mfma_rate_probe(int32_t n_workgroups, int32_t iters, float *sink, void *stream);

const char *pd_status_string(pd_status s);
const char *pd_last_error_message(void); /* thread-local detail of the last error */
const char *pd_version(void);

#ifdef __cplusplus
}
#endif
#endif /* PD_H */
