/*
 * comem_kv_evict.h -- which tokens of a context stay when it is cut, on AMD
 * Instinct MI355X (gfx950): the attention that each cached token was paid,
 * and the tokens that were paid the most.
 *
 * The paper bounds the cost of a step by bounding the context (Sec. 3.3) and
 * names eviction from the cache among the ways to do that. comem_kv_compact
 * (comem_kv_pages.h) cuts a row to a list of its tokens; these calls make the
 * list on the GPU. The attention calls return the log-sum-exp of every query
 * row, from which any one weight follows without the others:
 *
 *     w_i,h(t)   = exp(scale * dot(q[i, h, :], K_b[t, h / G, :]) - lse[i, h])
 *     weights[t] = decay * prior[t] + sum_i sum_h w_i,h(t)
 *
 * over the new tokens i of sequence b (a decode step's one, or a chunk of the
 * last M_b of its L_b tokens as in comem_prefill_attn.h: token i sees the
 * tokens t <= L_b - M_b + i) and all query heads h. A context's pages hold all
 * of its heads, so one sum serves them all. The new tokens themselves,
 * t >= L_b - M_b, were paid nothing before: their prior is 0, whatever the
 * buffer says, so that it needs no initialisation.
 *
 * Ownership, errors, streams and the device-side contract (lengths, block
 * tables) are those of the decode calls (comem_decode_attn.h). Same arguments
 * (workspaces of the same use among them), same bits.
 */
#ifndef COMEM_KV_EVICT_H
#define COMEM_KV_EVICT_H

#include "comem_decode_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* *workspace_bytes_out gets the bytes that a weights call with these bounds can
 * use (0: none). */
comem_status comem_attn_weights_workspace(const comem_decode_attn_plan* plan, int32_t batch, int32_t max_q_len,
                                          int64_t max_ctx_len, size_t* workspace_bytes_out);

/* Attention weights over a contiguous / ragged cache.
 *   q          [rows, h_q, d_h] dense, as in the attention calls; 16-byte aligned.
 *   lse        float32 [rows, h_q], what the attention call returned for q. A
 *              row of -inf (it saw no key with a weight) adds nothing. NaN
 *              queries, keys and lse make the weights that they meet NaN.
 *   q_start    device int64 [batch]: first row of each sequence's new tokens.
 *   q_lens     device int32 [batch]: M_b. Both NULL: one new token a sequence,
 *              row b.
 *   max_q_len  host bound >= every q_lens[b], 0 .. max_ctx_len; 1 when q_lens is NULL. With
 *              max_q_len = 0 or batch = 0 nothing is enqueued and no pointer
 *              is looked at.
 *   prior      float32 [batch, weights_stride] or NULL; weights itself, or not
 *              overlapping it. Not read with decay = 0.
 *   decay      finite, >= 0 (not looked at with prior NULL).
 *   weights    float32 [batch, weights_stride]: element (b, t), t < L_b, is
 *              written, the others are left as they were.
 *   weights_stride >= max_ctx_len.
 *   workspace  device memory, 256-byte aligned, of any size, or NULL; no
 *              initialisation, nothing kept between calls. With the bytes that
 *              comem_attn_weights_workspace says, many query rows over few
 *              tokens are shared by several workgroups, and a second kernel
 *              adds up their sums (another order of the same additions).
 * k, strides, seq_start, ctx_lens, batch and max_ctx_len as in
 * comem_decode_attn. A sequence with ctx_lens[b] outside [0, max_ctx_len], or
 * q_lens[b] outside [1, min(ctx_lens[b], max_q_len)], is left as it is. */
comem_status comem_attn_weights(const comem_decode_attn_plan* plan, const void* q, const float* lse,
                                const int64_t* q_start, const int32_t* q_lens, int32_t max_q_len, const void* k,
                                int64_t stride_token, int64_t stride_head, const int64_t* seq_start,
                                const int32_t* ctx_lens, int32_t batch, int64_t max_ctx_len, const float* prior,
                                float decay, float* weights, int64_t weights_stride, void* workspace,
                                size_t workspace_bytes, void* hip_stream);

/* Paged cache; pages, strides and block table as in comem_decode_attn_paged. */
comem_status comem_attn_weights_paged(const comem_decode_attn_plan* plan, const void* q, const float* lse,
                                      const int64_t* q_start, const int32_t* q_lens, int32_t max_q_len,
                                      const void* k_pages, int64_t stride_page, int64_t stride_token,
                                      int64_t stride_head, int32_t page_size, int64_t num_pages,
                                      const int32_t* block_table, int32_t max_pages_per_seq, const int32_t* ctx_lens,
                                      int32_t batch, int64_t max_ctx_len, const float* prior, float decay,
                                      float* weights, int64_t weights_stride, void* workspace,
                                      size_t workspace_bytes, void* hip_stream);

/* *workspace_bytes_out gets the bytes that a keep call for n rows can use (0:
 * none). */
comem_status comem_keep_tokens_workspace(const comem_decode_attn_plan* plan, int32_t n, int64_t max_ctx_len,
                                         size_t* workspace_bytes_out);

/* The tokens of row r = rows[i] (rows NULL: r = i) that stay: of its L =
 * ctx_lens[r] tokens the first `first`, the last `last` and, of those between,
 * the ones with the largest weights, min(L, budget) in all. Of equal weights
 * (0 and -0 are equal) the earlier token stays; NaN is above every number. The
 * lists are what comem_kv_compact takes: positions in ascending order.
 *   weights    float32, element (r, t) at weights[r * weights_stride + t] (may
 *              be NULL with max_ctx_len = 0).
 *   weights_stride >= max_ctx_len.
 *   ctx_lens   device int32 [num_rows]; num_rows 1 .. 65535.
 *   rows       device int32 [n], or NULL; 0 <= n <= num_rows (0: nothing is
 *              enqueued and no pointer looked at).
 *   budget     tokens that stay, >= first + last; first, last >= 0.
 *   budgets    device int32 [n], or NULL: entry i's own budget, taken as the
 *              nearest one in [first + last, budget].
 *   keep       int32 [n, keep_stride]: the list of entry i; what follows the
 *              list is left as it was. keep_stride >= min(budget, max_ctx_len);
 *              where that is 0, keep may be NULL.
 *   keep_start int64 [n] or NULL: gets i * keep_stride.
 *   keep_lens  int32 [n]: the list's length; -1, and no list, for a row outside
 *              [0, num_rows) or with a length outside [0, max_ctx_len]
 *              (comem_kv_compact leaves such an entry out).
 *   kept       float32 [n, keep_stride] or NULL: the weights of the tokens that
 *              stay, in the places they have after comem_kv_compact.
 *   workspace  device memory, 256-byte aligned, of any size, or NULL; no
 *              initialisation, nothing kept between calls. With the bytes that
 *              comem_keep_tokens_workspace says, long rows are shared by several
 *              workgroups (three kernels instead of one; the same results).
 * Of the plan only max_ctx_len and the device matter. Outputs may not overlap
 * the inputs. */
comem_status comem_keep_tokens(const comem_decode_attn_plan* plan, const float* weights, int64_t weights_stride,
                               const int32_t* ctx_lens, int32_t num_rows, const int32_t* rows, int32_t n,
                               int64_t max_ctx_len, int32_t budget, const int32_t* budgets, int32_t first,
                               int32_t last, int32_t* keep, int64_t keep_stride, int64_t* keep_start,
                               int32_t* keep_lens, float* kept, void* workspace, size_t workspace_bytes,
                               void* hip_stream);

#ifdef __cplusplus
}
#endif

#endif /* COMEM_KV_EVICT_H */
