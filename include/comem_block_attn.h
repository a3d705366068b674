/*
 * comem_block_attn.h -- decode attention over chosen blocks of a paged KV
 * cache on AMD Instinct MI355X (gfx950): a cheap score for every block, the
 * blocks with the largest, and attention over those alone.
 *
 * A decode step costs what it reads (paper Sec. 3.3: KV bytes over bandwidth).
 * A context may stay whole and a step still read little of it, where most
 * blocks hold no key that the step's queries score high. The blocks are the
 * cache's pages. For each page, KV head and element the least and the greatest
 * key are kept (comem_block_bounds), which bound every score in the page:
 *
 *     score[b, hk, n] = scale * max_h sum_d (max(q_hd, 0) hi_d + min(q_hd, 0) lo_d)
 *                    >= scale * q_h . k_t      for the keys t of block n
 *
 * over the G query heads h of KV head hk (FP8 caches: times k_scale). Scores are
 * computed as float32 sums, so the inequality holds up to their rounding: 2 d_h
 * 2^-23 of the sum of the products' magnitudes, and 2^-22 of the score. With
 * 2 / page_size of the keys' bytes that is what a step reads of the whole
 * context (comem_block_scores). Then each KV head of each sequence attends
 * over the blocks with its largest scores (comem_block_select,
 * comem_block_attn): out and lse as in comem_decode_attn, over their tokens.
 *
 * Four launches and the bounds' bytes instead of one and all of the keys' and
 * values': worth it for long contexts and for batches. A whole step of these
 * calls and comem_decode_attn_paged, us (graph; 8 KV heads of 128, pages of 64):
 * one sequence of 32 query heads, 64 blocks, bf16 16384 tokens 20.3 / 16.0, 32768
 * 21.7 / 25.6 (called eagerly through the torch wrapper 30 / 25), 65536 25.3 /
 * 43.6, FP8 32768 22.1 / 16.3, 65536 26.0 / 26.3, 131072 28.6 / 45.6; 8 sequences
 * of 64 heads and 131072 tokens, 128 blocks, bf16 77 / 632, FP8 57 / 339.
 *
 * Ownership, errors, streams and the device-side contract (lengths, block
 * tables) are those of the decode calls (comem_decode_attn.h); pages, strides
 * and block tables are those of comem_decode_attn_paged. Each call enqueues
 * one kernel; all but comem_block_attn need no workspace. Same arguments, same
 * bits.
 */
#ifndef COMEM_BLOCK_ATTN_H
#define COMEM_BLOCK_ATTN_H

#include "comem_decode_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Bounds of the pages that the last M_b tokens of each sequence lie in, from
 * the tokens that the pages hold (of the last page those below L_b): after
 * new tokens were stored, or (M_b = L_b) for a whole context, for instance
 * after comem_kv_compact moved it; after comem_kv_fork a child's last page
 * (M_b = 1). Least and greatest by the order of the values as bit patterns:
 * -NaN, -inf, ..., -0, +0, ..., inf, NaN.
 *   q_lens     device int32 [batch]: M_b; NULL: 1 each.
 *   max_q_len  host bound >= every q_lens[b], 0 .. max_ctx_len; 1 when q_lens is
 *              NULL. With max_q_len = 0 or batch = 0 nothing is enqueued and no
 *              pointer is looked at.
 *   bounds     [num_pages, h_kv, 2, d_h] dense, the cache's type (FP8: codes),
 *              16-byte aligned: the least and the greatest of each page and
 *              head. Other pages' bounds are left as they were.
 * A sequence with ctx_lens[b] outside [0, max_ctx_len], or q_lens[b] outside
 * [1, min(ctx_lens[b], max_q_len)], is skipped, and so is a page outside
 * [0, num_pages). Sequences that share a page hold the same tokens of it (as
 * after comem_kv_fork, which shares whole pages alone): each of them writes its
 * bounds. */
comem_status comem_block_bounds(const comem_decode_attn_plan* plan, const void* k_pages, int64_t stride_page,
                                int64_t stride_token, int64_t stride_head, int32_t page_size, int64_t num_pages,
                                const int32_t* block_table, int32_t max_pages_per_seq, const int32_t* ctx_lens,
                                const int32_t* q_lens, int32_t max_q_len, int32_t batch, int64_t max_ctx_len,
                                void* bounds, void* hip_stream);

/* The scores above for one new query token of each sequence.
 *   q          [batch, h_q, d_h] dense, as in comem_decode_attn.
 *   bounds     as above.
 *   scores     float32 [batch, h_kv, scores_stride]: element (b, hk, n), n <
 *              ceil(L_b / page_size), is written, the others are left as they
 *              were. scores_stride >= ceil(max_ctx_len / page_size); where that
 *              is 0, scores may be NULL, here and below.
 * A NaN in a bound or query that meets it makes the score NaN, and so does
 * the product of an infinity and a 0. */
comem_status comem_block_scores(const comem_decode_attn_plan* plan, const void* q, const void* bounds,
                                int32_t page_size, int64_t num_pages, const int32_t* block_table,
                                int32_t max_pages_per_seq, const int32_t* ctx_lens, int32_t batch,
                                int64_t max_ctx_len, float* scores, int64_t scores_stride, void* hip_stream);

/* For each KV head of each sequence the pages of min(budget, N) of its N =
 * ceil(L_b / page_size) blocks: the first `first`, the last `last` and, of those
 * between, the ones with the largest scores, in the context's order. Of equal
 * scores (0 and -0 are equal) the earlier block; NaN is above every number.
 *   first, last >= 0 and >= 1; first + last <= budget.
 *   table      int32 [batch, h_kv, max_blocks]: the pages, as the block table
 *              names them; what follows them is left as it was. max_blocks >=
 *              min(budget, ceil(max_ctx_len / page_size)); may be NULL with
 *              max_ctx_len = 0.
 *   lens       int32 [batch]: the tokens in them, the same for all heads (the
 *              last block is among them, the others are whole); 0 where L_b
 *              is 0, L_b being taken into [0, max_ctx_len] first. */
comem_status comem_block_select(const comem_decode_attn_plan* plan, const float* scores, int64_t scores_stride,
                                int32_t page_size, const int32_t* block_table, int32_t max_pages_per_seq,
                                const int32_t* ctx_lens, int32_t batch, int64_t max_ctx_len, int32_t budget,
                                int32_t first, int32_t last, int32_t* table, int32_t max_blocks, int32_t* lens,
                                void* hip_stream);

/* Decode attention with a block table for each KV head: head hk of sequence b
 * attends over the first lens[b] tokens of the pages table[b, hk, :].
 *   table      device int32 [batch, h_kv, max_blocks], max_blocks >=
 *              ceil(max_len / page_size).
 *   lens       device int32 [batch]; max_len the host's bound of them, at most
 *              the plan's max_ctx_len.
 * Other arguments, workspace (calls that share one do not overlap, decode calls
 * among them) and results as in comem_decode_attn_paged, but that the weights enter the matrix cores in three bf16 parts instead of two:
 * a weight is off by less than 2^-26 of itself. */
comem_status comem_block_attn(const comem_decode_attn_plan* plan, const void* q, const void* k_pages,
                              const void* v_pages, int64_t stride_page, int64_t stride_token, int64_t stride_head,
                              int32_t page_size, int64_t num_pages, const int32_t* table, int32_t max_blocks,
                              const int32_t* lens, int32_t batch, int64_t max_len, float* out, float* lse,
                              void* workspace, size_t workspace_bytes, void* hip_stream);

#ifdef __cplusplus
}
#endif

#endif /* COMEM_BLOCK_ATTN_H */
