/*
 * comem_prefill_fp8.h -- prefill attention over a cached prefix on AMD
 * Instinct MI355X (gfx950), for FP8 caches.
 *
 * The operation of comem_prefill_attn.h over the FP8 caches of
 * comem_decode_attn.h: new token i of sequence b attends over the cached
 * tokens 0 .. L_b - M_b + i, whose keys and values are E4M3 codes times the
 * plan's k_scale and v_scale; queries are bfloat16:
 *
 *     s_t = scale * k_scale * dot(q[i, h, :], Kcode_b[t, h / G, :])
 *     out = v_scale * sum_t softmax(s)_t * Vcode_b[t, h / G, :]
 *     lse = ln sum_t exp(s_t)
 *
 * Codes are exact on the matrix cores; scores and sums are fp32. The
 * probabilities enter as a sum of two f16 values: a weight is off by at most
 * 2^-23 of itself, or by 2^-34 of the row's largest weight where that is more.
 * A NaN code of K makes out and lse of the rows that see it NaN; a NaN code of
 * V the outputs at its place, and that of a new token may reach new tokens
 * before it too.
 *
 * The calls take a plan from comem_decode_attn_init whose dtype is
 * COMEM_FP8_E4M3 (others: COMEM_ERR_UNSUPPORTED); its heads, head_dim, scales,
 * max_batch and max_ctx_len apply, its chunk_tokens and variant do not.
 * Execution, ownership, errors and the device-side contract are those of
 * comem_prefill_attn.h.
 */
#ifndef COMEM_PREFILL_FP8_H
#define COMEM_PREFILL_FP8_H

#include "comem_decode_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* *workspace_bytes_out gets the bytes that a call with these bounds can use
 * (0: none), as comem_prefill_attn_workspace. */
comem_status comem_prefill_fp8_workspace(const comem_decode_attn_plan* plan, int32_t batch, int32_t max_q_len,
                                         int64_t max_ctx_len, size_t* workspace_bytes_out);

/* Contiguous / ragged cache. Arguments as in comem_prefill_attn_split; strides
 * count bytes. workspace: NULL or of any size, 256-byte aligned; with one of
 * comem_prefill_fp8_workspace's size, the keys of a few new tokens' blocks are
 * shared by several workgroups and a second kernel merges the results. */
comem_status comem_prefill_fp8_attn(const comem_decode_attn_plan* plan, const void* q, const int64_t* q_start,
                                    const int32_t* q_lens, int32_t max_q_len, const void* k, const void* v,
                                    int64_t stride_token, int64_t stride_head, const int64_t* seq_start,
                                    const int32_t* ctx_lens, int32_t batch, int64_t max_ctx_len, float* out,
                                    float* lse, void* workspace, size_t workspace_bytes, void* hip_stream);

/* Paged cache. Arguments as in comem_prefill_attn_split_paged. */
comem_status comem_prefill_fp8_attn_paged(const comem_decode_attn_plan* plan, const void* q, const int64_t* q_start,
                                          const int32_t* q_lens, int32_t max_q_len, const void* k_pages,
                                          const void* v_pages, int64_t stride_page, int64_t stride_token,
                                          int64_t stride_head, int32_t page_size, int64_t num_pages,
                                          const int32_t* block_table, int32_t max_pages_per_seq,
                                          const int32_t* ctx_lens, int32_t batch, int64_t max_ctx_len, float* out,
                                          float* lse, void* workspace, size_t workspace_bytes, void* hip_stream);

#ifdef __cplusplus
}
#endif

#endif /* COMEM_PREFILL_FP8_H */
