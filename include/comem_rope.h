/*
 * comem_rope.h -- new tokens' queries, keys and values on their way into the
 * attention calls: head norms, position rotation and the cache store in one
 * pass, on AMD Instinct MI355X (gfx950).
 *
 * Between a layer's projections and its attention (the paper's models are
 * grouped-query models of this kind, Sec. 2.2), every query and key head
 * x[0 .. d_h) of a new token is normalised over its elements (where the model
 * has such norms) and its first rot_dim elements are rotated to the token's
 * position; the key and the value then join the cache. With w the norm's
 * weight, p the position, R = rot_dim, and (c, s) the row p of the table of
 * cosines and sines:
 *
 *     y_j = x_j * w_j / sqrt(mean_i x_i^2 + eps)        (without a weight: y = x)
 *     z_j         = y_j c_j - y_{j + R/2} s_j           j = 0 .. R/2 - 1
 *     z_{j + R/2} = y_{j + R/2} c_j + y_j s_j
 *     z_j         = y_j                                 j = R .. d_h - 1
 *
 * or, with COMEM_ROPE_INTERLEAVED, the same for the pairs (y_2j, y_2j+1) in
 * the places 2j and 2j + 1. All of it is float32; q_out and the cache get the
 * result rounded once: to nearest in the plan's type, or, for FP8 caches, the
 * E4M3 code nearest to z * (1 / k_scale) (and v * (1 / v_scale)), reciprocal
 * and product in float32, magnitudes above 448 becoming 448 and NaN staying
 * NaN.
 *
 * Sequence b holds L_b = ctx_lens[b] tokens, of which the last M_b are the new
 * ones, as in the prefill calls (comem_prefill_attn.h): new token i becomes
 * cache token t = L_b - M_b + i. Its position is t, or what `positions` says
 * (after a cut of the context, comem_kv_compact, cache index and position
 * differ). With q_start and q_lens NULL every sequence has one new token, row
 * b, as in a decode step. A call stores the last M_b tokens of what ctx_lens
 * says: where a sequence may have been refused room (comem_kv_reserve), its
 * M_b must be 0, or tokens it holds are overwritten. q_lens may be the
 * lengths that comem_kv_reserve_granted left on the device.
 *
 * Both calls take a plan from comem_decode_attn_init: its heads, head_dim,
 * dtype (q, new keys and values and weights are float32 for COMEM_F32 plans
 * and bfloat16 otherwise), FP8 scales, max_batch and max_ctx_len apply. They
 * need no workspace, enqueue one kernel on the given stream and return. FP8
 * scales whose reciprocal is not a finite float32 give COMEM_ERR_UNSUPPORTED.
 * Ownership and errors are those of the decode calls.
 *
 * Device-side contract: 0 <= q_lens[b] <= ctx_lens[b] <= max_ctx_len and
 * q_lens[b] <= max_q_len; a sequence outside of it is skipped, nothing of it
 * is written. A token whose block-table entry lies outside [0, num_pages)
 * gets its q_out rows, its key and value are not stored. A position outside
 * [0, num_positions) is taken as the nearest one inside. Rows of q_out that
 * belong to no sequence are left as they were, like every cache element that
 * no new token goes to.
 */
#ifndef COMEM_ROPE_H
#define COMEM_ROPE_H

#include "comem_decode_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

#define COMEM_ROPE_INTERLEAVED 1u /* rotate the pairs (2j, 2j + 1) instead of (j, j + R/2) */

/* The model's side of a call. Device pointers, 16-byte aligned.
 *   q_weight, k_weight  [d_h] of the new rows' type, or NULL: no norm.
 *   cos_sin        float32 [num_positions, rot_dim]: rot_dim / 2 cosines,
 *                  then as many sines. NULL only with rot_dim = 0.
 *   num_positions  0 < num_positions < 2^31 (with rot_dim > 0).
 *   rot_dim        0 (no rotation) or a multiple of 16 up to d_h.
 *   eps            finite, >= 0.
 *   flags          0 or COMEM_ROPE_INTERLEAVED. */
typedef struct {
  const void* q_weight;
  const void* k_weight;
  const float* cos_sin;
  int64_t num_positions;
  int32_t rot_dim;
  float eps;
  uint32_t flags;
} comem_rope_config;

/* Contiguous / ragged cache.
 *   q, new_k, new_v  element (row, h, d) at q[row * q_stride + h * d_h + d];
 *              the strides count elements and are at least heads * d_h, so
 *              the three may be parts of one projection's output. 16-byte
 *              aligned, byte strides multiples of 16.
 *   q_start    device int64 [batch]: first row of each sequence's new tokens.
 *   q_lens     device int32 [batch]: M_b. (Both or neither may be NULL.)
 *   max_q_len  host bound >= every q_lens[b], 0 .. max_ctx_len; 1 when q_lens
 *              is NULL; COMEM_ERR_INVALID_SHAPE above 2^26 - 1. With max_q_len
 *              = 0 or batch = 0 nothing is enqueued and no pointer is looked at.
 *   positions  device int32, one for each row, or NULL.
 *   q_out      [rows, h_q, d_h] dense, q's type, 16-byte aligned. May be q
 *              itself where q is dense; no other overlap.
 *   k, v, stride_token, stride_head, seq_start, ctx_lens, batch, max_ctx_len:
 *              as in comem_decode_attn, k and v being written. */
comem_status comem_rope_append(const comem_decode_attn_plan* plan, const comem_rope_config* rope, const void* q,
                               int64_t q_stride, const void* new_k, int64_t k_stride, const void* new_v,
                               int64_t v_stride, const int64_t* q_start, const int32_t* q_lens, int32_t max_q_len,
                               const int32_t* positions, void* q_out, void* k, void* v, int64_t stride_token,
                               int64_t stride_head, const int64_t* seq_start, const int32_t* ctx_lens,
                               int32_t batch, int64_t max_ctx_len, void* hip_stream);

/* Paged cache; pages, strides and block table as in comem_decode_attn_paged. */
comem_status comem_rope_append_paged(const comem_decode_attn_plan* plan, const comem_rope_config* rope,
                                     const void* q, int64_t q_stride, const void* new_k, int64_t k_stride,
                                     const void* new_v, int64_t v_stride, const int64_t* q_start,
                                     const int32_t* q_lens, int32_t max_q_len, const int32_t* positions,
                                     void* q_out, void* k_pages, void* v_pages, int64_t stride_page,
                                     int64_t stride_token, int64_t stride_head, int32_t page_size,
                                     int64_t num_pages, const int32_t* block_table, int32_t max_pages_per_seq,
                                     const int32_t* ctx_lens, int32_t batch, int64_t max_ctx_len,
                                     void* hip_stream);

#ifdef __cplusplus
}
#endif

#endif /* COMEM_ROPE_H */
