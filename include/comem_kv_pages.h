/*
 * comem_kv_pages.h -- the pages of a paged KV cache, kept on the GPU, on AMD
 * Instinct MI355X (gfx950): pages for new tokens, a second sequence on the
 * same history, a context cut to the tokens that stay, pages given back.
 *
 * The paper's pipeline keeps an agent stepping on its history while a memory
 * model reads that history, and then replaces it by a summary and the recent
 * buffer (Algorithm 1, Sec. 3.2): the sequence is forked, and later compacted.
 * These calls do it on the block table that the paged attention calls read
 * (comem_decode_attn.h). All state lies in device memory and no call looks at
 * it from the host, so a decode loop that takes pages as it goes can be
 * captured in a graph. A row that gets no room keeps its length, and a call
 * after it that stores new tokens as the row's last ones would write over
 * tokens it holds, which forks may share: such a loop has to learn on the
 * device which rows grew (comem_kv_reserve_granted).
 *
 * State, the caller's (comem_kv_pages below): a block table of num_rows rows,
 * one sequence each, ctx_lens[r] tokens long, and refcounts[p], the number of
 * table entries that hold page p. A page with count 0 is free. The entries
 * i < ceil(ctx_lens[r] / page_size) of row r hold pages, the others nothing
 * (-1 by custom; what they say plays no part). To begin with: zero refcounts and
 * ctx_lens. A caller that keeps a page for itself sets its count to 1.
 *
 * A page that several rows hold is full in all of them: forks share whole
 * pages and copy the last, partly filled one, so that the rows' next tokens
 * go to pages of their own.
 *
 * Pages are given out lowest free page first, to the call's rows in their
 * order and to a row's entries in theirs: the same state and arguments always
 * give the same pages. A call that needs more pages than are free takes none,
 * changes nothing and stores the number it lacks in *missing, else 0.
 *
 * One block table may serve the caches of several layers: num_layers pools,
 * stride_layer apart, whose pages are copied together.
 *
 * Ownership, errors and streams are as for the decode calls: every argument
 * is checked on the host before any HIP call; the calls enqueue their kernels
 * on the given stream and return, and neither allocate nor synchronise. Calls
 * on one state change it and must be ordered, by one stream or by events, and
 * enqueued one after the other (a call is several kernels); the workspace
 * belongs to the state.
 *
 * Device-side contract: 0 <= ctx_lens[r] <= max_ctx_len; entries that hold
 * pages lie in [0, num_pages). A row outside the first part is left as it is.
 * An entry outside the pool is read as page 0 where tokens are copied from it,
 * and is not counted. What else a call leaves out is said there; no violation
 * leads to an access outside the given buffers.
 */
#ifndef COMEM_KV_PAGES_H
#define COMEM_KV_PAGES_H

#include "comem_decode_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Strides count elements of the plan's dtype (bytes for FP8 caches); those of
 * page, token and head as in comem_decode_attn_paged. Pointers are to device
 * memory. comem_kv_reserve and comem_kv_release do not look at the pools. */
typedef struct {
  void* k_pages;
  void* v_pages;
  int64_t stride_layer; /* from a layer's pool to the next; not looked at with one layer */
  int64_t stride_page;
  int64_t stride_token;
  int64_t stride_head;
  int32_t num_layers;   /* 1 .. 65535 */
  int32_t page_size;    /* a power of two, 1 .. 4096 */
  int64_t num_pages;    /* 1 .. 2^31 - 1 */
  int32_t* refcounts;   /* [num_pages] */
  int32_t* block_table; /* [num_rows, max_pages_per_seq] */
  int32_t* ctx_lens;    /* [num_rows] */
  int32_t num_rows;     /* 1 .. 65535; need not be the plan's max_batch */
  int32_t max_pages_per_seq; /* >= ceil(max_ctx_len / page_size) */
  int64_t max_ctx_len;  /* bound of every ctx_lens[r], <= plan max_ctx_len */
} comem_kv_pages;

/* *workspace_bytes_out gets the size of the workspace that every call on
 * `pages` fits in: device memory, 256-byte aligned, no initialisation, nothing
 * kept between calls. */
comem_status comem_kv_pages_workspace(const comem_decode_attn_plan* plan, const comem_kv_pages* pages,
                                      size_t* workspace_bytes_out);

/* Room for add_lens[r] more tokens in every row r: the row gets the pages that
 * ceil((ctx_lens[r] + add_lens[r]) / page_size) asks for besides those it has,
 * and ctx_lens[r] grows by add_lens[r]. A row with add_lens[r] < 0, or that
 * would grow past max_ctx_len, is left as it is and does not show in *missing.
 * Neither does *missing reach a call enqueued after this one: unless the
 * caller has looked at it, and knows that no row passes max_ctx_len, use
 * comem_kv_reserve_granted.
 *   add_lens   device int32 [num_rows].
 *   missing    device int32 [1]. */
comem_status comem_kv_reserve(const comem_decode_attn_plan* plan, const comem_kv_pages* pages,
                              const int32_t* add_lens, int32_t* missing, void* workspace,
                              size_t workspace_bytes, void* hip_stream);

/* The same, and granted[r] becomes the number of tokens that row r grew by:
 * add_lens[r], or 0 for a row that is left as it is (every row, where pages
 * are missing). It is the q_lens of the calls that follow: comem_rope_append
 * with q_lens = granted stores nothing for a row without room, prefill writes
 * nothing. comem_kv_append and the fused append have no such argument: give
 * them, and the attention, lengths that are 0 for those rows.
 *   granted    device int32 [num_rows], not overlapping add_lens. */
comem_status comem_kv_reserve_granted(const comem_decode_attn_plan* plan, const comem_kv_pages* pages,
                                      const int32_t* add_lens, int32_t* granted, int32_t* missing,
                                      void* workspace, size_t workspace_bytes, void* hip_stream);

/* Row children[i] becomes a second sequence on the tokens of row parents[i]:
 * it holds the parent's whole pages too, and of a last, partly filled one a
 * copy in a page of its own (K and V of its tokens, every layer; the rest of
 * that page is left as it was). A parent may be named several times. Children
 * are empty (ctx_lens 0) before the call; a child that is not empty or stands
 * earlier in the list, a row outside [0, num_rows) or a row as its own child
 * leaves that pair out.
 *   parents, children  device int32 [n], 0 <= n <= num_rows (0: nothing is
 *              enqueued, *missing is not written and no pointer looked at). */
comem_status comem_kv_fork(const comem_decode_attn_plan* plan, const comem_kv_pages* pages, const int32_t* parents,
                           const int32_t* children, int32_t n, int32_t* missing, void* workspace,
                           size_t workspace_bytes, void* hip_stream);

/* The context of row rows[i] is cut to keep_lens[i] of its tokens: token t
 * becomes what was token keep[keep_start[i] + t], for every layer. The list is
 * strictly increasing, so whole pages at its start whose tokens all stay in
 * place stay too, shared ones among them; from the first other page on the
 * tokens are copied to fresh pages (taken before the old ones are given back)
 * and the old entries are given up. The keys are copied as they are: their
 * rotation remains that of the position they were made at, and the positions
 * of later tokens (comem_rope_append) are the caller's to keep. This is also
 * the way to drop a row's last tokens (its list is then the first ones): a
 * ctx_lens entry lowered by hand would leave its pages counted.
 *   rows       device int32 [n]; 0 <= n <= num_rows (0: as above).
 *   keep       device int32 [keep_total] (NULL with keep_total = 0).
 *   keep_start device int64 [n]; keep_lens device int32 [n].
 * A row outside [0, num_rows), one that stands earlier in rows, one with more
 * kept tokens than it has, or with a list outside [0, keep_total) is left as
 * it is (of a row named twice the first list counts). A listed position outside
 * the row's tokens is taken as the nearest one. */
comem_status comem_kv_compact(const comem_decode_attn_plan* plan, const comem_kv_pages* pages, const int32_t* rows,
                              const int32_t* keep, int64_t keep_total, const int64_t* keep_start,
                              const int32_t* keep_lens, int32_t n, int32_t* missing, void* workspace,
                              size_t workspace_bytes, void* hip_stream);

/* The rows give up their pages: entries become -1, their counts go down by
 * one, ctx_lens become 0. Rows outside [0, num_rows) and empty rows are
 * skipped; a row may be named twice.
 *   rows       device int32 [n], 0 <= n <= num_rows (0: nothing is enqueued). */
comem_status comem_kv_release(const comem_decode_attn_plan* plan, const comem_kv_pages* pages, const int32_t* rows,
                              int32_t n, void* hip_stream);

#ifdef __cplusplus
}
#endif

#endif /* COMEM_KV_PAGES_H */
