// Host side of the block-attention C ABI (comem_block_attn.h): argument
// validation (before any HIP call) and launch of the kernels. comem_block_attn
// itself is a decode call and lives in api.cpp.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <cstring>

#include "blocks.h"
#include "comem_block_attn.h"
#include "comem_decode_attn.h"
#include "plan.h"

using namespace comem::host;

namespace {

constexpr int64_t kMostBlocks = int64_t{1} << 20;  // workgroups of a sequence; past them each takes several blocks

comem_status check_bounds(const comem_decode_attn_plan& p, int32_t batch, int64_t max_ctx_len) {
  if (batch < 0 || batch > p.cfg.max_batch) return COMEM_ERR_INVALID_SHAPE;
  return max_ctx_len < 0 || max_ctx_len > p.cfg.max_ctx_len ? COMEM_ERR_INVALID_SHAPE : COMEM_OK;
}

// The block table's part of validate_paged, for calls that look at no pages.
comem_status check_table(int32_t page_size, const int32_t* block_table, int32_t max_pages_per_seq,
                         int64_t max_ctx_len) {
  if (block_table == nullptr) return COMEM_ERR_NULL_POINTER;
  if (page_size <= 0 || page_size > 4096 || (page_size & (page_size - 1)) != 0) return COMEM_ERR_INVALID_SHAPE;
  if (max_pages_per_seq <= 0 || max_pages_per_seq < ceil_div(max_ctx_len, page_size)) return COMEM_ERR_INVALID_SHAPE;
  return aligned(block_table, 4) ? COMEM_OK : COMEM_ERR_MISALIGNED;
}

template <typename Params>
comem_status launched(void (*fn)(Params), dim3 grid, int threads, Params& a, void* stream) {
  if (fn == nullptr) return COMEM_ERR_UNSUPPORTED;
  void* argv[] = {&a};
  const hipError_t err = hipLaunchKernel(reinterpret_cast<const void*>(fn), grid, dim3(static_cast<unsigned>(threads)),
                                         argv, 0, static_cast<hipStream_t>(stream));
  return err == hipSuccess ? COMEM_OK : COMEM_ERR_HIP;
}

}  // namespace

extern "C" {

comem_status comem_block_bounds(const comem_decode_attn_plan* plan, const void* k_pages, int64_t stride_page,
                                int64_t stride_token, int64_t stride_head, int32_t page_size, int64_t num_pages,
                                const int32_t* block_table, int32_t max_pages_per_seq, const int32_t* ctx_lens,
                                const int32_t* q_lens, int32_t max_q_len, int32_t batch, int64_t max_ctx_len,
                                void* bounds, void* hip_stream) {
  const comem_decode_attn_plan* p = checked(plan);
  if (p == nullptr) return COMEM_ERR_BAD_HANDLE;
  comem_status st = check_bounds(*p, batch, max_ctx_len);
  if (st != COMEM_OK) return st;
  if (max_q_len < 0 || max_q_len > max_ctx_len) return COMEM_ERR_INVALID_SHAPE;
  if (batch == 0 || max_q_len == 0) return COMEM_OK;
  if (k_pages == nullptr || ctx_lens == nullptr || bounds == nullptr) return COMEM_ERR_NULL_POINTER;
  if (q_lens == nullptr && max_q_len != 1) return COMEM_ERR_INVALID_SHAPE;
  if (stride_token <= 0 || stride_head < 0) return COMEM_ERR_INVALID_SHAPE;
  if (p->cfg.num_kv_heads > 1 && stride_head == 0) return COMEM_ERR_INVALID_SHAPE;
  const int64_t e = elem_bytes(p->cfg);
  if (stride_token > kMaxTokenStrideBytes / e) return COMEM_ERR_INVALID_SHAPE;
  if ((stride_token * e) % 16 != 0 || (stride_head * e) % 16 != 0) return COMEM_ERR_MISALIGNED;
  if (!aligned(k_pages, 16) || !aligned(bounds, 16) || !aligned(ctx_lens, 4) || !aligned(q_lens, 4))
    return COMEM_ERR_MISALIGNED;
  st = validate_paged(*p, stride_page, page_size, num_pages, block_table, max_pages_per_seq, max_ctx_len);
  if (st != COMEM_OK) return st;
  if (p->device == COMEM_NO_DEVICE) return COMEM_ERR_NO_DEVICE;
  comem::BoundsParams a;
  std::memset(&a, 0, sizeof(a));
  a.k = static_cast<const char*>(k_pages);
  a.bounds = static_cast<char*>(bounds);
  a.ctx_lens = ctx_lens;
  a.q_lens = q_lens;
  a.block_table = block_table;
  a.stride_page = stride_page * e;
  a.stride_token = stride_token * e;
  a.stride_head = stride_head * e;
  a.num_pages = num_pages;
  a.max_pages = max_pages_per_seq;
  a.page_shift = log2_of(page_size);
  a.max_ctx = static_cast<int32_t>(max_ctx_len);
  a.max_q = max_q_len;
  const int64_t head_pieces = p->cfg.head_dim * e / 16;
  a.piece_shift = log2_of(static_cast<int32_t>(head_pieces));
  a.pieces = static_cast<int32_t>(p->cfg.num_kv_heads * head_pieces);
  // Pages that max_q_len tokens can lie in.
  const int64_t pages = std::min({ceil_div(max_q_len - 1, page_size) + 1, ceil_div(max_ctx_len, page_size), kMostBlocks});
  // A workgroup takes whole tokens; of few and long pages 512 bytes of each, so
  // that more workgroups share a page (us, 512 bytes / whole tokens of 2 KiB and,
  // FP8, 1 KiB: 64 pages of 64 tokens 4.2 / 6.0 and 6.1 / 6.9, of 128 5.1 / 9.0
  // and 7.6 / 9.8, of 16 4.2 / 3.6 and 6.1 / 5.5; 1024 of 64 25 / 23 and 26 / 20).
  const bool few = page_size >= 64 && pages * batch <= p->num_cus;
  a.width = std::min(a.pieces, few ? 32 : comem::kBoundsThreads);
  const dim3 grid(static_cast<unsigned>(pages), static_cast<unsigned>(batch),
                  static_cast<unsigned>(ceil_div(a.pieces, a.width)));
  return launched(comem::select_bounds_kernel(comem::cache_type(p->cfg)), grid, comem::kBoundsThreads, a, hip_stream);
}

comem_status comem_block_scores(const comem_decode_attn_plan* plan, const void* q, const void* bounds,
                                int32_t page_size, int64_t num_pages, const int32_t* block_table,
                                int32_t max_pages_per_seq, const int32_t* ctx_lens, int32_t batch,
                                int64_t max_ctx_len, float* scores, int64_t scores_stride, void* hip_stream) {
  const comem_decode_attn_plan* p = checked(plan);
  if (p == nullptr) return COMEM_ERR_BAD_HANDLE;
  comem_status st = check_bounds(*p, batch, max_ctx_len);
  if (st != COMEM_OK || batch == 0) return st;
  if (q == nullptr || bounds == nullptr || ctx_lens == nullptr || (scores == nullptr && max_ctx_len > 0))
    return COMEM_ERR_NULL_POINTER;
  st = check_table(page_size, block_table, max_pages_per_seq, max_ctx_len);
  if (st != COMEM_OK) return st;
  const int64_t blocks = ceil_div(max_ctx_len, page_size);
  if (num_pages <= 0 || scores_stride < blocks) return COMEM_ERR_INVALID_SHAPE;
  if (!aligned(q, 16) || !aligned(bounds, 16) || !aligned(ctx_lens, 4) || !aligned(scores, 4))
    return COMEM_ERR_MISALIGNED;
  if (p->device == COMEM_NO_DEVICE) return COMEM_ERR_NO_DEVICE;
  if (max_ctx_len == 0) return COMEM_OK;
  comem::ScoresParams a;
  std::memset(&a, 0, sizeof(a));
  a.q = static_cast<const char*>(q);
  a.bounds = static_cast<const char*>(bounds);
  a.ctx_lens = ctx_lens;
  a.block_table = block_table;
  a.scores = scores;
  a.scores_stride = scores_stride;
  a.num_pages = num_pages;
  a.max_pages = max_pages_per_seq;
  a.page_shift = log2_of(page_size);
  a.max_ctx = static_cast<int32_t>(max_ctx_len);
  a.num_kv_heads = p->cfg.num_kv_heads;
  a.group = group_of(p->cfg);
  a.scale = p->cfg.scale * (is_fp8(p->cfg) ? p->cfg.k_scale : 1.f);
  const dim3 grid(static_cast<unsigned>(std::min(ceil_div(blocks, comem::kScoresBlocks), kMostBlocks)),
                  static_cast<unsigned>(ceil_div(a.num_kv_heads, comem::kScoresWaves)), static_cast<unsigned>(batch));
  return launched(comem::select_scores_kernel(p->cfg.head_dim, comem::cache_type(p->cfg)), grid, 64 * comem::kScoresWaves, a,
                  hip_stream);
}

comem_status comem_block_select(const comem_decode_attn_plan* plan, const float* scores, int64_t scores_stride,
                                int32_t page_size, const int32_t* block_table, int32_t max_pages_per_seq,
                                const int32_t* ctx_lens, int32_t batch, int64_t max_ctx_len, int32_t budget,
                                int32_t first, int32_t last, int32_t* table, int32_t max_blocks, int32_t* lens,
                                void* hip_stream) {
  const comem_decode_attn_plan* p = checked(plan);
  if (p == nullptr) return COMEM_ERR_BAD_HANDLE;
  comem_status st = check_bounds(*p, batch, max_ctx_len);
  if (st != COMEM_OK || batch == 0) return st;
  if (first < 0 || last < 1 || int64_t{first} + last > budget) return COMEM_ERR_INVALID_SHAPE;
  if (ctx_lens == nullptr || lens == nullptr || (max_ctx_len > 0 && (scores == nullptr || table == nullptr)))
    return COMEM_ERR_NULL_POINTER;
  st = check_table(page_size, block_table, max_pages_per_seq, max_ctx_len);
  if (st != COMEM_OK) return st;
  const int64_t blocks = ceil_div(max_ctx_len, page_size);
  if (scores_stride < blocks || max_blocks < std::min<int64_t>(budget, blocks)) return COMEM_ERR_INVALID_SHAPE;
  if (!aligned(scores, 4) || !aligned(ctx_lens, 4) || !aligned(table, 4) || !aligned(lens, 4))
    return COMEM_ERR_MISALIGNED;
  const int64_t items = int64_t{batch} * p->cfg.num_kv_heads;
  const comem::ChooseForm form = comem::select_choose_kernel(true, blocks, items, p->num_cus);
  if (items > ((int64_t{1} << 32) - 1) / form.threads) return COMEM_ERR_INVALID_SHAPE;  // more than a launch holds
  if (p->device == COMEM_NO_DEVICE) return COMEM_ERR_NO_DEVICE;
  comem::ChooseParams a;
  std::memset(&a, 0, sizeof(a));
  a.scores = scores;
  a.scores_stride = scores_stride;
  a.lens = ctx_lens;
  a.max_len = static_cast<int32_t>(max_ctx_len);
  a.budget = budget;
  a.first = first;
  a.last = last;
  a.out = table;
  a.out_stride = max_blocks;
  a.out_lens = lens;
  a.block_table = block_table;
  a.max_pages = max_pages_per_seq;
  a.heads = p->cfg.num_kv_heads;
  a.page_shift = log2_of(page_size);
  return launched(form.fn, dim3(static_cast<unsigned>(items), static_cast<unsigned>(form.parts)), form.threads, a, hip_stream);
}

}  // extern "C"
