// Host side of the eviction C ABI (comem_kv_evict.h): argument validation
// (before any HIP call) and launch of the kernels.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <cstring>

#include "comem_decode_attn.h"
#include "comem_kv_evict.h"
#include "evict.h"
#include "plan.h"

using namespace comem::host;

namespace {

constexpr int64_t kMostTiles = int64_t{1} << 20;  // workgroups of a sequence; past them each takes several tiles

bool weights_is_empty(int32_t batch, int32_t max_q_len) { return batch == 0 || max_q_len == 0; }

// Checks of a weights call shared by both layouts; fills the kernel arguments.
comem_status prepare_weights(const comem_decode_attn_plan& p, const void* q, const float* lse, const int64_t* q_start,
                             const int32_t* q_lens, int32_t max_q_len, const void* k, int64_t stride_token,
                             int64_t stride_head, const int32_t* ctx_lens, int32_t batch, int64_t max_ctx_len,
                             const float* prior, float decay, float* weights, int64_t weights_stride,
                             comem::WeightsParams& a) {
  if (batch < 0 || batch > p.cfg.max_batch) return COMEM_ERR_INVALID_SHAPE;
  if (max_ctx_len < 0 || max_ctx_len > p.cfg.max_ctx_len) return COMEM_ERR_INVALID_SHAPE;
  if (max_q_len < 0 || max_q_len > max_ctx_len) return COMEM_ERR_INVALID_SHAPE;
  if (weights_is_empty(batch, max_q_len)) return COMEM_OK;
  if (q == nullptr || lse == nullptr || k == nullptr || ctx_lens == nullptr || weights == nullptr ||
      (q_start == nullptr) != (q_lens == nullptr))
    return COMEM_ERR_NULL_POINTER;
  if (q_lens == nullptr && max_q_len != 1) return COMEM_ERR_INVALID_SHAPE;
  if (prior != nullptr && (!std::isfinite(decay) || decay < 0)) return COMEM_ERR_INVALID_SHAPE;
  if (weights_stride < max_ctx_len || stride_token <= 0 || stride_head < 0) return COMEM_ERR_INVALID_SHAPE;
  if (p.cfg.num_kv_heads > 1 && stride_head == 0) return COMEM_ERR_INVALID_SHAPE;
  const int64_t e = elem_bytes(p.cfg);
  if (stride_token > kMaxTokenStrideBytes / e) return COMEM_ERR_INVALID_SHAPE;
  if ((stride_token * e) % 16 != 0 || (stride_head * e) % 16 != 0) return COMEM_ERR_MISALIGNED;
  if (!aligned(q, 16) || !aligned(k, 16) || !aligned(lse, 4) || !aligned(q_start, 8) || !aligned(q_lens, 4) ||
      !aligned(ctx_lens, 4) || !aligned(prior, 4) || !aligned(weights, 4))
    return COMEM_ERR_MISALIGNED;
  std::memset(&a, 0, sizeof(a));
  a.q = static_cast<const char*>(q);
  a.lse = lse;
  a.k = static_cast<const char*>(k);
  a.q_start = q_start;
  a.q_lens = q_lens;
  a.ctx_lens = ctx_lens;
  a.prior = decay != 0 ? prior : nullptr;
  a.weights = weights;
  a.weights_stride = weights_stride;
  a.stride_token = stride_token * e;
  a.stride_head = stride_head * e;
  a.max_ctx = static_cast<int32_t>(max_ctx_len);
  a.max_q = max_q_len;
  a.num_kv_heads = p.cfg.num_kv_heads;
  a.group_shift = log2_of(group_of(p.cfg));
  a.scale_log2 = p.cfg.scale * (is_fp8(p.cfg) ? p.cfg.k_scale : 1.f) * 1.4426950408889634f;
  a.decay = decay;
  return COMEM_OK;
}

comem_status launch_weights(const comem_decode_attn_plan& p, comem::WeightsParams& a, bool paged, int32_t batch,
                            void* stream) {
  int sub = p.cfg.dtype == COMEM_F32 ? 2 : 4;
  while (sub > 1 && batch * ceil_div(a.max_ctx, 16 * sub) < 2 * p.num_cus) sub /= 2;
  const comem::WeightsKernelFn fn = comem::select_weights_kernel(p.cfg.head_dim, comem::cache_type(p.cfg), paged, sub);
  if (fn == nullptr) return COMEM_ERR_UNSUPPORTED;
  const int64_t tiles = std::min(ceil_div(a.max_ctx, 16 * sub), kMostTiles);
  void* argv[] = {&a};
  const hipError_t err = hipLaunchKernel(reinterpret_cast<const void*>(fn),
                                         dim3(static_cast<unsigned>(tiles), static_cast<unsigned>(batch)),
                                         dim3(64 * comem::kWeightsWaves), argv, 0, static_cast<hipStream_t>(stream));
  return err == hipSuccess ? COMEM_OK : COMEM_ERR_HIP;
}

}  // namespace

extern "C" {

comem_status comem_attn_weights(const comem_decode_attn_plan* plan, const void* q, const float* lse,
                                const int64_t* q_start, const int32_t* q_lens, int32_t max_q_len, const void* k,
                                int64_t stride_token, int64_t stride_head, const int64_t* seq_start,
                                const int32_t* ctx_lens, int32_t batch, int64_t max_ctx_len, const float* prior,
                                float decay, float* weights, int64_t weights_stride, void* hip_stream) {
  const comem_decode_attn_plan* p = checked(plan);
  if (p == nullptr) return COMEM_ERR_BAD_HANDLE;
  comem::WeightsParams a;
  const comem_status st = prepare_weights(*p, q, lse, q_start, q_lens, max_q_len, k, stride_token, stride_head, ctx_lens,
                                          batch, max_ctx_len, prior, decay, weights, weights_stride, a);
  if (st != COMEM_OK || weights_is_empty(batch, max_q_len)) return st;
  if (seq_start == nullptr) return COMEM_ERR_NULL_POINTER;
  if (!aligned(seq_start, 8)) return COMEM_ERR_MISALIGNED;
  if (p->device == COMEM_NO_DEVICE) return COMEM_ERR_NO_DEVICE;
  a.seq_start = seq_start;
  return launch_weights(*p, a, false, batch, hip_stream);
}

comem_status comem_attn_weights_paged(const comem_decode_attn_plan* plan, const void* q, const float* lse,
                                      const int64_t* q_start, const int32_t* q_lens, int32_t max_q_len,
                                      const void* k_pages, int64_t stride_page, int64_t stride_token,
                                      int64_t stride_head, int32_t page_size, int64_t num_pages,
                                      const int32_t* block_table, int32_t max_pages_per_seq, const int32_t* ctx_lens,
                                      int32_t batch, int64_t max_ctx_len, const float* prior, float decay,
                                      float* weights, int64_t weights_stride, void* hip_stream) {
  const comem_decode_attn_plan* p = checked(plan);
  if (p == nullptr) return COMEM_ERR_BAD_HANDLE;
  comem::WeightsParams a;
  comem_status st = prepare_weights(*p, q, lse, q_start, q_lens, max_q_len, k_pages, stride_token, stride_head,
                                    ctx_lens, batch, max_ctx_len, prior, decay, weights, weights_stride, a);
  if (st != COMEM_OK || weights_is_empty(batch, max_q_len)) return st;
  st = validate_paged(*p, stride_page, page_size, num_pages, block_table, max_pages_per_seq, max_ctx_len);
  if (st != COMEM_OK) return st;
  if (p->device == COMEM_NO_DEVICE) return COMEM_ERR_NO_DEVICE;
  a.block_table = block_table;
  a.stride_page = stride_page * elem_bytes(p->cfg);
  a.num_pages = num_pages;
  a.max_pages = max_pages_per_seq;
  a.page_shift = log2_of(page_size);
  a.page_mask = page_size - 1;
  return launch_weights(*p, a, true, batch, hip_stream);
}

comem_status comem_keep_tokens(const comem_decode_attn_plan* plan, const float* weights, int64_t weights_stride,
                               const int32_t* ctx_lens, int32_t num_rows, const int32_t* rows, int32_t n,
                               int64_t max_ctx_len, int32_t budget, const int32_t* budgets, int32_t first,
                               int32_t last, int32_t* keep, int64_t keep_stride, int64_t* keep_start,
                               int32_t* keep_lens, float* kept, void* hip_stream) {
  const comem_decode_attn_plan* p = checked(plan);
  if (p == nullptr) return COMEM_ERR_BAD_HANDLE;
  if (num_rows < 1 || num_rows > kGridYZLimit || n < 0 || n > num_rows) return COMEM_ERR_INVALID_SHAPE;
  if (max_ctx_len < 0 || max_ctx_len > p->cfg.max_ctx_len) return COMEM_ERR_INVALID_SHAPE;
  if (first < 0 || last < 0 || int64_t{first} + last > budget) return COMEM_ERR_INVALID_SHAPE;
  if (n == 0) return COMEM_OK;
  const int64_t most = std::min<int64_t>(budget, max_ctx_len);
  if (weights_stride < max_ctx_len || keep_stride < most) return COMEM_ERR_INVALID_SHAPE;
  if ((weights == nullptr && max_ctx_len > 0) || ctx_lens == nullptr || (keep == nullptr && most > 0) ||
      keep_lens == nullptr)
    return COMEM_ERR_NULL_POINTER;
  if (!aligned(weights, 4) || !aligned(ctx_lens, 4) || !aligned(rows, 4) || !aligned(budgets, 4) ||
      !aligned(keep, 4) || !aligned(keep_start, 8) || !aligned(keep_lens, 4) || !aligned(kept, 4))
    return COMEM_ERR_MISALIGNED;
  if (p->device == COMEM_NO_DEVICE) return COMEM_ERR_NO_DEVICE;
  comem::ChooseParams a;
  std::memset(&a, 0, sizeof(a));
  a.scores = weights;
  a.scores_stride = weights_stride;
  a.lens = ctx_lens;
  a.rows = rows;
  a.budgets = budgets;
  a.num_rows = num_rows;
  a.max_len = static_cast<int32_t>(max_ctx_len);
  a.budget = budget;
  a.first = first;
  a.last = last;
  a.out = keep;
  a.out_stride = keep_stride;
  a.out_start = keep_start;
  a.out_lens = keep_lens;
  a.kept = kept;
  const comem::ChooseForm form = comem::select_choose_kernel(false, max_ctx_len, n, p->num_cus);
  void* argv[] = {&a};
  const hipError_t err =
      hipLaunchKernel(reinterpret_cast<const void*>(form.fn), dim3(static_cast<unsigned>(n), static_cast<unsigned>(form.parts)),
                      dim3(static_cast<unsigned>(form.threads)), argv, 0, static_cast<hipStream_t>(hip_stream));
  return err == hipSuccess ? COMEM_OK : COMEM_ERR_HIP;
}

}  // extern "C"
