// Host side of the rotate-and-store C ABI (comem_rope.h): argument validation
// (before any HIP call) and launch of the kernel.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <cstring>

#include "comem_decode_attn.h"
#include "comem_rope.h"
#include "plan.h"
#include "rope.h"

using namespace comem::host;

namespace {

bool rope_is_empty(int32_t batch, int32_t max_q_len) { return batch == 0 || max_q_len == 0; }

comem_status check_rope(const comem_decode_attn_plan& p, const comem_rope_config* r) {
  if (r == nullptr) return COMEM_ERR_NULL_POINTER;
  if ((r->flags & ~COMEM_ROPE_INTERLEAVED) != 0) return COMEM_ERR_UNSUPPORTED;
  if (r->rot_dim < 0 || r->rot_dim > p.cfg.head_dim || r->rot_dim % 16 != 0) return COMEM_ERR_INVALID_SHAPE;
  if (!std::isfinite(r->eps) || r->eps < 0) return COMEM_ERR_INVALID_SHAPE;
  if (r->rot_dim > 0) {
    if (r->num_positions <= 0 || r->num_positions > INT32_MAX) return COMEM_ERR_INVALID_SHAPE;
    if (r->cos_sin == nullptr) return COMEM_ERR_NULL_POINTER;
  }
  if (!aligned(r->cos_sin, 16) || !aligned(r->q_weight, 16) || !aligned(r->k_weight, 16)) return COMEM_ERR_MISALIGNED;
  return COMEM_OK;
}

// Checks of a call shared by both layouts; fills the kernel arguments.
comem_status prepare_rope(const comem_decode_attn_plan& p, const comem_rope_config* rope, const void* q,
                          int64_t q_stride, const void* new_k, int64_t k_stride, const void* new_v, int64_t v_stride,
                          const int64_t* q_start, const int32_t* q_lens, int32_t max_q_len, const int32_t* positions,
                          void* q_out, void* k, void* v, int64_t stride_token, int64_t stride_head,
                          const int32_t* ctx_lens, int32_t batch, int64_t max_ctx_len, comem::RopeParams& a) {
  if (batch < 0 || batch > p.cfg.max_batch) return COMEM_ERR_INVALID_SHAPE;
  if (max_ctx_len < 0 || max_ctx_len > p.cfg.max_ctx_len) return COMEM_ERR_INVALID_SHAPE;
  if (max_q_len < 0 || max_q_len > max_ctx_len) return COMEM_ERR_INVALID_SHAPE;
  if (rope_is_empty(batch, max_q_len)) return COMEM_OK;
  if (max_q_len >= (1 << 26)) return COMEM_ERR_INVALID_SHAPE;
  if (is_fp8(p.cfg) && !(std::isfinite(1.f / p.cfg.k_scale) && std::isfinite(1.f / p.cfg.v_scale)))
    return COMEM_ERR_UNSUPPORTED;
  comem_status st = check_rope(p, rope);
  if (st != COMEM_OK) return st;
  if (q == nullptr || new_k == nullptr || new_v == nullptr || q_out == nullptr || k == nullptr || v == nullptr ||
      ctx_lens == nullptr || (q_start == nullptr) != (q_lens == nullptr))
    return COMEM_ERR_NULL_POINTER;
  if (q_lens == nullptr && max_q_len != 1) return COMEM_ERR_INVALID_SHAPE;
  const int64_t e = elem_bytes(p.cfg), d = p.cfg.head_dim;
  const int64_t qe = p.cfg.dtype == COMEM_F32 ? 4 : 2;
  if (q_stride < p.cfg.num_q_heads * d || k_stride < p.cfg.num_kv_heads * d || v_stride < p.cfg.num_kv_heads * d)
    return COMEM_ERR_INVALID_SHAPE;
  const int64_t widest = std::max({q_stride, k_stride, v_stride});
  if (widest > kMaxTokenStrideBytes || stride_token <= 0 || stride_head < 0) return COMEM_ERR_INVALID_SHAPE;
  if (stride_token > kMaxTokenStrideBytes / e) return COMEM_ERR_INVALID_SHAPE;
  if (p.cfg.num_kv_heads > 1 && stride_head == 0) return COMEM_ERR_INVALID_SHAPE;
  if (q_out == q && q_stride != p.cfg.num_q_heads * d) return COMEM_ERR_INVALID_SHAPE;
  if ((q_stride * qe) % 16 != 0 || (k_stride * qe) % 16 != 0 || (v_stride * qe) % 16 != 0 ||
      (stride_token * e) % 16 != 0 || (stride_head * e) % 16 != 0)
    return COMEM_ERR_MISALIGNED;
  if (!aligned(q, 16) || !aligned(new_k, 16) || !aligned(new_v, 16) || !aligned(q_out, 16) || !aligned(k, 16) ||
      !aligned(v, 16) || !aligned(q_start, 8) || !aligned(q_lens, 4) || !aligned(positions, 4) ||
      !aligned(ctx_lens, 4))
    return COMEM_ERR_MISALIGNED;
  std::memset(&a, 0, sizeof(a));
  a.q = static_cast<const char*>(q);
  a.new_k = static_cast<const char*>(new_k);
  a.new_v = static_cast<const char*>(new_v);
  a.q_stride = q_stride * qe;
  a.k_stride = k_stride * qe;
  a.v_stride = v_stride * qe;
  a.q_out = static_cast<char*>(q_out);
  a.k = static_cast<char*>(k);
  a.v = static_cast<char*>(v);
  a.q_weight = static_cast<const char*>(rope->q_weight);
  a.k_weight = static_cast<const char*>(rope->k_weight);
  a.cos_sin = rope->cos_sin;
  a.positions = positions;
  a.q_start = q_start;
  a.q_lens = q_lens;
  a.ctx_lens = ctx_lens;
  a.stride_token = stride_token * e;
  a.stride_head = stride_head * e;
  a.num_positions = static_cast<int32_t>(rope->num_positions);
  a.max_ctx = static_cast<int32_t>(max_ctx_len);
  a.max_q = max_q_len;
  a.num_q_heads = p.cfg.num_q_heads;
  a.num_kv_heads = p.cfg.num_kv_heads;
  a.rot_dim = rope->rot_dim;
  a.interleaved = (rope->flags & COMEM_ROPE_INTERLEAVED) != 0 ? 1 : 0;
  a.eps = rope->eps;
  a.inv_k_scale = is_fp8(p.cfg) ? 1.f / p.cfg.k_scale : 1.f;
  a.inv_v_scale = is_fp8(p.cfg) ? 1.f / p.cfg.v_scale : 1.f;
  return COMEM_OK;
}

comem_status launch_rope(const comem_decode_attn_plan& p, comem::RopeParams& a, bool paged, int32_t batch,
                         void* stream) {
  const comem::RopeCache cache = p.cfg.dtype == COMEM_F32    ? comem::RopeCache::kF32
                                 : p.cfg.dtype == COMEM_BF16 ? comem::RopeCache::kBf16
                                                             : comem::RopeCache::kFp8;
  const int64_t heads = p.cfg.num_q_heads + 2 * int64_t{p.cfg.num_kv_heads};
  const int64_t passes = ceil_div(heads, 1024 / p.cfg.head_dim);
  const int64_t tokens = static_cast<int64_t>(batch) * a.max_q;
  // A token's heads are shared by several waves until there are 8 for every
  // compute unit.
  const int64_t want = std::max<int64_t>(1, 8 * p.num_cus / tokens);
  a.part_passes = static_cast<int32_t>(ceil_div(passes, std::min(want, passes)));
  a.parts = static_cast<int32_t>(ceil_div(passes, a.part_passes));
  // What the attention that follows reads again stays in the caches while it
  // fits the last one (256 MB); where it does not, the stores pass them by.
  // Measured (us, bf16 and FP8 caches, 32 + 16 heads of 128): 402 and 335 MB
  // written 166 and 150 -> 149 and 122 us; 201 and 168 MB 71 and 64, past the
  // caches 78 and 65. The lengths are on the device, so a ragged batch counts as
  // if every sequence had max_q_len tokens, and may pass the caches needlessly.
  const int64_t d = p.cfg.head_dim, qe = p.cfg.dtype == COMEM_F32 ? 4 : 2;
  const int64_t written = tokens * d * (p.cfg.num_q_heads * qe + 2 * int64_t{p.cfg.num_kv_heads} * elem_bytes(p.cfg));
  const comem::RopeKernelFn fn =
      comem::select_rope_kernel(p.cfg.head_dim, cache, paged, written > (int64_t{256} << 20));
  if (fn == nullptr) return COMEM_ERR_UNSUPPORTED;
  // A launch has less than 2^32 threads along a dimension: the last 3 of the
  // 2^26 - 1 tokens that a call may have take a second slice of the grid.
  const int64_t blocks = ceil_div(int64_t{a.max_q} * a.parts, comem::kRopeWaves);
  const int64_t slices = ceil_div(blocks, ((int64_t{1} << 32) - 1) / (64 * comem::kRopeWaves));
  void* argv[] = {&a};
  const hipError_t err =
      hipLaunchKernel(reinterpret_cast<const void*>(fn),
                      dim3(static_cast<unsigned>(ceil_div(blocks, slices)), static_cast<unsigned>(batch),
                           static_cast<unsigned>(slices)),
                      dim3(64 * comem::kRopeWaves), argv, 0, static_cast<hipStream_t>(stream));
  return err == hipSuccess ? COMEM_OK : COMEM_ERR_HIP;
}

}  // namespace

extern "C" {

comem_status comem_rope_append(const comem_decode_attn_plan* plan, const comem_rope_config* rope, const void* q,
                               int64_t q_stride, const void* new_k, int64_t k_stride, const void* new_v,
                               int64_t v_stride, const int64_t* q_start, const int32_t* q_lens, int32_t max_q_len,
                               const int32_t* positions, void* q_out, void* k, void* v, int64_t stride_token,
                               int64_t stride_head, const int64_t* seq_start, const int32_t* ctx_lens,
                               int32_t batch, int64_t max_ctx_len, void* hip_stream) {
  const comem_decode_attn_plan* p = checked(plan);
  if (p == nullptr) return COMEM_ERR_BAD_HANDLE;
  comem::RopeParams a;
  const comem_status st =
      prepare_rope(*p, rope, q, q_stride, new_k, k_stride, new_v, v_stride, q_start, q_lens, max_q_len, positions,
                   q_out, k, v, stride_token, stride_head, ctx_lens, batch, max_ctx_len, a);
  if (st != COMEM_OK || rope_is_empty(batch, max_q_len)) return st;
  if (seq_start == nullptr) return COMEM_ERR_NULL_POINTER;
  if (!aligned(seq_start, 8)) return COMEM_ERR_MISALIGNED;
  if (p->device == COMEM_NO_DEVICE) return COMEM_ERR_NO_DEVICE;
  a.seq_start = seq_start;
  return launch_rope(*p, a, false, batch, hip_stream);
}

comem_status comem_rope_append_paged(const comem_decode_attn_plan* plan, const comem_rope_config* rope,
                                     const void* q, int64_t q_stride, const void* new_k, int64_t k_stride,
                                     const void* new_v, int64_t v_stride, const int64_t* q_start,
                                     const int32_t* q_lens, int32_t max_q_len, const int32_t* positions,
                                     void* q_out, void* k_pages, void* v_pages, int64_t stride_page,
                                     int64_t stride_token, int64_t stride_head, int32_t page_size,
                                     int64_t num_pages, const int32_t* block_table, int32_t max_pages_per_seq,
                                     const int32_t* ctx_lens, int32_t batch, int64_t max_ctx_len,
                                     void* hip_stream) {
  const comem_decode_attn_plan* p = checked(plan);
  if (p == nullptr) return COMEM_ERR_BAD_HANDLE;
  comem::RopeParams a;
  comem_status st =
      prepare_rope(*p, rope, q, q_stride, new_k, k_stride, new_v, v_stride, q_start, q_lens, max_q_len, positions,
                   q_out, k_pages, v_pages, stride_token, stride_head, ctx_lens, batch, max_ctx_len, a);
  if (st != COMEM_OK || rope_is_empty(batch, max_q_len)) return st;
  st = validate_paged(*p, stride_page, page_size, num_pages, block_table, max_pages_per_seq, max_ctx_len);
  if (st != COMEM_OK) return st;
  if (p->device == COMEM_NO_DEVICE) return COMEM_ERR_NO_DEVICE;
  a.block_table = block_table;
  a.stride_page = stride_page * elem_bytes(p->cfg);
  a.num_pages = num_pages;
  a.max_pages = max_pages_per_seq;
  a.page_shift = log2_of(page_size);
  a.page_mask = page_size - 1;
  return launch_rope(*p, a, true, batch, hip_stream);
}

}  // extern "C"
