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

// How a weights call is shared out.
struct WeightsShape {
  int sub;         // 16-token slabs of a workgroup
  int waves;       // of a workgroup
  int64_t tiles;   // workgroups of a sequence
  int64_t splits;  // workgroups of a tile, each with a part of its query rows
  bool ring;       // query rows asked for groups ahead
};

// One or two groups of query rows (a decode step): memory bounds the call, so
// large tiles where there are tiles enough, small ones where the tokens must
// reach every unit (us, tile 32 / 64 / 96 tokens: 6001 tokens 5.9 / 8.1 / 10.7,
// 32768 15.0 / 14.1 / 18.6, 64 x 2048-16384 218 / 210 / 206).
//
// More rows: the least estimated time over the tile sizes and the shares of the
// rows. A turn of 8 waves on a unit (16 query rows each, two waves on a SIMD)
// takes 0.33 us and 0.11 for each slab (float32 2.4: 300 rows over 24300 take
// 513 us, 2.3 for each turn and unit, at 0.116 of the 0.152 PFLOP/s of a large
// product), a workgroup's start about 2 us and half a slab's more, adding the
// shares up 3. Once there are workgroups for two a unit they have 4 waves. Measured (us, the choice and the best of 48 forced
// ones): 300 rows over 24300 78.7 / 78.7, 64 over 2000 10.4 / 10.4, all of 300
// 11 / 11, of 2000 50 / 50, of 8192 394-431 / 394, 32-64 over 8 x 8000-16000
// FP8 58 / 58, 1-16 over 4 x 2000-12000 14.3 / 12.0.
WeightsShape weights_shape(const comem_decode_attn_plan& p, int64_t batch, int64_t max_q, int64_t max_ctx, bool split) {
  const int64_t heads = p.cfg.num_kv_heads, groups = ceil_div(max_q * group_of(p.cfg), 16), cus = p.num_cus;
  const bool f32 = p.cfg.dtype == COMEM_F32;
  WeightsShape s;
  s.ring = groups > 2;
  s.splits = 1;
  if (!s.ring) {
    const int64_t slabs = batch * ceil_div(max_ctx, 16);
    s.sub = f32 || slabs < 4 * cus ? 2 : slabs < 16 * cus ? 4 : 6;
    s.waves = static_cast<int>(std::min<int64_t>(heads, 4));
  } else {
    double least = INFINITY;
    for (int sub = 2; sub <= (f32 ? 2 : 6); sub += 2) {
      const int64_t tiles = batch * ceil_div(max_ctx, 16 * sub);
      const double turn = f32 ? 2.4 : 0.33 + 0.11 * sub;
      for (int64_t splits : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32}) {
        if (splits > (split ? groups : 1)) break;
        const int64_t workgroups = tiles * splits, waves = workgroups <= cus ? 8 : 4;
        const int64_t shares = std::max<int64_t>(1, waves / heads);
        const double rounds = static_cast<double>(workgroups) / static_cast<double>(cus * (8 / waves));
        const double turns = static_cast<double>(ceil_div(heads * shares, waves) * ceil_div(groups, splits * shares));
        const double us = (rounds < 4 ? std::ceil(rounds) : rounds) * (2 + 0.5 * sub + turns * turn) + (splits > 1 ? 3 : 0);
        if (us < least) {
          least = us;
          s.sub = sub;
          s.waves = static_cast<int>(waves);
          s.splits = splits;
        }
      }
    }
  }
  s.tiles = std::min(ceil_div(max_ctx, 16 * s.sub), kMostTiles);
  return s;
}

size_t weights_bytes(const WeightsShape& s, int64_t batch, int64_t max_ctx) {
  return s.splits > 1 ? align256(static_cast<size_t>(s.splits * batch * max_ctx) * 4) : 0;
}

comem_status launch_weights(const comem_decode_attn_plan& p, comem::WeightsParams& a, bool paged, int32_t batch,
                            void* workspace, size_t workspace_bytes, void* stream) {
  WeightsShape s = weights_shape(p, batch, a.max_q, a.max_ctx, true);
  if (s.splits > 1 && (workspace == nullptr || workspace_bytes < weights_bytes(s, batch, a.max_ctx)))
    s = weights_shape(p, batch, a.max_q, a.max_ctx, false);
  const comem::WeightsForm form =
      comem::select_weights_kernel(p.cfg.head_dim, comem::cache_type(p.cfg), paged, s.sub, s.ring);
  if (form.fn == nullptr) return COMEM_ERR_UNSUPPORTED;
  if (s.splits > 1) a.partial = static_cast<float*>(workspace);
  void* argv[] = {&a, nullptr};
  if (hipLaunchKernel(reinterpret_cast<const void*>(form.fn),
                      dim3(static_cast<unsigned>(s.tiles), static_cast<unsigned>(batch), static_cast<unsigned>(s.splits)),
                      dim3(static_cast<unsigned>(64 * s.waves)), argv, static_cast<size_t>(s.waves * form.wave_bytes),
                      static_cast<hipStream_t>(stream)) != hipSuccess)
    return COMEM_ERR_HIP;
  if (s.splits == 1) return COMEM_OK;
  int splits = static_cast<int>(s.splits);
  argv[1] = &splits;
  const int64_t blocks = std::min(ceil_div(a.max_ctx, 256), kMostTiles);
  const hipError_t err = hipLaunchKernel(reinterpret_cast<const void*>(comem::add_weights_kernel_fn()),
                                         dim3(static_cast<unsigned>(blocks), static_cast<unsigned>(batch)), dim3(256),
                                         argv, 0, static_cast<hipStream_t>(stream));
  return err == hipSuccess ? COMEM_OK : COMEM_ERR_HIP;
}

// Longest rows that one workgroup takes: the binding's KEEP_CHUNKS_MIN_CTX, below which it asks for no workspace.
constexpr int64_t kKeepChunksMinCtx = 49152;

// Rows of a keep call in chunks (comem_keep_tokens_workspace), or 0. us, a
// quarter kept, one workgroup a row / chunks: one row of 49152 entries 17.4 /
// 16.5, of 65536 20 / 16, of 262144 56 / 21; 32 rows of 131072 37 / 28, of
// 262144 63 / 62; 64 of 65536 25 / 25, of 131072 41 / 49. Every chunk adds up
// the counts of all of its row's, so many chunks of many rows lose; up to 49152
// entries an eager call's host time (three launches 18, one 10) would show.
int64_t keep_chunks(const comem_decode_attn_plan& p, int64_t n, int64_t max_ctx) {
  const int64_t chunks = ceil_div(max_ctx, comem::kChunkEntries);
  const bool few = 8 * n <= p.num_cus && n * chunks <= 4 * p.num_cus;
  return max_ctx > kKeepChunksMinCtx && chunks <= comem::kMostChunks && few ? chunks : 0;
}

size_t keep_bytes(const comem_decode_attn_plan& p, int64_t n, int64_t max_ctx) {
  const int64_t chunks = keep_chunks(p, n, max_ctx);
  return chunks > 0 ? static_cast<size_t>(n * comem::choose_item_bytes(chunks)) : 0;
}

}  // namespace

extern "C" {

comem_status comem_attn_weights_workspace(const comem_decode_attn_plan* plan, int32_t batch, int32_t max_q_len,
                                          int64_t max_ctx_len, size_t* workspace_bytes_out) {
  const comem_decode_attn_plan* p = checked(plan);
  if (p == nullptr) return COMEM_ERR_BAD_HANDLE;
  if (workspace_bytes_out == nullptr) return COMEM_ERR_NULL_POINTER;
  *workspace_bytes_out = 0;
  if (batch < 0 || batch > p->cfg.max_batch) return COMEM_ERR_INVALID_SHAPE;
  if (max_ctx_len < 0 || max_ctx_len > p->cfg.max_ctx_len) return COMEM_ERR_INVALID_SHAPE;
  if (max_q_len < 0 || max_q_len > max_ctx_len) return COMEM_ERR_INVALID_SHAPE;
  if (!weights_is_empty(batch, max_q_len))
    *workspace_bytes_out = weights_bytes(weights_shape(*p, batch, max_q_len, max_ctx_len, true), batch, max_ctx_len);
  return COMEM_OK;
}

comem_status comem_attn_weights(const comem_decode_attn_plan* plan, const void* q, const float* lse,
                                const int64_t* q_start, const int32_t* q_lens, int32_t max_q_len, const void* k,
                                int64_t stride_token, int64_t stride_head, const int64_t* seq_start,
                                const int32_t* ctx_lens, int32_t batch, int64_t max_ctx_len, const float* prior,
                                float decay, float* weights, int64_t weights_stride, void* workspace,
                                size_t workspace_bytes, void* hip_stream) {
  const comem_decode_attn_plan* p = checked(plan);
  if (p == nullptr) return COMEM_ERR_BAD_HANDLE;
  comem::WeightsParams a;
  const comem_status st = prepare_weights(*p, q, lse, q_start, q_lens, max_q_len, k, stride_token, stride_head, ctx_lens,
                                          batch, max_ctx_len, prior, decay, weights, weights_stride, a);
  if (st != COMEM_OK || weights_is_empty(batch, max_q_len)) return st;
  if (seq_start == nullptr) return COMEM_ERR_NULL_POINTER;
  if (!aligned(seq_start, 8) || !aligned(workspace, 256)) return COMEM_ERR_MISALIGNED;
  if (p->device == COMEM_NO_DEVICE) return COMEM_ERR_NO_DEVICE;
  a.seq_start = seq_start;
  return launch_weights(*p, a, false, batch, workspace, workspace_bytes, hip_stream);
}

comem_status comem_attn_weights_paged(const comem_decode_attn_plan* plan, const void* q, const float* lse,
                                      const int64_t* q_start, const int32_t* q_lens, int32_t max_q_len,
                                      const void* k_pages, int64_t stride_page, int64_t stride_token,
                                      int64_t stride_head, int32_t page_size, int64_t num_pages,
                                      const int32_t* block_table, int32_t max_pages_per_seq, const int32_t* ctx_lens,
                                      int32_t batch, int64_t max_ctx_len, const float* prior, float decay,
                                      float* weights, int64_t weights_stride, void* workspace,
                                      size_t workspace_bytes, void* hip_stream) {
  const comem_decode_attn_plan* p = checked(plan);
  if (p == nullptr) return COMEM_ERR_BAD_HANDLE;
  comem::WeightsParams a;
  comem_status st = prepare_weights(*p, q, lse, q_start, q_lens, max_q_len, k_pages, stride_token, stride_head,
                                    ctx_lens, batch, max_ctx_len, prior, decay, weights, weights_stride, a);
  if (st != COMEM_OK || weights_is_empty(batch, max_q_len)) return st;
  st = validate_paged(*p, stride_page, page_size, num_pages, block_table, max_pages_per_seq, max_ctx_len);
  if (st != COMEM_OK) return st;
  if (!aligned(workspace, 256)) return COMEM_ERR_MISALIGNED;
  if (p->device == COMEM_NO_DEVICE) return COMEM_ERR_NO_DEVICE;
  a.block_table = block_table;
  a.stride_page = stride_page * elem_bytes(p->cfg);
  a.num_pages = num_pages;
  a.max_pages = max_pages_per_seq;
  a.page_shift = log2_of(page_size);
  a.page_mask = page_size - 1;
  return launch_weights(*p, a, true, batch, workspace, workspace_bytes, hip_stream);
}

comem_status comem_keep_tokens_workspace(const comem_decode_attn_plan* plan, int32_t n, int64_t max_ctx_len,
                                         size_t* workspace_bytes_out) {
  const comem_decode_attn_plan* p = checked(plan);
  if (p == nullptr) return COMEM_ERR_BAD_HANDLE;
  if (workspace_bytes_out == nullptr) return COMEM_ERR_NULL_POINTER;
  *workspace_bytes_out = 0;
  if (n < 0 || n > kGridYZLimit) return COMEM_ERR_INVALID_SHAPE;
  if (max_ctx_len < 0 || max_ctx_len > p->cfg.max_ctx_len) return COMEM_ERR_INVALID_SHAPE;
  *workspace_bytes_out = keep_bytes(*p, n, max_ctx_len);
  return COMEM_OK;
}

comem_status comem_keep_tokens(const comem_decode_attn_plan* plan, const float* weights, int64_t weights_stride,
                               const int32_t* ctx_lens, int32_t num_rows, const int32_t* rows, int32_t n,
                               int64_t max_ctx_len, int32_t budget, const int32_t* budgets, int32_t first,
                               int32_t last, int32_t* keep, int64_t keep_stride, int64_t* keep_start,
                               int32_t* keep_lens, float* kept, void* workspace, size_t workspace_bytes,
                               void* hip_stream) {
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
      !aligned(keep, 4) || !aligned(keep_start, 8) || !aligned(keep_lens, 4) || !aligned(kept, 4) ||
      !aligned(workspace, 256))
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
  void* argv[] = {&a};
  auto launched = [&](comem::ChooseKernelFn fn, int64_t parts, int threads) {
    return hipLaunchKernel(reinterpret_cast<const void*>(fn),
                           dim3(static_cast<unsigned>(n), static_cast<unsigned>(parts)),
                           dim3(static_cast<unsigned>(threads)), argv, 0,
                           static_cast<hipStream_t>(hip_stream)) == hipSuccess;
  };
  const int64_t chunks = keep_chunks(*p, n, max_ctx_len);
  bool ok;
  if (chunks > 0 && workspace != nullptr && workspace_bytes >= keep_bytes(*p, n, max_ctx_len)) {
    a.workspace = static_cast<char*>(workspace);
    const comem::ChunkKernels k = comem::select_chunk_kernels();
    ok = launched(k.count, chunks, k.threads) && launched(k.list, chunks, k.threads) &&
         launched(k.put, chunks, k.threads);
  } else {
    const comem::ChooseForm form = comem::select_choose_kernel(false, max_ctx_len, n, p->num_cus);
    ok = launched(form.fn, form.parts, form.threads);
  }
  return ok ? COMEM_OK : COMEM_ERR_HIP;
}

}  // extern "C"
