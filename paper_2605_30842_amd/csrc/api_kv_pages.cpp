// Host side of the page C ABI (comem_kv_pages.h): argument validation (before
// any HIP call), the workspace's layout and the launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <cstring>

#include "comem_decode_attn.h"
#include "comem_kv_pages.h"
#include "kv_pages.h"
#include "plan.h"

using namespace comem::host;

namespace {

// Workgroups that move tokens in one call, at most, over all items.
constexpr int64_t kMovers = 8192;

comem_status check_state(const comem_decode_attn_plan& p, const comem_kv_pages* s) {
  if (s == nullptr) return COMEM_ERR_NULL_POINTER;
  if (s->page_size <= 0 || s->page_size > 4096 || (s->page_size & (s->page_size - 1)) != 0)
    return COMEM_ERR_INVALID_SHAPE;
  if (s->num_pages <= 0 || s->num_pages > INT32_MAX) return COMEM_ERR_INVALID_SHAPE;
  if (s->num_rows <= 0 || s->num_rows > kGridYZLimit) return COMEM_ERR_INVALID_SHAPE;
  if (s->max_ctx_len <= 0 || s->max_ctx_len > p.cfg.max_ctx_len) return COMEM_ERR_INVALID_SHAPE;
  if (s->max_pages_per_seq <= 0 || s->max_pages_per_seq < ceil_div(s->max_ctx_len, s->page_size))
    return COMEM_ERR_INVALID_SHAPE;
  if (s->refcounts == nullptr || s->block_table == nullptr || s->ctx_lens == nullptr) return COMEM_ERR_NULL_POINTER;
  if (!aligned(s->refcounts, 4) || !aligned(s->block_table, 4) || !aligned(s->ctx_lens, 4))
    return COMEM_ERR_MISALIGNED;
  return COMEM_OK;
}

// The pools of a call that copies tokens.
comem_status check_pools(const comem_decode_attn_plan& p, const comem_kv_pages& s) {
  if (s.k_pages == nullptr || s.v_pages == nullptr) return COMEM_ERR_NULL_POINTER;
  if (s.num_layers <= 0 || s.num_layers > kGridYZLimit) return COMEM_ERR_INVALID_SHAPE;
  if (s.num_layers > 1 && s.stride_layer <= 0) return COMEM_ERR_INVALID_SHAPE;
  if (s.stride_page <= 0 || s.stride_token <= 0 || s.stride_head < 0) return COMEM_ERR_INVALID_SHAPE;
  if (p.cfg.num_kv_heads > 1 && s.stride_head == 0) return COMEM_ERR_INVALID_SHAPE;
  const int64_t e = elem_bytes(p.cfg);
  if (s.stride_token > kMaxTokenStrideBytes / e) return COMEM_ERR_INVALID_SHAPE;
  if ((s.stride_page * e) % 16 != 0 || (s.stride_token * e) % 16 != 0 || (s.stride_head * e) % 16 != 0 ||
      (s.num_layers > 1 && (s.stride_layer * e) % 16 != 0))
    return COMEM_ERR_MISALIGNED;
  if (!aligned(s.k_pages, 16) || !aligned(s.v_pages, 16)) return COMEM_ERR_MISALIGNED;
  return COMEM_OK;
}

int32_t chunks_of(const comem_kv_pages& s) {
  return static_cast<int32_t>(ceil_div(s.num_pages, comem::kChunkPages));
}

// Bytes of the workspace's parts: items, the chunks' free pages, the fresh
// pages, the old entries.
struct Layout {
  size_t item, chunks, fresh, old;
  size_t total() const { return 256 + 7 * item + chunks + fresh + old; }
};

Layout layout_of(const comem_kv_pages& s) {
  const int64_t entries = static_cast<int64_t>(s.num_rows) * s.max_pages_per_seq;
  Layout l;
  l.item = align256(static_cast<size_t>(s.num_rows) * 4);
  l.chunks = align256(static_cast<size_t>(chunks_of(s)) * 4);
  l.fresh = align256(static_cast<size_t>(std::min(s.num_pages, entries)) * 4);
  l.old = align256(static_cast<size_t>(entries) * 4);
  return l;
}

comem::PageParams params_of(const comem_decode_attn_plan& p, const comem_kv_pages& s, int32_t n) {
  const int64_t e = elem_bytes(p.cfg);
  comem::PageParams a;
  std::memset(&a, 0, sizeof(a));
  a.num_pages = s.num_pages;
  a.max_ctx = s.max_ctx_len;
  a.refcounts = s.refcounts;
  a.block_table = s.block_table;
  a.ctx_lens = s.ctx_lens;
  a.num_rows = s.num_rows;
  a.max_pages = s.max_pages_per_seq;
  a.page_shift = log2_of(s.page_size);
  a.n = n;
  a.chunks = chunks_of(s);
  a.num_kv_heads = p.cfg.num_kv_heads;
  a.piece_shift = log2_of(static_cast<int32_t>(p.cfg.head_dim * e / 16));
  return a;
}

void set_pools(const comem_decode_attn_plan& p, const comem_kv_pages& s, comem::PageParams& a) {
  const int64_t e = elem_bytes(p.cfg);
  a.k = static_cast<char*>(s.k_pages);
  a.v = static_cast<char*>(s.v_pages);
  a.num_layers = s.num_layers;
  a.stride_layer = s.num_layers > 1 ? s.stride_layer * e : 0;
  a.stride_page = s.stride_page * e;
  a.stride_token = s.stride_token * e;
  a.stride_head = s.stride_head * e;
}

comem_status check_workspace(const comem_kv_pages& s, const int32_t* missing, const void* workspace, size_t bytes) {
  if (missing == nullptr || workspace == nullptr) return COMEM_ERR_NULL_POINTER;
  if (!aligned(missing, 4) || !aligned(workspace, 256)) return COMEM_ERR_MISALIGNED;
  return bytes < layout_of(s).total() ? COMEM_ERR_WORKSPACE_TOO_SMALL : COMEM_OK;
}

void set_workspace(const comem_kv_pages& s, void* workspace, comem::PageParams& a) {
  const Layout l = layout_of(s);
  char* at = static_cast<char*>(workspace);
  a.granted = reinterpret_cast<int32_t*>(at);
  at += 256;
  for (int32_t** item : {&a.items.row, &a.items.from, &a.items.len, &a.items.grown, &a.items.first, &a.items.need,
                         &a.items.base}) {
    *item = reinterpret_cast<int32_t*>(at);
    at += l.item;
  }
  a.free_counts = reinterpret_cast<int32_t*>(at);
  at += l.chunks;
  a.fresh = reinterpret_cast<int32_t*>(at);
  a.old = reinterpret_cast<int32_t*>(at + l.fresh);
}

bool launched(comem::PageKernelFn fn, dim3 grid, int threads, comem::PageParams& a, void* stream) {
  void* argv[] = {&a};
  return hipLaunchKernel(reinterpret_cast<const void*>(fn), grid, dim3(static_cast<unsigned>(threads)), argv, 0,
                         static_cast<hipStream_t>(stream)) == hipSuccess;
}

// `moved`: the most tokens of an item that a call may copy; `bytes`: the most
// that it may store in all (listed tokens that stay in place count too: the
// lists are on the device). Tokens that the last cache (256 MB) cannot hold for
// the attention that follows pass it by (us, compact calls that move 410 and
// 799 MB 206 and 362 -> 190 and 344; 70 MB 59.3, past the caches 60.3).
comem_status launch_pages(comem::PageOp op, comem::PageParams& a, int64_t moved, double bytes, void* stream) {
  using comem::PageOp;
  // A fork's item looks through the list before it, so past what one workgroup
  // finds at once the lists are looked through side by side (us, a fork and a
  // release, one workgroup / a find launch: 32 pairs 14.9 / 18.1, 1024 50.8 /
  // 52.7, 1025 68.5 / 53.9, 4096 305 / 188, 65534 44600 / 2890).
  const bool compact = op == PageOp::kCompact;
  const bool alone = a.chunks == 1 && !compact && (op == PageOp::kReserve || a.n <= comem::kPageThreads);
  bool ok = true;
  if (!alone) {
    const int64_t items = compact ? a.n : ceil_div(a.n, comem::kPageThreads);
    const int64_t blocks = items + (a.chunks > 1 ? a.chunks : 0);
    ok = launched(comem::select_page_find_kernel(op), dim3(static_cast<unsigned>(blocks)), comem::kPageThreads, a, stream);
  }
  ok = ok && launched(comem::select_page_give_kernel(op, alone), dim3(static_cast<unsigned>(a.chunks)),
                      comem::kPageThreads, a, stream);
  if (op != PageOp::kReserve) {
    const int64_t units = ceil_div(moved, comem::kMoveTokens) * a.num_layers;
    const int64_t movers = std::min(ceil_div(units, comem::kApplyThreads / 64), std::max<int64_t>(1, kMovers / a.n));
    ok = ok && launched(comem::select_page_apply_kernel(op, bytes > 256.0 * (1 << 20)),
                        dim3(static_cast<unsigned>(1 + movers), static_cast<unsigned>(a.n)), comem::kApplyThreads, a,
                        stream);
  }
  return ok ? COMEM_OK : COMEM_ERR_HIP;
}

// granted: nullptr where the caller does not ask for it.
comem_status reserve(const comem_decode_attn_plan* plan, const comem_kv_pages* pages, const int32_t* add_lens,
                     int32_t* granted, int32_t* missing, void* workspace, size_t workspace_bytes, void* hip_stream) {
  const comem_decode_attn_plan* p = checked(plan);
  if (p == nullptr) return COMEM_ERR_BAD_HANDLE;
  comem_status st = check_state(*p, pages);
  if (st != COMEM_OK) return st;
  if (add_lens == nullptr) return COMEM_ERR_NULL_POINTER;
  if (!aligned(add_lens, 4) || !aligned(granted, 4)) return COMEM_ERR_MISALIGNED;
  st = check_workspace(*pages, missing, workspace, workspace_bytes);
  if (st != COMEM_OK) return st;
  if (p->device == COMEM_NO_DEVICE) return COMEM_ERR_NO_DEVICE;
  comem::PageParams a = params_of(*p, *pages, pages->num_rows);
  set_workspace(*pages, workspace, a);
  a.add_lens = add_lens;
  a.given = granted;
  a.missing = missing;
  return launch_pages(comem::PageOp::kReserve, a, 0, 0, hip_stream);
}

}  // namespace

extern "C" {

comem_status comem_kv_pages_workspace(const comem_decode_attn_plan* plan, const comem_kv_pages* pages,
                                      size_t* workspace_bytes_out) {
  const comem_decode_attn_plan* p = checked(plan);
  if (p == nullptr) return COMEM_ERR_BAD_HANDLE;
  if (workspace_bytes_out == nullptr) return COMEM_ERR_NULL_POINTER;
  *workspace_bytes_out = 0;
  const comem_status st = check_state(*p, pages);
  if (st == COMEM_OK) *workspace_bytes_out = layout_of(*pages).total();
  return st;
}

comem_status comem_kv_reserve(const comem_decode_attn_plan* plan, const comem_kv_pages* pages,
                              const int32_t* add_lens, int32_t* missing, void* workspace,
                              size_t workspace_bytes, void* hip_stream) {
  return reserve(plan, pages, add_lens, nullptr, missing, workspace, workspace_bytes, hip_stream);
}

comem_status comem_kv_reserve_granted(const comem_decode_attn_plan* plan, const comem_kv_pages* pages,
                                      const int32_t* add_lens, int32_t* granted, int32_t* missing,
                                      void* workspace, size_t workspace_bytes, void* hip_stream) {
  if (checked(plan) == nullptr) return COMEM_ERR_BAD_HANDLE;
  if (granted == nullptr) return COMEM_ERR_NULL_POINTER;
  return reserve(plan, pages, add_lens, granted, missing, workspace, workspace_bytes, hip_stream);
}

comem_status comem_kv_fork(const comem_decode_attn_plan* plan, const comem_kv_pages* pages, const int32_t* parents,
                           const int32_t* children, int32_t n, int32_t* missing, void* workspace,
                           size_t workspace_bytes, void* hip_stream) {
  const comem_decode_attn_plan* p = checked(plan);
  if (p == nullptr) return COMEM_ERR_BAD_HANDLE;
  comem_status st = check_state(*p, pages);
  if (st != COMEM_OK) return st;
  if (n < 0 || n > pages->num_rows) return COMEM_ERR_INVALID_SHAPE;
  if (n == 0) return COMEM_OK;
  st = check_pools(*p, *pages);
  if (st != COMEM_OK) return st;
  if (parents == nullptr || children == nullptr) return COMEM_ERR_NULL_POINTER;
  if (!aligned(parents, 4) || !aligned(children, 4)) return COMEM_ERR_MISALIGNED;
  st = check_workspace(*pages, missing, workspace, workspace_bytes);
  if (st != COMEM_OK) return st;
  if (p->device == COMEM_NO_DEVICE) return COMEM_ERR_NO_DEVICE;
  comem::PageParams a = params_of(*p, *pages, n);
  set_pools(*p, *pages, a);
  set_workspace(*pages, workspace, a);
  a.rows = parents;
  a.children = children;
  a.missing = missing;
  return launch_pages(comem::PageOp::kFork, a, pages->page_size, 0, hip_stream);
}

comem_status comem_kv_compact(const comem_decode_attn_plan* plan, const comem_kv_pages* pages, const int32_t* rows,
                              const int32_t* keep, int64_t keep_total, const int64_t* keep_start,
                              const int32_t* keep_lens, int32_t n, int32_t* missing, void* workspace,
                              size_t workspace_bytes, void* hip_stream) {
  const comem_decode_attn_plan* p = checked(plan);
  if (p == nullptr) return COMEM_ERR_BAD_HANDLE;
  comem_status st = check_state(*p, pages);
  if (st != COMEM_OK) return st;
  if (n < 0 || n > pages->num_rows) return COMEM_ERR_INVALID_SHAPE;
  if (n == 0) return COMEM_OK;
  st = check_pools(*p, *pages);
  if (st != COMEM_OK) return st;
  if (keep_total < 0) return COMEM_ERR_INVALID_SHAPE;
  if (rows == nullptr || keep_start == nullptr || keep_lens == nullptr || (keep == nullptr && keep_total > 0))
    return COMEM_ERR_NULL_POINTER;
  if (!aligned(rows, 4) || !aligned(keep, 4) || !aligned(keep_start, 8) || !aligned(keep_lens, 4))
    return COMEM_ERR_MISALIGNED;
  st = check_workspace(*pages, missing, workspace, workspace_bytes);
  if (st != COMEM_OK) return st;
  if (p->device == COMEM_NO_DEVICE) return COMEM_ERR_NO_DEVICE;
  comem::PageParams a = params_of(*p, *pages, n);
  set_pools(*p, *pages, a);
  set_workspace(*pages, workspace, a);
  a.rows = rows;
  a.keep = keep;
  a.keep_total = keep_total;
  a.keep_start = keep_start;
  a.keep_lens = keep_lens;
  a.missing = missing;
  const double token = 2.0 * p->cfg.num_kv_heads * p->cfg.head_dim * elem_bytes(p->cfg) * pages->num_layers;
  return launch_pages(comem::PageOp::kCompact, a, std::min(keep_total, pages->max_ctx_len),
                      static_cast<double>(keep_total) * token, hip_stream);
}

comem_status comem_kv_release(const comem_decode_attn_plan* plan, const comem_kv_pages* pages, const int32_t* rows,
                              int32_t n, void* hip_stream) {
  const comem_decode_attn_plan* p = checked(plan);
  if (p == nullptr) return COMEM_ERR_BAD_HANDLE;
  const comem_status st = check_state(*p, pages);
  if (st != COMEM_OK) return st;
  if (n < 0 || n > pages->num_rows) return COMEM_ERR_INVALID_SHAPE;
  if (n == 0) return COMEM_OK;
  if (rows == nullptr) return COMEM_ERR_NULL_POINTER;
  if (!aligned(rows, 4)) return COMEM_ERR_MISALIGNED;
  if (p->device == COMEM_NO_DEVICE) return COMEM_ERR_NO_DEVICE;
  comem::PageParams a = params_of(*p, *pages, n);
  a.rows = rows;
  return launched(comem::page_release_kernel(), dim3(static_cast<unsigned>(n)), comem::kPageThreads, a, hip_stream)
             ? COMEM_OK
             : COMEM_ERR_HIP;
}

}  // extern "C"
