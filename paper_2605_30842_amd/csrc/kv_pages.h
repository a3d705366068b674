// Kernel arguments of the page kernels (host and device side).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace comem {

constexpr int kPageThreads = 1024;   // kernels that edit tables and counts
constexpr int kChunkPages = 8192;    // pages whose counts one workgroup looks through
constexpr int kApplyThreads = 256;   // the kernel that also moves tokens
constexpr int kMoveTokens = 4;       // tokens that a wave moves at a time

// One item of a call: a row and the table entries that get fresh pages,
// first .. first + need - 1. Workspace arrays, [num_rows] each.
struct PageItems {
  int32_t* row;    // table row that changes, -1: left out
  int32_t* from;   // row whose pages the tokens come from (fork)
  int32_t* len;    // its tokens before the call (fork: the parent's)
  int32_t* grown;  // its tokens after the call
  int32_t* first;
  int32_t* need;
  int32_t* base;   // place of the item's first page in `fresh` (fork, compact)
};

// Offsets and strides are in bytes.
struct PageParams {
  char* k;
  char* v;
  int64_t stride_layer;
  int64_t stride_page;
  int64_t stride_token;
  int64_t stride_head;
  int64_t num_pages;
  int64_t max_ctx;
  int32_t* refcounts;
  int32_t* block_table;
  int32_t* ctx_lens;
  int32_t num_layers;
  int32_t num_rows;
  int32_t max_pages;
  int32_t page_shift;
  int32_t n;                  // items
  int32_t chunks;             // of kChunkPages pages
  int32_t num_kv_heads;
  int32_t piece_shift;        // log2 of the 16-byte pieces of a head's row
  const int32_t* rows;        // compact, release; fork: the parents
  const int32_t* children;    // fork
  const int32_t* add_lens;    // reserve
  int32_t* given;             // reserve: the tokens that each row grew by, or nullptr
  const int32_t* keep;        // compact
  const int64_t* keep_start;
  const int32_t* keep_lens;
  int64_t keep_total;
  int32_t* missing;
  PageItems items;            // workspace from here on
  int32_t* granted;           // [1]: whether the call has its pages
  int32_t* free_counts;       // free pages of each chunk (more than one)
  int32_t* fresh;             // fork, compact: the pages given out, in order
  int32_t* old;               // compact: the rows' entries before the call, [n, max_pages]
};

enum class PageOp { kReserve, kFork, kCompact };

using PageKernelFn = void (*)(PageParams);
// Items and, of more than one chunk, the chunks' free pages: chunk_blocks +
// (compact: n, else ceil(n / kPageThreads)) workgroups.
PageKernelFn select_page_find_kernel(PageOp);
// One workgroup per chunk. ALONE: of one chunk, whose items are found here as
// well (reserve, and fork of at most kPageThreads pairs).
PageKernelFn select_page_give_kernel(PageOp, bool alone);
// Fork, compact: grid (1 + movers, n). stream (compact): tokens pass the caches by.
PageKernelFn select_page_apply_kernel(PageOp, bool stream);
PageKernelFn page_release_kernel();             // one workgroup per item

}  // namespace comem
