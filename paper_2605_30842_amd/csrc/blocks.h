// Kernel arguments of the block kernels (host and device side).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "evict.h"

namespace comem {

constexpr int kBoundsThreads = 512;
constexpr int kScoresWaves = 4;    // waves of a workgroup, a KV head each
constexpr int kScoresBlocks = 16;  // blocks of a workgroup

// Offsets and strides are in bytes.
struct BoundsParams {
  const char* k;
  char* bounds;                // [num_pages, Hkv, 2, D]
  const int32_t* ctx_lens;
  const int32_t* q_lens;       // nullptr: 1 each
  const int32_t* block_table;  // [B, max_pages]
  int64_t stride_page;
  int64_t stride_token;
  int64_t stride_head;
  int64_t num_pages;
  int32_t max_pages;
  int32_t page_shift;
  int32_t max_ctx;
  int32_t max_q;
  int32_t pieces;              // 16-byte pieces of a token's heads
  int32_t width;               // of them, a workgroup's
  int32_t piece_shift;         // log2 of those of one head
};

struct ScoresParams {
  const char* q;
  const char* bounds;
  const int32_t* ctx_lens;
  const int32_t* block_table;
  float* scores;
  int64_t scores_stride;
  int64_t num_pages;
  int32_t max_pages;
  int32_t page_shift;
  int32_t max_ctx;
  int32_t num_kv_heads;
  int32_t group;
  float scale;                 // times the K scale of an FP8 cache
};

using BoundsKernelFn = void (*)(BoundsParams);
BoundsKernelFn select_bounds_kernel(CacheType cache);
using ScoresKernelFn = void (*)(ScoresParams);
ScoresKernelFn select_scores_kernel(int head_dim, CacheType cache);

}  // namespace comem
