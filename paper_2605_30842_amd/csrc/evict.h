// Kernel arguments of the attention-weight and choice kernels (host and device side).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "comem_decode_attn.h"

namespace comem {

enum class CacheType { kF32, kBf16, kFp8 };

inline CacheType cache_type(const comem_decode_attn_config& c) {
  return c.dtype == COMEM_F32 ? CacheType::kF32 : c.dtype == COMEM_BF16 ? CacheType::kBf16 : CacheType::kFp8;
}

constexpr int kWeightsWaves = 8;  // most waves of a workgroup, on the same tokens

// Offsets and strides are in bytes, but for that of the weights.
struct WeightsParams {
  const char* q;               // [rows, Hq, D]
  const float* lse;            // [rows, Hq]
  const char* k;               // contiguous: [T, Hkv, D] rows; paged: page pool
  const int64_t* q_start;      // nullptr: one token per sequence
  const int32_t* q_lens;
  const int64_t* seq_start;    // contiguous layout
  const int32_t* ctx_lens;
  const int32_t* block_table;  // paged layout, [B, max_pages]
  const float* prior;          // or nullptr
  float* weights;
  float* partial;              // [splits, B, max_ctx], or nullptr: one workgroup has a tile's query rows
  int64_t weights_stride;
  int64_t stride_token;
  int64_t stride_head;
  int64_t stride_page;
  int64_t num_pages;
  int32_t max_pages;
  int32_t page_shift;
  int32_t page_mask;
  int32_t max_ctx;
  int32_t max_q;
  int32_t num_kv_heads;
  int32_t group_shift;         // log2(G)
  float scale_log2;            // scale * log2(e), times the K scale of an FP8 cache
  float decay;
};

using WeightsKernelFn = void (*)(WeightsParams);
struct WeightsForm {
  WeightsKernelFn fn;
  int wave_bytes;  // LDS that the launch gives each wave
};
// sub: 16-token slabs of a workgroup, 2, 4 or 6 (float32: 2). ring: for many
// groups of 16 query rows.
WeightsForm select_weights_kernel(int head_dim, CacheType cache, bool paged, int sub, bool ring);
using AddWeightsKernelFn = void (*)(WeightsParams, int);
AddWeightsKernelFn add_weights_kernel_fn();

// The largest entries of a row, in ascending order.
struct ChooseParams {
  const float* scores;
  int64_t scores_stride;
  const int32_t* lens;         // tokens of each row or sequence
  const int32_t* rows;         // tokens: row of each item, or nullptr
  const int32_t* budgets;      // tokens: each item's, or nullptr
  int32_t num_rows;
  int32_t max_len;             // bound of lens
  int32_t budget;
  int32_t first;
  int32_t last;
  int32_t* out;                // positions (tokens) or pages (blocks)
  int64_t out_stride;
  int64_t* out_start;          // tokens, or nullptr
  int32_t* out_lens;
  float* kept;                 // tokens, or nullptr
  const int32_t* block_table;  // blocks, [B, max_pages]
  int32_t max_pages;
  int32_t heads;               // items of a sequence
  int32_t page_shift;
  char* workspace;             // choose_item_bytes for each item of long rows in chunks
};

// Rows in chunks.
constexpr int kMostChunks = 64, kChunkEntries = 8192;

// Workspace of an item: 2048 counts a chunk; a header of 4 words; two counts and
// a list for each chunk.
__host__ __device__ inline int64_t choose_item_bytes(int64_t chunks) {
  return (4 * (2048 * chunks + 4 + 2 * chunks + kChunkEntries * chunks) + 255) / 256 * 256;
}

using ChooseKernelFn = void (*)(ChooseParams);
struct ChooseForm {
  ChooseKernelFn fn;
  int threads;
  int parts;  // grid (items, parts)
};
// For `items` rows of at most `most` entries on `cus` compute units.
ChooseForm select_choose_kernel(bool blocks, int64_t most, int64_t items, int cus);

// Tokens of long rows, one launch after the other, grid (items, chunks).
struct ChunkKernels {
  ChooseKernelFn count, list, put;
  int threads;
};
ChunkKernels select_chunk_kernels();

}  // namespace comem
