// Kernel arguments of the rotate-and-store kernel (host and device side).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace comem {

constexpr int kRopeWaves = 4;  // waves per workgroup, each with a token or a part of its heads
constexpr int kRopeBatch = 3;  // passes of a wave whose rows are in flight together

// Offsets and strides are in bytes.
struct RopeParams {
  const char* q;               // rows of Hq heads
  const char* new_k;           // rows of Hkv heads
  const char* new_v;
  int64_t q_stride;
  int64_t k_stride;
  int64_t v_stride;
  char* q_out;                 // dense
  char* k;                     // contiguous: [T, Hkv, D] rows; paged: page pool
  char* v;
  const char* q_weight;        // [D] of the new rows' type, or nullptr
  const char* k_weight;
  const float* cos_sin;        // [num_positions, rot_dim]
  const int32_t* positions;    // one per row, or nullptr: the cache index
  const int64_t* q_start;      // nullptr: one token per sequence
  const int32_t* q_lens;
  const int64_t* seq_start;    // contiguous layout
  const int32_t* ctx_lens;
  const int32_t* block_table;  // paged layout, [B, max_pages]
  int64_t stride_token;
  int64_t stride_head;
  int64_t stride_page;
  int64_t num_pages;
  int32_t num_positions;
  int32_t max_pages;
  int32_t page_shift;
  int32_t page_mask;
  int32_t max_ctx;
  int32_t max_q;
  int32_t num_q_heads;
  int32_t num_kv_heads;
  int32_t rot_dim;
  int32_t interleaved;
  int32_t parts;               // waves that share a token's heads
  int32_t part_passes;         // passes of each
  float eps;
  float inv_k_scale;           // FP8 caches: codes of value * inv_scale
  float inv_v_scale;
};

enum class RopeCache { kF32, kBf16, kFp8 };

using RopeKernelFn = void (*)(RopeParams);
// stream: q_out, and cache rows that are no codes, are stored past the caches.
RopeKernelFn select_rope_kernel(int head_dim, RopeCache cache, bool paged, bool stream);

}  // namespace comem
