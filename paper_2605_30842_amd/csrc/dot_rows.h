// Products of 16 cached rows with 16 query rows on the matrix cores (gfx950),
// for kernels that need the scores alone.
//
// A wave's lane 16 g + c holds a part of cached row c and of query row c; the
// result is the product of cached row 4 g + r and query row c in element r. The
// parts are any fixed division of the D elements among the four lane groups,
// the same for both operands: elements 32 i + 8 g .. + 8 of bf16 rows (64
// bytes of a row side by side in every load), 16 i + 4 g .. + 4 of float32
// rows, and for codes, of which a load brings 16, (D / 4) g + 16 i .. + 16.
// Products of bf16 are exact in the float32 sums; E4M3 codes are widened to
// bf16 exactly. float32 rows take the float32 products.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "evict.h"

namespace comem {

typedef uint32_t dot_u32x4 __attribute__((ext_vector_type(4)));
typedef float dot_f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 dot_bf16x8 __attribute__((ext_vector_type(8)));

// A lane's part of a query row, or of a widened cached row.
template <int D, CacheType C>
struct DotPart {
  static constexpr int kLoads = C == CacheType::kF32 ? D / 16 : D / 32;
  static constexpr int kStep = C == CacheType::kFp8 ? 16 : 64;  // bytes from one load to the next
  dot_u32x4 x[kLoads];
  static __device__ int lane_offset(int g) { return C == CacheType::kFp8 ? (D / 2) * g : 16 * g; }
  // row: the query row (of the cache's type, bf16 for codes).
  __device__ void load_query(const char* row, int g) {
    const char* at = row + lane_offset(g);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) x[i] = *reinterpret_cast<const dot_u32x4*>(at + kStep * i);
  }
};

// A lane's part of a cached row, as it lies in memory.
template <int D, CacheType C>
struct RowPart {
  static constexpr int kLoads = C == CacheType::kF32 ? D / 16 : C == CacheType::kBf16 ? D / 32 : D / 64;
  dot_u32x4 x[kLoads];
  static __device__ int lane_offset(int g) { return C == CacheType::kFp8 ? (D / 4) * g : 16 * g; }
  // at: the row, lane_offset added.
  __device__ void load(const char* at) {
    constexpr int kStep = C == CacheType::kFp8 ? 16 : 64;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) x[i] = *reinterpret_cast<const dot_u32x4*>(at + kStep * i);
  }
  __device__ DotPart<D, C> widened() const {
    DotPart<D, C> r;
    if constexpr (C == CacheType::kFp8) {
#pragma unroll
      for (int i = 0; i < kLoads; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t w = x[i][e];
          r.x[2 * i + e / 2][2 * (e & 1)] =
              __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, false));
          r.x[2 * i + e / 2][2 * (e & 1) + 1] =
              __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, true));
        }
    } else {
#pragma unroll
      for (int i = 0; i < kLoads; ++i) r.x[i] = x[i];
    }
    return r;
  }
};

template <int D, CacheType C>
__device__ inline dot_f32x4 dot_rows(const DotPart<D, C>& k, const DotPart<D, C>& q, dot_f32x4 acc) {
#pragma unroll
  for (int i = 0; i < DotPart<D, C>::kLoads; ++i) {
    if constexpr (C == CacheType::kF32) {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(k.x[i][e]), __uint_as_float(q.x[i][e]), acc, 0, 0, 0);
    } else {
      acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(dot_bf16x8, k.x[i]),
                                                    __builtin_bit_cast(dot_bf16x8, q.x[i]), acc, 0, 0, 0);
    }
  }
  return acc;
}

// x of the lane N places before, around the 16 lanes of a row.
template <int N>
__device__ inline uint32_t row_turned(uint32_t x) {
  return static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(x), 0x120 + N, 0xf, 0xf, true));
}

}  // namespace comem
