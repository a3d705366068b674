// Head norms, position rotation and the cache store of new tokens, one pass,
// gfx950.
//
// Every query and key head of a new token is scaled by the reciprocal root of
// its mean square and the norm's weight, and its first rot_dim elements are
// turned by the angles of the token's position: (a, b) -> (a c - b s,
// b c + a s). Queries go to q_out, keys and values to the cache row of the
// token, in the cache's type (FP8: the code nearest to value / scale).
//
// D / 16 lanes take a head, 16 elements each, 8 and 8, so that both elements
// of every rotated pair are in one lane and every access is 16 bytes wide
// (8 bytes for codes). The sum of squares crosses the head's lanes by
// data-parallel moves. A wave's lanes so hold 8 (16) heads of one token in a
// pass and keep the position's cosines and sines, which are 2 to 4 times as
// large as a head, in registers over all passes; kRopeBatch passes' rows are
// in flight together. The new rows are read past the caches, once and for all
// (16384 tokens of 32 + 16 bf16 heads of 128: 86 -> 71 us, 1024: 9.3 -> 8.2).
//
// Memory bounds it: 5.5 to 6.4 TB/s of reads and writes from 8192 tokens on
// with bf16 and FP8 caches (32768 tokens: 136 and 117 us), 4.9 with f32 (331
// us), whose lanes take 32 bytes at a time; a copy of the same size reaches 5.3.
// Below, the launch and the chain of length, block-table entry and rows.
#include <type_traits>

#include "rope.h"

namespace comem {
namespace {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

typedef float f32x8 __attribute__((ext_vector_type(8), aligned(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

struct F32Row {
  using Elem = float;
  using Raw = f32x8;  // 8 elements
  static __device__ f32x8 widen(Raw r) { return r; }
  static __device__ Raw narrow(f32x8 x) { return x; }
};

struct Bf16Row {
  using Elem = __bf16;
  using Raw = bf16x8;
  static __device__ f32x8 widen(Raw r) { return __builtin_convertvector(r, f32x8); }
  static __device__ Raw narrow(f32x8 x) { return __builtin_convertvector(x, bf16x8); }  // to nearest even
};

// The E4M3 codes nearest to 8 values; 448 is the largest magnitude, NaN stays NaN.
__device__ inline u32x2 fp8_codes(f32x8 x) {
  u32x2 r;
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = __builtin_fabsf(x[e]) > 448.f ? __builtin_copysignf(448.f, x[e]) : x[e];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i], x[4 * i + 1], 0, false);
    r[i] = static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i + 2], x[4 * i + 3], lo, true));
  }
  return r;
}

typedef float f32x4 __attribute__((ext_vector_type(4)));
__device__ inline f32x4 load4(const float* p) { return *reinterpret_cast<const f32x4*>(p); }
__device__ inline f32x8 load8(const float* p) { return *reinterpret_cast<const f32x8*>(p); }

// STREAM: past the caches (a form of its own: with both stores behind a
// branch the compiler makes one ordinary store of them).
template <bool STREAM, typename Raw>
__device__ inline void put(char* at, Raw x) {
  if constexpr (STREAM) {
    __builtin_nontemporal_store(x, reinterpret_cast<Raw*>(at));
  } else {
    *reinterpret_cast<Raw*>(at) = x;
  }
}

template <int CTRL>
__device__ inline float moved(float x) {
  return __uint_as_float(__builtin_amdgcn_update_dpp(0, static_cast<int>(__float_as_uint(x)), CTRL, 0xf, 0xf, true));
}

// Sum over the D / 16 lanes of a head (neighbours, pairs, the 8 mirrored).
template <int D>
__device__ inline float head_sum(float x) {
  x += moved<0xb1>(x);
  x += moved<0x4e>(x);
  if constexpr (D == 128) x += moved<0x141>(x);
  return x;
}

template <int D, RopeCache CACHE, bool PAGED, bool STREAM>
__global__ __launch_bounds__(64 * kRopeWaves) void rope_append_kernel(const RopeParams p) {
  using Row = typename std::conditional<CACHE == RopeCache::kF32, F32Row, Bf16Row>::type;
  using Raw = typename Row::Raw;
  using Elem = typename Row::Elem;
  constexpr int kLanes = D / 16;       // lanes of a head
  constexpr int kHeads = 64 / kLanes;  // heads of a pass
  constexpr int kRow = D * static_cast<int>(sizeof(Elem));
  const int b = blockIdx.y;
  const int lane = threadIdx.x & 63;
  const int block = blockIdx.z * gridDim.x + blockIdx.x;
  const int unit = __builtin_amdgcn_readfirstlane(block * kRopeWaves + (threadIdx.x >> 6));
  const int i = unit / p.parts;  // new token
  const int part = unit - i * p.parts;
  const int L = p.ctx_lens[b];
  const int M = p.q_lens == nullptr ? 1 : p.q_lens[b];
  if (L < 0 || L > p.max_ctx || M < 0 || M > L || M > p.max_q || i >= M) return;
  const int64_t row = p.q_lens == nullptr ? b : p.q_start[b] + i;
  const int t = L - M + i;

  // Cache row of the token, or negative: nothing to store.
  int64_t at;
  if constexpr (PAGED) {
    const int entry = t >> p.page_shift;
    const int32_t page = p.block_table[static_cast<int64_t>(b) * p.max_pages + entry];
    at = page < 0 || page >= p.num_pages
             ? -1
             : static_cast<int64_t>(page) * p.stride_page + static_cast<int64_t>(t & p.page_mask) * p.stride_token;
  } else {
    const int64_t start = p.seq_start[b];
    at = start < 0 ? -1 : (start + t) * p.stride_token;
  }

  // Elements of this lane: 8 from e0 on and 8 from e1 on. Neighbouring lanes
  // have neighbouring pieces of 16 bytes in either access.
  const int j = lane % kLanes;
  const int turned_lanes = p.rot_dim / 16;  // rotated in halves
  const bool halves = p.interleaved == 0 && j < turned_lanes;
  int e0, e1;
  if (p.interleaved != 0) {
    e0 = 8 * j;
    e1 = D / 2 + 8 * j;
  } else if (halves) {
    e0 = 8 * j;
    e1 = p.rot_dim / 2 + 8 * j;
  } else {
    e0 = p.rot_dim + 8 * (j - turned_lanes);
    e1 = e0 + (D - p.rot_dim) / 2;
  }
  // Interleaved: 4 angles for each piece that is rotated. (A piece that is not
  // is left out of the rotation: an infinity times a sine of 0 is NaN.)
  const bool turn0 = p.interleaved != 0 && e0 < p.rot_dim, turn1 = p.interleaved != 0 && e1 < p.rot_dim;
  f32x8 c{}, s{};
  if (p.rot_dim > 0) {
    const int32_t pos = min(max(p.positions == nullptr ? t : p.positions[row], 0), p.num_positions - 1);
    const float* angles = p.cos_sin + static_cast<int64_t>(pos) * p.rot_dim;
    const int half = p.rot_dim / 2;
    if (halves) {
      c = load8(angles + 8 * j);
      s = load8(angles + half + 8 * j);
    } else if (p.interleaved != 0) {
      if (turn0) {
        c.lo = load4(angles + e0 / 2);
        s.lo = load4(angles + half + e0 / 2);
      }
      if (turn1) {
        c.hi = load4(angles + e1 / 2);
        s.hi = load4(angles + half + e1 / 2);
      }
    }
  }
  Raw wq0{}, wq1{}, wk0{}, wk1{};
  if (p.q_weight != nullptr) {
    wq0 = *reinterpret_cast<const Raw*>(p.q_weight + e0 * sizeof(Elem));
    wq1 = *reinterpret_cast<const Raw*>(p.q_weight + e1 * sizeof(Elem));
  }
  if (p.k_weight != nullptr) {
    wk0 = *reinterpret_cast<const Raw*>(p.k_weight + e0 * sizeof(Elem));
    wk1 = *reinterpret_cast<const Raw*>(p.k_weight + e1 * sizeof(Elem));
  }

  // Heads in order: queries, keys, values.
  const int first_v = p.num_q_heads + p.num_kv_heads, heads = first_v + p.num_kv_heads;
  const int end = min((part + 1) * p.part_passes * kHeads, heads);
  for (int h0 = part * p.part_passes * kHeads + lane / kLanes; h0 < end; h0 += kHeads * kRopeBatch) {
    Raw r0[kRopeBatch], r1[kRopeBatch];
#pragma unroll
    for (int u = 0; u < kRopeBatch; ++u) {
      const int h = h0 + u * kHeads;
      r0[u] = Raw{};
      r1[u] = Raw{};
      if (h < end) {
        const char* src = h < p.num_q_heads ? p.q + row * p.q_stride + h * kRow
                          : h < first_v     ? p.new_k + row * p.k_stride + (h - p.num_q_heads) * kRow
                                            : p.new_v + row * p.v_stride + (h - first_v) * kRow;
        r0[u] = __builtin_nontemporal_load(reinterpret_cast<const Raw*>(src + e0 * sizeof(Elem)));
        r1[u] = __builtin_nontemporal_load(reinterpret_cast<const Raw*>(src + e1 * sizeof(Elem)));
      }
    }
#pragma unroll
    for (int u = 0; u < kRopeBatch; ++u) {
      const int h = h0 + u * kHeads;
      if (h >= end) continue;
      const bool is_q = h < p.num_q_heads, is_v = h >= first_v;
      f32x8 x0 = Row::widen(r0[u]), x1 = Row::widen(r1[u]);
      if (!is_v) {
        if ((is_q ? p.q_weight : p.k_weight) != nullptr) {
          float ss = 0.f;
#pragma unroll
          for (int e = 0; e < 8; ++e) ss += x0[e] * x0[e] + x1[e] * x1[e];
          const float r = rsqrtf(head_sum<D>(ss) * (1.f / D) + p.eps);
          x0 = x0 * r * Row::widen(is_q ? wq0 : wk0);
          x1 = x1 * r * Row::widen(is_q ? wq1 : wk1);
        }
        if (halves) {
          const f32x8 y0 = x0 * c - x1 * s;
          x1 = x1 * c + x0 * s;
          x0 = y0;
        } else if (p.interleaved != 0) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float a0 = x0[2 * e], a1 = x1[2 * e];
            const float b0 = x0[2 * e + 1], b1 = x1[2 * e + 1];
            x0[2 * e] = turn0 ? a0 * c[e] - b0 * s[e] : a0;
            x0[2 * e + 1] = turn0 ? b0 * c[e] + a0 * s[e] : b0;
            x1[2 * e] = turn1 ? a1 * c[e + 4] - b1 * s[e + 4] : a1;
            x1[2 * e + 1] = turn1 ? b1 * c[e + 4] + a1 * s[e + 4] : b1;
          }
        }
      }
      if (is_q) {
        char* dst = p.q_out + (row * p.num_q_heads + h) * kRow;
        put<STREAM>(dst + e0 * sizeof(Elem), Row::narrow(x0));
        put<STREAM>(dst + e1 * sizeof(Elem), Row::narrow(x1));
      } else if (at >= 0) {
        char* dst = (is_v ? p.v : p.k) + at + (h - (is_v ? first_v : p.num_q_heads)) * p.stride_head;
        if constexpr (CACHE == RopeCache::kFp8) {
          const float inv = is_v ? p.inv_v_scale : p.inv_k_scale;
          *reinterpret_cast<u32x2*>(dst + e0) = fp8_codes(x0 * inv);
          *reinterpret_cast<u32x2*>(dst + e1) = fp8_codes(x1 * inv);
        } else {
          put<STREAM>(dst + e0 * sizeof(Elem), is_v ? r0[u] : Row::narrow(x0));
          put<STREAM>(dst + e1 * sizeof(Elem), is_v ? r1[u] : Row::narrow(x1));
        }
      }
    }
  }
}

#define COMEM_ROPE_FORMS(D, C)                                                                   \
  template __global__ void rope_append_kernel<D, RopeCache::C, false, false>(const RopeParams); \
  template __global__ void rope_append_kernel<D, RopeCache::C, true, false>(const RopeParams);  \
  template __global__ void rope_append_kernel<D, RopeCache::C, false, true>(const RopeParams);  \
  template __global__ void rope_append_kernel<D, RopeCache::C, true, true>(const RopeParams);
COMEM_ROPE_FORMS(64, kF32)
COMEM_ROPE_FORMS(64, kBf16)
COMEM_ROPE_FORMS(64, kFp8)
COMEM_ROPE_FORMS(128, kF32)
COMEM_ROPE_FORMS(128, kBf16)
COMEM_ROPE_FORMS(128, kFp8)
#undef COMEM_ROPE_FORMS

template <int D, RopeCache CACHE>
RopeKernelFn rope_form(bool paged, bool stream) {
  if (stream) return paged ? rope_append_kernel<D, CACHE, true, true> : rope_append_kernel<D, CACHE, false, true>;
  return paged ? rope_append_kernel<D, CACHE, true, false> : rope_append_kernel<D, CACHE, false, false>;
}

template <int D>
RopeKernelFn rope_by_cache(RopeCache cache, bool paged, bool stream) {
  if (cache == RopeCache::kF32) return rope_form<D, RopeCache::kF32>(paged, stream);
  if (cache == RopeCache::kBf16) return rope_form<D, RopeCache::kBf16>(paged, stream);
  return rope_form<D, RopeCache::kFp8>(paged, stream);
}

}  // namespace

RopeKernelFn select_rope_kernel(int head_dim, RopeCache cache, bool paged, bool stream) {
  if (head_dim == 128) return rope_by_cache<128>(cache, paged, stream);
  if (head_dim == 64) return rope_by_cache<64>(cache, paged, stream);
  return nullptr;
}

}  // namespace comem
