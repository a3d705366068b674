// Bounds of a page's keys, and the scores that they allow (gfx950).
//
// Bounds. Least and greatest are taken on the bit patterns: a float's bits with
// all but the sign turned over where the sign is set order as signed integers,
// so that bf16 pairs take packed 16-bit minima, and nothing is rounded. A
// thread has one 16-byte piece of the tokens' heads and every slots-th token
// of the page; the slots meet in LDS. Bound by a launch, the table's and the
// keys' round trips until there is much to read: a step's 64 pages of 64 FP8
// tokens 6.1 us, 8 chunks of 128-2048 tokens in pages of 16, 17 MB, 6.6 us,
// 8 whole contexts of 8192, 134 MB (from the last cache), 25 us = 6 TB/s.
//
// Scores. max(q_d lo_d, q_d hi_d) = max(q_d, 0) hi_d + min(q_d, 0) lo_d, so the
// bound of 16 blocks with the G query heads is two matrix products, the
// negative parts of the queries with the least keys and the positive ones
// with the greatest; the largest over a KV head's queries is the score. A wave
// has 16 blocks of a head, which it reads once: 8 sequences of 131072 FP8
// tokens in pages of 64, 34 MB of bounds, 8.9 us = 3.9 TB/s, of which a launch
// and two dependent loads are about 3 (one sequence of 32768: 3.1 us).
#include "attn_common.h"
#include "blocks.h"
#include "dot_rows.h"

namespace comem {
namespace {

typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef unsigned short u16x8 __attribute__((ext_vector_type(8)));
typedef int s32x4 __attribute__((ext_vector_type(4)));

// Least and greatest of the elements of a 16-byte piece.
template <CacheType C>
struct Ends;
template <>
struct Ends<CacheType::kF32> {
  s32x4 lo, hi;
  __device__ void clear() {
    lo = s32x4(INT32_MAX);
    hi = ~lo;
  }
  static __device__ s32x4 order(s32x4 x) { return x ^ ((x >> 31) & 0x7fffffff); }
  __device__ void add(dot_u32x4 x) {
    const s32x4 v = order(__builtin_bit_cast(s32x4, x));
    lo = __builtin_elementwise_min(lo, v);
    hi = __builtin_elementwise_max(hi, v);
  }
  __device__ void join(const Ends& o) {
    lo = __builtin_elementwise_min(lo, o.lo);
    hi = __builtin_elementwise_max(hi, o.hi);
  }
  __device__ dot_u32x4 least() const { return __builtin_bit_cast(dot_u32x4, order(lo)); }
  __device__ dot_u32x4 greatest() const { return __builtin_bit_cast(dot_u32x4, order(hi)); }
};
template <>
struct Ends<CacheType::kBf16> {
  s16x8 lo, hi;
  __device__ void clear() {
    lo = s16x8(static_cast<short>(0x7fff));
    hi = ~lo;
  }
  static __device__ s16x8 order(s16x8 x) { return x ^ ((x >> 15) & static_cast<short>(0x7fff)); }
  __device__ void add(dot_u32x4 x) {
    const s16x8 v = order(__builtin_bit_cast(s16x8, x));
    lo = __builtin_elementwise_min(lo, v);
    hi = __builtin_elementwise_max(hi, v);
  }
  __device__ void join(const Ends& o) {
    lo = __builtin_elementwise_min(lo, o.lo);
    hi = __builtin_elementwise_max(hi, o.hi);
  }
  __device__ dot_u32x4 least() const { return __builtin_bit_cast(dot_u32x4, order(lo)); }
  __device__ dot_u32x4 greatest() const { return __builtin_bit_cast(dot_u32x4, order(hi)); }
};
// Codes: the even and the odd ones, each in the high byte of 16 bits.
template <>
struct Ends<CacheType::kFp8> {
  s16x8 lo0, lo1, hi0, hi1;
  __device__ void clear() {
    lo0 = lo1 = s16x8(static_cast<short>(0x7f00));
    hi0 = hi1 = s16x8(static_cast<short>(0x8000));
  }
  static __device__ s16x8 order(s16x8 x) { return x ^ ((x >> 15) & static_cast<short>(0x7f00)); }
  __device__ void add(dot_u32x4 x) {
    const s16x8 v = __builtin_bit_cast(s16x8, x);
    const s16x8 even = order(v << 8), odd = order(v & static_cast<short>(0xff00));
    lo0 = __builtin_elementwise_min(lo0, even);
    lo1 = __builtin_elementwise_min(lo1, odd);
    hi0 = __builtin_elementwise_max(hi0, even);
    hi1 = __builtin_elementwise_max(hi1, odd);
  }
  __device__ void join(const Ends& o) {
    lo0 = __builtin_elementwise_min(lo0, o.lo0);
    lo1 = __builtin_elementwise_min(lo1, o.lo1);
    hi0 = __builtin_elementwise_max(hi0, o.hi0);
    hi1 = __builtin_elementwise_max(hi1, o.hi1);
  }
  static __device__ dot_u32x4 codes(s16x8 even, s16x8 odd) {
    const u16x8 e = __builtin_bit_cast(u16x8, order(even)) >> 8, o = __builtin_bit_cast(u16x8, order(odd));
    return __builtin_bit_cast(dot_u32x4, e | o);
  }
  __device__ dot_u32x4 least() const { return codes(lo0, lo1); }
  __device__ dot_u32x4 greatest() const { return codes(hi0, hi1); }
};

template <CacheType C>
__global__ __launch_bounds__(kBoundsThreads) void block_bounds_kernel(const BoundsParams p) {
  __shared__ Ends<C> meet[kBoundsThreads];
  const int b = blockIdx.y, tid = threadIdx.x;
  const int L = uniform_i32(p.ctx_lens[b]);
  const int M = p.q_lens == nullptr ? 1 : uniform_i32(p.q_lens[b]);
  if (L > p.max_ctx || M < 1 || M > L || M > p.max_q) return;
  const int width = p.width;
  const int slots = kBoundsThreads / width;
  const int slot = tid / width;
  const int piece = blockIdx.z * width + tid % width;
  const bool works = slot < slots && piece < p.pieces;
  const int head = piece >> p.piece_shift, part = piece & ((1 << p.piece_shift) - 1);
  const int last = (L - 1) >> p.page_shift;
  for (int n = ((L - M) >> p.page_shift) + blockIdx.x; n <= last; n += gridDim.x) {
    const int32_t page = uniform_i32(p.block_table[static_cast<int64_t>(b) * p.max_pages + n]);
    if (page < 0 || page >= p.num_pages) continue;
    const int tokens = min(1 << p.page_shift, L - (n << p.page_shift));
    const char* k = p.k + static_cast<int64_t>(page) * p.stride_page + head * p.stride_head + 16 * part;
    Ends<C> ends;
    ends.clear();
    if (works) {
      // Four tokens at a time, the next four asked for ahead; past the last
      // token it is read again.
      dot_u32x4 x[4], next[4];
      auto ask = [&](int t, dot_u32x4 (&y)[4]) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          y[e] = *reinterpret_cast<const dot_u32x4*>(k + min(t + e * slots, tokens - 1) * p.stride_token);
      };
      ask(slot, x);
#pragma unroll 1
      for (int t = slot;;) {
        t += 4 * slots;
        if (t < tokens) ask(t, next);
#pragma unroll
        for (int e = 0; e < 4; ++e) ends.add(x[e]);
        if (t >= tokens) break;
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = next[e];
      }
    }
    // Slots with a token: halved until one is left.
    for (int live = min(slots, tokens); live > 1;) {
      const int half = (live + 1) >> 1;
      meet[tid] = ends;
      __syncthreads();
      if (works && slot < live - half) ends.join(meet[tid + half * width]);
      __syncthreads();
      live = half;
    }
    if (works && slot == 0) {
      const int64_t row = 16 << p.piece_shift;  // bytes of a head's row
      char* out = p.bounds + (static_cast<int64_t>(page) * (p.pieces >> p.piece_shift) + head) * 2 * row + 16 * part;
      *reinterpret_cast<dot_u32x4*>(out) = ends.least();
      *reinterpret_cast<dot_u32x4*>(out + row) = ends.greatest();
    }
  }
}

// A query row's negative and positive elements, 0 in the others' places.
template <int D, CacheType C>
__device__ inline void by_sign(const DotPart<D, C>& q, DotPart<D, C>& neg, DotPart<D, C>& pos) {
#pragma unroll
  for (int i = 0; i < DotPart<D, C>::kLoads; ++i) {
    dot_u32x4 below;
    if constexpr (C == CacheType::kF32) {
      below = __builtin_bit_cast(dot_u32x4, __builtin_bit_cast(s32x4, q.x[i]) >> 31);
    } else {
      below = __builtin_bit_cast(dot_u32x4, __builtin_bit_cast(s16x8, q.x[i]) >> 15);
    }
    neg.x[i] = q.x[i] & below;
    pos.x[i] = q.x[i] & ~below;
  }
}

__device__ inline int ordered(float x) {
  const int u = static_cast<int>(__float_as_uint(x == x ? x : __builtin_nanf("")));
  return u ^ ((u >> 31) & 0x7fffffff);
}
__device__ inline float unordered(int u) { return __uint_as_float(static_cast<uint32_t>(u ^ ((u >> 31) & 0x7fffffff))); }

template <int D, CacheType C>
__global__ __launch_bounds__(64 * kScoresWaves) void block_scores_kernel(const ScoresParams p) {
  constexpr int kElem = C == CacheType::kF32 ? 4 : C == CacheType::kBf16 ? 2 : 1;
  constexpr int kQueryBytes = D * (C == CacheType::kF32 ? 4 : 2);
  const int b = blockIdx.z;
  const int lane = threadIdx.x & 63, w = uniform_i32(threadIdx.x >> 6);
  const int hk = blockIdx.y * kScoresWaves + w;
  if (hk >= p.num_kv_heads) return;
  const int c = lane & 15, g = lane >> 4;
  const int L = min(max(uniform_i32(p.ctx_lens[b]), 0), p.max_ctx);
  const int blocks = static_cast<int>((static_cast<uint32_t>(L) + (1u << p.page_shift) - 1) >> p.page_shift);
  if (static_cast<int>(blockIdx.x) * kScoresBlocks >= blocks) return;
  DotPart<D, C> q, neg, pos;
  const int64_t row = (static_cast<int64_t>(b) * p.num_kv_heads + hk) * p.group + min(c, p.group - 1);
  q.load_query(p.q + row * kQueryBytes, g);
  by_sign<D, C>(q, neg, pos);
  float* out = p.scores + (static_cast<int64_t>(b) * p.num_kv_heads + hk) * p.scores_stride;
  for (int n0 = blockIdx.x * kScoresBlocks; n0 < blocks; n0 += gridDim.x * kScoresBlocks) {
    const int32_t entry = p.block_table[static_cast<int64_t>(b) * p.max_pages + min(n0 + c, blocks - 1)];
    const int64_t page = entry < 0 || entry >= p.num_pages ? 0 : entry;
    const char* at = p.bounds + (page * p.num_kv_heads + hk) * (2 * D * kElem) + RowPart<D, C>::lane_offset(g);
    RowPart<D, C> lo, hi;
    lo.load(at);
    hi.load(at + D * kElem);
    dot_f32x4 x = dot_rows<D, C>(lo.widened(), neg, dot_f32x4{0.f, 0.f, 0.f, 0.f});
    x = dot_rows<D, C>(hi.widened(), pos, x);
    // Columns past the group repeat its last query.
    float mine = 0.f;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      int v = ordered(x[r]);
      v = max(v, static_cast<int>(row_turned<8>(static_cast<uint32_t>(v))));
      v = max(v, static_cast<int>(row_turned<4>(static_cast<uint32_t>(v))));
      v = max(v, static_cast<int>(row_turned<2>(static_cast<uint32_t>(v))));
      v = max(v, static_cast<int>(row_turned<1>(static_cast<uint32_t>(v))));
      if (c == r) mine = unordered(v);
    }
    const int n = n0 + 4 * g + c;
    if (c < 4 && n < blocks) out[n] = p.scale * mine;
  }
}

template <int D>
ScoresKernelFn scores_by_cache(CacheType cache) {
  if (cache == CacheType::kF32) return block_scores_kernel<D, CacheType::kF32>;
  if (cache == CacheType::kBf16) return block_scores_kernel<D, CacheType::kBf16>;
  return block_scores_kernel<D, CacheType::kFp8>;
}

}  // namespace

BoundsKernelFn select_bounds_kernel(CacheType cache) {
  if (cache == CacheType::kF32) return block_bounds_kernel<CacheType::kF32>;
  if (cache == CacheType::kBf16) return block_bounds_kernel<CacheType::kBf16>;
  return block_bounds_kernel<CacheType::kFp8>;
}

ScoresKernelFn select_scores_kernel(int head_dim, CacheType cache) {
  if (head_dim == 128) return scores_by_cache<128>(cache);
  if (head_dim == 64) return scores_by_cache<64>(cache);
  return nullptr;
}

}  // namespace comem
