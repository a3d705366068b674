// Attention weights of cached tokens, summed over the query rows that see
// them (gfx950).
//
// The attention call's log-sum-exp makes every weight exp2(x - lse) (in log2
// units, x = scale log2(e) q.k) a value of its own, so a token's sum needs no
// other token: no running maximum, no split to merge. A workgroup takes
// 16 SUB tokens of a sequence and all of its query rows. Its waves share the
// tokens and divide the KV heads (and, of fewer heads than waves, a head's
// query rows): a wave keeps the tokens' keys of one head in registers and goes
// through the head's M G query rows, 16 at a time, as the other operand of the
// matrix cores. A lane then holds the scores of one query row with 4 SUB
// tokens, so the row's lse and causal limit are one value a lane, and its
// weights add up in 4 SUB registers over all rows and heads. The 16 lanes of
// a token and the four waves meet once, at the end, in a fixed order.
#include "attn_common.h"
#include "dot_rows.h"
#include "evict.h"

namespace comem {
namespace {

constexpr float kLog2e = 1.4426950408889634f;

__device__ inline float row_total(float x) {
  x += __uint_as_float(row_turned<8>(__float_as_uint(x)));
  x += __uint_as_float(row_turned<4>(__float_as_uint(x)));
  x += __uint_as_float(row_turned<2>(__float_as_uint(x)));
  x += __uint_as_float(row_turned<1>(__float_as_uint(x)));
  return x;
}

template <int D, CacheType C, bool PAGED, int SUB>
__global__ __launch_bounds__(64 * kWeightsWaves) void attn_weights_kernel(const WeightsParams p) {
  constexpr int kTile = 16 * SUB;
  constexpr int kQueryBytes = D * (C == CacheType::kF32 ? 4 : 2);
  __shared__ float part[kWeightsWaves][kTile];
  const int b = blockIdx.y;
  const int L = uniform_i32(p.ctx_lens[b]);
  const int M = p.q_lens == nullptr ? 1 : uniform_i32(p.q_lens[b]);
  if (L > p.max_ctx || M < 1 || M > L || M > p.max_q) return;
  const int64_t row0 = p.q_lens == nullptr ? b : uniform_i64(p.q_start[b]);
  const int64_t seq0 = PAGED ? 0 : uniform_i64(p.seq_start[b]);
  const int old = L - M;  // tokens that all new ones see
  const int lane = threadIdx.x & 63, w = uniform_i32(threadIdx.x >> 6);
  const int c = lane & 15, g = lane >> 4;
  const int G = 1 << p.group_shift, num_q_heads = p.num_kv_heads << p.group_shift;
  const int per = 16 >> p.group_shift;                              // new tokens of 16 query rows
  const int col_token = c >> p.group_shift, col_head = c & (G - 1);
  const int groups = (M + per - 1) / per;                           // of 16 query rows
  const int shares = max(1, kWeightsWaves / p.num_kv_heads);        // waves of a head

  for (int t0 = blockIdx.x * kTile; t0 < L; t0 += gridDim.x * kTile) {
    const int own = t0 + static_cast<int>(threadIdx.x);             // the token that this thread writes
    const bool writes = threadIdx.x < kTile && own < L;
    float* out = p.weights + b * p.weights_stride + own;
    float before = 0.f;
    if (p.prior != nullptr && writes && own < old) before = p.prior[b * p.weights_stride + own];

    const char* key[SUB];
#pragma unroll
    for (int s = 0; s < SUB; ++s) {
      const int t = min(t0 + 16 * s + c, L - 1);
      int64_t at;
      if constexpr (PAGED) {
        const int32_t page = p.block_table[static_cast<int64_t>(b) * p.max_pages + (t >> p.page_shift)];
        at = static_cast<int64_t>(page < 0 || page >= p.num_pages ? 0 : page) * p.stride_page +
             static_cast<int64_t>(t & p.page_mask) * p.stride_token;
      } else {
        at = (seq0 + t) * p.stride_token;
      }
      key[s] = p.k + at + RowPart<D, C>::lane_offset(g);
    }
    float sum[SUB][4] = {};
    // Rows of new tokens before the tile's first token see none of it.
    const int begin = max(0, t0 - old) / per;
    const int last = min(t0 + kTile, L) - 1;
    for (int u = w; u < p.num_kv_heads * shares; u += kWeightsWaves) {
      const int hk = u / shares;
      DotPart<D, C> k[SUB];
#pragma unroll
      for (int s = 0; s < SUB; ++s) {
        RowPart<D, C> r;
        r.load(key[s] + hk * p.stride_head);
        k[s] = r.widened();
      }
      for (int n = begin + u % shares; n < groups; n += shares) {
        const int i = n * per + col_token;
        const int64_t row = (row0 + min(i, M - 1)) * num_q_heads + hk * G + col_head;
        DotPart<D, C> q;
        q.load_query(p.q + row * kQueryBytes, g);
        const float lse = p.lse[row];
        const float below = -lse * kLog2e;
        const int limit = i < M && lse != -INFINITY ? old + i : -1;  // last token that this query row sees
        const bool all = __builtin_amdgcn_ballot_w64(limit < last) == 0;
#pragma unroll
        for (int s = 0; s < SUB; ++s) {
          const dot_f32x4 x = dot_rows<D, C>(k[s], q, dot_f32x4{0.f, 0.f, 0.f, 0.f});
          if (all) {
#pragma unroll
            for (int r = 0; r < 4; ++r) sum[s][r] += fast_exp2(fmaf(x[r], p.scale_log2, below));
          } else {
#pragma unroll
            for (int r = 0; r < 4; ++r)
              sum[s][r] += t0 + 16 * s + 4 * g + r <= limit ? fast_exp2(fmaf(x[r], p.scale_log2, below)) : 0.f;
          }
        }
      }
    }
#pragma unroll
    for (int s = 0; s < SUB; ++s)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float x = row_total(sum[s][r]);
        if (c == r) part[w][16 * s + 4 * g + r] = x;
      }
    __syncthreads();
    if (writes) {
      float x = 0.f;
#pragma unroll
      for (int i = 0; i < kWeightsWaves; ++i) x += part[i][threadIdx.x];
      *out = p.prior != nullptr && own < old ? fmaf(p.decay, before, x) : x;
    }
    __syncthreads();
  }
}

template <int D, CacheType C, bool PAGED>
WeightsKernelFn by_sub(int sub) {
  if (sub == 1) return attn_weights_kernel<D, C, PAGED, 1>;
  if (sub == 2) return attn_weights_kernel<D, C, PAGED, 2>;
  if constexpr (C != CacheType::kF32)
    if (sub == 4) return attn_weights_kernel<D, C, PAGED, 4>;
  return nullptr;
}

template <int D, bool PAGED>
WeightsKernelFn by_cache(CacheType cache, int sub) {
  if (cache == CacheType::kF32) return by_sub<D, CacheType::kF32, PAGED>(sub);
  if (cache == CacheType::kBf16) return by_sub<D, CacheType::kBf16, PAGED>(sub);
  return by_sub<D, CacheType::kFp8, PAGED>(sub);
}

}  // namespace

WeightsKernelFn select_weights_kernel(int head_dim, CacheType cache, bool paged, int sub) {
  if (head_dim == 128) return paged ? by_cache<128, true>(cache, sub) : by_cache<128, false>(cache, sub);
  if (head_dim == 64) return paged ? by_cache<64, true>(cache, sub) : by_cache<64, false>(cache, sub);
  return nullptr;
}

}  // namespace comem
