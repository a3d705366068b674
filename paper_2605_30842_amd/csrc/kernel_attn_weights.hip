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
// a token and the waves meet once, at the end, in a fixed order. Scores, weights
// and sums are float32; FP8 keys become bf16, which holds them exactly.
//
// A decode step (RING false) is bound by its keys: 64 sequences of 2048-16384
// tokens, 1.2 GB, 206-231 us, 5.2-5.9 TB/s; 8 sequences of 1000-7000 FP8
// tokens, 30 MB, 10 us, where a launch, the table's and the keys' round trips
// are half of it.
//
// A chunk (RING true) is bound by the matrix cores, the exponentials and what
// the two do not overlap: 300 rows over 24300 tokens with 32 heads of 128, 60
// GFLOP and 233 million exponentials, 75-78 us, 0.76-0.8 PFLOP/s (a large matrix
// product 1.19; the first 15 ms after the card was idle 84-86, before its clock
// has risen), FP8 74, float32 513 (0.116 of 0.152); matrix cores busy 35%, VALU
// 55% of the SIMDs' cycles. No one of them is the bound: when it took 86 us,
// leaving out the exponentials saved 3, the products 4, the requests for query
// rows 18. What costs beside them: bank conflicts (see QueryRing), and 24 scalar
// registers (31 paged) that the 96-token form with 237 of 256 vector registers
// keeps in lanes of those. Rows read from LDS a turn ahead as well: 2% less for
// 20 registers more; not kept.
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

// Where a wave keeps the query rows that it has asked for ahead: kSlots groups
// of 16 rows and their lse. A request brings 1 KiB of rows, each one whole; a
// row's pieces of 16 bytes lie at their place exclusive-or the row's three low
// bits: of the 16 rows of which a read takes one piece each, rows c and c + 8
// share their banks and no others do. (Conflicts are 0.46 of the LDS's active
// cycles at 300 rows over 24300 tokens; four bits, for rows of 16 pieces and
// more, took no less time.)
template <int D, CacheType C>
struct QueryRing {
  static constexpr int kLoads = DotPart<D, C>::kLoads;
  static constexpr int kSlots = kLoads > 4 ? 2 : 4;
  static constexpr int kWaits = (kSlots - 1) * (kLoads + 1);  // requests after the oldest group's
  static constexpr int kPieces = D * (C == CacheType::kF32 ? 4 : 2) / 16;  // of a row
  struct Slot {
    dot_u32x4 x[16 * kPieces];
    float lse[64];
  };
  static __device__ int turned(int row, int piece) { return piece ^ (row & 7); }
  // Place of load i of lane 16 g + c in a slot.
  static __device__ int place(int i, int c, int g) {
    const int piece = (DotPart<D, C>::lane_offset(g) + DotPart<D, C>::kStep * i) / 16;
    return c * kPieces + turned(c, piece);
  }
};

// 16 (4) bytes from each lane's address (`from` is uniform, `offset` the
// lane's) to consecutive places in LDS from `to` on. In assembly, since the
// compiler would wait for all of them before it reads any LDS.
__device__ inline void request_x4(const char* from, uint32_t offset, uint32_t to) {
  asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(offset), "s"(from), "{m0}"(to) : "memory");
}
__device__ inline void request_x1(const char* from, uint32_t offset, uint32_t to) {
  asm volatile("s_nop 0\n\tglobal_load_lds_dword %0, %1" ::"v"(offset), "s"(from), "{m0}"(to) : "memory");
}
__device__ inline uint32_t lds_address(const void* p) {
  return static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) const void*)p));
}

// RING: query rows come through LDS, asked for groups ahead (a load that one
// turn of products has to cover takes longer than the turn).
template <int D, CacheType C, bool PAGED, int SUB, bool RING>
__global__ __launch_bounds__(64 * kWeightsWaves, 2) void attn_weights_kernel(const WeightsParams p) {
  using Ring = QueryRing<D, C>;
  constexpr int kTile = 16 * SUB;
  constexpr int kQueryBytes = D * (C == CacheType::kF32 ? 4 : 2);
  extern __shared__ char shared[];  // the waves' rings
  __shared__ float part[kWeightsWaves][kTile];
  const int b = blockIdx.y;
  const int L = uniform_i32(p.ctx_lens[b]);
  const int M = p.q_lens == nullptr ? 1 : uniform_i32(p.q_lens[b]);
  if (L > p.max_ctx || M < 1 || M > L || M > p.max_q) return;
  const int64_t row0 = p.q_lens == nullptr ? b : uniform_i64(p.q_start[b]);
  const int64_t seq0 = PAGED ? 0 : uniform_i64(p.seq_start[b]);
  const int old = L - M;  // tokens that all new ones see
  const int waves = blockDim.x >> 6;
  const int lane = threadIdx.x & 63, w = uniform_i32(threadIdx.x >> 6);
  const int c = lane & 15, g = lane >> 4;
  const int G = 1 << p.group_shift, num_q_heads = p.num_kv_heads << p.group_shift;
  const int per = 16 >> p.group_shift;                        // new tokens of 16 query rows
  const int groups = (M + per - 1) / per;                     // of 16 query rows
  const int shares = max(1, waves / p.num_kv_heads);          // waves of a head

  for (int t0 = blockIdx.x * kTile; t0 < L; t0 += gridDim.x * kTile) {
    // The tokens that this thread writes, and what they had.
    constexpr int kOwn = (kTile + 63) / 64;
    float before[kOwn];
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
      const int own = threadIdx.x + i * blockDim.x;
      before[i] = p.prior != nullptr && p.partial == nullptr && own < kTile && t0 + own < old
                      ? p.prior[b * p.weights_stride + t0 + own]
                      : 0.f;
    }

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
    for (int u = w; u < p.num_kv_heads * shares; u += waves) {
      const int hk = u / shares;
      const int first = begin + blockIdx.z * shares + u % shares, step = gridDim.z * shares;
      if (first >= groups) continue;
      auto token_of = [&](int n) { return n * per + (c >> p.group_shift); };
      auto row_of = [&](int n) { return (row0 + min(token_of(n), M - 1)) * num_q_heads + hk * G + (c & (G - 1)); };
      DotPart<D, C> k[SUB];
      auto load_keys = [&] {
        RowPart<D, C> r[SUB];
#pragma unroll
        for (int s = 0; s < SUB; ++s) r[s].load(key[s] + hk * p.stride_head);
#pragma unroll
        for (int s = 0; s < SUB; ++s) k[s] = r[s].widened();
      };
      auto pay = [&](const DotPart<D, C>& q, float lse, int token) {
        const float below = -lse * kLog2e;
        // Last token that the lane's query row sees; a row that is none, or saw nothing, sees none.
        const int limit = token < M && lse != -INFINITY ? old + token : -1;
        const bool all = __builtin_amdgcn_ballot_w64(limit < last) == 0;
        if (all) {
          dot_f32x4 x[SUB];
#pragma unroll
          for (int s = 0; s < SUB; ++s) x[s] = dot_rows<D, C>(k[s], q, dot_f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
          for (int s = 0; s < SUB; ++s)
#pragma unroll
            for (int r = 0; r < 4; ++r) sum[s][r] += fast_exp2(fmaf(x[s][r], p.scale_log2, below));
          // A slab's products run beside the exponentials of the slab before the last.
          constexpr int kMfma = C == CacheType::kF32 ? D / 4 : D / 32;
          constexpr int kLead = SUB > 2 ? 2 : 1;
          __builtin_amdgcn_sched_group_barrier(0x8, kLead * kMfma, 0);
#pragma unroll
          for (int i = 0; i < 4 * (SUB - kLead); ++i) {
            __builtin_amdgcn_sched_group_barrier(0x8, kMfma / 4 > 0 ? kMfma / 4 : 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x402, 3, 0);
          }
          __builtin_amdgcn_sched_group_barrier(0x402, 12 * kLead, 0);
        } else {
#pragma unroll
          for (int s = 0; s < SUB; ++s) {
            const dot_f32x4 x = dot_rows<D, C>(k[s], q, dot_f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
            for (int r = 0; r < 4; ++r)
              sum[s][r] += t0 + 16 * s + 4 * g + r <= limit ? fast_exp2(fmaf(x[r], p.scale_log2, below)) : 0.f;
          }
        }
      };
      if constexpr (RING) {
        typename Ring::Slot* slots = reinterpret_cast<typename Ring::Slot*>(shared) + w * Ring::kSlots;
        // Offsets of the lane's pieces from a group's first row, and of its lse.
        const int64_t token_bytes = static_cast<int64_t>(num_q_heads) * kQueryBytes;  // 16 / G tokens: below 2^31
        auto row_offset_of = [&](int row, int most) {
          return static_cast<uint32_t>(min(row >> p.group_shift, most) * token_bytes + (row & (G - 1)) * kQueryBytes);
        };
        auto piece_offset = [&](int i, int most) {
          const int at = 64 * i + lane, row = at / Ring::kPieces;
          return row_offset_of(row, most) + 16 * Ring::turned(row, at % Ring::kPieces);
        };
        auto lse_offset = [&](int most) { return row_offset_of(c, most) / (kQueryBytes / 4); };
        uint32_t offset[Ring::kLoads];
#pragma unroll
        for (int i = 0; i < Ring::kLoads; ++i) offset[i] = piece_offset(i, per);
        const uint32_t offset_lse = lse_offset(per);
        auto request = [&](int n, int slot) {
          const int64_t row = uniform_i64((row0 + static_cast<int64_t>(n) * per) * num_q_heads + hk * G);
          const char* from = p.q + row * kQueryBytes;
          const char* from_lse = reinterpret_cast<const char*>(p.lse + row);
          const uint32_t to = uniform_i32(lds_address(&slots[slot]));
          const int most = M - 1 - n * per;  // the group's last token (rows past it repeat it)
          if (most >= per - 1) {
#pragma unroll
            for (int i = 0; i < Ring::kLoads; ++i) request_x4(from, offset[i], to + 1024 * i);
            request_x1(from_lse, offset_lse, to + 1024 * Ring::kLoads);
          } else {
#pragma unroll
            for (int i = 0; i < Ring::kLoads; ++i) request_x4(from, piece_offset(i, most), to + 1024 * i);
            request_x1(from_lse, lse_offset(most), to + 1024 * Ring::kLoads);
          }
        };
        // The groups, from another one on in every workgroup: those of an XCD
        // would else ask its L2 for the same lines at the same time.
        const int count = (groups - first + step - 1) / step, lead = blockIdx.x * 5 % count;
        auto group_at = [&](int i) {
          i = min(i, count - 1) + lead;
          return first + (i < count ? i : i - count) * step;
        };
#pragma unroll
        for (int i = 0; i < Ring::kSlots - 1; ++i) request(group_at(i), i);
        load_keys();
        // Here the compiler waits for the keys: in the loop it would wait for
        // every request in flight, of which it does not know.
#pragma unroll
        for (int s = 0; s < SUB; ++s)
#pragma unroll
          for (int i = 0; i < DotPart<D, C>::kLoads; ++i) asm volatile("" : "+v"(k[s].x[i]));
#pragma unroll 1
        for (int i = 0; i < count; ++i) {
          const int slot = i % Ring::kSlots;
          asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the slot that is asked for anew has been read
          request(group_at(i + Ring::kSlots - 1), (i + Ring::kSlots - 1) % Ring::kSlots);
          asm volatile("s_waitcnt vmcnt(%0)" ::"n"(Ring::kWaits) : "memory");
          DotPart<D, C> q;
#pragma unroll
          for (int j = 0; j < Ring::kLoads; ++j) q.x[j] = slots[slot].x[Ring::place(j, c, g)];
          pay(q, slots[slot].lse[lane], token_of(group_at(i)));
        }
        // What was asked for past the last group is in no one's way, and the last slot has been read before the next
        // head asks for it anew.
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
      } else {
        for (int n = first; n < groups; n += step) {
          const int64_t row = row_of(n);
          DotPart<D, C> q;
          q.load_query(p.q + row * kQueryBytes, g);
          const float lse = p.lse[row];
          if (n == first) load_keys();
          pay(q, lse, token_of(n));
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
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
      const int own = threadIdx.x + i * blockDim.x;
      if (own >= kTile || t0 + own >= L) continue;
      float x = 0.f;
      for (int v = 0; v < waves; ++v) x += part[v][own];
      if (p.partial != nullptr) {
        p.partial[(static_cast<int64_t>(blockIdx.z) * gridDim.y + b) * p.max_ctx + t0 + own] = x;
      } else {
        p.weights[b * p.weights_stride + t0 + own] = p.prior != nullptr && t0 + own < old ? fmaf(p.decay, before[i], x) : x;
      }
    }
    __syncthreads();
  }
}

// The sums of the `splits` workgroups that shared a sequence's query rows.
__global__ __launch_bounds__(256) void add_weights_kernel(const WeightsParams p, int splits) {
  const int b = blockIdx.y;
  const int L = uniform_i32(p.ctx_lens[b]);
  const int M = p.q_lens == nullptr ? 1 : uniform_i32(p.q_lens[b]);
  if (L > p.max_ctx || M < 1 || M > L || M > p.max_q) return;
  for (int t = blockIdx.x * 256 + threadIdx.x; t < L; t += gridDim.x * 256) {
    float* out = p.weights + b * p.weights_stride + t;
    const float before = p.prior != nullptr && t < L - M ? p.prior[b * p.weights_stride + t] : 0.f;
    float x = 0.f;
#pragma unroll 4
    for (int z = 0; z < splits; ++z) x += p.partial[(static_cast<int64_t>(z) * gridDim.y + b) * p.max_ctx + t];
    *out = p.prior != nullptr && t < L - M ? fmaf(p.decay, before, x) : x;
  }
}

template <int D, CacheType C, bool PAGED, bool RING>
WeightsKernelFn by_sub(int sub) {
  if (sub == 2) return attn_weights_kernel<D, C, PAGED, 2, RING>;
  if constexpr (C != CacheType::kF32) {
    if (sub == 4) return attn_weights_kernel<D, C, PAGED, 4, RING>;
    if (sub == 6) return attn_weights_kernel<D, C, PAGED, 6, RING>;
  }
  return nullptr;
}

template <int D, CacheType C>
WeightsForm form(bool paged, int sub, bool ring) {
  using Slot = typename QueryRing<D, C>::Slot;
  if (ring)
    return {paged ? by_sub<D, C, true, true>(sub) : by_sub<D, C, false, true>(sub),
            static_cast<int>(sizeof(Slot)) * QueryRing<D, C>::kSlots};
  return {paged ? by_sub<D, C, true, false>(sub) : by_sub<D, C, false, false>(sub), 0};
}

template <int D>
WeightsForm by_cache(CacheType cache, bool paged, int sub, bool ring) {
  if (cache == CacheType::kF32) return form<D, CacheType::kF32>(paged, sub, ring);
  if (cache == CacheType::kBf16) return form<D, CacheType::kBf16>(paged, sub, ring);
  return form<D, CacheType::kFp8>(paged, sub, ring);
}

}  // namespace

AddWeightsKernelFn add_weights_kernel_fn() { return add_weights_kernel; }

WeightsForm select_weights_kernel(int head_dim, CacheType cache, bool paged, int sub, bool ring) {
  if (head_dim == 128) return by_cache<128>(cache, paged, sub, ring);
  if (head_dim == 64) return by_cache<64>(cache, paged, sub, ring);
  return {nullptr, 0};
}

}  // namespace comem
