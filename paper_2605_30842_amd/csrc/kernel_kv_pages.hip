// The pages of a paged KV cache: giving out, sharing, compacting, giving back
// (gfx950). Nothing here computes; the tables take launches and round trips,
// the copied tokens memory bandwidth.
//
// A call that needs fresh pages runs in two launches. In the first, one
// workgroup finds what every item needs, adds it up in order and lists the
// lowest free pages, so that the result depends on the state alone. In the
// second, each item's first workgroup edits its table row and the counts, and
// the others move tokens. A compact call has a launch before these, a
// workgroup an item, that looks for the first token to move and copies the
// row's entries, which the second launch reads while it replaces them.
#include "kv_pages.h"

namespace comem {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

__device__ inline int32_t pages_for(int64_t tokens, int shift) {
  return static_cast<int32_t>((tokens + (int64_t{1} << shift) - 1) >> shift);
}

__device__ inline bool in_pool(const PageParams& p, int32_t page) { return page >= 0 && page < p.num_pages; }

// Inclusive sum over the lanes of a wave up to this one.
__device__ inline int64_t wave_scan(int64_t x, int lane) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int64_t y = __shfl_up(x, d);
    if (lane >= d) x += y;
  }
  return x;
}

__device__ inline int wave_scan(int x, int lane) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int y = __shfl_up(x, d);
    if (lane >= d) x += y;
  }
  return x;
}

// Sum of the workgroup's values before this thread's, and of all of them.
// `sums` is one of two buffers used in turn: a barrier stands between a
// buffer's reads and its next writes.
template <typename T>
__device__ inline T block_scan(T x, T* sums, T& total) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const T upto = wave_scan(x, lane);
  if (lane == 63) sums[w] = upto;
  __syncthreads();
  T before = 0, all = 0;
#pragma unroll
  for (int i = 0; i < kTakeThreads / 64; ++i) {
    const T s = sums[i];
    before += i < w ? s : 0;
    all += s;
  }
  total = all;
  return before + upto - x;
}

__global__ __launch_bounds__(kPageThreads) void page_scan(const PageParams p) {
  __shared__ int first_moved;
  const int i = blockIdx.x;
  const int r = p.rows[i];
  const int64_t n = p.keep_lens[i], start = p.keep_start[i];
  int64_t len = -1;
  if (r >= 0 && r < p.num_rows) len = p.ctx_lens[r];
  const bool valid = len >= 0 && len <= p.max_ctx && n >= 0 && n <= len && start >= 0 && start <= p.keep_total - n;
  if (threadIdx.x == 0) first_moved = static_cast<int>(valid ? n : 0);
  __syncthreads();
  if (!valid) {
    if (threadIdx.x == 0) {
      p.items.row[i] = -1;
      p.items.need[i] = 0;
    }
    return;
  }
  int moved = static_cast<int>(n);
  for (int t = threadIdx.x; t < n; t += kPageThreads) {
    if (p.keep[start + t] != t) {
      moved = t;
      break;
    }
  }
  atomicMin(&first_moved, moved);
  const int held = pages_for(len, p.page_shift);
  const int32_t* entries = p.block_table + static_cast<int64_t>(r) * p.max_pages;
  int32_t* old = p.old + static_cast<int64_t>(i) * p.max_pages;
  for (int e = threadIdx.x; e < held; e += kPageThreads) old[e] = entries[e];
  __syncthreads();
  if (threadIdx.x == 0) {
    const int first = first_moved >> p.page_shift;
    p.items.row[i] = r;
    p.items.len[i] = static_cast<int32_t>(len);
    p.items.grown[i] = static_cast<int32_t>(n);
    p.items.first[i] = first;
    p.items.need[i] = pages_for(n, p.page_shift) - first;
  }
}

// What item i of a call needs.
template <PageOp OP>
__device__ inline int find_item(const PageParams& p, int i) {
  if constexpr (OP == PageOp::kCompact) return p.items.need[i];
  int row = -1, from = -1, first = 0, need = 0;
  int64_t len = -1, grown = -1;
  if constexpr (OP == PageOp::kReserve) {
    const int64_t add = p.add_lens[i];
    len = p.ctx_lens[i];
    grown = len + add;
    if (len >= 0 && add >= 0 && grown <= p.max_ctx) {
      row = i;
      first = pages_for(len, p.page_shift);
      need = pages_for(grown, p.page_shift) - first;
    }
  } else {
    const int child = p.children[i];
    from = p.rows[i];
    if (from >= 0 && from < p.num_rows && child >= 0 && child < p.num_rows && child != from && p.ctx_lens[child] == 0)
      len = p.ctx_lens[from];
    if (len >= 0 && len <= p.max_ctx) {
      row = child;
      grown = len;
      first = static_cast<int>(len >> p.page_shift);
      need = pages_for(len, p.page_shift) - first;
    }
  }
  p.items.row[i] = row;
  p.items.from[i] = from;
  p.items.len[i] = static_cast<int32_t>(len);
  p.items.grown[i] = static_cast<int32_t>(grown);
  p.items.first[i] = first;
  p.items.need[i] = need;
  return need;
}

// Gives out the lowest free pages: items' needs summed in order, then the
// counts looked through from page 0 until there are enough zeros. A thread
// takes 16 neighbouring counts a step.
template <PageOp OP>
__global__ __launch_bounds__(kTakeThreads) void page_take(const PageParams p) {
  constexpr int kCounts = 16;
  constexpr int kStep = kCounts * kTakeThreads;
  __shared__ int64_t need_sums[2][kTakeThreads / 64];
  __shared__ int free_sums[2][kTakeThreads / 64];
  int64_t need_all = 0;
  int turn = 0;
  for (int i0 = 0; i0 < p.n; i0 += kTakeThreads, turn ^= 1) {
    const int i = i0 + static_cast<int>(threadIdx.x);
    const int64_t need = i < p.n ? find_item<OP>(p, i) : 0;
    int64_t total;
    const int64_t base = need_all + block_scan<int64_t>(need, need_sums[turn], total);
    // Past 2^31 the call has no pages and the base is not used.
    if (i < p.n) p.items.base[i] = static_cast<int32_t>(base);
    need_all += total;
  }
  int64_t found = 0;
  turn = 0;
  for (int64_t c0 = 0; c0 < p.num_pages && found < need_all; c0 += kStep, turn ^= 1) {
    const int64_t c = c0 + kCounts * static_cast<int64_t>(threadIdx.x);
    uint32_t zeros = 0;
    if (c + kCounts <= p.num_pages) {
      const int4* counts = reinterpret_cast<const int4*>(p.refcounts + c);
#pragma unroll
      for (int k = 0; k < kCounts / 4; ++k) {
        const int4 x = counts[k];
        zeros |= ((x.x == 0 ? 1u : 0u) | (x.y == 0 ? 2u : 0u) | (x.z == 0 ? 4u : 0u) | (x.w == 0 ? 8u : 0u)) << (4 * k);
      }
    } else {
      for (int k = 0; k < kCounts && c + k < p.num_pages; ++k) zeros |= (p.refcounts[c + k] == 0 ? 1u : 0u) << k;
    }
    int total;
    int64_t rank = found + block_scan<int>(__popc(zeros), free_sums[turn], total);
    while (zeros != 0 && rank < need_all) {
      const int k = __ffs(zeros) - 1;
      zeros &= zeros - 1;
      p.fresh[rank++] = static_cast<int32_t>(c + k);
    }
    found += total;
  }
  if (threadIdx.x == 0) {
    const int64_t missing = need_all > found ? need_all - found : 0;
    *p.granted = missing == 0 ? 1 : 0;
    *p.missing = static_cast<int32_t>(missing < INT32_MAX ? missing : INT32_MAX);
  }
}

template <PageOp OP>
__device__ inline void edit_table(const PageParams& p, int i, int row) {
  int32_t* entries = p.block_table + static_cast<int64_t>(row) * p.max_pages;
  const int len = p.items.len[i], grown = p.items.grown[i], first = p.items.first[i], need = p.items.need[i];
  const int32_t* fresh = p.fresh + p.items.base[i];
  if constexpr (OP == PageOp::kFork) {
    const int32_t* from = p.block_table + static_cast<int64_t>(p.items.from[i]) * p.max_pages;
    for (int e = threadIdx.x; e < first; e += kPageThreads) {
      const int32_t page = from[e];
      entries[e] = page;
      if (in_pool(p, page)) atomicAdd(p.refcounts + page, 1);
    }
  }
  if constexpr (OP == PageOp::kCompact) {
    const int32_t* old = p.old + static_cast<int64_t>(i) * p.max_pages;
    const int held = pages_for(len, p.page_shift);
    for (int e = first + static_cast<int>(threadIdx.x); e < held; e += kPageThreads) {
      if (in_pool(p, old[e])) atomicSub(p.refcounts + old[e], 1);
      if (e >= first + need) entries[e] = -1;
    }
  }
  for (int e = threadIdx.x; e < need; e += kPageThreads) {
    entries[first + e] = fresh[e];
    p.refcounts[fresh[e]] = 1;
  }
  if (threadIdx.x == 0) p.ctx_lens[row] = grown;
}

// The value of a lane (the same for the whole wave).
__device__ inline int64_t of_lane(int64_t x, int lane) {
  const uint32_t lo = __builtin_amdgcn_readlane(static_cast<uint32_t>(x), lane);
  const uint32_t hi = __builtin_amdgcn_readlane(static_cast<uint32_t>(static_cast<uint64_t>(x) >> 32), lane);
  return static_cast<int64_t>((static_cast<uint64_t>(hi) << 32) | lo);
}

// Tokens first << page_shift .. grown - 1 of item i to their fresh pages, K
// and V of every layer. A wave takes kMoveTokens tokens of a layer: lane l
// finds token l's rows, then the wave copies 4 tokens' pieces at a time.
template <PageOp OP>
__device__ inline void move_tokens(const PageParams& p, int i, int mover, int movers) {
  constexpr int kAtOnce = 4;
  const int lane = threadIdx.x & 63;
  const int first = p.items.first[i], grown = p.items.grown[i], len = p.items.len[i];
  const int t0 = first << p.page_shift;
  if (grown <= t0) return;
  const int groups = (grown - t0 + kMoveTokens - 1) / kMoveTokens;
  const int64_t units = static_cast<int64_t>(groups) * p.num_layers;
  const int mask = (1 << p.page_shift) - 1;
  const int32_t* fresh = p.fresh + p.items.base[i];
  const int32_t* pages = OP == PageOp::kFork ? p.block_table + static_cast<int64_t>(p.items.from[i]) * p.max_pages
                                             : p.old + static_cast<int64_t>(i) * p.max_pages;
  const int64_t start = OP == PageOp::kCompact ? p.keep_start[i] : 0;
  const int pieces = p.num_kv_heads << p.piece_shift;
  const int waves = kPageThreads / 64;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  for (int64_t u = static_cast<int64_t>(mover) * waves + wave; u < units; u += static_cast<int64_t>(movers) * waves) {
    const int layer = static_cast<int>(u / groups);
    const int g0 = t0 + static_cast<int>(u - static_cast<int64_t>(layer) * groups) * kMoveTokens;
    const int count = min(kMoveTokens, grown - g0);
    const int t = g0 + min(lane, count - 1);
    int from = t;
    if constexpr (OP == PageOp::kCompact) from = min(max(p.keep[start + t], 0), len - 1);
    int32_t page = pages[from >> p.page_shift];
    page = in_pool(p, page) ? page : 0;
    const int64_t at = layer * p.stride_layer;
    const int64_t src = at + page * p.stride_page + (from & mask) * p.stride_token;
    const int64_t dst = at + fresh[(t >> p.page_shift) - first] * p.stride_page + (t & mask) * p.stride_token;
    for (int k0 = 0; k0 < count; k0 += kAtOnce) {
      int64_t s[kAtOnce], d[kAtOnce];  // past the last token: that one again, not stored
#pragma unroll
      for (int a = 0; a < kAtOnce; ++a) {
        s[a] = of_lane(src, min(k0 + a, count - 1));
        d[a] = of_lane(dst, min(k0 + a, count - 1));
      }
      for (int c = lane; c < pieces; c += 64) {
        const int64_t piece = (c >> p.piece_shift) * p.stride_head + (c & ((1 << p.piece_shift) - 1)) * 16;
        u32x4 k[kAtOnce], v[kAtOnce];
#pragma unroll
        for (int a = 0; a < kAtOnce; ++a) {
          k[a] = *reinterpret_cast<const u32x4*>(p.k + s[a] + piece);
          v[a] = *reinterpret_cast<const u32x4*>(p.v + s[a] + piece);
        }
#pragma unroll
        for (int a = 0; a < kAtOnce; ++a) {
          if (k0 + a < count) {
            *reinterpret_cast<u32x4*>(p.k + d[a] + piece) = k[a];
            *reinterpret_cast<u32x4*>(p.v + d[a] + piece) = v[a];
          }
        }
      }
    }
  }
}

template <PageOp OP>
__global__ __launch_bounds__(kPageThreads) void page_apply(const PageParams p) {
  const int i = blockIdx.y;
  const int row = p.items.row[i];
  if (*p.granted == 0 || row < 0) return;
  if (blockIdx.x == 0) {
    edit_table<OP>(p, i, row);
  } else if constexpr (OP != PageOp::kReserve) {
    move_tokens<OP>(p, i, blockIdx.x - 1, gridDim.x - 1);
  }
}

// Entries are exchanged, so that of a row named twice each is counted once.
__global__ __launch_bounds__(kPageThreads) void page_release(const PageParams p) {
  const int r = p.rows[blockIdx.x];
  if (r < 0 || r >= p.num_rows) return;
  const int64_t len = p.ctx_lens[r];
  if (len <= 0 || len > p.max_ctx) return;
  int32_t* entries = p.block_table + static_cast<int64_t>(r) * p.max_pages;
  const int held = pages_for(len, p.page_shift);
  for (int e = threadIdx.x; e < held; e += kPageThreads) {
    const int32_t page = atomicExch(entries + e, -1);
    if (in_pool(p, page)) atomicSub(p.refcounts + page, 1);
  }
  __syncthreads();
  if (threadIdx.x == 0) p.ctx_lens[r] = 0;
}

}  // namespace

PageKernelFn page_scan_kernel() { return page_scan; }

PageKernelFn select_page_take_kernel(PageOp op) {
  if (op == PageOp::kReserve) return page_take<PageOp::kReserve>;
  return op == PageOp::kFork ? page_take<PageOp::kFork> : page_take<PageOp::kCompact>;
}

PageKernelFn select_page_apply_kernel(PageOp op) {
  if (op == PageOp::kReserve) return page_apply<PageOp::kReserve>;
  return op == PageOp::kFork ? page_apply<PageOp::kFork> : page_apply<PageOp::kCompact>;
}

PageKernelFn page_release_kernel() { return page_release; }

}  // namespace comem
