// The pages of a paged KV cache: giving out, sharing, compacting, giving back
// (gfx950). Nothing here computes; the tables take launches and round trips,
// the copied tokens memory bandwidth.
//
// Which pages a call gives out depends on the state alone: the lowest free
// ones, to its items in order. With a pool of one chunk (8192 pages) one
// workgroup finds the items' needs, ranks the free pages and hands them on.
// With more, a launch before counts each chunk's free pages and a workgroup
// per chunk hands out its own: the counts before it give its first rank. (That
// launch also finds the items of compact and of forks of over 1024 pairs.)
// Fork and compact calls then edit the tables and move tokens in one more
// launch: an item's first workgroup the tables, the others the tokens. The
// counts of given-up pages go down only there, after every look for free ones.
//
// Measured. A launch that only edits tables is its round trips to memory:
// page_release 2.1 to 4.5 us, page_find 4.6 to 4.8, page_give 4.6 (reserve),
// 5.1 to 7.7 (fork, compact), 7.1 over five chunks. A release and two reserves
// of 64 rows over 40960 pages took 38.9 us where one workgroup looked at all of
// them, 22.6 with a workgroup per chunk; of 8 rows over one chunk 28.6 with a
// separate find, 19.9 without. The copies: fork, the last pages of 32 rows over
// 4 layers (40 MB read and written) 10.3 us; compact, one row to 5471 tokens
// (37 MB) 9.4 us, eight rows to 6800 over 4 layers (0.79 GB) 152 us, 5.2 TB/s,
// the rate of a large copy.
#include "kv_pages.h"

namespace comem {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

__device__ inline int32_t pages_for(int64_t tokens, int shift) {
  return static_cast<int32_t>((tokens + (int64_t{1} << shift) - 1) >> shift);
}

__device__ inline bool in_pool(const PageParams& p, int32_t page) { return page >= 0 && page < p.num_pages; }

template <int CTRL, int ROWS>
__device__ inline uint32_t dpp_add(uint32_t x) {
  return x + static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(x), CTRL, ROWS, 0xf, false));
}

// Inclusive sum over the lanes of a wave up to this one (within each row of
// 16, then the rows' last lanes on to the next rows).
__device__ inline uint32_t wave_scan(uint32_t x) {
  x = dpp_add<0x111, 0xf>(x);
  x = dpp_add<0x112, 0xf>(x);
  x = dpp_add<0x114, 0xf>(x);
  x = dpp_add<0x118, 0xf>(x);
  x = dpp_add<0x142, 0xa>(x);
  return dpp_add<0x143, 0xc>(x);
}

// Minimum over the wave, in its last lane.
template <int CTRL, int ROWS>
__device__ inline int dpp_min(int x) {
  const int y = __builtin_amdgcn_update_dpp(INT32_MAX, x, CTRL, ROWS, 0xf, false);
  return x < y ? x : y;
}

__device__ inline int wave_min(int x) {
  x = dpp_min<0x111, 0xf>(x);
  x = dpp_min<0x112, 0xf>(x);
  x = dpp_min<0x114, 0xf>(x);
  x = dpp_min<0x118, 0xf>(x);
  x = dpp_min<0x142, 0xa>(x);
  return dpp_min<0x143, 0xc>(x);
}

// Pages needed: sums of up to 2^31 each pass 32 bits, so they are summed in
// two parts of which no workgroup's sum does.
constexpr int kLowBits = 20;
struct NeedSums {
  uint32_t low[kPageThreads / 64], high[kPageThreads / 64];
};

// Sum of the workgroup's values before this thread's, and of all of them.
// `sums` is one of two buffers used in turn: a barrier stands between a
// buffer's reads and its next writes.
__device__ inline int64_t block_scan(int64_t x, NeedSums& sums, int64_t& total) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const uint32_t low = static_cast<uint32_t>(x) & ((1u << kLowBits) - 1), high = static_cast<uint32_t>(x >> kLowBits);
  const uint32_t lo = wave_scan(low), hi = wave_scan(high);
  if (lane == 63) {
    sums.low[w] = lo;
    sums.high[w] = hi;
  }
  __syncthreads();
  uint32_t lo_before = 0, hi_before = 0, lo_all = 0, hi_all = 0;
#pragma unroll
  for (int i = 0; i < kPageThreads / 64; ++i) {
    lo_before += i < w ? sums.low[i] : 0;
    hi_before += i < w ? sums.high[i] : 0;
    lo_all += sums.low[i];
    hi_all += sums.high[i];
  }
  total = (static_cast<int64_t>(hi_all) << kLowBits) + lo_all;
  return (static_cast<int64_t>(hi_before + hi - high) << kLowBits) + (lo_before + lo - low);
}

// A thread's reference counts of a chunk, and the wave's free pages as masks:
// bit l of mask k of a wave is page 64 (kMasks w' + k) + l of the chunk, w' the
// wave's place. (Two steps, so that the counts can be on their way early.)
constexpr int kMasks = kChunkPages / kPageThreads;
__device__ inline void load_counts(const PageParams& p, int chunk, int32_t (&x)[kMasks]) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int64_t c0 = static_cast<int64_t>(chunk) * kChunkPages + w * (64 * kMasks) + lane;
#pragma unroll
  for (int k = 0; k < kMasks; ++k) x[k] = c0 + 64 * k < p.num_pages ? p.refcounts[c0 + 64 * k] : 1;
}

// Returns the wave's count.
__device__ inline int free_masks(const int32_t (&x)[kMasks], uint64_t (&mask)[kMasks]) {
  int count = 0;
#pragma unroll
  for (int k = 0; k < kMasks; ++k) {
    mask[k] = __builtin_amdgcn_ballot_w64(x[k] == 0);
    count += __popcll(mask[k]);
  }
  return count;
}

struct Item {
  int row, grown, first, need;
};

__device__ inline Item read_item(const PageParams& p, int i) {
  return Item{p.items.row[i], p.items.grown[i], p.items.first[i], p.items.need[i]};
}

// Whether a list names x = list[i] at a place before i, for the workgroup's
// i = i0 + thread together: earlier entries pass through LDS.
__device__ inline bool named_before(const int32_t* list, int x, int i0, int n) {
  __shared__ int32_t names[kPageThreads];
  const int tid = threadIdx.x, i = i0 + tid;
  bool found = false;
  for (int j0 = 0; j0 <= i0; j0 += kPageThreads) {
    const int y = j0 == i0 ? x : list[j0 + tid];
    __syncthreads();
    names[tid] = y;
    __syncthreads();
    const int end = i >= n ? 0 : j0 == i0 ? tid : kPageThreads;
#pragma unroll 8
    for (int k = 0; k < end; ++k) found |= names[k] == x;
  }
  return found;
}

// Item i of a reserve or fork call, all of whose threads come here together
// with i = i0 + thread.
template <PageOp OP>
__device__ inline Item find_item(const PageParams& p, int i0) {
  const int i = i0 + static_cast<int>(threadIdx.x);
  Item item{-1, -1, 0, 0};
  if constexpr (OP == PageOp::kReserve) {
    if (i >= p.n) return Item{};
    const int64_t add = p.add_lens[i], len = p.ctx_lens[i];
    if (len >= 0 && add >= 0 && len + add <= p.max_ctx) {
      item.row = i;
      item.grown = static_cast<int>(len + add);
      item.first = pages_for(len, p.page_shift);
      item.need = pages_for(len + add, p.page_shift) - item.first;
    }
  } else {
    const int child = i < p.n ? p.children[i] : -1, from = i < p.n ? p.rows[i] : -1;
    const bool rows = from >= 0 && from < p.num_rows && child >= 0 && child < p.num_rows && child != from;
    // On their way while the list is looked through.
    const int64_t child_len = p.ctx_lens[rows ? child : 0], from_len = p.ctx_lens[rows ? from : 0];
    const bool again = named_before(p.children, child, i0, p.n);
    if (i >= p.n) return Item{};
    const bool taken = rows && !again && child_len == 0 && from_len >= 0 && from_len <= p.max_ctx;
    if (taken) {
      item.row = child;
      item.grown = static_cast<int>(from_len);
      item.first = static_cast<int>(from_len >> p.page_shift);
      item.need = pages_for(from_len, p.page_shift) - item.first;
    }
    p.items.from[i] = from;
    p.items.len[i] = taken ? static_cast<int32_t>(from_len) : -1;
  }
  p.items.row[i] = item.row;
  p.items.grown[i] = item.grown;
  p.items.first[i] = item.first;
  p.items.need[i] = item.need;
  return item;
}

// Item i of a compact call, by a whole workgroup: the first token that moves,
// and the row's entries, which are replaced later, while tokens are read
// through them.
__device__ inline void find_cut(const PageParams& p, int i) {
  __shared__ int first_moved;
  constexpr int kAtOnce = 4;
  const int r = p.rows[i];
  const int64_t n = p.keep_lens[i], start = p.keep_start[i];
  if (threadIdx.x == 0) first_moved = INT32_MAX;
  bool again = false;
  for (int j = threadIdx.x; j < i; j += kPageThreads) again |= p.rows[j] == r;
  again = __syncthreads_or(again) != 0;
  // The list, the row's length and its entries (as many as a row can have)
  // are asked for together: none waits for another.
  const bool listed = n >= 0 && n <= p.max_ctx && start >= 0 && start <= p.keep_total - n;
  const bool has_row = !again && r >= 0 && r < p.num_rows;
  const int32_t* entries = p.block_table + static_cast<int64_t>(has_row ? r : 0) * p.max_pages;
  int32_t* old = p.old + static_cast<int64_t>(i) * p.max_pages;
  const int64_t len = has_row ? p.ctx_lens[r] : -1;
  const int most = has_row ? pages_for(p.max_ctx, p.page_shift) : 0;
  const int kept = listed ? static_cast<int>(n) : 0;
  int moved = kept;
  const int tid = threadIdx.x;
  for (int64_t t0 = tid; t0 < (kept > most ? kept : most); t0 += kAtOnce * kPageThreads) {
    int32_t at[kAtOnce], page[kAtOnce];
#pragma unroll
    for (int a = 0; a < kAtOnce; ++a) {
      const int64_t t = t0 + a * kPageThreads;
      at[a] = t < moved ? p.keep[start + t] : 0;
      page[a] = t < most ? entries[t] : 0;
    }
#pragma unroll
    for (int a = 0; a < kAtOnce; ++a) {
      const int64_t t = t0 + a * kPageThreads;
      if (t < moved && at[a] != t) moved = static_cast<int>(t);
      if (t < most) old[t] = page[a];
    }
  }
  moved = wave_min(moved);
  if ((tid & 63) == 63) atomicMin(&first_moved, moved);
  const bool valid = has_row && listed && len >= 0 && len <= p.max_ctx && n <= len;
  __syncthreads();
  if (threadIdx.x == 0) {
    const int first = valid ? first_moved >> p.page_shift : 0;
    p.items.row[i] = valid ? r : -1;
    p.items.len[i] = static_cast<int32_t>(len);
    p.items.grown[i] = static_cast<int32_t>(n);
    p.items.first[i] = first;
    p.items.need[i] = valid ? pages_for(n, p.page_shift) - first : 0;
  }
}

template <PageOp OP>
__global__ __launch_bounds__(kPageThreads) void page_find(const PageParams p) {
  const int counted = p.chunks > 1 ? p.chunks : 0;
  if (static_cast<int>(blockIdx.x) < counted) {
    __shared__ int32_t waves[kPageThreads / 64];
    int32_t x[kMasks];
    uint64_t mask[kMasks];
    load_counts(p, blockIdx.x, x);
    const int count = free_masks(x, mask);
    if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = count;
    __syncthreads();
    if (threadIdx.x == 0) {
      int all = 0;
      for (int w = 0; w < kPageThreads / 64; ++w) all += waves[w];
      p.free_counts[blockIdx.x] = all;
    }
  } else if constexpr (OP == PageOp::kCompact) {
    find_cut(p, blockIdx.x - counted);
  } else {
    find_item<OP>(p, static_cast<int>(blockIdx.x - counted) * kPageThreads);
  }
}

// Hands the chunk's free pages to the items whose places fall to them: into
// the table (reserve) or the list of fresh pages (fork, compact).
template <PageOp OP, bool ALONE>
__global__ __launch_bounds__(kPageThreads) void page_give(const PageParams p) {
  constexpr int kWaves = kPageThreads / 64;
  __shared__ NeedSums sums[2];
  __shared__ int32_t wave_free[kWaves];
  __shared__ int64_t tile_base[kPageThreads];
  __shared__ int32_t tile_need[kPageThreads], tile_first[kPageThreads];
  __shared__ int32_t pages[kChunkPages];  // the chunk's free pages in order
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int chunk = ALONE ? 0 : blockIdx.x;
  int32_t counts[kMasks];
  load_counts(p, chunk, counts);
  // The first tile of items stays in registers: with up to 1024 items no
  // other is looked at.
  Item item{};
  if constexpr (ALONE) {
    item = find_item<OP>(p, 0);
  } else if (static_cast<int>(threadIdx.x) < p.n) {
    item = read_item(p, threadIdx.x);
  }
  uint64_t mask[kMasks];
  const int mine = free_masks(counts, mask);
  if (lane == 0) wave_free[w] = mine;
  int64_t need_all, tile;
  int64_t base = block_scan(item.need, sums[0], need_all);
  tile = need_all;
  int place = 0, own = 0;  // the wave's place among the chunk's free pages, and their number
#pragma unroll
  for (int i = 0; i < kWaves; ++i) {
    place += i < w ? wave_free[i] : 0;
    own += wave_free[i];
  }
  if (p.n > kPageThreads) {
    int64_t more = 0, all;
    for (int i0 = kPageThreads; i0 < p.n; i0 += kPageThreads) {
      const int i = i0 + static_cast<int>(threadIdx.x);
      if constexpr (ALONE) {
        more += find_item<OP>(p, i0).need;
      } else if (i < p.n) {
        more += p.items.need[i];
      }
    }
    block_scan(more, sums[1], all);
    need_all += all;
    __syncthreads();
  }
  // Free pages of the chunks before this one and of all.
  int64_t before = 0, free_all = own;
  if (!ALONE && p.chunks > 1) {
    int64_t f = 0, b = 0;
    for (int c = threadIdx.x; c < p.chunks; c += kPageThreads) {
      f += p.free_counts[c];
      b += c < chunk ? p.free_counts[c] : 0;
    }
    block_scan(b, sums[1], before);
    block_scan(f, sums[0], free_all);
  }
  const int64_t missing = need_all > free_all ? need_all - free_all : 0;
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    *p.granted = missing == 0 ? 1 : 0;
    *p.missing = static_cast<int32_t>(missing < INT32_MAX ? missing : INT32_MAX);
  }
  if (missing != 0) {
    if constexpr (OP == PageOp::kReserve) {
      if (blockIdx.x == 0 && p.given != nullptr)
        for (int i = threadIdx.x; i < p.n; i += kPageThreads) p.given[i] = 0;
    }
    return;
  }

#pragma unroll
  for (int k = 0; k < kMasks; ++k) {
    if ((mask[k] >> lane) & 1) {
      const int64_t page = static_cast<int64_t>(chunk) * kChunkPages + (w * kMasks + k) * 64 + lane;
      pages[place + __popcll(mask[k] & ((uint64_t{1} << lane) - 1))] = static_cast<int32_t>(page);
    }
    place += __popcll(mask[k]);
  }
  const int64_t end = before + own < need_all ? before + own : need_all;  // places [before, end) are this chunk's
  if constexpr (OP != PageOp::kReserve) {
    __syncthreads();
    for (int64_t r = before + static_cast<int64_t>(threadIdx.x); r < end; r += kPageThreads) p.fresh[r] = pages[r - before];
    if (blockIdx.x != 0) return;
  }
  // Items in tiles of 1024. Reserve: each wave fills the entries of its items.
  int64_t tile_start = 0;
  int turn = 1;
  for (int i0 = 0;;) {
    const int i = i0 + static_cast<int>(threadIdx.x);
    if constexpr (OP == PageOp::kReserve) {
      tile_base[threadIdx.x] = base;
      tile_need[threadIdx.x] = item.need;
      tile_first[threadIdx.x] = item.first;
      if (blockIdx.x == 0 && i < p.n) {
        if (item.row >= 0) p.ctx_lens[i] = item.grown;
        if (p.given != nullptr) p.given[i] = item.row >= 0 ? p.add_lens[i] : 0;
      }
      __syncthreads();
      for (int k = w; k < kPageThreads && i0 + k < p.n; k += kWaves) {
        const int64_t b = tile_base[k];
        const int64_t lo = b > before ? b : before, hi = b + tile_need[k] < end ? b + tile_need[k] : end;
        if (lo >= hi) continue;
        int32_t* entries = p.block_table + static_cast<int64_t>(i0 + k) * p.max_pages + tile_first[k];
        for (int64_t r = lo + lane; r < hi; r += 64) {
          const int32_t page = pages[r - before];
          entries[r - b] = page;
          p.refcounts[page] = 1;
        }
      }
    } else if (i < p.n) {
      p.items.base[i] = static_cast<int32_t>(base);
    }
    i0 += kPageThreads;
    tile_start += tile;
    // Of the other chunks' workgroups, those whose places are filled stop.
    if (i0 >= p.n || (blockIdx.x != 0 && tile_start >= end)) return;
    __syncthreads();
    const int next = i0 + static_cast<int>(threadIdx.x);
    item = next < p.n ? read_item(p, next) : Item{};
    base = tile_start + block_scan(item.need, sums[turn], tile);
    turn ^= 1;
  }
}

template <PageOp OP>
__device__ inline void edit_table(const PageParams& p, int i, int row) {
  int32_t* entries = p.block_table + static_cast<int64_t>(row) * p.max_pages;
  const int len = p.items.len[i], grown = p.items.grown[i], first = p.items.first[i], need = p.items.need[i];
  const int32_t* fresh = p.fresh + p.items.base[i];
  if constexpr (OP == PageOp::kFork) {
    const int32_t* from = p.block_table + static_cast<int64_t>(p.items.from[i]) * p.max_pages;
    for (int e = threadIdx.x; e < first; e += kApplyThreads) {
      const int32_t page = from[e];
      entries[e] = page;
      if (in_pool(p, page)) atomicAdd(p.refcounts + page, 1);
    }
  }
  if constexpr (OP == PageOp::kCompact) {
    const int32_t* old = p.old + static_cast<int64_t>(i) * p.max_pages;
    const int held = pages_for(len, p.page_shift);
    for (int e = first + static_cast<int>(threadIdx.x); e < held; e += kApplyThreads) {
      if (in_pool(p, old[e])) atomicSub(p.refcounts + old[e], 1);
      if (e >= first + need) entries[e] = -1;
    }
  }
  for (int e = threadIdx.x; e < need; e += kApplyThreads) {
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

// STREAM: past the caches.
template <bool STREAM>
__device__ inline u32x4 get16(const char* p) {
  if constexpr (STREAM) return __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p));
  return *reinterpret_cast<const u32x4*>(p);
}
template <bool STREAM>
__device__ inline void put16(char* p, u32x4 x) {
  if constexpr (STREAM) {
    __builtin_nontemporal_store(x, reinterpret_cast<u32x4*>(p));
  } else {
    *reinterpret_cast<u32x4*>(p) = x;
  }
}

// Tokens first << page_shift .. grown - 1 of item i to their fresh pages, K
// and V of every layer. A wave takes kMoveTokens tokens of a layer: lane l
// finds token l's rows, then the wave copies 4 tokens' pieces at a time.
template <PageOp OP, bool STREAM>
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
  const int waves = kApplyThreads / 64;
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
          k[a] = get16<STREAM>(p.k + s[a] + piece);
          v[a] = get16<STREAM>(p.v + s[a] + piece);
        }
#pragma unroll
        for (int a = 0; a < kAtOnce; ++a) {
          if (k0 + a < count) {
            put16<STREAM>(p.k + d[a] + piece, k[a]);
            put16<STREAM>(p.v + d[a] + piece, v[a]);
          }
        }
      }
    }
  }
}

template <PageOp OP, bool STREAM>
__global__ __launch_bounds__(kApplyThreads) void page_apply(const PageParams p) {
  const int i = blockIdx.y;
  const int row = p.items.row[i];
  if (*p.granted == 0 || row < 0) return;
  if (blockIdx.x == 0) {
    edit_table<OP>(p, i, row);
  } else {
    move_tokens<OP, STREAM>(p, i, blockIdx.x - 1, gridDim.x - 1);
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

PageKernelFn select_page_find_kernel(PageOp op) {
  if (op == PageOp::kReserve) return page_find<PageOp::kReserve>;
  return op == PageOp::kFork ? page_find<PageOp::kFork> : page_find<PageOp::kCompact>;
}

PageKernelFn select_page_give_kernel(PageOp op, bool alone) {
  if (op == PageOp::kReserve) return alone ? page_give<PageOp::kReserve, true> : page_give<PageOp::kReserve, false>;
  if (op == PageOp::kFork) return alone ? page_give<PageOp::kFork, true> : page_give<PageOp::kFork, false>;
  return page_give<PageOp::kCompact, false>;
}

PageKernelFn select_page_apply_kernel(PageOp op, bool stream) {
  if (op == PageOp::kFork) return page_apply<PageOp::kFork, false>;
  return stream ? page_apply<PageOp::kCompact, true> : page_apply<PageOp::kCompact, false>;
}

PageKernelFn page_release_kernel() { return page_release; }

}  // namespace comem
