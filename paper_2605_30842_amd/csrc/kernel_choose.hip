// The largest entries of a row of scores, in the row's order (gfx950).
//
// Scores become 32-bit keys of the same order (NaN above all, and entries that
// always stay above NaN), and the K-th largest key is found some bits at a time
// from the top: a histogram of the digit over the keys that share the digits
// found so far, then the digit at which the counts from the top reach K. Keys
// above it stay, and as many of the equal ones as are still missing, the first
// ones. Every wave has a run of the row, so an entry's place is what the runs
// before hold plus a count of lane masks within its own: nothing depends on the
// order of atomics, which only count.
//
// Three forms, by the longest row: one wave, one workgroup, and three launches
// with a workgroup for each 8192 entries (which asks for a workspace).
// Histograms are kept 4 times, for a quarter of the lanes each: score digits
// cluster (a sign and an exponent have few values), and counts that meet in one
// word are added one after another.
#include <algorithm>
#include <type_traits>

#include "attn_common.h"
#include "evict.h"

namespace comem {
namespace {

typedef int s32x4 __attribute__((ext_vector_type(4)));
typedef int s32x2 __attribute__((ext_vector_type(2)));

constexpr uint32_t kForced = 0xffffffffu, kNaN = 0xfffffffeu;

// Keys order as the scores do; 0 is below every score's.
__device__ inline uint32_t key_of(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);  // -0 becomes 0
  return x == x ? (static_cast<int32_t>(u) < 0 ? ~u : u | 0x80000000u) : kNaN;
}

// One item of a call: its row's entries, how many of them stay, where they go.
template <bool BLOCKS>
struct Item {
  const float* scores;
  const int32_t* table;
  int32_t* out;
  float* kept;
  int n, count, first, last;

  // The first lane of the first workgroup of an item also writes its length.
  __device__ Item(const ChooseParams& p, int item, bool writes) : first(p.first), last(p.last) {
    int row;
    if constexpr (BLOCKS) {
      row = item / p.heads;
      const int L = min(max(uniform_i32(p.lens[row]), 0), p.max_len);
      const int page = 1 << p.page_shift;
      n = static_cast<int>((static_cast<uint32_t>(L) + page - 1) >> p.page_shift);
      count = min(n, p.budget);
      if (writes && item == row * p.heads) p.out_lens[row] = n == 0 ? 0 : (count - 1) * page + L - (n - 1) * page;
      table = p.block_table + static_cast<int64_t>(row) * p.max_pages;
      kept = nullptr;
    } else {
      row = p.rows == nullptr ? item : uniform_i32(p.rows[item]);
      n = row < 0 || row >= p.num_rows ? -1 : uniform_i32(p.lens[row]);
      if (n > p.max_len) n = -1;
      int budget = p.budget;
      if (p.budgets != nullptr) budget = min(max(uniform_i32(p.budgets[item]), p.first + p.last), p.budget);
      count = n < 0 ? -1 : min(n, budget);
      if (writes) {
        p.out_lens[item] = count;
        if (p.out_start != nullptr) p.out_start[item] = item * p.out_stride;
      }
      table = nullptr;
      kept = p.kept == nullptr ? nullptr : p.kept + item * p.out_stride;
    }
    scores = p.scores + static_cast<int64_t>(BLOCKS ? item : row) * p.scores_stride;
    out = p.out + item * p.out_stride;
  }
  __device__ float score_at(int i) const { return scores[min(i, n - 1)]; }
  // Of entry i, whose score is x.
  __device__ uint32_t key(int i, float x) const {
    const uint32_t k = i < first || i >= n - last ? kForced : key_of(x);
    return i < n ? k : 0;
  }
  __device__ void put(int at, int i) const { put(at, i, kept != nullptr ? scores[i] : 0.f); }
  // x: its score.
  __device__ void put(int at, int i, float x) const {
    if constexpr (BLOCKS) {
      out[at] = table[i];
    } else {
      out[at] = i;
      if (kept != nullptr) kept[at] = x;
    }
  }
};

// What stays: keys from `least` on, and the first `ties` keys that are `tie`.
struct Limit {
  uint32_t least, tie;
  int ties;
};

// The keys from `found` on stay, where the digits below it were not needed to
// part them; else those above it and `need` of the equal ones.
__device__ inline Limit limit_of(uint32_t found, int need, bool all) {
  return all ? Limit{found, 0, 0} : Limit{found + 1, found, need};
}

__device__ inline int lanes_before(uint64_t mask) {
  return static_cast<int>(__builtin_amdgcn_mbcnt_hi(static_cast<uint32_t>(mask >> 32),
                                                    __builtin_amdgcn_mbcnt_lo(static_cast<uint32_t>(mask), 0)));
}

// Entries of one step (64 side by side) before and among those that stay.
struct Places {
  int above = 0, equal = 0;
  // Where the lane's entry goes, -1: it does not stay. equals: it is one of
  // those of which the first `ties` stay.
  __device__ int next(bool stays, bool equals, int ties) {
    const uint64_t over = __builtin_amdgcn_ballot_w64(stays);
    int at = above + lanes_before(over);
    if (ties > 0) {
      const uint64_t same = __builtin_amdgcn_ballot_w64(equals);
      const int e = equal + lanes_before(same);
      at += min(e, ties);
      stays = stays || (equals && e < ties);
      equal += __builtin_popcountll(same);
    }
    above += __builtin_popcountll(over);
    return stays ? at : -1;
  }
};

// Sum of x over the lanes up to this one.
template <int CTRL, int ROWS>
__device__ inline int moved(int x) {
  return __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xf, false);
}
__device__ inline int upto_lane(int x) {
  x += moved<0x111, 0xf>(x);  // 1, 2, 4, 8 lanes before, within a row of 16
  x += moved<0x112, 0xf>(x);
  x += moved<0x114, 0xf>(x);
  x += moved<0x118, 0xf>(x);
  x += moved<0x142, 0xa>(x);  // the last of the row before; of the half before
  x += moved<0x143, 0xc>(x);
  return x;
}

__device__ inline int wave_sum(int x) { return __builtin_amdgcn_readlane(upto_lane(x), 63); }

// 4 bytes from each lane's address to consecutive places in LDS. (The caller
// waits for vector memory before it reads them.)
__device__ inline void load_to_lds(const void* from, uint32_t* to) {
  __builtin_amdgcn_global_load_lds(reinterpret_cast<const __attribute__((address_space(1))) uint32_t*>(
                                       reinterpret_cast<uintptr_t>(from)),
                                   (__attribute__((address_space(3))) uint32_t*)to, 4, 0, 0);
}

// Short rows (which ones, says `form` below): one wave each, which needs no
// barrier and holds at most kWaveEntries of them in LDS. 8 bits at a time, 4
// copies of the histogram, 4 bins a lane. The loops are rolled: the code is cold
// at every launch. 8 rows of 512 blocks 5.5 us, 512 rows of
// 128-1024 9.5 us; latency.
constexpr int kWaveEntries = 2048, kWaveCopies = 4;

__device__ inline void wave_lds_done() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup"); }

template <bool BLOCKS>
__global__ __launch_bounds__(64) void choose_wave_kernel(const ChooseParams p) {
  __shared__ s32x4 hist[256];  // the copies of a bin side by side
  __shared__ uint32_t keys[kWaveEntries];
  __shared__ uint32_t pages[BLOCKS ? kWaveEntries : 1];
  const int lane = threadIdx.x;
  const Item<BLOCKS> item(p, blockIdx.x, lane == 0);
  if (item.count <= 0) return;
  if (item.count == item.n) {
    for (int i = lane; i < item.n; i += 64) item.put(i, i);
    return;
  }
  // From memory straight into LDS, all of them in flight together; the first
  // pass makes keys of the scores.
#pragma unroll 1
  for (int g = 0; g < item.n; g += 64) {
    const int i = min(g + lane, item.n - 1);
    load_to_lds(item.scores + i, &keys[g]);
    if constexpr (BLOCKS) load_to_lds(item.table + i, &pages[g]);
  }
  wait_stores_done();
  uint32_t found = 0;
  int need = item.count;
  bool all = false;
#pragma unroll 1
  for (int shift = 24; shift >= 0 && !all; shift -= 8) {
#pragma unroll
    for (int i = 0; i < 4; ++i) hist[64 * i + lane] = s32x4{0, 0, 0, 0};
    wave_lds_done();
    const uint32_t mask = shift == 24 ? 0u : ~0u << (shift + 8);
    // Keys past the row are 0. In the first digit they are counted with -inf and scores below -1.7e38: that bin's size
    // then is no reason to stop (`all`), and the second digit parts them (0, and 0x7f or more).
#pragma unroll 1
    for (int g = 0; g < item.n; g += 256) {
      uint32_t k[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) k[e] = keys[g + 64 * e + lane];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (shift == 24) {
          k[e] = item.key(g + 64 * e + lane, __uint_as_float(k[e]));
          keys[g + 64 * e + lane] = k[e];
        }
        if ((k[e] & mask) == found)
          atomicAdd(reinterpret_cast<int*>(&hist[(k[e] >> shift) & 255u]) + (lane & (kWaveCopies - 1)), 1);
      }
    }
    wave_lds_done();
    // The lane's bins from the top down, and the entries of the lanes before it.
    int v[4], total = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const s32x4 x = hist[255 - 4 * lane - e];
      v[e] = x[0] + x[1] + x[2] + x[3];
      total += v[e];
    }
    int above = upto_lane(total) - total, digit = -1, at = 0, size = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (above < need && need <= above + v[e]) {
        digit = 255 - 4 * lane - e;
        at = above;
        size = v[e];
      }
      above += v[e];
    }
    const int from = __builtin_ctzll(__builtin_amdgcn_ballot_w64(digit >= 0));
    found |= static_cast<uint32_t>(__builtin_amdgcn_readlane(digit, from)) << shift;
    need -= __builtin_amdgcn_readlane(at, from);
    all = need == __builtin_amdgcn_readlane(size, from);
  }
  const Limit limit = limit_of(found, need, all);
  Places places;
#pragma unroll 1
  for (int g = 0; g < item.n; g += 256) {  // keys past the row are 0, which stays nowhere
    const int i0 = g + lane;
    uint32_t k[4];
    int32_t page[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      k[e] = keys[i0 + 64 * e];
      if constexpr (BLOCKS) page[e] = static_cast<int32_t>(pages[i0 + 64 * e]);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int at = places.next(k[e] >= limit.least, k[e] == limit.tie, limit.ties);
      if constexpr (BLOCKS) {
        if (at >= 0) item.out[at] = page[e];
      } else {
        if (at >= 0) item.put(at, i0 + 64 * e);
      }
    }
  }
}

// Sum of x[0 .. w - 1], for w < 16.
__device__ inline int waves_before(const int* x, int w, int lane) {
  const int upto = upto_lane(x[lane & 15]);
  return w > 0 ? __builtin_amdgcn_readlane(upto, w - 1) : 0;
}

// Longer rows (see `form`): a workgroup of 16 waves, each with a run of the row,
// which it reads three times, 8 groups of 64 entries a turn and the next turn's scores
// asked for ahead. The first time it counts the top 11 bits of the scores
// (4 copies of the histogram, so that lanes with one digit do not all wait for
// one word), which gives the digit that holds the limit. The second time it
// counts what lies above that digit and lists the scores that have it, a few
// percent of the row, each lane its own; the other digits, 11 and 10 bits,
// follow from the lists (where one overflows, from the row again). The third
// time it puts what stays. `gridDim.y` workgroups do the first two for a row,
// with the same results, and share the third.
//
// One compute unit's instructions bound it (24300 entries 12.1-12.8 us: launch 2.0,
// first count 2.7, its digit 1.4, the lists 3, the rest 3), so turns without
// NaN between the entries that always stay compare scores as floats, and only
// the others, and the lists, make keys. Rows held in LDS between the readings
// took 13.5: LDS holds fewer lists then, and the loads were hidden.
constexpr int kThreadsWide = 1024, kWavesWide = kThreadsWide / 64;
constexpr int kBins = 2048, kCopies = 4;  // of the histogram
constexpr int kTurn = 8;                  // groups of a turn
constexpr int kListed = 30;               // scores of a lane's list

// The least score whose key is k or more (a NaN, which no comparison holds for,
// where there is no such number).
__device__ inline float score_of(uint32_t k) {
  const uint32_t lowest = 0x007fffffu;  // the key of -inf
  k = max(k, lowest);
  return __uint_as_float(static_cast<int32_t>(k) < 0 ? k & 0x7fffffffu : ~k);
}

// Of a turn: numbers to choose among; entries that all stay; none; anything else.
enum class Turn { kPlain, kForced, kEmpty, kMixed };

// Orders LDS accesses alone: scores asked for ahead stay in flight.
__device__ inline void lds_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// A row as the kernels for long rows read it. Between `begin` and `end` it is
// chosen; what lies outside, and in the row, stays.
template <bool BLOCKS>
struct Row {
  const Item<BLOCKS>& item;
  int begin, end, lane;
  __device__ Row(const Item<BLOCKS>& it, int l)
      : item(it), begin(min(it.first, it.n)), end(max(it.n - it.last, begin)), lane(l) {}
  __device__ int missing() const { return item.count - begin - (item.n - end); }  // entries to choose
  __device__ bool chosen(int i) const { return i >= begin && i < end; }
  __device__ bool forced(int i) const { return i < begin || (i >= end && i < item.n); }
  __device__ uint32_t key(int i, float x) const { return forced(i) ? kForced : chosen(i) ? key_of(x) : 0; }

  __device__ void ask(int at, float (&x)[kTurn]) const {
    if (at + 64 * kTurn <= item.n) {
      const float* from = item.scores + at + lane;
#pragma unroll
      for (int e = 0; e < kTurn; ++e) x[e] = from[64 * e];
    } else {
#pragma unroll
      for (int e = 0; e < kTurn; ++e) x[e] = item.score_at(at + 64 * e + lane);
    }
  }
  __device__ Turn kind(int at, const float (&x)[kTurn]) const {
    const int to = at + 64 * kTurn;
    if (at >= item.n) return Turn::kEmpty;
    if (to > item.n) return Turn::kMixed;
    if (at >= end || to <= begin) return Turn::kForced;
    if (at < begin || to > end) return Turn::kMixed;
#pragma unroll
    for (int e = 0; e < kTurn; e += 2)
      if (__builtin_amdgcn_ballot_w64(__builtin_isunordered(x[e], x[e + 1])) != 0) return Turn::kMixed;
    return Turn::kPlain;
  }
  // f(first entry of the turn, its scores, its kind) for the turns from .. to - 1
  // of the run that starts at entry `run`. `next` holds turn `from`'s scores, and
  // at the end those of turn `after`.
  template <typename F>
  __device__ void for_turns(int run, int from, int to, int after, float (&next)[kTurn], F&& f) const {
    float x[kTurn];
#pragma unroll 1
    for (int j = from; j < to; ++j) {
      const int at = run + 64 * kTurn * j;
#pragma unroll
      for (int e = 0; e < kTurn; ++e) x[e] = next[e];
      ask(run + 64 * kTurn * (j + 1 < to ? j + 1 : after), next);
      f(at, x, kind(at, x));
    }
  }

  // f(PLAIN) for the kinds of turns apart (one body for both branches at every
  // entry: 24300 entries 14.0 us instead of 12.1).
  template <typename F>
  __device__ static void by_kind(Turn kind, F&& f) {
    if (kind == Turn::kPlain) {
      f(std::true_type());
    } else {
      f(std::false_type());
    }
  }

  // Counts a turn's first digits, by the bits as they are; -0 as 0, NaN as one of them.
  template <typename Add>
  __device__ void count(int at, const float (&x)[kTurn], Turn kind, Add&& add) const {
    if (kind == Turn::kForced || kind == Turn::kEmpty) return;
    by_kind(kind, [&](auto plain) {
#pragma unroll
      for (int e = 0; e < kTurn; ++e) {
        uint32_t u = __float_as_uint(x[e] + 0.f);
        if constexpr (plain) {
          add(static_cast<int>(u >> 21));
        } else {
          u = x[e] == x[e] ? u : 0x7fffffffu;
          if (chosen(at + 64 * e + lane)) add(static_cast<int>(u >> 21));
        }
      }
    });
  }
  // Adds the lane's entries of a turn above digit `top` to `above`, and lists
  // those that have it: store(listed, score, true) for the lane's `listed`-th
  // one, and with false for the others.
  template <typename Store>
  __device__ void list(int at, const float (&x)[kTurn], Turn kind, uint32_t top, float least, float over, int& above,
                       int& listed, Store&& store) const {
    if (kind == Turn::kForced) above += kTurn;
    if (kind == Turn::kForced || kind == Turn::kEmpty) return;
    by_kind(kind, [&](auto plain) {
#pragma unroll
      for (int e = 0; e < kTurn; ++e) {
        bool more, same;
        if constexpr (plain) {
          more = x[e] >= over;
          same = (x[e] >= least) != more;  // `over` is above `least`
        } else {
          const int i = at + 64 * e + lane;
          const uint32_t digit = key_of(x[e]) >> 21;
          more = forced(i) || (chosen(i) && digit > top);
          same = chosen(i) && digit == top;
        }
        store(listed, x[e], same);
        above += more ? 1 : 0;
        listed += same ? 1 : 0;
      }
    });
  }
  // Puts a turn's entries that stay.
  __device__ void put(int at, const float (&x)[kTurn], Turn kind, const Limit& limit, float least, float tie,
                      Places& places) const {
    if (kind == Turn::kEmpty) return;
    by_kind(kind, [&](auto plain) {
#pragma unroll
      for (int e = 0; e < kTurn; ++e) {
        const int i = at + 64 * e + lane;
        bool stays, equals;
        if constexpr (plain) {
          stays = x[e] >= least;
          equals = x[e] == tie;
        } else {
          const uint32_t k = key(i, x[e]);
          stays = k >= limit.least;
          equals = limit.ties > 0 && k == limit.tie;
        }
        const int to = places.next(stays, equals, limit.ties);
        if (to >= 0) item.put(to, i, x[e]);
      }
    });
  }
};

// Where the first digit's counts lie: digits in the order of the scores, bins by
// their bits.
__device__ inline int first_bin(int digit) { return digit >= kBins / 2 ? digit - kBins / 2 : kBins - 1 - digit; }

// The limit as the digits are found.
struct Search {
  uint32_t found = 0;  // the digits found so far
  int need;            // entries still missing among the keys that begin with them
  bool all;            // all of those stay
  __device__ explicit Search(int missing) : need(missing), all(missing <= 0) {}
  // One more digit: it holds the need-th entry from the top, `above` lie above it, `size` have it.
  __device__ void add(int digit, int above, int size, int shift) {
    if (all) {
      found = ~0u;  // only what always stays
      return;
    }
    found |= static_cast<uint32_t>(digit) << shift;
    need -= above;
    all = need == size;
  }
  __device__ Limit limit() const { return limit_of(found, need, all); }
  __device__ float tie() const { return all ? __builtin_nanf("") : score_of(found); }
};

// What a workgroup of 16 waves finds with.
struct Found {
  int wave_total[kWavesWide];
  int result[3];
};
// Adds the digit that holds the need-th entry from the top: thread tid has the
// counts v of the digits kBins - 1 - 2 tid and the one below. The barriers of
// two calls have one between them.
__device__ inline void find_digit(Search& search, int shift, const int (&v)[2], Found& f, int tid, int lane, int w) {
  const int upto = upto_lane(v[0] + v[1]);
  if (lane == 63) f.wave_total[w] = upto;
  if (tid == 0) f.result[0] = f.result[1] = f.result[2] = 0;
  lds_barrier();
  int before = upto - v[0] - v[1] + waves_before(f.wave_total, w, lane);
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    if (before < search.need && search.need <= before + v[e]) {
      f.result[0] = kBins - 1 - 2 * tid - e;
      f.result[1] = before;
      f.result[2] = v[e];
    }
    before += v[e];
  }
  lds_barrier();
  search.add(uniform_i32(f.result[0]), uniform_i32(f.result[1]), uniform_i32(f.result[2]), shift);
}

// The histogram: the copies of a bin side by side.
__device__ inline void count_one(s32x4* hist, int bin, int lane) {
  atomicAdd(reinterpret_cast<int*>(&hist[bin]) + (lane & (kCopies - 1)), 1);
}
__device__ inline int taken(s32x4* bin) {
  const s32x4 x = *bin;
  *bin = s32x4{0, 0, 0, 0};
  return x[0] + x[1] + x[2] + x[3];
}

template <bool BLOCKS>
__global__ __launch_bounds__(kThreadsWide) void choose_kernel(const ChooseParams p) {
  __shared__ s32x4 hist[kBins];
  __shared__ float list[kWavesWide][kListed + 1][64];  // (the last place: those past the end)
  __shared__ Found found;
  __shared__ int wave_above[kWavesWide], wave_equal[kWavesWide];
  __shared__ int too_long;
  const int tid = threadIdx.x, lane = tid & 63, w = uniform_i32(tid >> 6);
  const int part = blockIdx.y, parts = gridDim.y;
  const Item<BLOCKS> item(p, blockIdx.x, tid == 0 && part == 0);
  if (item.count <= 0) return;
  if (item.count == item.n) {
    for (int i = part * kThreadsWide + tid; i < item.n; i += parts * kThreadsWide) item.put(i, i);
    return;
  }
  const Row<BLOCKS> row(item, lane);
  const int turns = (item.n + kTurn * kThreadsWide - 1) / (kTurn * kThreadsWide);
  const int run = w * turns * kTurn * 64;  // the wave's first entry
  auto add = [&](int bin) { count_one(hist, bin, lane); };

  float next[kTurn];
  row.ask(run, next);
#pragma unroll
  for (int i = 0; i < kBins; i += kThreadsWide) hist[i + tid] = s32x4{0, 0, 0, 0};
  if (tid == 0) too_long = 0;
  lds_barrier();
  Search search(row.missing());
  bool overflow = false;
  int above = 0, listed = 0, own_above = 0, own_listed = 0;
  const int part_begin = turns * part / parts, part_end = turns * (part + 1) / parts;
#pragma unroll 1
  for (int shift = 21;;) {
    const int bits = shift == 0 ? 10 : 11;
    const uint32_t low = (1u << bits) - 1;
    auto add_key = [&](uint32_t k) {
      if ((k ^ search.found) >> (shift + bits) == 0) add(static_cast<int>((k >> shift) & low));
    };
    if (shift == 21) {
      row.for_turns(run, 0, turns, 0, next,
                    [&](int at, const float (&x)[kTurn], Turn kind) { row.count(at, x, kind, add); });
    } else if (overflow) {
      row.for_turns(run, 0, turns, 0, next, [&](int at, const float (&x)[kTurn], Turn) {
#pragma unroll
        for (int e = 0; e < kTurn; ++e)
          if (row.chosen(at + 64 * e + lane)) add_key(key_of(x[e]));
      });
    } else {
#pragma unroll 1
      for (int i = 0; i < listed; ++i) add_key(key_of(list[w][i][lane]));
    }
    lds_barrier();
    int v[2];  // of a thread's two digits, from the top down
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int digit = kBins - 1 - 2 * tid - e;
      v[e] = taken(&hist[shift != 21 ? digit : first_bin(digit)]);
    }
    find_digit(search, shift, v, found, tid, lane, w);
    if (shift == 21) {
      const uint32_t top = search.found >> 21;
      const float least = score_of(top << 21), over = top == kBins - 1 ? __builtin_nanf("") : score_of((top + 1) << 21);
      row.for_turns(run, 0, turns, 0, next, [&](int at, const float (&x)[kTurn], Turn kind) {
        if (at == run + 64 * kTurn * part_begin) {
          own_above = above;
          own_listed = listed;
        }
        row.list(at, x, kind, top, least, over, above, listed,
                 // One that has another digit is written over by the next.
                 [&](int place, float score, bool) { list[w][min(place, kListed)][lane] = score; });
      });
      if (listed > kListed) too_long = 1;
      lds_barrier();
      overflow = uniform_i32(too_long) != 0;
    }
    if (search.all || shift == 0) break;
    shift = shift == 21 ? 10 : 0;
  }
  const Limit limit = search.limit();
  const float least = score_of(limit.least), tie = search.tie();

  // What each lane of a run, and before this workgroup's part of it, has of what stays.
  int equal = 0, own_equal = 0;
  if (overflow) {
    above = own_above = 0;
    row.for_turns(run, 0, turns, 0, next, [&](int at, const float (&x)[kTurn], Turn) {
      if (at == run + 64 * kTurn * part_begin) {
        own_above = above;
        own_equal = equal;
      }
#pragma unroll
      for (int e = 0; e < kTurn; ++e) {
        const uint32_t k = row.key(at + 64 * e + lane, x[e]);
        above += k >= limit.least ? 1 : 0;
        equal += k == limit.tie ? 1 : 0;
      }
    });
  } else {
#pragma unroll 1
    for (int i = 0; i < listed; ++i) {
      const uint32_t k = key_of(list[w][i][lane]);
      const int more = k >= limit.least ? 1 : 0, same = k == limit.tie ? 1 : 0, mine = i < own_listed ? 1 : 0;
      above += more;
      equal += same;
      own_above += more & mine;
      own_equal += same & mine;
    }
  }
  const int all_above = wave_sum(above), all_equal = wave_sum(equal);
  if (lane == 0) {
    wave_above[w] = all_above;
    wave_equal[w] = all_equal;
  }
  lds_barrier();
  Places own{wave_sum(own_above) + waves_before(wave_above, w, lane), wave_sum(own_equal) + waves_before(wave_equal, w, lane)};
  if (part_begin != 0) row.ask(run + 64 * kTurn * part_begin, next);
  row.for_turns(run, part_begin, part_end, part_begin, next, [&](int at, const float (&x)[kTurn], Turn kind) {
    row.put(at, x, kind, limit, least, tie, own);
  });
}

// The longest rows, with a workspace: the same three readings as three
// launches, each with a workgroup for every chunk of a row, a turn for each of
// its waves. The first leaves the chunk's counts; in the second every workgroup
// adds up those of the row's chunks, finds the digit and lists its chunk's
// scores that have it; in the third every workgroup goes through the lists for
// the other digits and for what stays before its chunk, and puts the chunk's.
// Latency bounds them: 8 rows of 32768-131072, 4.1 MB in and out, 18.3 us in
// all (traced one launch at a time 3.8, 6.6 and 9.5), where one workgroup a row
// takes 34. (A workgroup of 4 waves for a chunk, each
// wave with four turns and a list of its own, took 31: too few instructions at
// once in the lists.)
static_assert(kChunkEntries == kThreadsWide * kTurn);

// An item's part of the workspace.
struct ChunkSpace {
  int32_t* counts;  // [chunks][kBins]
  int32_t* header;  // first digit, entries missing among those that have it, whether all of them stay
  int32_t* above;   // [chunks]: entries above the digit
  int32_t* listed;  // [chunks]
  float* lists;     // [chunks][kChunkEntries]
  __device__ ChunkSpace(const ChooseParams& p, int item, int chunks)
      : counts(reinterpret_cast<int32_t*>(p.workspace + item * choose_item_bytes(chunks))),
        header(counts + chunks * kBins),
        above(header + 4),
        listed(above + chunks),
        lists(reinterpret_cast<float*>(listed + chunks)) {}
};

__global__ __launch_bounds__(kThreadsWide) void chunk_count_kernel(const ChooseParams p) {
  __shared__ s32x4 hist[kBins];
  const int tid = threadIdx.x, lane = tid & 63, w = uniform_i32(tid >> 6), chunk = blockIdx.y;
  const Item<false> item(p, blockIdx.x, tid == 0 && chunk == 0);
  const int at = chunk * kChunkEntries + w * 64 * kTurn;
  if (item.count <= 0 || item.count == item.n || chunk * kChunkEntries >= item.n) return;
  const Row<false> row(item, lane);
  float x[kTurn];
  row.ask(at, x);
#pragma unroll
  for (int i = 0; i < kBins; i += kThreadsWide) hist[i + tid] = s32x4{0, 0, 0, 0};
  lds_barrier();
  row.count(at, x, row.kind(at, x), [&](int bin) { count_one(hist, bin, lane); });
  lds_barrier();
  int32_t* counts = ChunkSpace(p, blockIdx.x, gridDim.y).counts + chunk * kBins;
  *reinterpret_cast<s32x2*>(counts + 2 * tid) = s32x2{taken(&hist[2 * tid]), taken(&hist[2 * tid + 1])};
}

__global__ __launch_bounds__(kThreadsWide) void chunk_list_kernel(const ChooseParams p) {
  __shared__ Found found;
  __shared__ int wave_above[kWavesWide], wave_listed[kWavesWide];
  const int tid = threadIdx.x, lane = tid & 63, w = uniform_i32(tid >> 6), chunk = blockIdx.y;
  const Item<false> item(p, blockIdx.x, false);
  const int at = chunk * kChunkEntries + w * 64 * kTurn;
  if (item.count <= 0 || item.count == item.n || chunk * kChunkEntries >= item.n) return;
  const Row<false> row(item, lane);
  float x[kTurn];
  row.ask(at, x);
  const ChunkSpace space(p, blockIdx.x, gridDim.y);
  const int chunks = (item.n + kChunkEntries - 1) / kChunkEntries;
  // The thread's two digits, side by side, upwards above 0 and downwards below.
  const int digit = kBins - 1 - 2 * tid;
  const bool up = digit >= kBins / 2;
  const int32_t* from = space.counts + (up ? first_bin(digit - 1) : first_bin(digit));
  s32x2 sum = {0, 0};
#pragma unroll 8
  for (int i = 0; i < chunks; ++i) sum += *reinterpret_cast<const s32x2*>(from + i * kBins);
  const int v[2] = {up ? sum[1] : sum[0], up ? sum[0] : sum[1]};
  Search search(row.missing());
  find_digit(search, 21, v, found, tid, lane, w);
  const uint32_t top = search.found >> 21;
  const float least = score_of(top << 21), over = top == kBins - 1 ? __builtin_nanf("") : score_of((top + 1) << 21);
  const Turn kind = row.kind(at, x);
  int above = 0, listed = 0;
  row.list(at, x, kind, top, least, over, above, listed, [](int, float, bool) {});
  const int upto = upto_lane(listed), all_above = wave_sum(above);
  if (lane == 63) {
    wave_above[w] = all_above;
    wave_listed[w] = upto;
  }
  lds_barrier();
  if (tid == 0) {
    if (chunk == 0) {
      space.header[0] = static_cast<int32_t>(search.found);
      space.header[1] = search.need;
      space.header[2] = search.all ? 1 : 0;
    }
  }
  if (w == 0) {
    const int chunk_above = waves_before(wave_above, kWavesWide, lane);
    const int chunk_listed = waves_before(wave_listed, kWavesWide, lane);
    if (lane == 0) {
      space.above[chunk] = chunk_above;
      space.listed[chunk] = chunk_listed;
    }
  }
  listed = waves_before(wave_listed, w, lane) + upto - listed;
  float* list = space.lists + static_cast<int64_t>(chunk) * kChunkEntries;
  row.list(at, x, kind, top, least, over, above, listed, [&](int place, float score, bool has) {
    if (has) list[place] = score;
  });
}

__global__ __launch_bounds__(kThreadsWide) void chunk_put_kernel(const ChooseParams p) {
  __shared__ s32x4 hist[kBins];
  __shared__ Found found;
  __shared__ int listed_of[kMostChunks], above_of[kMostChunks], equal_of[kMostChunks];  // what stays, of each chunk
  __shared__ int wave_above[kWavesWide], wave_equal[kWavesWide];
  const int tid = threadIdx.x, lane = tid & 63, w = uniform_i32(tid >> 6), chunk = blockIdx.y;
  const Item<false> item(p, blockIdx.x, false);
  const int at = chunk * kChunkEntries + w * 64 * kTurn;
  if (item.count <= 0 || chunk * kChunkEntries >= item.n) return;
  if (item.count == item.n) {
    for (int i = chunk * kChunkEntries + tid; i < min(item.n, (chunk + 1) * kChunkEntries); i += kThreadsWide)
      item.put(i, i);
    return;
  }
  const Row<false> row(item, lane);
  float x[kTurn];
  row.ask(at, x);
  const ChunkSpace space(p, blockIdx.x, gridDim.y);
  const int chunks = (item.n + kChunkEntries - 1) / kChunkEntries;
  Search search(0);
  search.found = static_cast<uint32_t>(uniform_i32(space.header[0]));
  search.need = uniform_i32(space.header[1]);
  search.all = uniform_i32(space.header[2]) != 0;
#pragma unroll
  for (int i = 0; i < kBins; i += kThreadsWide) hist[i + tid] = s32x4{0, 0, 0, 0};
  if (tid < chunks) {
    listed_of[tid] = space.listed[tid];
    above_of[tid] = space.above[tid];
    equal_of[tid] = 0;
  }
  lds_barrier();
  // f(chunk, key or 0 past the end): a chunk's list is one wave's.
  auto for_lists = [&](auto&& f) {
#pragma unroll 1
    for (int c = w; c < chunks; c += kWavesWide) {
      const int n = uniform_i32(listed_of[c]);
      const float* list = space.lists + static_cast<int64_t>(c) * kChunkEntries;
#pragma unroll 1
      for (int i = lane; i - lane < n; i += 256) {
        float y[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = i + 64 * e < n ? list[i + 64 * e] : 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) f(c, i + 64 * e < n ? key_of(y[e]) : 0);
      }
    }
  };
#pragma unroll 1
  for (int shift = 10; !search.all; shift = 0) {
    const int bits = shift == 0 ? 10 : 11;
    for_lists([&](int, uint32_t k) {
      if (k != 0 && (k ^ search.found) >> (shift + bits) == 0)
        count_one(hist, static_cast<int>((k >> shift) & ((1u << bits) - 1)), lane);
    });
    lds_barrier();
    const int v[2] = {taken(&hist[kBins - 1 - 2 * tid]), taken(&hist[kBins - 2 - 2 * tid])};
    find_digit(search, shift, v, found, tid, lane, w);
    if (shift == 0) break;
  }
  const Limit limit = search.limit();
  const float least = score_of(limit.least), tie = search.tie();
  for_lists([&](int c, uint32_t k) {
    const uint64_t more = __builtin_amdgcn_ballot_w64(k >= limit.least);
    const uint64_t same = limit.ties > 0 ? __builtin_amdgcn_ballot_w64(k == limit.tie) : 0;
    if (lane == 0) {
      above_of[c] += __builtin_popcountll(more);
      equal_of[c] += __builtin_popcountll(same);
    }
  });
  // The wave's own turn, and what stays before it in the chunk and in the row.
  const Turn kind = row.kind(at, x);
  int above = 0, equal = 0;
  if (kind != Turn::kEmpty) {
#pragma unroll
    for (int e = 0; e < kTurn; ++e) {
      const uint32_t k = row.key(at + 64 * e + lane, x[e]);
      above += __builtin_popcountll(__builtin_amdgcn_ballot_w64(k >= limit.least));
      if (limit.ties > 0) equal += __builtin_popcountll(__builtin_amdgcn_ballot_w64(k == limit.tie));
    }
  }
  if (lane == 0) {
    wave_above[w] = above;
    wave_equal[w] = equal;
  }
  lds_barrier();
  Places own;
  own.above = waves_before(wave_above, w, lane) +
              wave_sum(lane < chunk ? above_of[lane] : 0);
  own.equal = waves_before(wave_equal, w, lane) +
              wave_sum(lane < chunk ? equal_of[lane] : 0);
  row.put(at, x, kind, limit, least, tie, own);
}

template <bool BLOCKS>
ChooseForm form(int64_t most, int64_t items, int cus) {
  // One wave, or one workgroup while there are compute units enough (us, 64 rows
  // of 1025 entries 8.7 / 9.8, 1200 9.8 / 9.9, 1536 11.3 / 9.8, 2048 12.7 / 10.0;
  // 256 of 2048 14.1 / 11.0; 300 of 2049 in workgroups 18.4, 512 of 2048 in waves 14.3).
  if (most <= 1280 || (most <= kWaveEntries && items > cus)) return {choose_wave_kernel<BLOCKS>, 64, 1};
  const int64_t parts = std::min<int64_t>(8, std::max<int64_t>(1, cus / items));
  return {choose_kernel<BLOCKS>, kThreadsWide, static_cast<int>(parts)};
}

}  // namespace

ChooseForm select_choose_kernel(bool blocks, int64_t most, int64_t items, int cus) {
  return blocks ? form<true>(most, items, cus) : form<false>(most, items, cus);
}

ChunkKernels select_chunk_kernels() {
  return {chunk_count_kernel, chunk_list_kernel, chunk_put_kernel, kThreadsWide};
}

}  // namespace comem
