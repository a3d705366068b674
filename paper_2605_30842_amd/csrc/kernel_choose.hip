// The largest entries of a row of scores, in the row's order (gfx950).
//
// One workgroup per row. Scores become 32-bit keys of the same order (NaN above
// all, and entries that always stay above NaN), and the K-th largest key is
// found 8 bits at a time from the top: a histogram of the digit over the keys
// that share the digits found so far, then the digit at which the counts from
// the top reach K. Keys above it stay, and as many of the equal ones as are
// still missing, the first ones. Every wave has a run of the row, so an entry's
// place is what the runs before hold plus a count of lane masks within its own.
//
// The histogram is kept 32 times, one copy for each of 32 lanes: score digits
// cluster (a sign and an exponent have few values), and counts that meet in one
// word are added one after another.
#include "attn_common.h"
#include "evict.h"

namespace comem {
namespace {

constexpr uint32_t kForced = 0xffffffffu, kNaN = 0xfffffffeu;
constexpr int kCopies = 32, kBins = 256;

// Keys order as the scores do; 0 is below every score's.
__device__ inline uint32_t key_of(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);  // -0 becomes 0
  return x == x ? (static_cast<int32_t>(u) < 0 ? ~u : u | 0x80000000u) : kNaN;
}

// The digit that holds the need-th entry from the top, the entries above it and
// those of it; every wave looks for it by itself.
struct Digit {
  int digit, above, count;
};
__device__ inline Digit find_digit(const int* sums, int need, int lane) {
  int v[4], total = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    v[e] = sums[kBins - 1 - 4 * lane - e];
    total += v[e];
  }
  int upto = total;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int x = __shfl_up(upto, o);
    if (lane >= o) upto += x;
  }
  int above = upto - total, digit = -1, count = 0, at = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if (above < need && need <= above + v[e]) {
      digit = kBins - 1 - 4 * lane - e;
      at = above;
      count = v[e];
    }
    above += v[e];
  }
  const int from = __builtin_ctzll(__builtin_amdgcn_ballot_w64(digit >= 0));
  return {__builtin_amdgcn_readlane(digit, from), __builtin_amdgcn_readlane(at, from),
          __builtin_amdgcn_readlane(count, from)};
}

// REGS: entries of a lane that are kept in registers; those past them are read again.
template <bool BLOCKS, int THREADS, int REGS>
__global__ __launch_bounds__(THREADS) void choose_kernel(const ChooseParams p) {
  constexpr int kWavesHere = THREADS / 64;
  __shared__ int hist[kBins * kCopies];
  __shared__ int sums[kBins];
  __shared__ int wave_above[kWavesHere], wave_equal[kWavesHere];
  const int tid = threadIdx.x, lane = tid & 63, w = uniform_i32(tid >> 6);
  const int item = blockIdx.x;
  int n, count, row;
  if constexpr (BLOCKS) {
    row = item / p.heads;
    const int L = min(max(uniform_i32(p.lens[row]), 0), p.max_len);
    const int page = 1 << p.page_shift;
    n = static_cast<int>((static_cast<uint32_t>(L) + page - 1) >> p.page_shift);
    count = min(n, p.budget);
    if (item - row * p.heads == 0 && tid == 0)
      p.out_lens[row] = n == 0 ? 0 : (count - 1) * page + L - (n - 1) * page;
  } else {
    row = p.rows == nullptr ? item : uniform_i32(p.rows[item]);
    n = row < 0 || row >= p.num_rows ? -1 : uniform_i32(p.lens[row]);
    if (n > p.max_len) n = -1;
    int budget = p.budget;
    if (p.budgets != nullptr) budget = min(max(uniform_i32(p.budgets[item]), p.first + p.last), p.budget);
    count = n < 0 ? -1 : min(n, budget);
    if (tid == 0) {
      p.out_lens[item] = count;
      if (p.out_start != nullptr) p.out_start[item] = item * p.out_stride;
    }
  }
  if (count <= 0) return;
  const float* scores = p.scores + static_cast<int64_t>(BLOCKS ? item : row) * p.scores_stride;
  int32_t* out = p.out + item * p.out_stride;
  const int32_t* table = BLOCKS ? p.block_table + static_cast<int64_t>(row) * p.max_pages : nullptr;
  auto put = [&](int at, int i) {
    if constexpr (BLOCKS) {
      out[at] = table[i];
    } else {
      out[at] = i;
      if (p.kept != nullptr) p.kept[item * p.out_stride + at] = scores[i];
    }
  };
  if (count == n) {
    for (int i = tid; i < n; i += THREADS) put(i, i);
    return;
  }

  // The wave's run of the row, 64 entries a step.
  const int steps = (n + THREADS - 1) / THREADS;
  const int run = w * steps * 64 + lane;
  auto key_at = [&](int j) -> uint32_t {
    const int i = run + 64 * j;
    if (i >= n) return 0;
    return i < p.first || i >= n - p.last ? kForced : key_of(scores[i]);
  };
  uint32_t key[REGS];
#pragma unroll
  for (int j = 0; j < REGS; ++j) key[j] = j < steps ? key_at(j) : 0;
  auto for_all = [&](auto&& f) {
#pragma unroll
    for (int j = 0; j < REGS; ++j)
      if (j < steps) f(j, key[j]);
    for (int j = REGS; j < steps; ++j) f(j, key_at(j));
  };

  for (int i = tid; i < kBins * kCopies; i += THREADS) hist[i] = 0;
  __syncthreads();
  uint32_t least = 0;       // the digits found so far
  int need = count;         // entries still missing among the keys that begin with them
  bool all = false;         // all of those stay
#pragma unroll 1
  for (int shift = 24; shift >= 0 && !all; shift -= 8) {
    const uint32_t mask = shift == 24 ? 0u : ~0u << (shift + 8);
    for_all([&](int, uint32_t k) {
      if (k != 0 && (k & mask) == least) atomicAdd(&hist[((k >> shift) & 255u) * kCopies + (lane & 31)], 1);
    });
    __syncthreads();
    if (tid < kBins) {
      int s = 0;
#pragma unroll
      for (int i = 0; i < kCopies; ++i) {
        int* at = &hist[tid * kCopies + ((i + tid) & 31)];
        s += *at;
        *at = 0;
      }
      sums[tid] = s;
    }
    __syncthreads();
    const Digit d = find_digit(sums, need, lane);
    least |= static_cast<uint32_t>(d.digit) << shift;
    need -= d.above;
    all = need == d.count;
  }
  if (all) need = INT32_MAX;

  int above = 0, equal = 0;
  const uint32_t top = least;
  // Keys that begin with the digits found: equal to `top` where all digits were
  // needed, else all of them stay, as those above do.
  auto masks = [&](uint32_t k, uint64_t& over, uint64_t& same) {
    over = __builtin_amdgcn_ballot_w64(all ? k >= top && k != 0 : k > top);
    same = all ? 0 : __builtin_amdgcn_ballot_w64(k == top);
  };
  for_all([&](int, uint32_t k) {
    uint64_t over, same;
    masks(k, over, same);
    above += __builtin_popcountll(over);
    equal += __builtin_popcountll(same);
  });
  if (lane == 0) {
    wave_above[w] = above;
    wave_equal[w] = equal;
  }
  __syncthreads();
  above = 0;
  equal = 0;
  for (int i = 0; i < w; ++i) {
    above += wave_above[i];
    equal += wave_equal[i];
  }
  const uint64_t before = (uint64_t{1} << lane) - 1;
  for_all([&](int j, uint32_t k) {
    uint64_t over, same;
    masks(k, over, same);
    const int a = above + __builtin_popcountll(over & before), e = equal + __builtin_popcountll(same & before);
    const bool stays = ((over >> lane) & 1) != 0 || (((same >> lane) & 1) != 0 && e < need);
    if (stays) put(a + min(e, need), run + 64 * j);
    above += __builtin_popcountll(over);
    equal += __builtin_popcountll(same);
  });
}

template <bool BLOCKS>
ChooseForm form(int64_t most) {
  if (most <= 2048) return {choose_kernel<BLOCKS, 256, 8>, 256};
  return {choose_kernel<BLOCKS, 1024, 32>, 1024};
}

}  // namespace

ChooseForm select_choose_kernel(bool blocks, int64_t most) { return blocks ? form<true>(most) : form<false>(most); }

}  // namespace comem
