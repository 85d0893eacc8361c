// Pruning: a sequence of more than `budget` tokens keeps its first ones (sinks), its
// last ones (recent) and, of those between, the ones whose attention weights add up to
// the most; ties go to the earlier token. The moves are those of kv_keep.hip; here the
// tokens are chosen, one workgroup per sequence:
//
//   the weights as whole numbers of the same order; the k-th largest of them by its
//   digits, three counts of 11, 11 and 10 bits; then, in the tokens' order, those above
//   it and the first of those equal to it.
//
// Bound by the counts in LDS and the chain of their scans: 2000 of up to 16384 tokens each
// of 32 sequences take 24 us (67 with 256 threads), 256 of up to 1200 of 8 sequences 13
// (16 with 256 threads), of 522 and 23 us that the moves take.
#include "block_common.h"
#include "kv.h"

namespace semsched {

namespace {

constexpr int kBins = 2048;
constexpr int NT = 1024;    // threads of a sequence
constexpr int kCopies = 4;  // of the counters, for lanes in turn: few lanes then meet at one
constexpr int kEach = 4;    // neighbouring tokens of a thread
// Rounds of them whose weights stay in registers (2, 4 or 8: 32 sequences of 8192 tokens to
// 512 in one layer 62, 64, 66 us in all, of 16384 78, 75, 77, of 32768 102, 99, 94).
constexpr int kHeld = 4;

// Numbers in the order of floats; NaN comes before all.
__device__ __forceinline__ uint32_t order_of(float x) {
  const uint32_t u = __float_as_uint(x + 0.0f);  // (minus zero becomes zero)
  if (x != x) return 0u;
  return u >> 31 ? ~u : u | 0x80000000u;
}

__global__ __launch_bounds__(NT) void kv_prune_plan(KvPruneArgs a) {
  constexpr int kRound = kEach * NT;    // tokens
  constexpr int kMine = kBins / NT;     // digits of a thread
  __shared__ alignas(16) uint32_t bins[kBins * kCopies];
  __shared__ uint32_t scratch[NT / kWave + 1];
  __shared__ uint32_t digit_found, above_found, wrong;
  __shared__ int32_t gap;  // the first token that leaves
  const KvView& c = a.k.c;
  const int64_t i = blockIdx.x;
  const int t = threadIdx.x;
  const int32_t s = a.k.seqs[i];
  const int64_t room = (int64_t)c.max_blocks << c.page_shift;
  const int64_t len64 = (uint32_t)s < (uint32_t)c.slots ? c.lens[s] : -1;
  KvKept kept = {-1, 0, 0, 0, 0, 0};
  if (len64 < 0 || len64 > room || len64 <= a.budget) {
    if (t == 0) {
      if (len64 < 0 || len64 > room) atomicOr(c.flags, kFlagInval);
      a.k.kept[i] = kept;
    }
    return;
  }
  // (A sequence is listed once; otherwise the first counts. Two would change each other's
  // weights while they are counted.)
  bool again = false;
  for (int64_t k = t; k < i; k += NT) again |= a.k.seqs[k] == s;
  if (t == 0) wrong = 0;
  block_sync();
  if (again) wrong = 1;
  block_sync();
  if (wrong) {
    if (t == 0) {
      atomicOr(c.flags, kFlagInval);
      a.k.kept[i] = kept;
    }
    return;
  }
  const int len = (int)len64, budget = (int)a.budget;
  const int sinks = (int)min(a.sinks, (int64_t)budget);
  const int recent = (int)min(a.recent, (int64_t)(budget - sinks));
  float* const mass = a.mass + s * a.mass_stride;
  const int low = sinks, high = len - recent;  // the tokens between
  uint32_t want = (uint32_t)(budget - sinks - recent);
  const bool any = want > 0;
  const int64_t rounds = ((int64_t)len + kRound - 1) / kRound;

  // Round r's weights: neighbouring tokens of a thread, the first rounds' from registers.
  uint32_t held[kHeld][kEach];
  auto fetch = [&](int64_t r, uint32_t (&key)[kEach]) __attribute__((always_inline)) {
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
      const int64_t j = r * kRound + kEach * t + k;
      key[k] = j >= low && j < high ? order_of(mass[j]) : 0u;
    }
  };
  auto each_round = [&](auto work) __attribute__((always_inline)) {
#pragma unroll
    for (int r = 0; r < kHeld; ++r)
      if (r < rounds) work(r, held[r]);
    for (int64_t r = kHeld; r < rounds; ++r) {
      uint32_t key[kEach];
      fetch(r, key);
      work(r, key);
    }
  };
  if (any) {
#pragma unroll
    for (int r = 0; r < kHeld; ++r) fetch(r, held[r]);
  }

  // The want-th largest of them: its digits from the first on.
  uint32_t edge = 0;
  if (any) {
    constexpr int kShift[3] = {21, 10, 0};
    uint32_t known = 0;  // bits of the edge that are found
    for (int b = t; b < kBins * kCopies; b += NT) bins[b] = 0;
    block_sync();
#pragma unroll 1
    for (int p = 0; p < 3; ++p) {
      const int shift = p == 0 ? kShift[0] : p == 1 ? kShift[1] : kShift[2];
      const uint32_t digits = p == 2 ? 1024u : 2048u;
      each_round([&](int64_t r, const uint32_t (&key)[kEach]) __attribute__((always_inline)) {
#pragma unroll
        for (int k = 0; k < kEach; ++k) {
          const int64_t j = r * kRound + kEach * t + k;
          const bool mine = j >= low && j < high && (key[k] & known) == (edge & known);
          const uint32_t digit = (key[k] >> shift) & (digits - 1u);
          // (equal weights are common, and a counter takes one lane at a time)
          const uint64_t all = __ballot(mine);
          if (all == 0) continue;
          const int one = __ffsll((unsigned long long)all) - 1;
          const uint32_t first = (uint32_t)__builtin_amdgcn_readlane((int)digit, one);
          if (__ballot(mine && digit != first) == 0) {
            if (lane_id() == one) atomicAdd(&bins[first * kCopies], (uint32_t)__popcll(all));
          } else if (mine) {
            atomicAdd(&bins[digit * kCopies + lane_id() % kCopies], 1u);
          }
        }
      });
      block_sync();
      // from the largest digit down, some to a thread
      uint32_t count[kMine], own = 0;
#pragma unroll
      for (int k = 0; k < kMine; ++k) {
        uint4* at = reinterpret_cast<uint4*>(bins + (kBins - 1 - kMine * t - k) * kCopies);
        const uint4 n = *at;
        *at = make_uint4(0, 0, 0, 0);  // for the next digit
        count[k] = n.x + n.y + n.z + n.w;
        own += count[k];
      }
      uint32_t sum;
      uint32_t above = block_excl_scan_u32<NT>(own, scratch, sum);
#pragma unroll
      for (int k = 0; k < kMine; ++k) {
        if (above < want && want <= above + count[k]) {
          digit_found = kBins - 1 - kMine * t - k;
          above_found = above;
        }
        above += count[k];
      }
      block_sync();
      edge |= digit_found << shift;
      want -= above_found;
      known |= (digits - 1u) << shift;
      block_sync();
    }
  }

  // `want` of those equal to the edge stay, the first ones.
  if (t == 0) gap = INT32_MAX;
  block_sync();
  int32_t* const source = a.k.pages + i * budget;  // (the tokens at first)
  uint32_t more = 0, equal = 0;  // before this round
  int32_t leaves = INT32_MAX;
  each_round([&](int64_t r, const uint32_t (&key)[kEach]) __attribute__((always_inline)) {
    const int64_t first = r * kRound + kEach * t;
    uint32_t is_more = 0, is_equal = 0;
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
      const int64_t j = first + k;
      if (j >= len) continue;
      if (j < low || j >= high) {
        is_more |= 1u << k;
      } else if (any) {
        if (key[k] > edge) is_more |= 1u << k;
        else if (key[k] == edge) is_equal |= 1u << k;
      }
    }
    uint32_t sum;
    const uint32_t before = block_excl_scan_u32<NT>(
        (uint32_t)__popc(is_more) | (uint32_t)__popc(is_equal) << 16, scratch, sum);
    uint32_t m = more + (before & 0xffffu), e = equal + (before >> 16);
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
      const int64_t j = first + k;
      const bool stays = (is_more >> k & 1) || ((is_equal >> k & 1) && e < want);
      if (stays) source[m + min(e, want)] = (int32_t)j;
      else if (j < len) leaves = min(leaves, (int32_t)j);
      m += is_more >> k & 1;
      e += is_equal >> k & 1;
    }
    more += sum & 0xffffu;
    equal += sum >> 16;
  });
  const uint32_t lowest = wave_min_u32((uint32_t)leaves);
  if (lane_id() == 0) atomicMin(&gap, (int32_t)lowest);
  wait_stores();
  block_sync();

  // The blocks that are written, none where only the end leaves.
  const bool moves = gap < budget;
  const int begin = moves ? gap >> c.page_shift : 0;
  const auto blocks_of = [&](int tokens) {
    return (int)(((uint32_t)tokens + (uint32_t)c.page_tokens - 1) >> c.page_shift);
  };
  const int end = moves ? blocks_of(budget) : 0;
  const int blocks = blocks_of(len);
  const int32_t* table = c.tables + (int64_t)s * c.max_blocks;
  for (int b = (moves ? begin : budget >> c.page_shift) + t; b < blocks; b += NT) {
    const int32_t page = table[b];
    if ((uint32_t)page >= (uint64_t)c.num_pages) wrong = 1;
    else if (b >= begin && b < end && c.refs[page] != 1) wrong = 1;
  }
  block_sync();
  if (wrong) {
    if (t == 0) {
      atomicOr(c.flags, kFlagInval);
      a.k.kept[i] = kept;
    }
    return;
  }
  // The tokens' pages and places, and their weights. Sources lie at their tokens or
  // behind, so a round's weights are read before any of them is written.
  for (int64_t j0 = moves ? begin << c.page_shift : budget; j0 < budget; j0 += kEach * NT) {
    int from[kEach];
    float x[kEach];
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
      const int64_t j = j0 + k * NT + t;
      from[k] = j < budget ? source[j] : 0;
    }
#pragma unroll
    for (int k = 0; k < kEach; ++k) x[k] = mass[from[k]];
    block_sync();
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
      const int64_t j = j0 + k * NT + t;
      if (j >= budget) continue;
      mass[j] = x[k];
      write_source(a.k, i * budget + j, table[from[k] >> c.page_shift],
                   from[k] & (c.page_tokens - 1));
    }
  }
  wait_stores();
  block_sync();
  for (int64_t j = budget + t; j < len; j += NT) mass[j] = 0.0f;
  if (t == 0) {
    kept.seq = s;
    kept.now = budget;
    kept.begin = begin;
    kept.end = end;
    kept.source = i * budget + ((int64_t)begin << c.page_shift);
    kept.scales = i * blocks_of(budget);
    a.k.kept[i] = kept;
  }
}

}  // namespace

hipError_t launch_kv_prune(const KvPruneArgs& a, hipStream_t st) {
  if (a.k.n == 0) return hipSuccess;
  if (!kv_kept_fits(a.k) || !grid_fits(a.k.n, NT)) return hipErrorInvalidConfiguration;
  const dim3 grid((unsigned)a.k.n);
  hipLaunchKernelGGL(kv_prune_plan, grid, dim3(NT), 0, st, a);
  return launch_kv_kept(a.k, a.k.n * a.budget, st);
}

}  // namespace semsched
