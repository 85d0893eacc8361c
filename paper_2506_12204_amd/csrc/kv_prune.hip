// Pruning: a sequence of more than `budget` tokens keeps its first ones (sinks), its
// last ones (recent) and, of those between, the ones whose attention weights add up to
// the most; ties go to the earlier token. The moves are those of kv_keep.hip; here the
// tokens are chosen, one workgroup per sequence:
//
//   the weights as whole numbers of the same order; the k-th largest of them by its
//   digits, three counts of 11, 11 and 10 bits; then, in the tokens' order, those above
//   it and the first of those equal to it.
#include "block_common.h"
#include "kv.h"

namespace semsched {

namespace {

constexpr int PT = 1024;
constexpr int kBins = 2048;
constexpr int kEach = 4;  // neighbouring tokens of a thread

// Numbers in the order of floats; NaN comes before all.
__device__ __forceinline__ uint32_t order_of(float x) {
  const uint32_t u = __float_as_uint(x + 0.0f);  // (minus zero becomes zero)
  if (x != x) return 0u;
  return u >> 31 ? ~u : u | 0x80000000u;
}

__global__ __launch_bounds__(PT) void kv_prune_plan(KvPruneArgs a) {
  __shared__ uint32_t bins[kBins];
  __shared__ uint32_t scratch[PT / kWave + 1];
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
  const int len = (int)len64, budget = (int)a.budget;
  const int sinks = (int)min(a.sinks, (int64_t)budget);
  const int recent = (int)min(a.recent, (int64_t)(budget - sinks));
  float* const mass = a.mass + s * a.mass_stride;
  const int low = sinks, high = len - recent;  // the tokens between
  uint32_t want = (uint32_t)(budget - sinks - recent);

  // The want-th largest of them: its digits from the first on.
  uint32_t edge = 0;
  if (want > 0) {
    constexpr int kShift[3] = {21, 10, 0};
    uint32_t known = 0;  // bits of the edge that are found
#pragma unroll 1
    for (int p = 0; p < 3; ++p) {
      const int shift = kShift[p];
      const uint32_t digits = p == 2 ? 1024u : 2048u;
      bins[t] = 0;
      bins[t + PT] = 0;
      block_sync();
      for (int64_t j0 = low; j0 < high; j0 += kEach * PT) {
        uint32_t key[kEach];
#pragma unroll
        for (int k = 0; k < kEach; ++k) {
          const int64_t j = j0 + k * PT + t;
          key[k] = j < high ? order_of(mass[j]) : 0u;
        }
#pragma unroll
        for (int k = 0; k < kEach; ++k) {
          const bool mine = j0 + k * PT + t < high && (key[k] & known) == (edge & known);
          const uint32_t digit = (key[k] >> shift) & (digits - 1u);
          // (equal weights are common, and a counter takes one lane at a time)
          const uint64_t all = __ballot(mine);
          if (all == 0) continue;
          const int one = __ffsll((unsigned long long)all) - 1;
          const uint32_t first = (uint32_t)__builtin_amdgcn_readlane((int)digit, one);
          if (__ballot(mine && digit != first) == 0) {
            if (lane_id() == one) atomicAdd(&bins[first], (uint32_t)__popcll(all));
          } else if (mine) {
            atomicAdd(&bins[digit], 1u);
          }
        }
      }
      block_sync();
      // from the largest digit down, two to a thread
      const uint32_t d1 = kBins - 1u - 2u * t, d0 = d1 - 1u;
      const uint32_t n1 = bins[d1], n0 = bins[d0];
      uint32_t sum;
      const uint32_t above = block_excl_scan_u32<PT>(n1 + n0, scratch, sum);
      if (above < want && want <= above + n1) {
        digit_found = d1;
        above_found = above;
      } else if (above + n1 < want && want <= above + n1 + n0) {
        digit_found = d0;
        above_found = above + n1;
      }
      block_sync();
      edge |= digit_found << shift;
      want -= above_found;
      known |= (digits - 1u) << shift;
      block_sync();
    }
  }

  // `want` of those equal to the edge stay, the first ones.
  if (t == 0) {
    gap = INT32_MAX;
    wrong = 0;
  }
  block_sync();
  int32_t* const source = a.k.pages + i * budget;  // (the tokens at first)
  const bool any = budget - sinks - recent > 0;
  uint32_t more = 0, equal = 0;  // before this round
  for (int64_t j0 = 0; j0 < len; j0 += kEach * PT) {
    const int64_t first = j0 + kEach * t;
    uint32_t mine = 0, is_more = 0, is_equal = 0;
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
      const int64_t j = first + k;
      if (j >= len) continue;
      if (j < low || j >= high) {
        is_more |= 1u << k;
      } else if (any) {
        const uint32_t key = order_of(mass[j]);
        if (key > edge) is_more |= 1u << k;
        else if (key == edge) is_equal |= 1u << k;
      }
    }
    mine = (uint32_t)__popc(is_more) | (uint32_t)__popc(is_equal) << 16;
    uint32_t sum;
    const uint32_t before = block_excl_scan_u32<PT>(mine, scratch, sum);
    uint32_t m = more + (before & 0xffffu), e = equal + (before >> 16);
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
      const int64_t j = first + k;
      const bool stays = (is_more >> k & 1) || ((is_equal >> k & 1) && e < want);
      if (stays) source[m + min(e, want)] = (int32_t)j;
      else if (j < len) atomicMin(&gap, (int32_t)j);
      m += is_more >> k & 1;
      e += is_equal >> k & 1;
    }
    more += sum & 0xffffu;
    equal += sum >> 16;
  }
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
  for (int b = (moves ? begin : budget >> c.page_shift) + t; b < blocks; b += PT) {
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
  for (int64_t j0 = moves ? begin << c.page_shift : budget; j0 < budget; j0 += PT) {
    const int64_t j = j0 + t;
    int from = 0;
    float x = 0.0f;
    if (j < budget) {
      from = source[j];
      x = mass[from];
    }
    block_sync();
    if (j < budget) {
      mass[j] = x;
      write_source(a.k, i * budget + j, table[from >> c.page_shift], from & (c.page_tokens - 1));
    }
  }
  wait_stores();
  block_sync();
  for (int64_t j = budget + t; j < len; j += PT) mass[j] = 0.0f;
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
  if (!kv_kept_fits(a.k) || !grid_fits(a.k.n, PT)) return hipErrorInvalidConfiguration;
  hipLaunchKernelGGL(kv_prune_plan, dim3((unsigned)a.k.n), dim3(PT), 0, st, a);
  const int64_t pt = a.k.c.page_tokens;
  return launch_kv_kept(a.k, a.k.n * ((a.budget + pt - 1) / pt), st);
}

}  // namespace semsched
