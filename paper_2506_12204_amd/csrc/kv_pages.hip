// The page tables of the KV cache: fork, reserve (with copies of shared last
// pages), free and compact. Pages are named by number; every result is defined
// by ascending page numbers and by the order of the caller's lists, never by
// the order in which workgroups run, so page numbers are reproducible. The
// only atomics are integer additions and bit operations, which commute.
//
// Bound by latency where few pages are touched (16 forks with their copies 16 us
// in three launches, which the host's time per launch is about; the kernels are 4
// to 6 us each) and by the copies where many are: 96 of 256 sequences freed and
// the cache compacted (4096 pages of 512 KiB) in 223 us, 4.7 TB/s, and 256
// branches of up to 64 tokens in 59 us, 4.4 TB/s.
#include <algorithm>

#include "block_common.h"
#include "kv.h"

namespace semsched {

namespace {

constexpr int PT = 256;           // threads of the per-sequence kernels
constexpr int ST = 1024;          // threads of the one-workgroup planners
constexpr uint32_t kNoPage = ~0u;
constexpr int kCopyUnit = 16384;  // bytes of a page that a workgroup copies at a time

__device__ __forceinline__ void flag(const KvView& c, uint32_t bit) { atomicOr(c.flags, bit); }

__device__ __forceinline__ bool bad_page(const KvView& c, int32_t page) {
  return (uint32_t)page >= (uint64_t)c.num_pages;
}

__device__ __forceinline__ int blocks_of(const KvView& c, int tokens) {
  return (int)(((uint32_t)tokens + (uint32_t)c.page_tokens - 1) >> c.page_shift);
}

// A sequence's length, 0 if it is not one that the table can hold.
__device__ __forceinline__ int checked_len(const KvView& c, int s) {
  const int n = c.lens[s];
  if (n < 0 || (int64_t)n > ((int64_t)c.max_blocks << c.page_shift)) {
    flag(c, kFlagInval);
    return 0;
  }
  return n;
}

// One workgroup per pair. Every thread has read both lengths before one of
// them writes the new sequence's.
__global__ __launch_bounds__(PT) void kv_fork(KvForkArgs a) {
  const KvView& c = a.c;
  const int64_t i = blockIdx.x;
  const int32_t s = a.src[i], d = a.dst[i];
  if ((uint32_t)s >= (uint32_t)c.slots || (uint32_t)d >= (uint32_t)c.slots || s == d) {
    if (threadIdx.x == 0) flag(c, kFlagInval);
    return;
  }
  int n = checked_len(c, s);
  const bool taken = c.lens[d] != 0;
  if (a.tokens) {
    const int t = a.tokens[i];
    if (t < 0 && threadIdx.x == 0) flag(c, kFlagRange);
    n = min(n, max(t, 0));
  }
  block_sync();
  if (taken) {  // the new sequence has to be empty
    if (threadIdx.x == 0) flag(c, kFlagInval);
    return;
  }
  const int nb = blocks_of(c, n);
  const int32_t* from = c.tables + (int64_t)s * c.max_blocks;
  int32_t* to = c.tables + (int64_t)d * c.max_blocks;
  for (int b = threadIdx.x; b < nb; b += PT) {
    const int32_t page = from[b];
    if (bad_page(c, page)) {
      flag(c, kFlagInval);
      continue;
    }
    to[b] = page;
    atomicAdd(c.refs + page, 1);
  }
  if (threadIdx.x == 0) c.lens[d] = n;
}

// One workgroup per sequence: its blocks beyond those that `keep` tokens need.
__global__ __launch_bounds__(PT) void kv_free(KvFreeArgs a) {
  const KvView& c = a.c;
  const int64_t i = blockIdx.x;
  const int32_t s = a.seqs[i];
  if ((uint32_t)s >= (uint32_t)c.slots) {
    if (threadIdx.x == 0) flag(c, kFlagInval);
    return;
  }
  const int n = checked_len(c, s);
  int keep = 0;
  if (a.keep) {
    keep = a.keep[i];
    if (keep < 0) {
      if (threadIdx.x == 0) flag(c, kFlagRange);
      return;
    }
    keep = min(keep, n);
  }
  block_sync();
  const int nb = blocks_of(c, n);
  int32_t* table = c.tables + (int64_t)s * c.max_blocks;
  for (int b = blocks_of(c, keep) + threadIdx.x; b < nb; b += PT) {
    const int32_t page = table[b];
    if (bad_page(c, page)) {
      flag(c, kFlagInval);
      continue;
    }
    const int32_t old = atomicSub(c.refs + page, 1);
    if (old == 1) {
      atomicAnd(c.live + (page >> 5), ~(1u << (page & 31)));
    } else if (old <= 0) {  // not a page in use: nothing was there to give back
      atomicAdd(c.refs + page, 1);
      flag(c, kFlagInval);
    }
    table[b] = -1;
  }
  if (threadIdx.x == 0) c.lens[s] = keep;
}

// A listed sequence's needs.
struct Growth {
  int32_t seq, len, grow, tail;  // tail: its last page, if that is copied
  uint32_t shared, need;         // whether it is; pages in all
  uint32_t wrong;                // error bits
};

__device__ __forceinline__ Growth growth_of(const KvReserveArgs& a, int64_t i) {
  const KvView& c = a.c;
  Growth g = {a.seqs[i], 0, a.grow[i], 0, 0, 0, 0};
  if ((uint32_t)g.seq >= (uint32_t)c.slots) {
    g.wrong = kFlagInval;
    return g;
  }
  if (g.grow < 0) {
    g.wrong = kFlagRange;
    return g;
  }
  g.len = c.lens[g.seq];
  const int64_t want = (int64_t)g.len + g.grow;
  if (g.len < 0 || want > ((int64_t)c.max_blocks << c.page_shift)) {
    g.wrong = kFlagInval;  // not a length, or the sequence's table is full
    return g;
  }
  const int have = blocks_of(c, g.len);
  g.need = (uint32_t)(blocks_of(c, (int)want) - have);
  if (g.grow > 0 && (g.len & (c.page_tokens - 1)) != 0) {
    g.tail = c.tables[(int64_t)g.seq * c.max_blocks + have - 1];
    if (bad_page(c, g.tail)) g.wrong = kFlagInval;
    else g.shared = c.refs[g.tail] > 1 ? 1u : 0u;
    g.need += g.shared;
  }
  return g;
}

// Room for grow[i] more tokens of each listed sequence, in one workgroup: needs
// are counted and summed, the free pages listed in ascending order, and only
// if there are enough of them is anything changed. Bound by its chain of loads
// (sequence, length, table, count, then the free pages): 5 us for 16 sequences,
// 11 us for 256 that grow by up to 64 tokens. Up to 1024 sequences keep their
// needs in registers.
__global__ __launch_bounds__(ST) void kv_reserve_plan(KvReserveArgs a) {
  __shared__ uint64_t sums[ST / kWave + 1];
  __shared__ uint32_t scratch[ST / kWave + 1];
  __shared__ uint32_t bad;
  const KvView& c = a.c;
  const int t = threadIdx.x;
  if (t == 0) {
    bad = 0;
    *a.ncopies = 0;
  }
  block_sync();
  Growth mine = {};
  uint32_t first = 0;  // of the thread's last sequence in `fresh`
  uint64_t total = 0;
  for (int64_t i0 = 0; i0 < a.n; i0 += ST) {
    const int64_t i = i0 + t;
    mine = Growth{};
    if (i < a.n) {
      mine = growth_of(a, i);
      if (mine.wrong) {
        flag(c, mine.wrong);
        atomicOr(&bad, 1u);
        mine.need = 0;
      }
    }
    uint64_t sum;  // (a need may be 2^27 pages, and there are 1024 of them)
    first = (uint32_t)(total + block_excl_scan_u64<ST>(mine.need, sums, sum));
    if (i < a.n) a.begin[i] = first | (mine.shared << 31);
    total += sum;
    if (total > (uint64_t)a.room) break;  // more than the pool has; uniform
  }
  wait_stores();
  block_sync();
  if (bad) return;
  // the lowest free pages
  uint64_t found = 0;
  if (total <= (uint64_t)a.room) {
    const int64_t words = (c.num_pages + 31) >> 5;
    for (int64_t w0 = 0; w0 < words && found < total; w0 += ST) {
      const int64_t w = w0 + t;
      uint32_t open = 0;
      if (w < words) {
        open = ~c.live[w];
        if ((w + 1) * 32 > c.num_pages) open &= (1u << (c.num_pages & 31)) - 1u;
      }
      uint32_t sum;
      uint64_t at = found + block_excl_scan_u32<ST>((uint32_t)__popc(open), scratch, sum);
      while (open && at < total) {
        const int b = __ffs(open) - 1;
        a.fresh[at++] = (uint32_t)(w * 32 + b);
        open &= open - 1;
      }
      found += sum;
    }
  }
  wait_stores();
  block_sync();
  if (found < total) {
    if (t == 0) flag(c, kFlagNoMem);
    return;
  }
  for (int64_t i = t; i < a.n; i += ST) {
    if (a.n > ST) {  // not in registers
      mine.seq = a.seqs[i];
      mine.grow = a.grow[i];
      mine.len = (int)min((int64_t)c.lens[mine.seq], (int64_t)c.max_blocks << c.page_shift);
      mine.shared = a.begin[i] >> 31;  // (as it was before any count changed)
      first = a.begin[i] & 0x7fffffffu;
      if (mine.shared)
        mine.tail = c.tables[(int64_t)mine.seq * c.max_blocks + blocks_of(c, mine.len) - 1];
      if (mine.shared && bad_page(c, mine.tail)) mine.shared = 0;
    }
    int32_t* table = c.tables + (int64_t)mine.seq * c.max_blocks;
    uint32_t at = first;
    int b = blocks_of(c, mine.len);
    // a sequence listed twice breaks the contract: its pages are then wrong, but
    // the bounds keep every access inside the tables and lists
    const int end = (int)min((int64_t)blocks_of(c, mine.len + mine.grow), (int64_t)c.max_blocks);
    if (mine.shared && at < total) {
      const uint32_t page = a.fresh[at++];
      a.copies[atomicAdd(a.ncopies, 1u)] = (uint64_t)(uint32_t)mine.tail | ((uint64_t)page << 32);
      table[b - 1] = (int32_t)page;
      c.refs[page] = 1;
      atomicOr(c.live + (page >> 5), 1u << (page & 31));
      // when all its sharers take copies in this call the page becomes free
      if (atomicSub(c.refs + mine.tail, 1) == 1)
        atomicAnd(c.live + (mine.tail >> 5), ~(1u << (mine.tail & 31)));
    }
    for (; b < end && at < total; ++b) {
      const uint32_t page = a.fresh[at++];
      table[b] = (int32_t)page;
      c.refs[page] = 1;
      atomicOr(c.live + (page >> 5), 1u << (page & 31));
    }
    c.lens[mine.seq] = mine.len + mine.grow;
  }
}

// Copies `bytes` (a multiple of 16) with one workgroup.
__device__ __forceinline__ void copy_bytes(const uint8_t* from, uint8_t* to, int bytes) {
  const uint4* f = reinterpret_cast<const uint4*>(from);
  uint4* t = reinterpret_cast<uint4*>(to);
  const int n = bytes / 16;
  int i = threadIdx.x;
  for (; i + 3 * PT < n; i += 4 * PT) {
    const uint4 x0 = f[i], x1 = f[i + PT], x2 = f[i + 2 * PT], x3 = f[i + 3 * PT];
    t[i] = x0;
    t[i + PT] = x1;
    t[i + 2 * PT] = x2;
    t[i + 3 * PT] = x3;
  }
  for (; i < n; i += PT) t[i] = f[i];
}

// Unit u of a list of page copies: kCopyUnit bytes of a page; a page's first
// unit copies its scales too.
__device__ __forceinline__ void copy_unit(const KvView& c, const uint64_t* list, int64_t u,
                                          int units) {
  const uint64_t m = list[u / units];
  const int part = (int)(u % units);
  const int64_t from = (uint32_t)m, to = (int64_t)(m >> 32);
  const int64_t off = (int64_t)part * kCopyUnit;
  const int64_t left = c.page_bytes - off;
  copy_bytes(c.data + from * c.page_bytes + off, c.data + to * c.page_bytes + off,
             (int)(left < kCopyUnit ? left : kCopyUnit));
  if (part == 0) {
    for (int i = threadIdx.x; i < c.page_scales; i += PT)
      c.scale[to * c.page_scales + i] = c.scale[from * c.page_scales + i];
  }
}

__global__ __launch_bounds__(PT) void kv_copy(KvView c, const uint64_t* list,
                                              const uint32_t* count) {
  const int units = (int)((c.page_bytes + kCopyUnit - 1) / kCopyUnit);
  const int64_t total = (int64_t)*count * units;
  for (int64_t u = blockIdx.x; u < total; u += gridDim.x) copy_unit(c, list, u, units);
}

// One workgroup: with L live pages, the live pages from L on and the free ones
// below L, both ascending, are paired; then the live bits become those of the
// compacted pool.
__global__ __launch_bounds__(ST) void kv_compact_plan(KvCompactArgs a) {
  __shared__ uint32_t scratch[ST / kWave + 1];
  const KvView& c = a.c;
  const int t = threadIdx.x;
  const int64_t words = (c.num_pages + 31) >> 5;
  // (bits past the last page are not pages, whatever they hold)
  auto live_word = [&](int64_t w) {
    const uint32_t all = (w + 1) * 32 > c.num_pages ? (1u << (c.num_pages & 31)) - 1u : ~0u;
    return c.live[w] & all;
  };
  uint32_t mine = 0;
  for (int64_t w = t; w < words; w += ST) mine += (uint32_t)__popc(live_word(w));
  uint32_t alive;
  block_excl_scan_u32<ST>(mine, scratch, alive);
  uint32_t holes = 0, far = 0;
  // (the halves of an entry are written by different threads)
  uint32_t* half = reinterpret_cast<uint32_t*>(a.moves);
  for (int64_t w0 = 0; w0 < words; w0 += ST) {
    const int64_t w = w0 + t;
    uint32_t hole = 0, high = 0, dead = 0;
    if (w < words) {
      const uint32_t live = live_word(w);
      const int64_t first = w * 32;
      const uint32_t below = first + 32 <= (int64_t)alive ? ~0u
                             : first >= (int64_t)alive    ? 0u
                                                          : (1u << (alive - (uint32_t)first)) - 1u;
      hole = ~live & below;
      high = live & ~below;
      dead = ~live & ~below;
      if (first + 32 > c.num_pages) dead &= (1u << (c.num_pages & 31)) - 1u;
    }
    for (; dead; dead &= dead - 1) a.remap[w * 32 + __ffs(dead) - 1] = kNoPage;
    uint32_t sum;
    uint32_t at = holes + block_excl_scan_u32<ST>((uint32_t)__popc(hole), scratch, sum);
    holes += sum;
    for (; hole; hole &= hole - 1) half[2 * at++ + 1] = (uint32_t)(w * 32 + __ffs(hole) - 1);
    at = far + block_excl_scan_u32<ST>((uint32_t)__popc(high), scratch, sum);
    far += sum;
    for (; high; high &= high - 1) {
      const uint32_t page = (uint32_t)(w * 32 + __ffs(high) - 1);
      a.remap[page] = at;  // its place in the list, for now
      half[2 * at++] = page;
    }
  }
  wait_stores();
  block_sync();
  for (uint32_t k = t; k < far; k += ST) a.remap[half[2 * k]] = half[2 * k + 1];
  for (int64_t w = t; w < words; w += ST) {
    const int64_t first = w * 32;
    c.live[w] = first + 32 <= (int64_t)alive ? ~0u
                : first >= (int64_t)alive    ? 0u
                                             : (1u << (alive - (uint32_t)first)) - 1u;
  }
  if (t == 0) {
    a.counts[0] = far;
    a.counts[1] = alive;
  }
}

// The moves of the plan and, in the same launch, the page numbers of the tables.
__global__ __launch_bounds__(PT) void kv_compact_move(KvCompactArgs a) {
  const KvView& c = a.c;
  const int units = (int)((c.page_bytes + kCopyUnit - 1) / kCopyUnit);
  const uint32_t moves = a.counts[0], alive = a.counts[1];
  if (moves == 0) return;
  const int64_t copies = (int64_t)moves * units;
  const int64_t entries = (int64_t)c.slots * c.max_blocks;
  const int64_t rows = (entries + 4 * PT - 1) / (4 * PT);
  for (int64_t u = blockIdx.x; u < copies + rows; u += gridDim.x) {
    if (u < copies) {
      copy_unit(c, a.moves, u, units);
      if (u % units == 0 && threadIdx.x == 0) {
        const uint64_t m = a.moves[u / units];
        c.refs[m >> 32] = c.refs[(uint32_t)m];
        c.refs[(uint32_t)m] = 0;
      }
      continue;
    }
    const int64_t e0 = (u - copies) * 4 * PT + threadIdx.x;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int64_t e = e0 + k * PT;
      if (e >= entries) continue;
      const int32_t page = c.tables[e];
      if (page < (int32_t)alive) continue;  // (-1 too)
      const uint32_t to = bad_page(c, page) ? kNoPage : a.remap[page];
      if (to == kNoPage) flag(c, kFlagInval);  // a table that names a free page
      else c.tables[e] = (int32_t)to;
    }
  }
}

}  // namespace

hipError_t launch_kv_fork(const KvForkArgs& a, hipStream_t st) {
  if (!grid_fits(a.n, PT)) return hipErrorInvalidConfiguration;
  if (a.n > 0) hipLaunchKernelGGL(kv_fork, dim3((unsigned)a.n), dim3(PT), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_kv_free(const KvFreeArgs& a, hipStream_t st) {
  if (!grid_fits(a.n, PT)) return hipErrorInvalidConfiguration;
  if (a.n > 0) hipLaunchKernelGGL(kv_free, dim3((unsigned)a.n), dim3(PT), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_kv_reserve(const KvReserveArgs& a, hipStream_t st) {
  if (a.n == 0) return hipSuccess;
  hipLaunchKernelGGL(kv_reserve_plan, dim3(1), dim3(ST), 0, st, a);
  const int64_t units = a.n * ((a.c.page_bytes + kCopyUnit - 1) / kCopyUnit);
  hipLaunchKernelGGL(kv_copy, dim3((unsigned)std::min<int64_t>(units, 2048)), dim3(PT), 0, st, a.c,
                     a.copies, a.ncopies);
  return hipGetLastError();
}

hipError_t launch_kv_compact(const KvCompactArgs& a, hipStream_t st) {
  hipLaunchKernelGGL(kv_compact_plan, dim3(1), dim3(ST), 0, st, a);
  hipLaunchKernelGGL(kv_compact_move, dim3(2048), dim3(PT), 0, st, a);
  return hipGetLastError();
}

}  // namespace semsched
