// Keeping some tokens of a sequence: the chosen ones move together, in order, and
// the pages behind them are given back.
//
// Token t of the new sequence is token source(t) >= t of the old one, ascending. A
// block (a page's K or V of one head) whose tokens change gets the scale
//
//   s' = max of the scales of the blocks that its tokens come from
//   c  <- round(c * s / s')    for the codes of a block of scale s
//
// (quotients and products in 32 bits, each rounded once, as append has them; codes
// of a block of the same scale stay as they are). No maximum over the values is
// taken: a code never grows.
//
// Three launches: a plan (one workgroup per sequence: the lists are looked at, every
// token's page and place written down), the codes (a wave per block of every layer
// and head), and the pages, lengths and scales. A sequence moves within its own
// pages: a wave takes its blocks one after the other, first reads all sources of a
// block and then writes it, and the sources of later blocks lie behind it. Different
// waves share no codes, and the scales that they read are only replaced afterwards.
#include <algorithm>

#include "block_common.h"
#include "kv.h"
#include "kv_codes.h"

namespace semsched {

namespace {

constexpr int KT = 256;  // threads of the per-sequence kernels
constexpr int MW = 4;    // waves of a workgroup of the moves

__device__ __forceinline__ bool block_any(bool x, uint32_t* scratch) {
  if (threadIdx.x == 0) *scratch = 0;
  block_sync();
  if (__ballot(x) && lane_id() == 0) atomicOr(scratch, 1u);
  block_sync();
  const bool any = *scratch != 0;
  block_sync();
  return any;
}

// Looks at one sequence's list and writes its plan.
__global__ __launch_bounds__(KT) void kv_keep_plan(KvKeepArgs a) {
  __shared__ uint32_t scratch;
  __shared__ int32_t lowest;
  const KvView& c = a.c;
  const int64_t i = blockIdx.x;
  const int t = threadIdx.x;
  auto wrong = [&] { atomicOr(c.flags, kFlagInval); };
  KvKept kept = {-1, 0, 0, 0, 0, 0};
  const int64_t row0 = a.cu[i], count = (int64_t)a.cu[i + 1] - row0;
  const int32_t s = a.seqs[i], last = a.last[i];
  const int64_t room = (int64_t)c.max_blocks << c.page_shift;
  const int64_t len = (uint32_t)s < (uint32_t)c.slots ? c.lens[s] : -1;
  if (i == 0 && t == 0 && (a.cu[0] != 0 || a.cu[a.n] != a.total)) wrong();
  if (t == 0) lowest = INT32_MAX;
  if (row0 < 0 || count < 0 || row0 + count > a.total || len < 0 || len > room || last < 0 ||
      last > len || count > last) {
    if (t == 0) {
      wrong();
      a.kept[i] = kept;
    }
    return;
  }
  block_sync();
  const int first = (int)len - last;  // of the tokens that the list is about
  bool bad = false;
  for (int64_t k = t; k < count; k += KT) {
    const int32_t at = a.index[row0 + k];
    bad |= at >= last || at <= (k ? a.index[row0 + k - 1] : -1);
    if (at != k) atomicMin(&lowest, (int32_t)k);
  }
  bad = block_any(bad, &scratch);
  const int now = first + (int)count;
  // The blocks that are written: none where only the end leaves.
  const bool moves = lowest < count;
  const int begin = moves ? (first + lowest) >> c.page_shift : 0;
  const int end = moves ? (now + c.page_tokens - 1) >> c.page_shift : 0;
  const int32_t* table = c.tables + (int64_t)(bad ? 0 : s) * c.max_blocks;
  const int blocks = ((int)len + c.page_tokens - 1) >> c.page_shift;
  bool shared = false;
  if (!bad && now < len) {
    const int from = moves ? begin : now >> c.page_shift;
    for (int b = from + t; b < blocks; b += KT) {
      const int32_t page = table[b];
      if ((uint32_t)page >= (uint64_t)c.num_pages) shared = true;
      else if (b >= begin && b < end && c.refs[page] != 1) shared = true;
    }
  }
  bad = block_any(bad || shared, &scratch);
  if (bad) {
    if (t == 0) {
      wrong();
      a.kept[i] = kept;
    }
    return;
  }
  const int64_t at = row0 + i * c.page_tokens;
  if (moves) {
    for (int64_t k = (begin << c.page_shift) + t; k < now; k += KT) {
      const int from = k < first ? (int)k : first + a.index[row0 + k - first];
      a.source[at + k - (begin << c.page_shift)] =
          ((int64_t)table[from >> c.page_shift] << c.page_shift) + (from & (c.page_tokens - 1));
    }
  }
  if (t == 0) {
    kept.seq = now < len ? s : -1;
    kept.now = now;
    kept.begin = begin;
    kept.end = end;
    kept.source = at;
    kept.scales = (row0 >> c.page_shift) + 2 * i;
    a.kept[i] = kept;
  }
}

// Four codes of a block of scale `was` on the scale that `q` divides by. (The scale is
// brought to its middle range first, so that no product leaves 32 bits.)
template <int FMT>
__device__ __forceinline__ uint32_t again(uint32_t codes, float was, const Quotient& q) {
  const float held = was * q.lift;
  float f[4];
#pragma unroll
  for (int k = 0; k < 4; ++k)
    f[k] = q.of_lifted(code_to_float<FMT>(codes >> (8 * k) & 0xffu) * held);
  return pack_codes<FMT>(f[0], f[1], f[2], f[3]);
}

// A wave: 64 channels (slice `blockIdx.y`) of a block of every page that changes.
template <int D, int FMT>
__global__ __launch_bounds__(MW* kWave) void kv_keep_move(KvKeepArgs a) {
  const KvView& c = a.c;
  const int64_t unit = (int64_t)blockIdx.x * MW +
                       __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int64_t i = unit / c.page_scales;
  if (i >= a.n) return;
  const int which = (int)(unit % c.page_scales), lane = lane_id(), slice = blockIdx.y;
  const bool value = which / c.kv_heads % 2 != 0;
  const KvKept kept = a.kept[i];
  if (kept.seq < 0) return;
  const int64_t block_bytes = (int64_t)c.page_tokens * D;
  uint8_t* const data = c.data + which * block_bytes;
  const float* const scale = c.scale + which;
  const int32_t* const table = c.tables + (int64_t)kept.seq * c.max_blocks;
  const int in_page = c.page_tokens - 1;
  for (int b = kept.begin; b < kept.end; ++b) {
    const int t0 = b << c.page_shift, n = min(kept.now - t0, c.page_tokens);
    const int64_t* source = a.source + kept.source + (t0 - (kept.begin << c.page_shift));
    float now = 0.0f;
    for (int t = lane; t < n; t += kWave)
      now = fmaxf(now, scale[(source[t] >> c.page_shift) * c.page_scales]);
    now = __uint_as_float(wave_max_u32(__float_as_uint(now)));
    if (lane == 0 && slice == 0)
      a.scales[(kept.scales + b - kept.begin) * c.page_scales + which] = now;
    const Quotient q(now > 0.0f ? now : 1.0f);
    uint8_t* const block = data + table[b] * c.page_bytes;
    for (int t1 = 0; t1 < n; t1 += kKvTile) {
      uint8_t* const tile = block + t1 * D;
      if (!value) {
        // 16 channels (group lane / 16 of the slice) of token lane % 16
        const int t = t1 + lane % 16;
        if (t < n) {
          const int64_t from = source[t];
          const int64_t page = from >> c.page_shift;
          const int in = (int)(from & in_page);
          const int group = (slice * 4 + lane / 16) * 256;
          const float was = scale[page * c.page_scales];
          uint4 u = *reinterpret_cast<const uint4*>(data + page * c.page_bytes + in / 16 * 16 * D +
                                                    group + in % 16 * 16);
          if (was != now) {
            u.x = again<FMT>(u.x, was, q);
            u.y = again<FMT>(u.y, was, q);
            u.z = again<FMT>(u.z, was, q);
            u.w = again<FMT>(u.w, was, q);
          }
          asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
          *reinterpret_cast<uint4*>(tile + group + lane % 16 * 16) = u;
        }
      } else {
        // 16 tokens of channel `lane` of the slice
        const int ch = slice * kWave + lane, m = min(n - t1, kKvTile);
        uint32_t w[4] = {0, 0, 0, 0};
        for (int k = 0; k < m; ++k) {
          const int64_t from = source[t1 + k];
          const int64_t page = from >> c.page_shift;
          const int in = (int)(from & in_page);
          const float was = scale[page * c.page_scales];
          uint32_t code = data[page * c.page_bytes + in / 16 * 16 * D + ch * 16 + in % 16];
          if (was != now) code = again<FMT>(code, was, q) & 0xffu;
          w[k / 4] |= code << (8 * (k % 4));
        }
        uint8_t* to = tile + ch * 16;
        if (m == kKvTile) {
          *reinterpret_cast<uint4*>(to) = make_uint4(w[0], w[1], w[2], w[3]);
        } else {
          for (int k = 0; k < m; ++k) to[k] = (uint8_t)(w[k / 4] >> (8 * (k % 4)));
        }
      }
      wait_stores();
    }
  }
}

// The scales of the blocks that changed, the pages behind the sequence, its length.
__global__ __launch_bounds__(KT) void kv_keep_finish(KvKeepArgs a) {
  const KvView& c = a.c;
  const KvKept kept = a.kept[blockIdx.x];
  if (kept.seq < 0) return;
  int32_t* table = c.tables + (int64_t)kept.seq * c.max_blocks;
  const int64_t changed = (int64_t)(kept.end - kept.begin) * c.page_scales;
  for (int64_t k = threadIdx.x; k < changed; k += KT) {
    const int b = (int)(k / c.page_scales), which = (int)(k % c.page_scales);
    c.scale[(int64_t)table[kept.begin + b] * c.page_scales + which] =
        a.scales[(kept.scales + b) * c.page_scales + which];
  }
  const int len = c.lens[kept.seq];
  const int blocks = (len + c.page_tokens - 1) >> c.page_shift;
  block_sync();
  for (int b = ((kept.now + c.page_tokens - 1) >> c.page_shift) + threadIdx.x; b < blocks; b += KT) {
    const int32_t page = table[b];
    const int32_t old = atomicSub(c.refs + page, 1);
    if (old == 1) {
      atomicAnd(c.live + (page >> 5), ~(1u << (page & 31)));
    } else if (old <= 0) {  // not a page in use: nothing was there to give back
      atomicAdd(c.refs + page, 1);
      atomicOr(c.flags, kFlagInval);
    }
    table[b] = -1;
  }
  if (threadIdx.x == 0) c.lens[kept.seq] = kept.now;
}

template <int D>
void launch_move(const KvKeepArgs& a, unsigned grid, hipStream_t st) {
  if (a.c.format == SEM_KV_INT8)
    hipLaunchKernelGGL((kv_keep_move<D, SEM_KV_INT8>), dim3(grid, D / 64), dim3(MW * kWave), 0, st,
                       a);
  else
    hipLaunchKernelGGL((kv_keep_move<D, SEM_KV_FP8>), dim3(grid, D / 64), dim3(MW * kWave), 0, st,
                       a);
}

}  // namespace

// The moves of a plan and what follows them.
hipError_t launch_kv_kept(const KvKeepArgs& a, hipStream_t st) {
  const int64_t grid = (a.n * a.c.page_scales + MW - 1) / MW;
  switch (a.c.head_dim) {
    case 64: launch_move<64>(a, (unsigned)grid, st); break;
    case 128: launch_move<128>(a, (unsigned)grid, st); break;
    default: launch_move<256>(a, (unsigned)grid, st);
  }
  hipLaunchKernelGGL(kv_keep_finish, dim3((unsigned)a.n), dim3(KT), 0, st, a);
  return hipGetLastError();
}

bool kv_kept_fits(const KvKeepArgs& a) {
  return grid_fits((a.n * a.c.page_scales + MW - 1) / MW, MW * kWave) && grid_fits(a.n, KT);
}

hipError_t launch_kv_keep(const KvKeepArgs& a, hipStream_t st) {
  if (a.n == 0) return hipSuccess;
  if (!kv_kept_fits(a)) return hipErrorInvalidConfiguration;
  hipLaunchKernelGGL(kv_keep_plan, dim3((unsigned)a.n), dim3(KT), 0, st, a);
  return launch_kv_kept(a, st);
}

}  // namespace semsched
