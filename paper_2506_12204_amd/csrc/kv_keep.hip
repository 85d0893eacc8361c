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
// token's page and place written down), the codes (a wave per 64 channels of a block of
// every layer and head), and the pages, lengths and scales. A sequence moves within its
// own pages: a wave takes its tokens in order, 16 at a time read before they are
// written, and later ones' sources lie behind. Different waves share no codes, and the
// scales that they read are only replaced afterwards.
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
  __shared__ int32_t lowest, filled;
  const KvView& c = a.c;
  const int64_t i = blockIdx.x;
  const int t = threadIdx.x;
  auto wrong = [&] { atomicOr(c.flags, kFlagInval); };
  auto blocks_of = [&](int tokens) {
    return (int)(((uint32_t)tokens + (uint32_t)c.page_tokens - 1) >> c.page_shift);
  };
  KvKept kept = {-1, 0, 0, 0, 0, 0};
  const int64_t row0 = a.cu[i], listed = (int64_t)a.cu[i + 1] - row0;
  const int32_t s = a.seqs[i], last = a.last[i];
  const int64_t room = (int64_t)c.max_blocks << c.page_shift;
  const int64_t len = (uint32_t)s < (uint32_t)c.slots ? c.lens[s] : -1;
  if (i == 0 && t == 0 && (a.cu[0] != 0 || a.cu[a.n] != a.total)) wrong();
  if (t == 0) lowest = filled = INT32_MAX;
  if (row0 < 0 || listed < 0 || row0 + listed > a.total || len < 0 || len > room || last < 0 ||
      last > len) {
    if (t == 0) {
      wrong();
      a.kept[i] = kept;
    }
    return;
  }
  block_sync();
  const int first = (int)len - last;  // of the tokens that the list is about
  bool bad = false;
  // (a sequence is listed once, and lists do not overlap: the first ones count)
  for (int64_t k = t; k < i; k += KT) bad |= a.seqs[k] == s || a.cu[k + 1] > row0;
  for (int64_t k = t; k < listed; k += KT) {
    const int32_t at = a.index[row0 + k], before = k ? a.index[row0 + k - 1] : 0;
    if (at >= 0) {
      bad |= at >= last || (k > 0 && (before < 0 || at <= before));
      if (at != k) atomicMin(&lowest, (int32_t)k);
    } else {  // the list is filled up from here on
      bad |= at != -1;
      if (before >= 0) atomicMin(&filled, (int32_t)k);
    }
  }
  bad = block_any(bad, &scratch);
  const int64_t count = min(listed, (int64_t)filled);
  const int now = first + (int)count;
  // The blocks that are written: none where only the end leaves.
  const bool moves = lowest < count;
  const int begin = moves ? (first + lowest) >> c.page_shift : 0;
  const int end = moves ? blocks_of(now) : 0;
  const int32_t* table = c.tables + (int64_t)(bad ? 0 : s) * c.max_blocks;
  const int blocks = blocks_of((int)len);
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
      write_source(a, at + k - ((int64_t)begin << c.page_shift), table[from >> c.page_shift],
                   from & (c.page_tokens - 1));
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

// Four codes, of a block whose scale times q's power of two is `held`, on the scale that
// q divides by. (The scale is lifted first, so that no product leaves 32 bits.)
template <int FMT>
__device__ __forceinline__ uint32_t again(uint32_t codes, float held, const Quotient& q) {
  float f[4];
#pragma unroll
  for (int k = 0; k < 4; ++k)
    f[k] = q.of_lifted(code_to_float<FMT>(codes >> (8 * k) & 0xffu) * held);
  return pack_codes<FMT>(f[0], f[1], f[2], f[3]);
}

__device__ __forceinline__ int64_t lane_i64(int64_t v, int lane) {
  return (int64_t)lane_u64((uint64_t)v, lane);
}
__device__ __forceinline__ float lane_float(float v, int lane) {
  return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(v), lane));
}

// The sources of a step of 64 tokens, a lane each, and where they go.
struct Step {
  int64_t from;  // the place that plans write
  int32_t page;  // -1: the token is not there
  int32_t to;    // its new page
  float was;     // the scale of the block that it comes from
};

template <int FMT>
__device__ __forceinline__ float number_of(int32_t code) {
  return FMT == SEM_KV_INT8 ? (float)code : code_to_float<FMT>((uint32_t)code);
}

// A wave's block of every page of a sequence that changes, 64 tokens at a time.
template <int D>
struct Mover {
  const KvKeepArgs& a;
  const KvKept& kept;
  const int which, lane = lane_id(), in_page = a.c.page_tokens - 1;
  // (rounds of 64 may end past 31 bits)
  const uint32_t first = (uint32_t)kept.begin << a.c.page_shift, end = (uint32_t)kept.now;
  const float* const scale = a.c.scale + which;
  const int32_t* const table = a.c.tables + (int64_t)kept.seq * a.c.max_blocks;
  const int64_t* const source = a.source + kept.source - first;
  const int32_t* const pages = a.pages + kept.source - first;
  Step s, next, later;
  float now = 0.0f;  // scale of the lane's block
  // of a step: what its tokens are divided by, what their codes are multiplied by before,
  // whether they stay on their scale, the tile that they go to
  Quotient q{1.0f};
  float held = 0.0f;
  bool same = false;
  int64_t to = 0;
  uint64_t moving = 0;

  __device__ __forceinline__ void look_up(uint32_t t0, Step& s) const {
    const uint32_t t = t0 + lane;
    s.from = 0;
    s.page = -1;
    s.to = 0;
    if (t < end) {
      s.page = pages[t];
      s.from = source[t];
      s.to = table[t >> a.c.page_shift];
    }
  }
  __device__ __forceinline__ void scale_of(Step& s) const {
    s.was = s.page >= 0 ? scale[(int64_t)s.page * a.c.page_scales] : 0.0f;
  }
  __device__ __forceinline__ void begin() {
    look_up(first, s);
    look_up(first + kWave, next);
    scale_of(s);
  }
  // Step t0: everything but its codes. The next two steps' loads are on their way.
  __device__ __forceinline__ void step(uint32_t t0) {
    const KvView& c = a.c;
    if (c.page_tokens <= kWave) {
      now = s.was;
      for (int off = 1; off < c.page_tokens; off *= 2) now = fmaxf(now, __shfl_xor(now, off, kWave));
    } else if (((t0 - first) & in_page) == 0) {
      now = s.was;
      const uint32_t stop = min(t0 + (uint32_t)c.page_tokens, end);
      for (uint32_t t = t0 + kWave + lane; t < stop; t += kWave)
        now = fmaxf(now, scale[(int64_t)pages[t] * c.page_scales]);
      now = __uint_as_float(wave_max_u32(__float_as_uint(now)));
    }
    const uint32_t t = t0 + lane;
    if (blockIdx.y == 0 && (t & in_page) == 0 && t < end)
      a.scales[(kept.scales + (t >> c.page_shift) - kept.begin) * c.page_scales + which] = now;
    q = Quotient(now > 0.0f ? now : 1.0f);
    held = s.was * q.lift;
    same = s.was == now;
    to = s.to * c.page_bytes + (int64_t)((t & in_page) / kKvTile * (kKvTile * D));
    moving = __ballot(s.page >= 0 && (s.from != to + lane % 16 || !same));
    scale_of(next);
    look_up(t0 + 2 * kWave, later);
  }
  __device__ __forceinline__ void advance() {
    s = next;
    next = later;
  }
  // The tokens of tile x that are not where they stay.
  __device__ __forceinline__ uint32_t in_tile(int x) const {
    return (uint32_t)(moving >> (x * 16)) & 0xffffu;
  }
  __device__ __forceinline__ int tokens_of(uint32_t at) const {
    return at < end ? (int)min(end - at, (uint32_t)kKvTile) : 0;
  }
};

// K: a lane has 16 channels of token lane % 16 of a tile.
template <int D, int FMT>
__device__ __forceinline__ void move_keys(Mover<D>& m, uint8_t* data) {
  constexpr int TILES = kWave / kKvTile;
  const int lane = lane_id();
  uint4 u[TILES], ahead[TILES];
  auto load = [&](const Step& of, uint64_t which, uint4 (&u)[TILES])
      __attribute__((always_inline)) {
#pragma unroll
    for (int x = 0; x < TILES; ++x) {
      if ((which >> (x * 16) & 0xffff) == 0) continue;
      const int mine = x * 16 + lane % 16;
      const int64_t from = __shfl(of.from, mine, kWave);
      if (which >> mine & 1)
        u[x] = *reinterpret_cast<const uint4*>(data + (from & ~15ll) + (from & 15) * 16 +
                                               lane / 16 * 256);
    }
  };
  for (uint32_t t0 = m.first; t0 < m.end; t0 += kWave, m.advance()) {
    m.step(t0);
    if (t0 == m.first) load(m.s, m.moving, u);
    if (m.end - t0 > (uint32_t)kWave) load(m.next, __ballot(m.next.page >= 0), ahead);
#pragma unroll
    for (int x = 0; x < TILES; ++x) {
      if (m.in_tile(x) == 0) continue;
      const int mine = x * 16 + lane % 16;
      Quotient by = m.q;  // the token's
      by.by = __shfl(m.q.by, mine, kWave);
      by.inv = __shfl(m.q.inv, mine, kWave);
      const float was = __shfl(m.held, mine, kWave);
      const bool stays = __shfl((int)m.same, mine, kWave);
      uint8_t* p = data + lane_i64(m.to, x * 16) + lane / 16 * 256 + lane % 16 * 16;
      if (m.moving >> mine & 1) {
        uint32_t w[4] = {u[x].x, u[x].y, u[x].z, u[x].w};
        if (!stays) {
#pragma unroll
          for (int k = 0; k < 4; ++k) w[k] = again<FMT>(w[k], was, by);
        }
        *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
      }
    }
#pragma unroll
    for (int x = 0; x < TILES; ++x) u[x] = ahead[x];
  }
}

// V: a lane has a channel and fetches its tokens' bytes one by one, at addresses whose
// bases are scalar: of a tile in which more than SOME tokens move all of them, a tile
// ahead, of others the ones that move.
template <int D, int FMT, int SOME>
__device__ __forceinline__ void move_values(Mover<D>& m, uint8_t* data) {
  constexpr int TILES = kWave / kKvTile;
  const int lane = lane_id();
  int32_t even[16], odd[16];
  // (tokens that are not there: the last one that is)
  auto load = [&](int64_t from, int x, int n, int32_t (&code)[16])
      __attribute__((always_inline)) {
#pragma unroll
    for (int k = 0; k < 16; ++k) {
      const uint8_t* p = data + lane_i64(from, x * 16 + min(k, n - 1)) + lane * 16;
      code[k] = FMT == SEM_KV_INT8 ? (int32_t) * reinterpret_cast<const int8_t*>(p) : (int32_t)*p;
    }
  };
  auto store = [&](int x, int n, const int32_t (&code)[16]) __attribute__((always_inline)) {
    Quotient by = m.q;
    by.by = lane_float(m.q.by, x * 16);
    by.inv = lane_float(m.q.inv, x * 16);
    uint8_t* p = data + lane_i64(m.to, x * 16) + lane * 16;
    const uint32_t still = (uint32_t)(__ballot(m.same) >> (x * 16)) & 0xffffu;
    uint32_t w[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      float f[4];
#pragma unroll
      for (int j = 0; j < 4; ++j)
        f[j] = by.of_lifted(number_of<FMT>(code[4 * k + j]) *
                            lane_float(m.held, x * 16 + 4 * k + j));
      w[k] = pack_codes<FMT>(f[0], f[1], f[2], f[3]);
    }
    if (still) {  // codes on the same scale stay as they are
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        uint32_t raw = 0, keep = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          raw |= ((uint32_t)code[4 * k + j] & 0xffu) << (8 * j);
          if (still >> (4 * k + j) & 1) keep |= 0xffu << (8 * j);
        }
        w[k] = (raw & keep) | (w[k] & ~keep);
      }
    }
    if (n == kKvTile) {
      *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    } else {  // the bytes behind the sequence stay
      for (int k = 0; k < n; ++k) {
        const uint32_t word = k < 8 ? (k < 4 ? w[0] : w[1]) : (k < 12 ? w[2] : w[3]);
        p[k] = (uint8_t)(word >> (8 * (k & 3)));
      }
    }
  };
  // A tile in which few tokens move: those alone, four at a time.
  auto some = [&](int x) __attribute__((always_inline)) {
    uint8_t* p = data + lane_i64(m.to, x * 16) + lane * 16;
    Quotient by = m.q;
    by.by = lane_float(m.q.by, x * 16);
    by.inv = lane_float(m.q.inv, x * 16);
    const uint64_t still = __ballot(m.same);
#pragma unroll 1
    for (uint32_t left = m.in_tile(x); left != 0;) {
      const int count = min(4, (int)__popc(left));
      int at[4];
      int32_t code[4];
      float f[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        at[j] = left ? x * 16 + __ffs(left) - 1 : at[j ? j - 1 : 0];
        left &= left - 1;
        const uint8_t* from = data + lane_i64(m.s.from, at[j]) + lane * 16;
        code[j] = FMT == SEM_KV_INT8 ? (int32_t) * reinterpret_cast<const int8_t*>(from)
                                     : (int32_t)*from;
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        f[j] = by.of_lifted(number_of<FMT>(code[j]) * lane_float(m.held, at[j]));
      }
      const uint32_t w = pack_codes<FMT>(f[0], f[1], f[2], f[3]);
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (j < count)
          p[at[j] % 16] = (uint8_t)(still >> at[j] & 1 ? (uint32_t)code[j] : w >> (8 * j));
    }
  };
  for (uint32_t t0 = m.first; t0 < m.end; t0 += kWave, m.advance()) {
    m.step(t0);
    auto n = [&](int x) __attribute__((always_inline)) { return m.tokens_of(t0 + x * 16); };
    auto many = [&](int x) __attribute__((always_inline)) {
      return __popc(m.in_tile(x)) > SOME;
    };
    if (t0 == m.first && many(0)) load(m.s.from, 0, n(0), even);
#pragma unroll 1
    for (int x = 0; x < TILES; x += 2) {
      if (many(x + 1)) load(m.s.from, x + 1, n(x + 1), odd);
      if (many(x)) store(x, n(x), even);
      else some(x);
      if (x + 2 < TILES) {
        if (many(x + 2)) load(m.s.from, x + 2, n(x + 2), even);
      } else if (m.end - t0 > (uint32_t)kWave) {
        load(m.next.from, 0, n(TILES), even);
      }
      if (many(x + 1)) store(x + 1, n(x + 1), odd);
      else some(x + 1);
    }
  }
}

// A wave: 64 channels (part blockIdx.y) of a block of every page that changes. Loads run
// ahead: sources two steps of 64 tokens, scales and codes one (V: a tile of 16). A token
// that stays where it is on the same scale is not touched, and a tile of 16 of them
// neither.
//
// Bound by memory: of the pages that tokens are taken from, every line that one of them
// lies in is read (128 bytes hold eight tokens' sixteen channels of K, or 16 tokens' eight
// channels of V). 32 sequences of 2048 to 16384 tokens pruned to 2000, 4 layers of 8 heads
// of 128 channels: 1.05 GB are moved, 1.97 GB in lines, which a copy's rate takes 418 us
// for; 522 us (K alone 227, V alone 320 and 303 without its conversions). Short lists are
// bound by the instructions and the chain of loads of a wave: the accepted tokens of a
// tree of 16 to 64 each of 64 sequences, 32 layers, 0.12 GB by the counters, 41 us.
template <int D, int FMT, int SOME>
__global__ __launch_bounds__(MW* kWave, 4) void kv_keep_move(KvKeepArgs a) {
  const KvView& c = a.c;
  const uint32_t scales = (uint32_t)c.page_scales, groups = (scales + MW - 1) / MW;
  const uint32_t i = blockIdx.x / groups;
  const uint32_t pair = (blockIdx.x - i * groups) * MW +
                        (uint32_t)__builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  if (pair >= scales) return;
  // K and V of a head side by side: V takes longer, and the dies deal out workgroups in turn
  const uint32_t both = 2 * (uint32_t)c.kv_heads, first = pair / both * both;
  const int which = (int)(first + pair % 2 * (uint32_t)c.kv_heads + (pair - first) / 2);
  const KvKept kept = a.kept[i];
  if (kept.seq < 0 || kept.begin >= kept.end) return;
  uint8_t* const data = c.data + which * ((int64_t)c.page_tokens * D) + blockIdx.y * 1024;
  Mover<D> m{a, kept, which};
  m.begin();
  if (pair % 2 == 0) move_keys<D, FMT>(m, data);
  else move_values<D, FMT, SOME>(m, data);
}

// The scales of the blocks that changed, the pages behind the sequence, its length.
// (In parts, blockIdx.y, where there are many scales; the first does the rest.)
__global__ __launch_bounds__(KT) void kv_keep_finish(KvKeepArgs a) {
  const KvView& c = a.c;
  const KvKept kept = a.kept[blockIdx.x];
  if (kept.seq < 0) return;
  int32_t* table = c.tables + (int64_t)kept.seq * c.max_blocks;
  const int64_t changed = (int64_t)(kept.end - kept.begin) * c.page_scales;
  for (int64_t k = (int64_t)blockIdx.y * KT + threadIdx.x; k < changed; k += gridDim.y * KT) {
    const int b = (int)(k / c.page_scales), which = (int)(k % c.page_scales);
    c.scale[(int64_t)table[kept.begin + b] * c.page_scales + which] =
        a.scales[(kept.scales + b) * c.page_scales + which];
  }
  if (blockIdx.y > 0) return;
  const int len = c.lens[kept.seq];
  const int blocks = (int)(((uint32_t)len + (uint32_t)c.page_tokens - 1) >> c.page_shift);
  block_sync();
  for (int b = (int)(((uint32_t)kept.now + (uint32_t)c.page_tokens - 1) >> c.page_shift) +
               (int)threadIdx.x;
       b < blocks; b += KT) {
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

// Workgroups of a sequence's moves.
int64_t groups_of(const KvKeepArgs& a) { return ((int64_t)a.c.page_scales + MW - 1) / MW; }

template <int D, int FMT>
void launch_move(const KvKeepArgs& a, int64_t tokens, hipStream_t st) {
  const dim3 grid((unsigned)(a.n * groups_of(a)), D / 64);
  // Without tiles that are loaded ahead a wave holds fewer registers. 4, 16, 32, 64 of 128
  // tokens of each of 64 sequences, 8 layers of 8 heads of 128 channels: 22, 34, 46, 74 us;
  // with them (where more than 8 tokens move) 27, 38, 48, 66 us. The host knows the room of
  // all lists alone, so the rule goes by their average: 1000 of 1200 tokens beside 63 lists
  // of 4 take 172 us, where 111 were possible; 4000 of 8000 beside them take 383 (or 657).
  if (tokens <= 32 * a.n)
    hipLaunchKernelGGL((kv_keep_move<D, FMT, kKvTile>), grid, dim3(MW * kWave), 0, st, a);
  else
    hipLaunchKernelGGL((kv_keep_move<D, FMT, 8>), grid, dim3(MW * kWave), 0, st, a);
}

template <int D>
void launch_format(const KvKeepArgs& a, int64_t tokens, hipStream_t st) {
  if (a.c.format == SEM_KV_INT8) launch_move<D, SEM_KV_INT8>(a, tokens, st);
  else launch_move<D, SEM_KV_FP8>(a, tokens, st);
}

}  // namespace

// The moves of a plan of so many kept tokens, and what follows them.
hipError_t launch_kv_kept(const KvKeepArgs& a, int64_t tokens, hipStream_t st) {
  switch (a.c.head_dim) {
    case 64: launch_format<64>(a, tokens, st); break;
    case 128: launch_format<128>(a, tokens, st); break;
    default: launch_format<256>(a, tokens, st);
  }
  const int64_t blocks = tokens / a.n / a.c.page_tokens + 2;  // of a sequence
  const int64_t parts = blocks * a.c.page_scales / (8 * KT);
  hipLaunchKernelGGL(kv_keep_finish,
                     dim3((unsigned)a.n, (unsigned)std::max<int64_t>(1, std::min<int64_t>(parts, 64))),
                     dim3(KT), 0, st, a);
  return hipGetLastError();
}

bool kv_kept_fits(const KvKeepArgs& a) {
  return grid_fits(a.n * groups_of(a), MW * kWave) && grid_fits(a.n, KT);
}

hipError_t launch_kv_keep(const KvKeepArgs& a, hipStream_t st) {
  if (a.n == 0) return hipSuccess;
  if (!kv_kept_fits(a)) return hipErrorInvalidConfiguration;
  hipLaunchKernelGGL(kv_keep_plan, dim3((unsigned)a.n), dim3(KT), 0, st, a);
  return launch_kv_kept(a, a.total, st);
}

}  // namespace semsched
