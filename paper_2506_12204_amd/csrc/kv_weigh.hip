// What the cached tokens weigh: the softmax weights that query rows give to every
// key, added up over rows and heads.
//
//   mass[j] += sum over rows r that see key j of exp(scale * ks_j (q_r . kc_j) - lse_r)
//
// with the logarithms of the sums that attention of the same rows returned, so one
// pass over the keys is enough and no values are read. The product runs on the matrix
// cores in the queries' own type, in which 8-bit codes are exact; sums and weights are
// in 32 bits. A key belongs to one workgroup, which adds its weights in an order that
// sizes and lengths alone decide: results do not depend on the run.
//
// A wave has 64 keys of a head in registers and goes through the row tiles. As in
// attention the product is K q^T: a lane ends up with the scores of one row (lane % 16)
// and 16 consecutive keys, whose weights it adds up in registers over all rows and heads
// that it takes.
//
// Few rows are bound by memory: 251 requests of 16 to 4096 keys, 32 heads on 8 of 128
// channels, take 41 us, of which reading the keys (203 MB) at 6 TB/s is 34. Many rows are
// bound by the latency of a tile, whose exponentials (256 cycles) and products (256) wait
// for its queries with two waves on a SIMD: 32 rows each of four contexts of 8192 to 32768
// keys, the same heads, take 70 us where the keys take 17 and the products 21. (Queries
// that run two tiles ahead do not fit the registers and took 75.)
//
// A wave goes through all rows of its keys' sequence: tiles that see none of them are
// multiplied, too, and their weights masked. So all 4096 rows of a prompt take 0.95 ms with
// a window of 512 as without, and 2048 rows beside 250 single tokens take 7.5 ms, as work is
// shared out by keys alone.
#include <algorithm>

#include "device_common.h"
#include "kv.h"
#include "kv_codes.h"

namespace semsched {

namespace {

constexpr int WW = 8;       // waves of a workgroup, one of which fills a compute unit
constexpr int kChunk = 64;  // keys of a wave
constexpr int kRows = 16;   // of a tile
typedef float float4_t __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));

// A listed sequence: its rows, keys and the chunks of 64 keys that its rows see.
// (units: of those chunks, what work goes by)
struct Seen {
  int32_t row0, fresh, slot, len, c0, c1;
  uint32_t units;
};

// (`bad` where the cache cannot hold it; it then counts as empty)
__device__ __forceinline__ Seen seen_of(const KvWeighArgs& a, int64_t i, bool& bad) {
  const KvView& c = a.c;
  Seen s = {0, 0, 0, 0, 0, 0, 0};
  if (i >= a.n) return s;
  const int64_t row0 = a.cu ? a.cu[i] : i;
  const int64_t fresh = a.cu ? (int64_t)a.cu[i + 1] - row0 : 1;
  const int32_t slot = a.seqs[i];
  const bool known = (uint32_t)slot < (uint32_t)c.slots;
  const int64_t len = known ? c.lens[slot] : -1;
  if (fresh < 0 || row0 < 0 || row0 + fresh > a.tokens || len < 0 ||
      len > ((int64_t)c.max_blocks << c.page_shift) || (len > 0 && c.num_pages == 0)) {
    bad = true;
    return s;
  }
  if (fresh == 0 || len == 0) return s;
  s.row0 = (int)row0;
  s.fresh = (int)fresh;
  s.slot = slot;
  s.len = (int)len;
  const int64_t first = len - fresh;  // position of the first row
  const int64_t low = a.window > 0 && first >= a.window ? first + 1 - a.window : 0;
  s.c0 = (int)(low / kChunk);
  s.c1 = (int)((len + kChunk - 1) / kChunk);
  s.units = (uint32_t)(s.c1 - s.c0);
  return s;
}

__device__ __forceinline__ Seen lane_seen(const Seen& s, int lane) {
  auto get = [&](int32_t v) { return __builtin_amdgcn_readlane(v, lane); };
  return {get(s.row0), get(s.fresh), get(s.slot), get(s.len),
          get(s.c0), get(s.c1), (uint32_t)get((int32_t)s.units)};
}

// Sixteen codes as two operands of the queries' type.
template <int FMT>
__device__ __forceinline__ void operands(uint4 w, half8_t& lo, half8_t& hi) {
  codes_to_operands<FMT>(w, lo, hi);
}
template <int FMT>
__device__ __forceinline__ void operands(uint4 w, bf16x8_t& lo, bf16x8_t& hi) {
  uint32_t p[8];
  codes_to_bf16<FMT>(w.x, p[0], p[1]);
  codes_to_bf16<FMT>(w.y, p[2], p[3]);
  codes_to_bf16<FMT>(w.z, p[4], p[5]);
  codes_to_bf16<FMT>(w.w, p[6], p[7]);
  lo = __builtin_bit_cast(bf16x8_t, make_uint4(p[0], p[1], p[2], p[3]));
  hi = __builtin_bit_cast(bf16x8_t, make_uint4(p[4], p[5], p[6], p[7]));
}
__device__ __forceinline__ float4_t product(half8_t a, half8_t b, float4_t c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ float4_t product(bf16x8_t a, bf16x8_t b, float4_t c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// A lane's row: its token and its head in the group, 16 rows further each time.
struct Row {
  uint32_t at, token, head;
  __device__ __forceinline__ Row(uint32_t r, uint32_t group)
      : at(r), token(r / group), head(r % group) {}
  __device__ __forceinline__ void next(uint32_t tokens, uint32_t heads, uint32_t group) {
    at += kRows;
    token += tokens;
    head += heads;
    if (head >= group) {
      head -= group;
      ++token;
    }
  }
};

// The sums of sixteen numbers over the sixteen lanes of a group: lane r gets the r-th. In
// each step a lane gives half of its numbers away and adds what it gets to the others.
template <int OFF>
__device__ __forceinline__ void halve(float (&x)[16], int r) {
  const bool upper = (r & OFF) != 0;
#pragma unroll
  for (int k = 0; k < OFF; ++k) {
    const float give = upper ? x[k] : x[k + OFF], keep = upper ? x[k + OFF] : x[k];
    x[k] = keep + __shfl_xor(give, OFF, kWave);
  }
}
__device__ __forceinline__ float sum_of_rows(float (&x)[16], int r) {
  halve<8>(x, r);
  halve<4>(x, r);
  halve<2>(x, r);
  halve<1>(x, r);
  return x[0];
}

// Whether a sequence is listed twice, which all workgroups find alike: its rows would be
// added to the same sums at once. The list marks its sequences' bits, some sequences at a
// time where there are very many. (Eight contexts of 4096 keys take 11.6 us with it, 11.1
// without; 251 ragged requests 41.2 and 40.9, 1024 73 and 74.)
constexpr int kBits = 1 << 17;
__device__ __forceinline__ bool listed_twice(const KvWeighArgs& a, uint32_t* bits, uint32_t* any) {
  if (a.n < 2) return false;
  constexpr int kThreads = WW * kWave;
  const uint32_t slots = (uint32_t)a.c.slots;
  if (threadIdx.x == 0) *any = 0;
  for (uint32_t base = 0; base < slots; base += kBits) {
    const uint32_t here = min(slots - base, (uint32_t)kBits);
    for (uint32_t k = threadIdx.x; k < (here + 31) / 32; k += kThreads) bits[k] = 0;
    block_sync();
    for (int64_t i = threadIdx.x; i < a.n; i += kThreads) {
      const uint32_t at = (uint32_t)a.seqs[i] - base;  // (others are not below `here`)
      if (at < here && (atomicOr(&bits[at / 32], 1u << (at % 32)) >> (at % 32) & 1)) *any = 1;
    }
    block_sync();
  }
  return *any != 0;
}

// Where a wave is on the line of units (64 keys of a sequence each, all heads).
struct Cursor {
  Seen s;
  int64_t index;
  uint32_t unit;  // of the sequence
  uint64_t u;     // of the line
  __device__ __forceinline__ int chunk() const { return s.c0 + (int)unit; }
  __device__ __forceinline__ void advance(const KvWeighArgs& a, uint64_t stop) {
    if (++u >= stop) return;
    ++unit;
    bool bad;  // (has been looked at)
    while (unit >= s.units) {
      if (++index >= a.n) {  // (lengths that change meanwhile end no later)
        u = stop;
        return;
      }
      unit = 0;
      s = lane_seen(seen_of(a, index, bad), 0);
    }
  }
};

// The waves of a team: the more, the shorter the piece that ends last, but each round of
// units has a join, which takes about half as long as a head. One token each, 32 heads on
// 8 of 128 channels, teams of 1, 2, 4, 8 waves: a context of 777 keys 20, 13, 9, 8 us;
// eight of 4096 20, 14, 11, 12 us; 251 of 16 to 4096 45, 41, 45, 50 us; 256 of 4096 204,
// 217, 236, 272 us.
__device__ __forceinline__ int team_of(uint64_t units, uint32_t waves, uint32_t heads) {
  uint32_t least = 0xffffffffu;
  int best = 1;
  if (units >= 16ull * waves) return best;  // (many rounds: their number is about the same)
  for (uint32_t share = 1; share <= WW && share <= heads; share *= 2) {
    const uint32_t teams = waves / share, rounds = ((uint32_t)units + teams - 1) / teams;
    const uint32_t cost = rounds * (2 * ((heads + share - 1) / share) + 1);
    if (cost < least) {
      best = (int)share;
      least = cost;
    }
  }
  return best;
}

// The line is cut into equal pieces of neighbours, one for each team of waves; a team's
// waves share the heads of its units and join through LDS. Loads run ahead: page numbers
// two units, codes one head or unit, queries one tile.
//
// FEW: for one tile of rows a sequence (any number is right): 16 keys at a time are
// turned into operands and used. Otherwise all 64 are, once for all tiles. (One token of
// each of 256 contexts of 4096 keys 204 us instead of 214.)
template <int D, int FMT, bool BF16, bool FEW>
__global__ __launch_bounds__(WW* kWave, 2) void kv_weigh(KvWeighArgs a) {
  using Operand = std::conditional_t<BF16, bf16x8_t, half8_t>;
  constexpr int N = D / 32;         // operands of a row or key
  constexpr bool AHEAD = D <= 128;  // (the registers hold no more codes of 256 channels)
  __shared__ float sums[2][WW][kChunk];
  __shared__ uint32_t bits[kBits / 32], any;
  const KvView& c = a.c;
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int r = lane % 16, g = lane / 16;
  if (a.cu && blockIdx.x == 0 && threadIdx.x == 0 && (a.cu[0] != 0 || a.cu[a.n] != a.tokens))
    atomicOr(c.flags, kFlagInval);
  if (listed_twice(a, bits, &any)) {
    if (blockIdx.x == 0 && threadIdx.x == 0) atomicOr(c.flags, kFlagInval);
    return;
  }
  // The units of all sequences, 64 at a time; the first ones' are kept for the search. (64,
  // 256 or 512 of them: a context of 777 keys 8.0, 8.4, 8.7 us; 251 ragged requests 41 each,
  // 4096 of 64 keys 119, 119, 113.)
  constexpr int kKept = 4;
  uint32_t units[kKept];
  bool bad = false;
#pragma unroll
  for (int k = 0; k < kKept; ++k) units[k] = seen_of(a, k * kWave + lane, bad).units;
  uint64_t total = 0;
#pragma unroll
  for (int k = 0; k < kKept; ++k) total += wave_add_u32(units[k]);
  for (int64_t at = kKept * kWave; at < a.n; at += kWave)
    total += wave_add_u32(seen_of(a, at + lane, bad).units);
  if (__ballot(bad) && blockIdx.x == 0 && lane == 0) atomicOr(c.flags, kFlagInval);
  const int share = team_of(total, gridDim.x * WW, (uint32_t)c.kv_heads);
  const int head_slot = wave % share;
  const uint64_t teams = (uint64_t)gridDim.x * (WW / share);
  const uint64_t self = (uint64_t)blockIdx.x * (WW / share) + wave / share;
  const uint64_t stop = total * (self + 1) / teams;
  // (all teams of a workgroup go through as many rounds)
  const uint32_t rounds = (uint32_t)((total + teams - 1) / teams);
  Cursor now = {{}, 0, 0, total * self / teams};
  if (now.u < stop) {
    uint64_t before = 0;
    // whether the piece starts among 64 sequences from `at` on
    auto starts = [&](int64_t at, uint32_t mine) __attribute__((always_inline)) {
      const uint32_t upto = wave_incl_scan_u32(mine);
      const uint64_t beyond = __ballot(before + upto > now.u);
      if (beyond) {
        const int first = __ffsll((unsigned long long)beyond) - 1;
        now.index = at + first;
        now.unit = (uint32_t)(now.u - before -
                              (uint32_t)__builtin_amdgcn_readlane((int)(upto - mine), first));
      }
      before += (uint32_t)__builtin_amdgcn_readlane((int)upto, kWave - 1);
      return beyond != 0;
    };
    bool found = false;
#pragma unroll
    for (int k = 0; k < kKept; ++k)
      if (!found) found = starts(k * kWave, units[k]);
    for (int64_t at = kKept * kWave; !found && at < a.n; at += kWave)
      found = starts(at, seen_of(a, at + lane, bad).units);
    if (found) now.s = lane_seen(seen_of(a, now.index, bad), 0);
    if (now.unit >= now.s.units) now.u = stop;  // (lengths that change meanwhile)
  }
  const int64_t block_bytes = (int64_t)c.page_tokens * D;
  const int in_page = c.page_tokens - 1;
  const uint32_t group = (uint32_t)a.group, step_tokens = kRows / group, step_heads = kRows % group;
  const Row first_row(r, group);
  bool wrong = false;

  // The pages of a unit: of this lane's K rows, and of its 16 keys.
  struct Entries {
    int32_t k, v;
  };
  auto entries = [&](const Cursor& at) __attribute__((always_inline)) {
    const int32_t* table = c.tables + (int64_t)at.s.slot * c.max_blocks;
    const int t0 = at.chunk() * kChunk, last_block = (at.s.len - 1) >> c.page_shift;
    return Entries{table[min((t0 + r / 4 * kKvTile) >> c.page_shift, last_block)],
                   table[min((t0 + g * kKvTile) >> c.page_shift, last_block)]};
  };
  const uint8_t* keys = nullptr;  // of the unit whose codes are loaded
  const float* scale = nullptr;
  auto find = [&](const Cursor& at, Entries e) __attribute__((always_inline)) {
    const bool bad =
        (uint32_t)e.k >= (uint64_t)c.num_pages || (uint32_t)e.v >= (uint64_t)c.num_pages;
    wrong |= bad;
    scale = c.scale + ((int64_t)(bad ? 0 : e.v) * c.layers + a.layer) * 2 * c.kv_heads;
    keys = c.data + (bad ? 0 : e.k) * c.page_bytes +
           (int64_t)a.layer * 2 * c.kv_heads * block_bytes +
           ((at.chunk() * kChunk + r / 4 * kKvTile) & in_page) * D + (r % 4) * 16 + g * 256;
  };
  uint4 raw[4][D / 64];
  float ks = 0.0f;
  auto load = [&](int kh) __attribute__((always_inline)) {
    ks = scale[kh];
#pragma unroll
    for (int x = 0; x < 4; ++x)
#pragma unroll
      for (int j = 0; j < D / 64; ++j)
        raw[x][j] = *reinterpret_cast<const uint4*>(keys + kh * block_bytes + x * 64 + j * 1024);
  };
  uint4 asked[N];
  float lse = 0.0f;
  auto ask = [&](const Seen& s, int kh, const Row& row, uint32_t rows)
      __attribute__((always_inline)) {
    const bool there = row.at < rows;  // (else the sequence's first)
    const int64_t token = s.row0 + (there ? row.token : 0u);
    const int head = kh * a.group + (int)(there ? row.head : 0u);
    const uint16_t* q = a.q + token * a.q_token + head * a.q_head + g * 16;
    lse = a.lse[token * a.heads + head];
#pragma unroll
    for (int j = 0; j < N; ++j)  // (rows need not be 16-byte aligned)
      __builtin_memcpy(&asked[j], q + j / 2 * 64 + j % 2 * 8, 16);
  };
  Cursor next = now;
  Entries ahead = {0, 0};
  if (now.u < stop) {
    find(now, entries(now));
    if (AHEAD) load(head_slot);
    next.advance(a, stop);
    if (next.u < stop) ahead = entries(next);
  }
  for (uint32_t round = 0; round < rounds; ++round) {
    float sum[16];
#pragma unroll
    for (int k = 0; k < 16; ++k) sum[k] = 0.0f;
    const bool live = now.u < stop;
    const Seen s = now.s;
    const int t0 = now.chunk() * kChunk, vt = t0 + g * kKvTile;
    float* const mass = a.mass + s.slot * a.mass_stride + min(t0 + lane, max(s.len, 1) - 1);
    float was = 0.0f;
    if (live && head_slot == 0) was = *mass;
    if (live) {
      const uint32_t rows = (uint32_t)s.fresh * group;
      for (int kh = head_slot; kh < c.kv_heads; kh += share) {
        Row row = first_row;
        if (!AHEAD) load(kh);
        ask(s, kh, row, rows);
        uint4 codes[4][D / 64];
        Operand key[FEW ? 1 : 4][N];
        const float f = ks * a.scale_log2;
#pragma unroll
        for (int x = 0; x < 4; ++x)
#pragma unroll
          for (int j = 0; j < D / 64; ++j) {
            if (FEW) codes[x][j] = raw[x][j];
            else operands<FMT>(raw[x][j], key[FEW ? 0 : x][2 * j], key[FEW ? 0 : x][2 * j + 1]);
          }
        if (kh + share < c.kv_heads) {
          if (AHEAD) load(kh + share);
        } else if (next.u < stop) {
          find(next, ahead);
          if (AHEAD) load(head_slot);
        }
        for (; row.at - r < rows;) {
          Operand query[N];
#pragma unroll
          for (int j = 0; j < N; ++j) query[j] = __builtin_bit_cast(Operand, asked[j]);
          // Rows that see no key, are not numbers, or are not there weigh nothing.
          const bool counts = row.at < rows && fabsf(lse) < __builtin_inff();
          const float base = lse * 1.4426950408889634f;
          const int pos = s.len - s.fresh + (int)row.token;
          const int seen = a.causal ? min(pos + 1, s.len) : s.len, high = counts ? seen : 0;
          const int low = a.window > 0 && pos >= a.window ? pos + 1 - a.window : 0;
          const bool hides = __ballot(low > t0 || high < t0 + kChunk) != 0;
          row.next(step_tokens, step_heads, group);
          if (!FEW) ask(s, kh, row, rows);  // (behind the last row: the first one again)
          float4_t t[4];
#pragma unroll
          for (int x = 0; x < 4; ++x) t[x] = float4_t{0.0f, 0.0f, 0.0f, 0.0f};
          if (FEW) {
#pragma unroll
            for (int x = 0; x < 4; ++x) {
#pragma unroll
              for (int j = 0; j < D / 64; ++j)
                operands<FMT>(codes[x][j], key[0][2 * j], key[0][2 * j + 1]);
#pragma unroll
              for (int j = 0; j < N; ++j) t[x] = product(key[0][j], query[j], t[x]);
            }
          } else {
#pragma unroll
            for (int j = 0; j < N; ++j)
#pragma unroll
              for (int x = 0; x < 4; ++x) t[x] = product(key[FEW ? 0 : x][j], query[j], t[x]);
          }
          float p[16];
#pragma unroll
          for (int k = 0; k < 16; ++k)
            p[k] = __builtin_amdgcn_exp2f(__builtin_fmaf(t[k / 4][k % 4], f, -base));
          if (hides) {
            asm volatile("");  // (a branch: selects in every tile would cost more)
#pragma unroll
            for (int k = 0; k < 16; ++k) p[k] = vt + k >= low && vt + k < high ? p[k] : 0.0f;
          }
#pragma unroll
          for (int k = 0; k < 16; ++k) sum[k] += p[k];
          if (FEW && row.at - r < rows) ask(s, kh, row, rows);
        }
      }
    }
    now = next;
    next.advance(a, stop);
    if (next.u < stop) ahead = entries(next);
    // the sixteen lanes of a group each hold other rows: lane r gets key r's sum
    const float whole = sum_of_rows(sum, r);
    float (&joined)[WW][kChunk] = sums[round & 1];  // (the other may still be read)
    if (share > 1) {
      if (head_slot > 0) joined[wave][lane] = whole;
      block_sync();
    }
    if (live && head_slot == 0) {
      float x = whole;
      for (int k = 1; k < share; ++k) x += joined[wave + k][lane];
      if (t0 + lane < s.len) *mass = was + x;
    }
  }
  if (__ballot(wrong) && lane == 0) atomicOr(c.flags, kFlagInval);
}

template <int D, int FMT, bool BF16>
void launch_rows(const KvWeighArgs& a, bool few, unsigned grid, hipStream_t st) {
  if (few)
    hipLaunchKernelGGL((kv_weigh<D, FMT, BF16, true>), dim3(grid), dim3(WW * kWave), 0, st, a);
  else
    hipLaunchKernelGGL((kv_weigh<D, FMT, BF16, false>), dim3(grid), dim3(WW * kWave), 0, st, a);
}

template <int D, int FMT>
void launch_type(const KvWeighArgs& a, bool few, unsigned grid, hipStream_t st) {
  if (a.bf16) launch_rows<D, FMT, true>(a, few, grid, st);
  else launch_rows<D, FMT, false>(a, few, grid, st);
}

template <int D>
void launch_dim(const KvWeighArgs& a, bool few, unsigned grid, hipStream_t st) {
  if (a.c.format == SEM_KV_INT8) launch_type<D, SEM_KV_INT8>(a, few, grid, st);
  else launch_type<D, SEM_KV_FP8>(a, few, grid, st);
}

}  // namespace

hipError_t launch_kv_weigh(const KvWeighArgs& args, int64_t max_new, int64_t max_len,
                           hipStream_t st) {
  if (args.n == 0) return hipSuccess;  // (without tokens the offsets are looked at)
  KvWeighArgs a = args;
  const bool few = max_new * a.group <= kRows;
  const int64_t units = std::max<int64_t>(1, a.n * ((max_len + kChunk - 1) / kChunk));
  constexpr int64_t kGroups = 256;
  const int64_t waves = units * std::min<int64_t>(WW, a.c.kv_heads);
  const unsigned grid = (unsigned)std::min<int64_t>(kGroups, (waves + WW - 1) / WW);
  switch (a.c.head_dim) {
    case 64: launch_dim<64>(a, few, grid, st); break;
    case 128: launch_dim<128>(a, few, grid, st); break;
    default: launch_dim<256>(a, few, grid, st);
  }
  return hipGetLastError();
}

}  // namespace semsched
