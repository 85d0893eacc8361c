// Attention of new tokens over the 8-bit KV cache.
//
// For a query row q (a token and a head) and the keys j that it sees, with the
// 8-bit codes kc, vc and the scales ks, vs of their pages' blocks:
//
//   x_j = scale * ks_j * (q . kc_j),  m = max x_j,  l = sum exp(x_j - m)
//   o   = (1 / l) sum exp(x_j - m) vs_j vc_j,       lse = m + log l
//
// in one pass over the keys with a running m, l and o in 32 bits. Both products
// run on the matrix cores in half precision with 32-bit sums: codes are exact
// there, and so are the queries (a bf16 row is first multiplied by a power of
// two that brings its largest element to 2^14, which is undone in the scale).
// The weights exp(x - m) vs are rounded to half precision relative to the
// largest vs of the keys that the row has seen, 2^6 above, so that weights down to
// 2^-20 of the largest keep 11 bits and smaller ones lose at most 2^-31 of it. Sums,
// maxima and outputs are in 32 bits.
#include <algorithm>
#include <cstdlib>

#include "device_common.h"
#include "kv.h"
#include "kv_codes.h"

namespace semsched {

namespace {

typedef float float4_t __attribute__((ext_vector_type(4)));

constexpr int kRows = 16;            // rows of a tile: a token and a head each
constexpr int kChunk = 64;           // keys a wave takes at a time
constexpr float kLift = 64.0f;       // 2^6
constexpr float kNone = -__builtin_inff();
// What the largest V scale met starts from, the least normal number: the
// reciprocal of a smaller one is not finite, and blocks of such scales (of values
// below 3.7e-37) count relative to this one.
constexpr float kLeastScale = 0x1p-126f;
constexpr int kMostParts = 128;      // of the key axis
// The running maximum is raised only when a score passes it by this much (in
// powers of two), which is seldom: most steps then need no rescaling of the
// outputs. Weights stay below kLift * 2^kSlack, which half precision holds.
constexpr float kSlack = 8.0f;

struct Sequence {
  const int32_t* table;
  int64_t row0;           // first query token
  int index, fresh, len;  // its number in the call, query tokens, keys
};

// The sequence of row tile u (all but its keys) and the tile's number in it;
// false if there is no such tile. Tiles are numbered sequence by sequence. The
// grid's size is a bound, and its workgroups without work have to be the last
// ones: the device deals workgroups to its parts in turn, and idle ones at
// regular places would leave the same parts without work. So every wave counts
// the tiles of all sequences, 64 at a time (n / 64 rounds of independent loads,
// where a search would take log n dependent ones).
__device__ __forceinline__ bool find_tile(const KvAttendArgs& a, uint32_t u, int rows, Sequence& q,
                                          int& tile) {
  const KvView& c = a.c;
  int64_t i = -1;
  if (a.cu) {
    const int lane = lane_id();
    uint32_t before = 0;
    for (int64_t at = 0; at < a.n; at += kWave) {
      uint32_t mine = 0;
      if (at + lane < a.n) {
        const int64_t fresh = (int64_t)a.cu[at + lane + 1] - a.cu[at + lane];
        if (fresh > 0 && fresh <= a.tokens) mine = (uint32_t)((fresh * a.group + rows - 1) / rows);
      }
      const uint32_t upto = before + wave_incl_scan_u32(mine);
      const uint64_t beyond = __ballot(upto > u);
      if (beyond) {
        const int first = __ffsll((unsigned long long)beyond) - 1;
        i = at + first;
        tile = (int)u - __builtin_amdgcn_readlane((int)(upto - mine), first);
        break;
      }
      before = (uint32_t)__builtin_amdgcn_readlane((int)upto, kWave - 1);
    }
    if (blockIdx.x == 0 && (a.cu[0] != 0 || a.cu[a.n] != a.tokens) && threadIdx.x == 0)
      atomicOr(c.flags, kFlagInval);
    if (i < 0) return false;
  } else {
    const uint32_t each = (uint32_t)(a.group + rows - 1) / (uint32_t)rows;
    i = u / each;
    tile = (int)(u % each);
  }
  q.row0 = a.cu ? a.cu[i] : i;
  const int64_t fresh = a.cu ? (int64_t)a.cu[i + 1] - q.row0 : 1;
  if (fresh < 0 || q.row0 < 0 || q.row0 + fresh > a.tokens) {
    if (threadIdx.x == 0) atomicOr(c.flags, kFlagInval);
    return false;
  }
  q.fresh = (int)fresh;
  q.index = (int)i;
  return true;
}

// The sequence's keys; none if the cache cannot hold them.
__device__ __forceinline__ void find_keys(const KvAttendArgs& a, Sequence& q) {
  const KvView& c = a.c;
  const int32_t s = a.seqs[q.index];
  const bool known = (uint32_t)s < (uint32_t)c.slots;
  q.table = c.tables + (known ? (int64_t)s * c.max_blocks : 0);
  q.len = known ? c.lens[s] : -1;
  if (q.len < 0 || (int64_t)q.len > ((int64_t)c.max_blocks << c.page_shift) ||
      (q.len > 0 && c.num_pages == 0)) {
    if (threadIdx.x == 0) atomicOr(c.flags, kFlagInval);
    q.len = 0;
  }
}

// Keys [low, high) that query token i of the sequence sees.
__device__ __forceinline__ void visible(const KvAttendArgs& a, const Sequence& q, int i, int& low,
                                        int& high) {
  const int pos = q.len - q.fresh + i;
  high = a.causal ? max(min(pos + 1, q.len), 0) : q.len;
  // (a negative position less a large window passes 32 bits)
  low = a.window > 0 && pos >= a.window ? pos + 1 - a.window : 0;
}

// Parts that chunks [c0, c1) of the keys are split into, of equal sizes (larger
// ones where the caller's bound on the length does not hold).
__device__ __forceinline__ int parts_of(const KvAttendArgs& a, int c0, int c1) {
  return max(1, min((c1 - c0 + a.part_chunks - 1) / a.part_chunks, a.parts));
}
__device__ __forceinline__ int part_start(int c0, int c1, int parts, int part) {
  return c0 + (int)((uint32_t)max(c1 - c0, 0) * (uint64_t)part / (uint32_t)parts);
}

// Two values in the outputs' type, rounded to the nearest.
template <bool BF16>
__device__ __forceinline__ uint32_t pack_pair(float x, float y) {
  const float2_t v = {x, y};
  if (BF16) {
    typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2_t));
  }
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, half2_t));
}
__device__ __forceinline__ uint32_t pack_pair(float x, float y, int bf16) {
  return bf16 ? pack_pair<true>(x, y) : pack_pair<false>(x, y);
}

// A row's query, as the lane's D / (8 G) operands of eight: of G = 4 lane groups,
// group g holds channels (4 j + g) * 16 .. + 15 in operands 2 j and 2 j + 1; of
// G = 2, channels 16 j + 8 g .. + 7 in operand j. Loaded first, so that finding
// the keys and their pages takes place meanwhile.
template <int D, int G>
struct Query {
  static constexpr int N = D / (8 * G);
  uint16_t e[N][8];

  __device__ __forceinline__ void load(const KvAttendArgs& a, const uint16_t* row, int g) {
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const uint16_t* p = row + (G == 4 ? (4 * (j / 2) + g) * 16 + j % 2 * 8 : 16 * j + 8 * g);
      if (a.wide) {
        *reinterpret_cast<uint4*>(e[j]) = *reinterpret_cast<const uint4*>(p);
      } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) e[j][k] = p[k];
      }
    }
  }

  // In halves. Returns what the scores have to be multiplied by, which is not
  // negative (a negative scale changes the query's sign).
  __device__ __forceinline__ float convert(const KvAttendArgs& a, half8_t (&q)[N]) const {
    const float sign = a.scale_log2 < 0.0f ? -1.0f : 1.0f;
    float up = 1.0f, undo = 1.0f;
    if (a.bf16) {
      float top = 0.0f;
#pragma unroll
      for (int j = 0; j < N; ++j)
#pragma unroll
        for (int k = 0; k < 8; ++k) top = fmaxf(top, fabsf(load16(e[j][k], 1)));
      if (G == 4) top = fmaxf(top, __shfl_xor(top, 16, kWave));
      top = fmaxf(top, __shfl_xor(top, 32, kWave));
      // 2^(14 - exponent), between 2^-126 and 2^126; rows of zeros or with an
      // infinity stay as they are
      const int e2 = (int)(__float_as_uint(top) >> 23);
      const int shift = top > 0.0f && e2 < 255 ? min(max(14 - (e2 - 127), -126), 126) : 0;
      up = __uint_as_float((uint32_t)(127 + shift) << 23);
      undo = __uint_as_float((uint32_t)(127 - shift) << 23);
    }
#pragma unroll
    for (int j = 0; j < N; ++j)
#pragma unroll
      for (int k = 0; k < 8; ++k) q[j][k] = (_Float16)(load16(e[j][k], a.bf16) * (up * sign));
    return undo * fabsf(a.scale_log2);
  }
};

// Sixteen codes as two operands of eight halves.
template <int FMT>
__device__ __forceinline__ void codes_to_operands(uint4 w, half8_t& lo, half8_t& hi) {
  half2_t p[8];
  codes_to_half<FMT>(w.x, p[0], p[1]);
  codes_to_half<FMT>(w.y, p[2], p[3]);
  codes_to_half<FMT>(w.z, p[4], p[5]);
  codes_to_half<FMT>(w.w, p[6], p[7]);
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    lo[2 * k] = p[k][0];
    lo[2 * k + 1] = p[k][1];
    hi[2 * k] = p[4 + k][0];
    hi[2 * k + 1] = p[4 + k][1];
  }
}

// Zeroes the codes from the n-th on.
__device__ __forceinline__ uint32_t keep_bytes(uint32_t w, int n) {
  return n >= 4 ? w : n <= 0 ? 0u : w & ((1u << (8 * n)) - 1u);
}

// The value of the lane 32 away.
__device__ __forceinline__ float other_half(float x) {
  const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false,
                                                  false);
  return __uint_as_float(lane_id() < 32 ? p[1] : p[0]);
}

// Writes a row that is joined: a lane holds D / 64 channels, not divided by the
// sum yet.
template <int D>
__device__ __forceinline__ void finish_row(const KvAttendArgs& a, int64_t token, int64_t head,
                                           float most, float total, const float (&o)[D / 64]) {
  constexpr int W = D / 64;
  const bool some = total > 0.0f || total != total;
  const float inv = some ? 1.0f / total : 0.0f;
  uint16_t* out = a.out + token * a.out_token + head * a.out_head + lane_id() * W;
#pragma unroll
  for (int j = 0; j < W; j += 2) {
    const uint32_t p = pack_pair(o[j] * inv, W > 1 ? o[(j + 1) % W] * inv : 0.0f, a.bf16);
    if (W == 1) {
      out[0] = (uint16_t)p;
    } else if (a.wide_out) {
      *reinterpret_cast<uint32_t*>(out + j) = p;
    } else {
      out[j] = (uint16_t)p;
      out[j + 1] = (uint16_t)(p >> 16);
    }
  }
  if (a.lse && lane_id() == 0)
    a.lse[token * a.heads + head] =
        some ? (most + __builtin_amdgcn_logf(total)) * 0.6931471805599453f : kNone;
}

// Joins a row's parts with one wave. They were written by workgroups of this
// kernel, and are read past the L2 caches.
template <int D>
__device__ __forceinline__ void join_row(const KvAttendArgs& a, int64_t token, int64_t head,
                                         int parts) {
  constexpr int W = D / 64;
  const int64_t all = a.tokens * a.heads, at = token * a.heads + head;
  const int lane = lane_id();
  // lane k has parts k and k + 64
  static_assert(kMostParts == 2 * kWave, "two parts per lane");
  const int far = kWave + lane;
  const float* ml = a.part_ml + 2 * at;
  const float m0 = lane < parts ? load_agent(ml + 2 * lane * all) : kNone;
  const float l0 = lane < parts ? load_agent(ml + 2 * lane * all + 1) : 0.0f;
  const float m1 = far < parts ? load_agent(ml + 2 * far * all) : kNone;
  const float l1 = far < parts ? load_agent(ml + 2 * far * all + 1) : 0.0f;
  float most = fmaxf(m0, m1);
#pragma unroll
  for (int off = 32; off > 0; off /= 2) most = fmaxf(most, __shfl_xor(most, off, kWave));
  const float base = most == kNone ? 0.0f : most;
  const float w0 = __builtin_amdgcn_exp2f(m0 - base), w1 = __builtin_amdgcn_exp2f(m1 - base);
  float total = l0 * w0 + l1 * w1;
#pragma unroll
  for (int off = 32; off > 0; off /= 2) total += __shfl_xor(total, off, kWave);
  float o[W];
#pragma unroll
  for (int j = 0; j < W; ++j) o[j] = 0.0f;
  const float* from = a.part_o + at * D + lane * W;
#pragma unroll 8
  for (int k = 0; k < parts; ++k) {
    const float w = __shfl(k < kWave ? w0 : w1, k % kWave, kWave);
#pragma unroll
    for (int j = 0; j < W; ++j) o[j] += load_agent(from + k * all * D + j) * w;
  }
  finish_row<D>(a, token, head, most, total, o);
}

// Few rows. One workgroup: a tile of 16 rows of one KV head over one part of the
// key axis; its waves take chunks of 64 keys in turn and join at the end. The
// last part of a tile to finish joins the parts, in their order.
//
// The score product is taken as K q^T, so that a lane ends up with scores of
// one row (lane % 16) and of 16 consecutive keys (tile lane / 16 of the chunk),
// which is what the second product V^T P^T wants of it: weights go from one to
// the other in registers. The cache's tiles are laid out for these operands: a
// lane's 16-byte load is 16 channels of a key or 16 keys of a channel, and no
// LDS is used before the join. A lane's 16 keys lie in one page, so the scales
// are one number each per lane and chunk.
//
// Bound by reading the cache where contexts are long: four of 100001 to 131072
// tokens (64 heads, 8 KV heads, 128 channels) take 170 us, 5.6 TB/s; 251 ragged
// requests of 16 to 4096 tokens 86 us, 4.4 TB/s. A single token over 777 keys
// takes 10 us, most of it the launch and the chain of loads before the first
// product (the sequence, its length, its table, the page).
template <int D, int FMT, int NW>
__global__ __launch_bounds__(NW* kWave) void kv_attend_rows(KvAttendArgs a) {
  constexpr int PITCH = D + 4;
  constexpr int W = D / 64;  // channels of a lane in the joins
  __shared__ float join_o[NW][kRows][PITCH];
  __shared__ float join_m[NW][kRows], join_l[NW][kRows];
  __shared__ int last;
  const KvView& c = a.c;
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int r = lane % 16, g = lane / 16;
  // The workgroups behind the tiles look for offsets that fall, as a tile's own
  // search ends where it finds the tile.
  if (blockIdx.x >= a.tiles) {
    const int64_t pair = (int64_t)(blockIdx.x - a.tiles) * (NW * kWave) + threadIdx.x;
    if (blockIdx.y == 0 && pair < a.n && a.cu[pair + 1] < a.cu[pair])
      atomicOr(c.flags, kFlagInval);
    return;
  }
  // heads side by side: the dies take workgroups in turn, and so get an equal
  // share of every sequence
  const int kh = blockIdx.x % c.kv_heads;
  Sequence q;
  int tile;
  if (!find_tile(a, blockIdx.x / c.kv_heads, kRows, q, tile)) return;
  const int rows = q.fresh * a.group;
  const uint32_t row = (uint32_t)min(tile * kRows + r, rows - 1);
  const int token = (int)(row / (uint32_t)a.group);
  const int head = kh * a.group + (int)(row % (uint32_t)a.group);
  Query<D, 4> raw;
  raw.load(a, a.q + (q.row0 + token) * a.q_token + head * a.q_head, g);
  find_keys(a, q);
  int low, high;
  visible(a, q, token, low, high);
  // the keys that any row of the tile sees, and those that all see
  int from, to, all_from, all_to;
  visible(a, q, (int)((uint32_t)(tile * kRows) / (uint32_t)a.group), from, all_to);
  visible(a, q, (int)((uint32_t)(min(tile * kRows + kRows, rows) - 1) / (uint32_t)a.group),
          all_from, to);
  const int c0 = from / kChunk, c1 = (to + kChunk - 1) / kChunk;
  const int parts = parts_of(a, c0, c1), part = blockIdx.y;
  if (part >= parts) return;
  const int begin = part_start(c0, c1, parts, part), stop = part_start(c0, c1, parts, part + 1);

  float m = kNone, l = 0.0f, vref = kLeastScale;
  float4_t acc[D / 16];
#pragma unroll
  for (int y = 0; y < D / 16; ++y) acc[y] = float4_t{0.0f, 0.0f, 0.0f, 0.0f};
  const int64_t block_bytes = (int64_t)c.page_tokens * D;
  const int64_t k_off =
      ((int64_t)a.layer * 2 * c.kv_heads + kh) * block_bytes + (r % 4) * 16 + g * 256;
  const int64_t v_off =
      (((int64_t)a.layer * 2 + 1) * c.kv_heads + kh) * block_bytes + r * 16;
  const int in_page = c.page_tokens - 1;
  const int last_block = (q.len - 1) >> c.page_shift;
  bool wrong = false;
  auto checked = [&](int32_t entry) __attribute__((always_inline)) -> int64_t {
    const bool bad = (uint32_t)entry >= (uint32_t)c.num_pages;
    wrong |= bad;
    return bad ? 0 : entry;
  };
  // Loads run ahead: table entries two of this wave's chunks, then K (and the
  // scales) and V one, each as soon as the registers of the last are free. They
  // return in order, so the entries that the next loads wait for go first.
  int32_t kentry = 0, ventry = 0;  // of the pages of this lane's K rows and of its 16 keys
  uint4 kc[4][D / 64], vc[D / 16];
  float kscale = 0.0f, vscale = 0.0f;
  auto look_up = [&](int ch) __attribute__((always_inline)) {
    const int t0 = min(ch, stop - 1) * kChunk;
    kentry = q.table[min((t0 + r / 4 * kKvTile) >> c.page_shift, last_block)];
    ventry = q.table[min((t0 + g * kKvTile) >> c.page_shift, last_block)];
  };
  auto load_k = [&](int ch, int64_t kpage, int64_t vpage) __attribute__((always_inline)) {
    const float* sp = c.scale + (vpage * c.layers + a.layer) * 2 * c.kv_heads + kh;
    kscale = sp[0];
    vscale = sp[c.kv_heads];
    const uint8_t* kp = c.data + kpage * c.page_bytes + k_off +
                        ((ch * kChunk + r / 4 * kKvTile) & in_page) * D;
#pragma unroll
    for (int x = 0; x < 4; ++x)
#pragma unroll
      for (int j = 0; j < D / 64; ++j)
        kc[x][j] = *reinterpret_cast<const uint4*>(kp + x * 64 + j * 1024);
  };
  auto load_v = [&](int ch, int64_t vpage) __attribute__((always_inline)) {
    const uint8_t* vp = c.data + vpage * c.page_bytes + v_off +
                        ((ch * kChunk + g * kKvTile) & in_page) * D;
#pragma unroll
    for (int y = 0; y < D / 16; ++y) vc[y] = *reinterpret_cast<const uint4*>(vp + y * 256);
  };
  if (begin + wave < stop) {
    look_up(begin + wave);
    const int64_t kpage = checked(kentry), vpage = checked(ventry);
    look_up(begin + wave + NW);
    load_k(begin + wave, kpage, vpage);
    load_v(begin + wave, vpage);
  }
  half8_t query[D / 32];
  const float factor = raw.convert(a, query);
  for (int ch = begin + wave; ch < stop; ch += NW) {
    const int t0 = ch * kChunk, vt = t0 + g * kKvTile;
    const bool more = ch + NW < stop;
    // (not zero, so that a hidden key's minus infinity stays one)
    const float f = fmaxf(kscale * factor, 1e-30f);
    float vs = vscale;
    const int64_t kpage = checked(kentry), vpage = checked(ventry);
    look_up(ch + 2 * NW);
    float s[16];
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      float4_t t = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int j = 0; j < D / 64; ++j) {
        half8_t lo, hi;
        codes_to_operands<FMT>(kc[x][j], lo, hi);
        t = __builtin_amdgcn_mfma_f32_16x16x32_f16(lo, query[2 * j], t, 0, 0, 0);
        t = __builtin_amdgcn_mfma_f32_16x16x32_f16(hi, query[2 * j + 1], t, 0, 0, 0);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) s[4 * x + i] = t[i];
    }
    if (more) load_k(ch + NW, kpage, vpage);
    if (t0 < all_from || t0 + kChunk > all_to) {
      // keys that some rows do not see (whatever is held there)
#pragma unroll
      for (int k = 0; k < 16; ++k) s[k] = vt + k >= low && vt + k < high ? s[k] : kNone;
      if (vt >= high || vt + kKvTile <= low) vs = vref;  // the row sees none of these 16
      const int n = q.len - vt;
#pragma unroll
      for (int y = 0; y < D / 16; ++y) {
        vc[y].x = keep_bytes(vc[y].x, n);
        vc[y].y = keep_bytes(vc[y].y, n - 4);
        vc[y].z = keep_bytes(vc[y].z, n - 8);
        vc[y].w = keep_bytes(vc[y].w, n - 12);
      }
    }
    float top = s[0];
#pragma unroll
    for (int k = 1; k < 16; ++k) top = fmaxf(top, s[k]);
    top *= f;
    top = fmaxf(top, __shfl_xor(top, 16, kWave));
    top = fmaxf(top, other_half(top));
    // weights are relative to the largest V scale that the row has seen
    float vmax = fmaxf(vs, __shfl_xor(vs, 16, kWave));
    vmax = fmaxf(fmaxf(vmax, other_half(vmax)), vref);
    const float inv = __builtin_amdgcn_rcpf(vmax);
    const bool raise = top > m + kSlack;
    const float next = raise ? top : m;
    const float shrink = raise ? __builtin_amdgcn_exp2f(m - next) : 1.0f;
    const float fade = vmax > vref ? shrink * (vref * inv) : shrink;
    m = next;
    vref = vmax;
    l *= shrink;
    if (__ballot(fade != 1.0f)) {
#pragma unroll
      for (int y = 0; y < D / 16; ++y) acc[y] *= fade;
    }
    const float base = next == kNone ? 0.0f : next;  // no key so far: exp2(-inf) = 0
    const float rel = vs * inv * kLift;
    half8_t w[2];
#pragma unroll
    for (int k = 0; k < 16; ++k) {
      const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[k], f, -base));
      l += p;
      w[k / 8][k % 8] = (_Float16)(p * rel);
    }
#pragma unroll
    for (int y = 0; y < D / 16; ++y) {
      half8_t lo, hi;
      codes_to_operands<FMT>(vc[y], lo, hi);
      acc[y] = __builtin_amdgcn_mfma_f32_16x16x32_f16(lo, w[0], acc[y], 0, 0, 0);
      acc[y] = __builtin_amdgcn_mfma_f32_16x16x32_f16(hi, w[1], acc[y], 0, 0, 0);
    }
    if (more) load_v(ch + NW, vpage);
  }
  if (__ballot(wrong) && lane == 0) atomicOr(c.flags, kFlagInval);
  // the four lane groups of a row each hold a quarter of its sum
  l += __shfl_xor(l, 16, kWave);
  l += other_half(l);
  const int busy = max(min(stop - begin, NW), 0);  // waves that had keys
  if (wave < busy) {
    if (g == 0) {
      join_m[wave][r] = m;
      join_l[wave][r] = l;
    }
#pragma unroll
    for (int y = 0; y < D / 16; ++y) {
      const float4_t o = acc[y] * (1.0f / kLift) * vref;  // (their product may not be normal)
      *reinterpret_cast<float4_t*>(&join_o[wave][r][y * 16 + g * 4]) = o;
    }
  }
  block_sync();
  // a wave joins every NW-th row, a lane its W channels of it
  const int64_t all = a.tokens * a.heads;
  for (int i = wave; i < kRows; i += NW) {
    const int rr = tile * kRows + i;
    if (rr >= rows) break;
    float most = kNone;
    for (int w = 0; w < busy; ++w) most = fmaxf(most, join_m[w][i]);
    const float base = most == kNone ? 0.0f : most;
    float total = 0.0f, o[W];
#pragma unroll
    for (int j = 0; j < W; ++j) o[j] = 0.0f;
    for (int w = 0; w < busy; ++w) {
      const float e = __builtin_amdgcn_exp2f(join_m[w][i] - base);
      total += join_l[w][i] * e;
#pragma unroll
      for (int j = 0; j < W; ++j) o[j] += join_o[w][i][lane * W + j] * e;
    }
    const int64_t tok = q.row0 + (uint32_t)rr / (uint32_t)a.group;
    const int64_t hd = kh * a.group + (uint32_t)rr % (uint32_t)a.group;
    if (parts == 1) {
      finish_row<D>(a, tok, hd, most, total, o);
    } else {
      // past the L2 caches, for the part that joins: it may run on another die
      const int64_t at = (int64_t)part * all + tok * a.heads + hd;
#pragma unroll
      for (int j = 0; j < W; ++j) store_agent(a.part_o + at * D + lane * W + j, o[j]);
      if (lane == 0) {
        store_agent(a.part_ml + 2 * at, most);
        store_agent(a.part_ml + 2 * at + 1, total);
      }
    }
  }
  if (parts == 1) return;
  wait_stores();
  block_sync();
  if (threadIdx.x == 0) {
    uint32_t* count = a.counts + blockIdx.x;
    last = atomicAdd(count, 1u) == (uint32_t)parts - 1;
    if (last) store_agent(count, 0u);  // for the next call
  }
  block_sync();
  if (!last) return;
  for (int i = wave; i < kRows; i += NW) {
    const int rr = tile * kRows + i;
    if (rr >= rows) break;
    join_row<D>(a, q.row0 + (uint32_t)rr / (uint32_t)a.group,
                kh * a.group + (uint32_t)rr % (uint32_t)a.group, parts);
  }
}

// ---------------------------------------------------------------------------
// Many rows: tiles of NW * 32 rows of one KV head.
//
// A wave holds 32 rows (their queries and outputs in registers) and goes
// through the keys 32 at a time; the workgroup turns their codes into halves
// once and keeps them in LDS in operand order, so that every operand is one
// 16-byte LDS read without bank conflicts. As above, scores are taken as K q^T:
// a lane has the scores of one row (lane % 32) and, by the order in which keys
// are fed, of 16 consecutive keys, which the second product takes from
// registers.
//
// A step's instructions do not wait for each other: step j takes the scores of
// keys j + 1, the weights of keys j and the outputs of keys j - 1. Codes are loaded
// four steps ahead and put into LDS two steps ahead. (Six or eight steps ahead
// measured the same.)
//
// Bound by the matrix and vector instructions of a step, which still run almost
// one after the other: 16 matrix instructions (512 cycles) and about 150 vector
// ones (about 800, the 16 exponentials at a quarter of the rate) per wave and 32
// keys (128 channels), two waves on a SIMD that meet at a barrier each step. Of
// the cycles of a prompt of 16384 tokens (32 heads of 128 channels) matrix
// instructions take 42% and vector ones about 64%: 2.34 to 2.50 ms by card, 880 to
// 940 TFLOP/s, where a large matrix product reaches 1300; 6.07 ms where the three
// parts of a step depended on each other.
constexpr int kWide = 32;  // rows of a matrix tile, and keys of a step
typedef float float16_t __attribute__((ext_vector_type(16)));

// How the tiles are shared out. All of a call's work is laid out as one line: a
// KV head's tiles after the other's, sequence by sequence, each as long as the
// keys that it takes plus kTileCost for its start and end. The line is cut into
// equal pieces, one per workgroup (one of which fills a compute unit), wherever
// the cuts fall; tiles that are cut are joined afterwards. So no compute unit
// waits for another, whatever the sequences' lengths, and at most two partial
// tiles per workgroup are written. Chunks of 300 to 512 queries of four sequences
// of 2048 to 8192 keys (32 heads, 8 KV heads, 128 channels) take 118 us, of which
// the join 15; parts of equal length dealt out in turn took 160 us, as long as
// the longest of them.
// Whole tiles are dealt in turn instead where that costs less by the lines'
// lengths, as for equal sequences whose tiles go into the compute units without
// rest: 2048 rows each of four sequences over 4096 keys take 158 us, 195 us cut.
// Where there are tiles for six rounds (kWholeRounds) each has a workgroup of its
// own, which the device places as compute units become free: 64 such sequences
// take 2.49 ms, dealt in turn 2.60 ms, cut 2.66 ms; ragged ones (64 to 448
// queries, 512 to 8192 keys, about eight rounds) 1.03 ms in either way, and of
// four rounds 0.50 ms whole and 0.40 ms cut.
constexpr int kPieces = kKvPieces;
constexpr int kTileCost = 256;    // in keys; 256 to 448 measure alike
constexpr int kLeastPiece = 512;  // pieces are not cut shorter than this
constexpr int kCutCost = 640;     // of the cuts and the join, as keys of every piece
constexpr int kWholeRounds = 6;

// A sequence's share of the line: tile t is first + rise * (t + 1) long.
struct Share {
  uint64_t first;
  uint32_t tiles, rise;
  int32_t row0, fresh, slot, len;  // the sequence's first query, queries, place, keys
  __device__ __forceinline__ uint64_t before(uint32_t t) const {
    return t * first + (uint64_t)rise * ((uint64_t)t * (t + 1) / 2);
  }
  __device__ __forceinline__ uint64_t of(uint32_t t) const {
    return first + (uint64_t)rise * (t + 1);
  }
};

template <int ROWS>
__device__ __forceinline__ Share share_of(const KvAttendArgs& a, int64_t i) {
  const KvView& c = a.c;
  Share s = {1, 0, 0, 0, 0, 0, 0};
  if (i >= a.n) return s;
  const int64_t row0 = a.cu ? a.cu[i] : i;
  const int64_t fresh = a.cu ? (int64_t)a.cu[i + 1] - row0 : 1;
  const int32_t slot = a.seqs[i];
  const bool known = (uint32_t)slot < (uint32_t)c.slots;
  int64_t len = known ? c.lens[slot] : -1;
  s.row0 = (int)row0;
  s.fresh = (int)fresh;
  s.slot = known ? slot : 0;
  bool wrong = fresh < 0 || row0 < 0 || row0 + fresh > a.tokens;
  if (!wrong) s.tiles = (uint32_t)((fresh * a.group + ROWS - 1) / ROWS);
  if (len < 0 || len > ((int64_t)c.max_blocks << c.page_shift) ||
      (len > 0 && c.num_pages == 0)) {
    wrong |= s.tiles > 0;
    len = 0;
  }
  s.len = (int)len;
  if (wrong && blockIdx.x == 0) atomicOr(c.flags, kFlagInval);
  const uint32_t group = min((uint32_t)a.group, (uint32_t)ROWS);
  if (a.causal && a.window == 0) {
    len = max(len - fresh, (int64_t)0);
    s.rise = ROWS;
  } else if (a.window > 0) {
    len = min(len, (int64_t)a.window + ROWS / (int)group);
  }
  s.first = group * (uint64_t)(len + kTileCost);
  return s;
}

__device__ __forceinline__ uint64_t lane_u64(uint64_t v, int lane) {
  return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, lane) |
         (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32;
}

__device__ __forceinline__ Share lane_share(const Share& s, int lane) {
  auto get = [&](uint32_t v) { return __builtin_amdgcn_readlane((int)v, lane); };
  return {lane_u64(s.first, lane), (uint32_t)get(s.tiles), (uint32_t)get(s.rise), get(s.row0),
          get(s.fresh), get(s.slot), get(s.len)};
}

// A place on the line: the tile there, and where it starts.
struct Place {
  uint64_t start;
  Share share;
  int head, index;
  uint32_t tile;
};

template <int ROWS>
struct Line {
  uint64_t each = 0;  // length of a KV head's part
  uint64_t size, rest;  // of a piece; so many are one longer
  uint32_t tiles = 0;   // of a KV head
  uint32_t pieces;
  bool dealt;           // whole tiles are
  Share mine;  // of the lane's sequence among the first 64

  __device__ __forceinline__ bool measure(const KvAttendArgs& a) {
    const int lane = lane_id();
    const uint32_t group = (uint32_t)min(a.group, ROWS);
    uint32_t longest = 0;  // tile, in keys
    mine = share_of<ROWS>(a, lane);
    for (int64_t at = 0; at < a.n; at += kWave) {
      const Share s = at == 0 ? mine : share_of<ROWS>(a, at + lane);
      each += last_lane_u64(wave_incl_scan_u64(s.before(s.tiles)));
      tiles += wave_add_u32(s.tiles);
      longest = max(longest, s.tiles ? (uint32_t)(s.of(s.tiles - 1) / group) : 0u);
    }
    longest = wave_max_u32(longest);
    if (tiles == 0) return false;
    const uint64_t total = each * a.c.kv_heads;
    const uint64_t whole = (uint64_t)tiles * a.c.kv_heads, keys = total / group;
    dealt = a.whole || (whole + kPieces - 1) / kPieces * longest < keys / kPieces + kCutCost;
    pieces = (uint32_t)min(max(whole, keys / kLeastPiece), (uint64_t)kPieces);
    size = total / pieces;
    rest = total - size * pieces;
    return true;
  }
  __device__ __forceinline__ uint64_t cut(uint32_t g) const {
    return size * g + min((uint64_t)g, rest);
  }
  __device__ __forceinline__ uint32_t piece_of(uint64_t x) const {
    const uint64_t longer = rest * (size + 1);
    return (uint32_t)(x < longer ? x / (size + 1) : rest + (x - longer) / size);
  }
  __device__ __forceinline__ bool find(const KvAttendArgs& a, uint64_t x, Place& p) const {
    const int lane = lane_id();
    p.head = (int)(x / each);
    uint64_t start = p.head * each;
    for (int64_t at = 0; at < a.n; at += kWave) {
      const Share s = at == 0 ? mine : share_of<ROWS>(a, at + lane);
      const uint64_t own = s.before(s.tiles), upto = start + wave_incl_scan_u64(own);
      const uint64_t beyond = __ballot(upto > x);
      if (beyond) {
        const int at_lane = __ffsll((unsigned long long)beyond) - 1;
        p.index = (int)at + at_lane;
        p.share = lane_share(s, at_lane);
        start = lane_u64(upto - own, at_lane);
        uint32_t low = 0, high = p.share.tiles;  // before(low) <= x - start
        while (high - low > 1) {
          const uint32_t mid = (low + high) / 2;
          if (p.share.before(mid) <= x - start) low = mid;
          else high = mid;
        }
        p.tile = low;
        p.start = start + p.share.before(low);
        return true;
      }
      start = last_lane_u64(upto);
    }
    return false;
  }
  // Tile u of all, KV heads side by side and the line's last tiles first (the
  // later a causal tile, the more keys its rows see).
  __device__ __forceinline__ bool deal(const KvAttendArgs& a, uint64_t u, Place& p) const {
    p.head = (int)(u % (uint32_t)a.c.kv_heads);
    u /= (uint32_t)a.c.kv_heads;
    if (u >= tiles) return false;
    u = tiles - 1 - u;
    const int lane = lane_id();
    uint32_t before = 0;
    for (int64_t at = 0; at < a.n; at += kWave) {
      const Share s = at == 0 ? mine : share_of<ROWS>(a, at + lane);
      const uint32_t upto = before + wave_incl_scan_u32(s.tiles);
      const uint64_t beyond = __ballot(upto > u);
      if (beyond) {
        const int at_lane = __ffsll((unsigned long long)beyond) - 1;
        p.index = (int)at + at_lane;
        p.share = lane_share(s, at_lane);
        p.tile = (uint32_t)u - (uint32_t)__builtin_amdgcn_readlane((int)(upto - s.tiles), at_lane);
        p.start = 0;
        return true;
      }
      before = (uint32_t)__builtin_amdgcn_readlane((int)upto, kWave - 1);
    }
    return false;
  }
  // The next tile of the line; false behind its end.
  __device__ __forceinline__ bool next(const KvAttendArgs& a, Place& p) const {
    p.start += p.share.of(p.tile);
    if (++p.tile < p.share.tiles) return true;
    p.tile = 0;
    do {
      if (++p.index >= (int)a.n) {
        p.index = 0;
        if (++p.head >= a.c.kv_heads) return false;
      }
      p.share = lane_share(share_of<ROWS>(a, p.index), 0);
    } while (p.share.tiles == 0);
    return true;
  }
};

__device__ __forceinline__ Sequence sequence_of(const KvAttendArgs& a, const Place& p) {
  return {a.c.tables + (int64_t)p.share.slot * a.c.max_blocks, p.share.row0, p.index,
          p.share.fresh, p.share.len};
}

template <int D, int FMT, int NW>
__global__ __launch_bounds__(NW* kWave, NW / 4) void kv_attend_tile(KvAttendArgs a) {
  constexpr int NT = NW * kWave;
  constexpr int KS = D / 16;       // matrix steps of the score product
  constexpr int DY = D / 32;       // output tiles
  constexpr int UNITS = 4 * D;     // 16-byte units of a step's K and V
  constexpr int PER = UNITS > NT ? UNITS / NT : 1;  // of them per thread
  constexpr int ROWS = NW * kWide;
  static_assert(NT * PER % UNITS == 0, "whole rounds of units");
  // Two waves per SIMD hold everything in vector registers; one has to keep
  // outputs and queries in the accumulation registers.
  constexpr bool PINNED = NW == 4;
  constexpr int KEYS = 2 * KS * kWave;      // [buffer][step][lane]
  constexpr int VALS = 4 * 2 * DY * kWave;  // [buffer][8 keys of either half][tile][lane]
  constexpr int PITCH = D / 8 + 1;          // of an output row at the end
  constexpr int OUTS = ROWS * PITCH;
  __shared__ half8_t pool[KEYS + VALS > OUTS ? KEYS + VALS : OUTS];
  __shared__ float scales[4 * 4];  // [buffer][K tile 0, 1, V tile 0, 1]
  half8_t* const keys = pool;
  half8_t* const vals = pool + KEYS;
  const KvView& c = a.c;
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int r = lane % kWide, h = lane / kWide;
  if (!a.whole && threadIdx.x == 0) a.cuts[blockIdx.x].parts = 0;
  Line<ROWS> line;
  const bool any = line.measure(a);
  if (a.cu && blockIdx.x == 0 && threadIdx.x == 0 && (a.cu[0] != 0 || a.cu[a.n] != a.tokens))
    atomicOr(c.flags, kFlagInval);
  if (!any) return;
  // a die's workgroups (every eighth) take neighbouring pieces: the same KV head
  const uint32_t piece = line.pieces == kPieces
                             ? blockIdx.x % 8 * (kPieces / 8) + blockIdx.x / 8
                             : blockIdx.x;
  // One of a SIMD's two waves goes first, so that they drift into different halves
  // of a step (the chunks at kPieces 118 us, 125 us without).
  if (wave >= 4) __builtin_amdgcn_s_setprio(1);
  uint64_t turn = blockIdx.x, x0 = 0, x1 = 0;
  Place at;
  if (line.dealt) {
    if (!line.deal(a, turn, at)) return;
  } else {
    if (piece >= line.pieces) return;
    x0 = line.cut(piece);
    x1 = line.cut(piece + 1);
    if (!line.find(a, x0, at)) return;
  }
  for (;;) {
    const int kh = at.head, tile = (int)at.tile;
    const Sequence q = sequence_of(a, at);
    const int rows = q.fresh * a.group;
    const int row0 = tile * ROWS + wave * kWide;
    const uint32_t row = (uint32_t)min(row0 + r, rows - 1);
    const bool live = row0 + r < rows;
    const int token = (int)(row / (uint32_t)a.group);
    const int head = kh * a.group + (int)(row % (uint32_t)a.group);
    Query<D, 2> asked;
    asked.load(a, a.q + (q.row0 + token) * a.q_token + head * a.q_head, h);
    // the keys that the workgroup's rows see
    int from, to, unused;
    visible(a, q, (int)((uint32_t)(tile * ROWS) / (uint32_t)a.group), from, unused);
    visible(a, q, (int)((uint32_t)(min(tile * ROWS + ROWS, rows) - 1) / (uint32_t)a.group), unused,
            to);
    const int c0 = from / kChunk, c1 = max((to + kChunk - 1) / kChunk, c0);
    const uint64_t width = at.share.of(at.tile), end = at.start + width;
    if (line.dealt) {
      x0 = at.start;
      x1 = end;
    }
    const bool whole = x0 == at.start && end <= x1;
    auto chunk_at = [&](uint64_t x) __attribute__((always_inline)) {
      const uint64_t n = (uint64_t)(c1 - c0), each = width / max(n, (uint64_t)1) + 1;
      return c0 + (int)min(n, (x - at.start) / each);
    };
    const int begin = 2 * (x0 == at.start ? c0 : chunk_at(x0));
    const int stop = 2 * (end <= x1 ? c1 : chunk_at(x1));
    int low, high;
    visible(a, q, token, low, high);
    if (!live) high = 0;
    // the keys that all of this wave's rows see
    int all_from = 0, all_to = 0;
    if (row0 + kWide <= rows) {
      visible(a, q, (int)((uint32_t)row0 / (uint32_t)a.group), unused, all_to);
      visible(a, q, (int)((uint32_t)(row0 + kWide - 1) / (uint32_t)a.group), all_from, unused);
      if (all_from >= all_to) all_to = 0;
    }

    const int64_t block_bytes = (int64_t)c.page_tokens * D;
    const int64_t k_off = ((int64_t)a.layer * 2 * c.kv_heads + kh) * block_bytes;
    const int64_t v_off = k_off + c.kv_heads * block_bytes;
    const int in_page = c.page_tokens - 1;
    const int last_block = (q.len - 1) >> c.page_shift;
    bool wrong = false;
    auto checked = [&](int32_t entry) __attribute__((always_inline)) -> uint32_t {
      const bool bad = (uint32_t)entry >= (uint32_t)c.num_pages;
      wrong |= bad;
      return bad ? 0u : (uint32_t)entry;
    };
    // A thread's 16-byte units of a step: the first half of all are K, the rest V;
    // a wave's lie side by side in one tile of 16 keys, so all of their address
    // but the lane is scalar. Pages are looked up a step before their codes are
    // loaded (even lanes the first tile's, odd lanes the second's), and those two
    // steps before they are put into LDS.
    auto unit_of = [&](int k) __attribute__((always_inline)) {
      return (wave * kWave + k * NT) % UNITS;  // of lane 0
    };
    auto is_key = [&](int k) __attribute__((always_inline)) { return unit_of(k) < UNITS / 2; };
    auto unit_tile = [&](int k) __attribute__((always_inline)) { return unit_of(k) / D & 1; };
    int64_t unit_off[PER];  // where a unit is in a tile's page
    int unit_to[PER];       // and where its operands go
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      const int in = unit_of(k) % D + lane, tl = unit_tile(k), tok = in % 16;
      unit_off[k] = (is_key(k) ? k_off : v_off) + unit_of(k) % D * 16;
      // K: 16 channels (step in / 16) of key in % 16; V: 16 keys of channel `in`
      unit_to[k] = is_key(k) ? in / 16 * kWave + tok / 4 * 8 + tl * 4 + tok % 4
                             : in / 32 * kWave + tl * kWide + in % 32;
    }
    const float* const scale_at =
        c.scale + ((int64_t)a.layer * 2 + lane / 2 % 2) * c.kv_heads + kh;
    auto look_up = [&](int j) __attribute__((always_inline)) {
      return q.table[min((min(j, stop - 1) * kWide + lane % 2 * kKvTile) >> c.page_shift,
                         last_block)];
    };
    // (all threads load and store one of the four scales: no branch)
    auto fetch = [&](int j, int32_t entry, uint4 (&to)[PER], float& sc)
        __attribute__((always_inline)) {
      const int t0 = min(j, stop - 1) * kWide;
      const uint32_t mine = checked(entry);
      const uint32_t both[2] = {(uint32_t)__builtin_amdgcn_readlane((int)mine, 0),
                                (uint32_t)__builtin_amdgcn_readlane((int)mine, 1)};
      sc = scale_at[(int64_t)mine * c.page_scales];
#pragma unroll
      for (int k = 0; k < PER; ++k) {
        const int t = t0 + unit_tile(k) * kKvTile;
        const uint8_t* p = c.data + (int64_t)both[unit_tile(k)] * c.page_bytes +
                           (t & in_page) * D + unit_off[k];
        to[k] = reinterpret_cast<const uint4*>(p)[lane];
      }
    };
    // V codes beyond the length may be anything (K ones are hidden later).
    auto hide = [&](int j, uint4 (&w)[PER]) __attribute__((always_inline)) {
      if ((j + 1) * kWide <= q.len) return;
#pragma unroll
      for (int k = 0; k < PER; ++k) {
        const int n = is_key(k) ? 16 : q.len - j * kWide - unit_tile(k) * kKvTile;
        w[k].x = keep_bytes(w[k].x, n);
        w[k].y = keep_bytes(w[k].y, n - 4);
        w[k].z = keep_bytes(w[k].z, n - 8);
        w[k].w = keep_bytes(w[k].w, n - 12);
      }
    };
    auto stage = [&](int j, const uint4 (&from)[PER], float sc) __attribute__((always_inline)) {
      scales[(j & 3) * 4 + lane % 4] = sc;
#pragma unroll
      for (int k = 0; k < PER; ++k) {
        half8_t lo, hi;
        codes_to_operands<FMT>(from[k], lo, hi);
        half8_t* to = is_key(k) ? keys + (j & 1) * (KS * kWave) : vals + (j & 3) * (2 * DY * kWave);
        to[unit_to[k]] = lo;
        to[unit_to[k] + (is_key(k) ? kWide : DY * kWave)] = hi;
      }
    };

    half8_t query[KS];
    float factor = 0.0f;
    float m = kNone, l = 0.0f, vref = kLeastScale;
    float16_t acc[DY], s0, s1;
    half8_t w0[2], w1[2];
#pragma unroll
    for (int y = 0; y < DY; ++y)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[y][i] = 0.0f;
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int i = 0; i < 8; ++i) w1[x][i] = (_Float16)0.0f;
    auto read_key = [&](int j, int k) __attribute__((always_inline)) {
      return keys[(j & 1) * (KS * kWave) + k * kWave + lane];
    };
    auto score = [&](int k, half8_t key, float16_t& s) __attribute__((always_inline)) {
      s = __builtin_amdgcn_mfma_f32_32x32x16_f16(key, query[k], s, 0, 0, 0);
    };
    auto output = [&](int x, const half8_t (&vf)[DY], const half8_t (&w)[2])
        __attribute__((always_inline)) {
#pragma unroll
      for (int y = 0; y < DY; ++y)
        acc[y] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf[y], w[x], acc[y], 0, 0, 0);
    };
    auto read_vals = [&](int j, int x, half8_t (&vf)[DY]) __attribute__((always_inline)) {
#pragma unroll
      for (int y = 0; y < DY; ++y)
        vf[y] = vals[(j & 3) * (2 * DY * kWave) + (x * DY + y) * kWave + lane];
    };

    int32_t page = 0;  // of the next step's loads
    // Step j: scores of keys j + 1 into nxt, weights of keys j from cur, outputs of
    // keys j - 1. The first half's matrix instructions each get a share of the
    // weights' vector ones (the compiler would put them all behind).
    auto step = [&](int j, float16_t& cur, float16_t& nxt, const half8_t (&wp)[2], half8_t (&wc)[2],
                    uint4 (&rw)[PER], float& sc) __attribute__((always_inline)) {
      const float ks = scales[(j & 3) * 4 + h];
      float vs0 = scales[(j & 3) * 4 + 2], vs1 = scales[(j & 3) * 4 + 3];
      if (j * kWide < all_from || (j + 1) * kWide > all_to) {  // keys that some rows do not see
        const int t0 = j * kWide, t1 = t0 + kKvTile, t = h ? t1 : t0;
#pragma unroll
        for (int i = 0; i < 16; ++i)
          cur[i] = t + i >= low && t + i < high ? cur[i] : kNone;
        if (t0 >= high || t1 <= low) vs0 = vref;  // none of these 16
        if (t1 >= high || t1 + kKvTile <= low) vs1 = vref;
      }
      hide(j + 2, rw);
#pragma unroll
      for (int i = 0; i < 16; ++i) nxt[i] = 0.0f;
      __builtin_amdgcn_sched_barrier(0);
      half8_t kf[KS];
#pragma unroll
      for (int k = 0; k < 4; ++k) kf[k] = read_key(j + 1, k);
      float top = cur[0];
#pragma unroll
      for (int i = 1; i < 16; ++i) top = __builtin_elementwise_maximum(top, cur[i]);
      __builtin_amdgcn_sched_barrier(0);
      score(0, kf[0], nxt);
      // weights are relative to the largest V scale that the row has seen; one of
      // zero is taken for 2^-60 of it, whose weights are 0 in half precision
      const float vmax = fmaxf(fmaxf(vs0, vs1), vref);
      const float inv = __builtin_amdgcn_rcpf(vmax);
      const float rel = fmaxf((h ? vs1 : vs0) * inv, 0x1p-60f) * kLift;
      const float unrel = __builtin_amdgcn_rcpf(rel);
      // (not zero, so that a hidden key's minus infinity stays one)
      const float f = fmaxf(ks * factor, 1e-30f);
      top *= f;
      top = __builtin_elementwise_maximum(top, other_half(top));
      __builtin_amdgcn_sched_barrier(0);
      score(1, kf[1], nxt);
      const bool raise = top > m + kSlack;
      const float next = raise ? top : m;
      const float shrink = raise ? __builtin_amdgcn_exp2f(m - next) : 1.0f;
      const float fade = vmax > vref ? shrink * (vref * inv) : shrink;
      vref = vmax;
      m = next;
      const float b = __builtin_amdgcn_logf(rel) - (next == kNone ? 0.0f : next);
      float sum[2] = {0.0f, 0.0f};
      half8_t vf[DY], vg[DY];
      constexpr int SHARES = KS / 2 - 1;  // of the weights
#pragma unroll
      for (int i = 0; i < SHARES; ++i) {
        __builtin_amdgcn_sched_barrier(0);
        score(2 * i + 2, kf[2 * i + 2], nxt);
        score(2 * i + 3, kf[2 * i + 3], nxt);
        if (2 * i + 4 < KS) {
          kf[2 * i + 4] = read_key(j + 1, 2 * i + 4);
          kf[2 * i + 5] = read_key(j + 1, 2 * i + 5);
        } else {
          read_vals(max(j - 1, begin), 0, vf);
        }
#pragma unroll
        for (int k = 16 * i / SHARES; k < 16 * (i + 1) / SHARES; ++k) {
          const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(cur[k], f, b));
          sum[k % 2] += p;
          wc[k / 8][k % 8] = (_Float16)p;
        }
      }
      l = l * shrink + (sum[0] + sum[1]) * unrel;
      asm volatile("" : "+v"(wc[0]), "+v"(wc[1]), "+v"(l));  // here, not where they are used
      __builtin_amdgcn_sched_barrier(0);
      read_vals(max(j - 1, begin), 1, vg);
      output(0, vf, wp);
      output(1, vg, wp);
      stage(j + 2, rw, sc);
      // the next look-up goes first: loads return in order, and the next step
      // needs it before these
      const int32_t entry = page;
      page = look_up(j + 5);
      fetch(j + 4, entry, rw, sc);
#pragma unroll
      for (int i = 0; i < 2 * DY; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);  // a matrix instruction,
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);  // an operand read
        __builtin_amdgcn_sched_group_barrier(0x002, 6, 0);  // and vector ones
      }
      __builtin_amdgcn_sched_barrier(0);
      if (__ballot(fade != 1.0f)) {
#pragma unroll
        for (int y = 0; y < DY; ++y) {
          // one after the other: all of them at once in the vector registers
          // would push out other values
          if (PINNED) asm volatile("" : "+a"(acc[y]));
          acc[y] *= fade;
          if (PINNED) asm volatile("" : "+a"(acc[y]));
        }
      }
      block_sync();
    };
    if (begin < stop) {
      int32_t entry[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) entry[i] = look_up(begin + i);
      page = look_up(begin + 4);
      factor = asked.convert(a, query);
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        if (PINNED) asm volatile("" : "+a"(query[k]));
        else asm volatile("" : "+v"(query[k]));
      }
      uint4 early[2][PER], raw[2][PER];
      float searly[2], sraw[2];
      fetch(begin, entry[0], early[0], searly[0]);
      fetch(begin + 1, entry[1], early[1], searly[1]);
      fetch(begin + 2, entry[2], raw[0], sraw[0]);
      fetch(begin + 3, entry[3], raw[1], sraw[1]);
      hide(begin, early[0]);
      hide(begin + 1, early[1]);
      stage(begin, early[0], searly[0]);
      stage(begin + 1, early[1], searly[1]);
      block_sync();
#pragma unroll
      for (int i = 0; i < 16; ++i) s0[i] = 0.0f;
#pragma unroll
      for (int k = 0; k < KS; ++k) score(k, read_key(begin, k), s0);
      block_sync();  // step `begin` puts keys begin + 2 where these were
      for (int j = begin; j < stop; j += 2) {
        step(j, s0, s1, w1, w0, raw[0], sraw[0]);
        step(j + 1, s1, s0, w0, w1, raw[1], sraw[1]);
      }
      half8_t vf[DY], vg[DY];
      read_vals(stop - 1, 0, vf);
      read_vals(stop - 1, 1, vg);
      output(0, vf, w1);
      output(1, vg, w1);
    }
    block_sync();  // the buffers are free
    if (__ballot(wrong) && lane == 0) atomicOr(c.flags, kFlagInval);
    l += other_half(l);
    if (!whole) {
      // a piece's first tile and its last one may be cut
      const int64_t slot = (int64_t)(2 * piece + (x0 == at.start)) * ROWS + wave * kWide + r;
      float* o = a.part_o + slot * D;
#pragma unroll
      for (int y = 0; y < DY; ++y)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float4_t x = {acc[y][4 * k], acc[y][4 * k + 1], acc[y][4 * k + 2],
                              acc[y][4 * k + 3]};
          *reinterpret_cast<float4_t*>(o + y * 32 + k * 8 + h * 4) = x * (1.0f / kLift) * vref;
        }
      if (h == 0) {
        a.part_ml[2 * slot] = m;
        a.part_ml[2 * slot + 1] = l;
      }
      if (x0 == at.start && threadIdx.x == 0)  // the first part tells how to join them
        a.cuts[blockIdx.x] = {(int32_t)(line.piece_of(end - 1) - piece) + 1, (int32_t)piece,
                              (int32_t)q.row0, rows, tile, kh};
    } else {
      const bool some = l > 0.0f || l != l;
      const float inv = some ? (1.0f / kLift) / l : 0.0f;
      // through LDS, so that rows are written whole
      uint2* const mine = reinterpret_cast<uint2*>(pool + (wave * kWide + r) * PITCH);
#pragma unroll
      for (int y = 0; y < DY; ++y)
#pragma unroll
        for (int k = 0; k < 4; ++k)
          mine[y * 8 + k * 2 + h] =
              make_uint2(pack_pair(acc[y][4 * k] * inv * vref, acc[y][4 * k + 1] * inv * vref, a.bf16),
                         pack_pair(acc[y][4 * k + 2] * inv * vref, acc[y][4 * k + 3] * inv * vref,
                                   a.bf16));
      if (a.lse && h == 0 && live)
        a.lse[(q.row0 + token) * a.heads + head] =
            some ? (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f : kNone;
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // (a wave reads what it wrote)
      constexpr int LANES = D / 8;  // of a row
#pragma unroll 2
      for (int i = lane / LANES; i < kWide; i += kWave / LANES) {
        const int rr = row0 + i;
        if (rr >= rows) break;
        const uint32_t tok = (uint32_t)rr / (uint32_t)a.group;
        const int64_t hd = kh * a.group + (int)((uint32_t)rr - tok * a.group);
        uint16_t* o = a.out + (q.row0 + tok) * a.out_token + hd * a.out_head + lane % LANES * 8;
        const uint4 x = __builtin_bit_cast(uint4, pool[(wave * kWide + i) * PITCH + lane % LANES]);
        if (a.wide_out) {
          *reinterpret_cast<uint4*>(o) = x;
        } else {
          const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
          for (int j = 0; j < 8; ++j) o[j] = (uint16_t)(w[j / 2] >> (16 * (j % 2)));
        }
      }
    }
    block_sync();  // the buffers are free
    if (line.dealt) {
      turn += gridDim.x;
      if (!line.deal(a, turn, at)) break;
    } else {
      x0 = end;
      if (x0 >= x1 || !line.next(a, at)) break;
    }
  }
}

// Joins the tiles that were cut: sixteen lanes per row, kJoinRows rows after
// each other.
constexpr int kJoinRows = 64;  // of a workgroup
template <int D, int ROWS>
__global__ __launch_bounds__(256) void kv_attend_join(KvAttendArgs a) {
  constexpr int W = D / 16;  // channels of a lane
  const KvCut cut = a.cuts[blockIdx.x];
  const int parts = cut.parts;
  if (parts == 0) return;
  // (the first part is its piece's last tile, the others are their pieces' first)
  for (int mine = blockIdx.y * kJoinRows + threadIdx.x / 16;
       mine < (int)(blockIdx.y + 1) * kJoinRows; mine += 16) {
    const int row = cut.tile * ROWS + mine;
    if (row >= cut.rows) return;
    auto slot = [&](int k) __attribute__((always_inline)) {
      return (int64_t)(2 * (cut.piece + k) + (k == 0)) * ROWS + mine;
    };
    const int64_t token = cut.row0 + (uint32_t)row / (uint32_t)a.group;
    const int64_t head = cut.head * a.group + (uint32_t)row % (uint32_t)a.group;
    const int lane = threadIdx.x % 16;
    const float2_t* ml = reinterpret_cast<const float2_t*>(a.part_ml);
    float most = kNone;
#pragma unroll 4
    for (int k = 0; k < parts; ++k) most = fmaxf(most, ml[slot(k)][0]);
    const float base = most == kNone ? 0.0f : most;
    float total = 0.0f;
    float4_t o[W / 4];
#pragma unroll
    for (int j = 0; j < W / 4; ++j) o[j] = float4_t{0.0f, 0.0f, 0.0f, 0.0f};
    const float* part = a.part_o + lane * W;
#pragma unroll 4
    for (int k = 0; k < parts; ++k) {
      const float2_t p = ml[slot(k)];
      const float w = __builtin_amdgcn_exp2f(p[0] - base);
      total += p[1] * w;
#pragma unroll
      for (int j = 0; j < W / 4; ++j)
        o[j] += *reinterpret_cast<const float4_t*>(part + slot(k) * D + 4 * j) * w;
    }
    const bool some = total > 0.0f || total != total;
    const float inv = some ? 1.0f / total : 0.0f;
    uint16_t* out = a.out + token * a.out_token + head * a.out_head + lane * W;
#pragma unroll
    for (int j = 0; j < W / 4; ++j) {
      const uint32_t x = pack_pair(o[j][0] * inv, o[j][1] * inv, a.bf16);
      const uint32_t y = pack_pair(o[j][2] * inv, o[j][3] * inv, a.bf16);
      if (a.wide_out) {
        *reinterpret_cast<uint2*>(out + 4 * j) = make_uint2(x, y);
      } else {
        out[4 * j] = (uint16_t)x;
        out[4 * j + 1] = (uint16_t)(x >> 16);
        out[4 * j + 2] = (uint16_t)y;
        out[4 * j + 3] = (uint16_t)(y >> 16);
      }
    }
    if (a.lse && lane == 0)
      a.lse[token * a.heads + head] =
          some ? (most + __builtin_amdgcn_logf(total)) * 0.6931471805599453f : kNone;
  }
}

// Waves of the tile kernel's workgroups, each with one tile of 32 rows.
template <int D>
constexpr int tile_waves() { return D > 128 ? 4 : 8; }
template <int D>
constexpr int tile_rows() { return tile_waves<D>() * kWide; }

template <int D, int FMT>
hipError_t launch_rows(KvAttendArgs a, hipStream_t st) {
  const int64_t tiles = a.cu ? a.tokens * a.group / kRows + a.n  // at most
                             : a.n * ((a.group + kRows - 1) / kRows);
  const int64_t checks = a.cu ? (a.n + a.waves * kWave - 1) / (a.waves * kWave) : 0;
  if (!grid_fits(tiles * a.c.kv_heads + checks, a.waves * kWave))
    return hipErrorInvalidConfiguration;
  a.tiles = (uint32_t)(tiles * a.c.kv_heads);
  const dim3 grid((unsigned)(a.tiles + checks), (unsigned)a.parts);
  if (D <= 128 && a.waves == 8)
    hipLaunchKernelGGL((kv_attend_rows<D, FMT, D <= 128 ? 8 : 4>), grid, dim3(8 * kWave), 0, st, a);
  else
    hipLaunchKernelGGL((kv_attend_rows<D, FMT, 4>), grid, dim3(4 * kWave), 0, st, a);
  return hipGetLastError();
}

template <int D, int FMT>
hipError_t launch(const KvAttendArgs& a, hipStream_t st) {
  if (!a.tiled) return launch_rows<D, FMT>(a, st);
  constexpr int ROWS = tile_rows<D>(), THREADS = tile_waves<D>() * kWave;
  const int64_t tiles = a.tokens * a.group / ROWS + a.n;  // at most
  const int64_t grid = a.whole ? tiles * a.c.kv_heads : kPieces;
  if (!grid_fits(grid, THREADS)) return hipErrorInvalidConfiguration;
  hipLaunchKernelGGL((kv_attend_tile<D, FMT, tile_waves<D>()>), dim3((unsigned)grid),
                     dim3(THREADS), 0, st, a);
  if (!a.whole)
    hipLaunchKernelGGL((kv_attend_join<D, ROWS>), dim3(kPieces, ROWS / kJoinRows), dim3(256), 0,
                       st, a);
  return hipGetLastError();
}

template <int D>
hipError_t launch_dim(const KvAttendArgs& a, hipStream_t st) {
  return a.c.format == SEM_KV_INT8 ? launch<D, SEM_KV_INT8>(a, st) : launch<D, SEM_KV_FP8>(a, st);
}

}  // namespace

// Which kernel, and how many parts of the key axis. Rules measured on MI355X:
//   * The kernel of few rows takes cost_few ns of the whole device per tile of 16
//     rows and chunk of 64 keys, the tile kernel cost_tile ns per tile and 32 keys
//     (256 rows, 128 for 256 channels), and 20 us more for its longer start and
//     end: 16 sequences of 128 rows over 4096 keys (8 KV heads, 128 channels) take
//     78 us with the one and 105 us with the other, of 256 rows 139 and 97 us.
//   * Few rows: parts only where there are fewer workgroups than compute units,
//     then as many as those; each is eight waves with long runs of keys (four
//     contexts of 131072 tokens take 175 us with 256 workgroups, 187 us with 768),
//     and not for fewer than 24 chunks (a single token over 1024 keys takes 10 us
//     in one part; two add 3 us of joining). With more workgroups than compute
//     units four waves each, without parts (256 ragged requests: 87 us, 95 us with
//     parts of 2048 keys). Equal contexts of 32768 keys, 8 KV heads, are read at
//     5.3 to 5.7 TB/s (8 to 17 sequences), 6.0 (24 to 32, 64) and 5.0 (40, a second
//     round that does not fill the device). Unequal ones are not balanced: 31
//     sequences of 1024 keys and one of 131072 take 942 us, as long as eight
//     workgroups need for the long one, where the bytes take 60.
//   * Tiles: see kPieces.
KvSplit kv_attend_split(int dim, int64_t n, int64_t tokens, int heads, int kv_heads,
                        int64_t max_new, int64_t max_len) {
  KvSplit s = {};
  const int group = heads / kv_heads;
  const int64_t chunks = std::max<int64_t>((max_len + kChunk - 1) / kChunk, 1);
  // row tiles of the grid, and what there are of them if max_new holds
  auto grid_of = [&](int64_t rows) { return tokens * group / rows + n; };
  auto tiles_of = [&](int64_t rows) {
    return std::min(grid_of(rows), n * ((max_new * group + rows - 1) / rows));
  };
  const int tile = dim == 256 ? tile_rows<256>() : tile_rows<128>();
  const double cost_few = dim == 64 ? 0.7 : dim == 128 ? 1.0 : 2.8;
  const double cost_tile = dim == 64 ? 3.7 : dim == 128 ? 4.6 : 5.4;
  const double each = (double)kv_heads * (double)chunks;
  s.tiled = cost_tile * 2 * each * (double)tiles_of(tile) + 20e3 <
            cost_few * each * (double)tiles_of(kRows);
  // SEMSCHED_KV_TILES=0 or 1 takes one kernel for all sizes, so that both stay
  // testable on small ones.
  const char* forced = std::getenv("SEMSCHED_KV_TILES");
  if (forced && (forced[0] == '0' || forced[0] == '1')) s.tiled = forced[0] == '1';
  if (s.tiled) {
    s.whole = tokens * group / tile * kv_heads >= kWholeRounds * kPieces;
    if (!s.whole) s.part_rows = 2 * kPieces * tile;
    return s;
  }
  const int64_t groups = std::max<int64_t>(tiles_of(kRows) * kv_heads, 1);
  s.waves = groups < 256 && dim <= 128 ? 8 : 4;
  const int64_t least = 2 * s.waves;  // chunks of a part
  // (a tile with parts needs a counter)
  const int64_t want = chunks <= 3 * s.waves || grid_of(kRows) * kv_heads > kKvCounts ? 1 : 256;
  const int64_t parts = std::max<int64_t>(1, std::min<int64_t>(want / groups, kMostParts));
  s.part_chunks = (int)std::max<int64_t>(least, (chunks + parts - 1) / parts);
  s.parts = (int)((chunks + s.part_chunks - 1) / s.part_chunks);
  if (s.parts > 1) s.part_rows = s.parts * tokens * heads;
  return s;
}

hipError_t launch_kv_attend(const KvAttendArgs& a, hipStream_t st) {
  if (a.n == 0) return hipSuccess;  // (without tokens the offsets are looked at)
  switch (a.c.head_dim) {
    case 64: return launch_dim<64>(a, st);
    case 128: return launch_dim<128>(a, st);
    default: return launch_dim<256>(a, st);
  }
}

}  // namespace semsched
