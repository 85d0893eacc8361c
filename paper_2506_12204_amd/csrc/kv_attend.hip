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
// largest vs seen, 2^14 above, so that weights down to 2^-28 of the largest
// keep 11 bits.
#include <algorithm>
#include <type_traits>

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
constexpr int kMostParts = 128;      // of the key axis
// The running maximum is raised only when a score passes it by this much (in
// powers of two), which is seldom: most steps then need no rescaling of the
// outputs. Weights stay below kLift * 2^kSlack, which half precision holds.
constexpr float kSlack = 8.0f;

struct Sequence {
  const int32_t* table;
  int64_t row0;     // first query token
  int fresh, len;   // query tokens, keys
};

// The sequence of row tile u and the tile's number in it; false if there is no
// such tile. Tiles are numbered sequence by sequence, LATE ones (whose causal
// rows see most keys) first where that is asked for. The grid's size is a bound,
// and its workgroups without work have to be the last or first ones: the device
// deals workgroups to its parts in turn, and idle ones at regular places would
// leave the same parts without work. So every wave counts the tiles of all
// sequences, 64 at a time (n / 64 rounds of independent loads, where a search
// would take log n dependent ones).
template <bool LATE>
__device__ __forceinline__ bool find_sequence(const KvAttendArgs& a, uint32_t u, int rows,
                                              Sequence& q, int64_t& tile) {
  const KvView& c = a.c;
  int64_t i = -1;
  if (a.cu) {
    const int lane = lane_id();
    auto count = [&](int64_t at) __attribute__((always_inline)) -> uint32_t {
      if (at >= a.n) return 0;
      const int64_t fresh = (int64_t)a.cu[at + 1] - a.cu[at];
      return fresh > 0 && fresh <= a.tokens ? (uint32_t)((fresh * a.group + rows - 1) / rows) : 0u;
    };
    uint32_t total = 0;
    if (LATE) {
      for (int64_t at = 0; at < a.n; at += kWave) total += wave_add_u32(count(at + lane));
      if (u >= total) return false;
      u = total - 1 - u;
    }
    uint32_t before = 0;
    for (int64_t at = 0; at < a.n; at += kWave) {
      const uint32_t mine = count(at + lane), upto = before + wave_incl_scan_u32(mine);
      const uint64_t beyond = __ballot(upto > u);
      if (beyond) {
        const int first = __ffsll((unsigned long long)beyond) - 1;
        i = at + first;
        tile = u - (uint32_t)__builtin_amdgcn_readlane((int)(upto - mine), first);
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
    tile = u % each;
  }
  q.row0 = a.cu ? a.cu[i] : i;
  const int64_t fresh = a.cu ? (int64_t)a.cu[i + 1] - q.row0 : 1;
  if (fresh < 0 || q.row0 < 0 || q.row0 + fresh > a.tokens) {
    if (threadIdx.x == 0) atomicOr(c.flags, kFlagInval);
    return false;
  }
  q.fresh = (int)fresh;
  const int32_t s = a.seqs[i];
  q.len = 0;
  q.table = c.tables;
  if ((uint32_t)s >= (uint32_t)c.slots) {
    if (threadIdx.x == 0) atomicOr(c.flags, kFlagInval);
    return true;  // its rows see no key
  }
  q.table += (int64_t)s * c.max_blocks;
  q.len = c.lens[s];
  if (q.len < 0 || (int64_t)q.len > ((int64_t)c.max_blocks << c.page_shift)) {
    if (threadIdx.x == 0) atomicOr(c.flags, kFlagInval);
    q.len = 0;
  }
  return true;
}

// Keys [low, high) that query token i of the sequence sees.
__device__ __forceinline__ void visible(const KvAttendArgs& a, const Sequence& q, int i, int& low,
                                        int& high) {
  const int pos = q.len - q.fresh + i;
  high = a.causal ? max(min(pos + 1, q.len), 0) : q.len;
  low = a.window > 0 ? max(pos + 1 - a.window, 0) : 0;
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

// A row's query in halves, as the lane's D / (8 G) operands of eight: of G = 4
// lane groups, group g holds channels (4 j + g) * 16 .. + 15 in operands 2 j and
// 2 j + 1; of G = 2, channels 16 j + 8 g .. + 7 in operand j. Returns what the
// scores have to be multiplied by, which is not negative (a negative scale
// changes the query's sign).
template <int D, int G>
__device__ __forceinline__ float load_query(const KvAttendArgs& a, const uint16_t* row, int g,
                                            half8_t (&q)[D / (8 * G)]) {
  constexpr int N = D / (8 * G);
  uint16_t e[N][8];
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

// Joins a row's parts with one wave.
// ALIVE: written by workgroups of this kernel, to be read past the L2 caches.
template <int D, bool ALIVE>
__device__ __forceinline__ void join_row(const KvAttendArgs& a, int64_t token, int64_t head,
                                         int parts) {
  constexpr int W = D / 64;
  const int64_t all = a.tokens * a.heads, at = token * a.heads + head;
  const int lane = lane_id();
  // lane k has parts k and k + 64
  static_assert(kMostParts == 2 * kWave, "two parts per lane");
  const int far = kWave + lane;
  const float* ml = a.part_ml + 2 * at;
  auto load = [](const float* p) __attribute__((always_inline)) {
    return ALIVE ? load_agent(p) : *p;
  };
  const float m0 = lane < parts ? load(ml + 2 * lane * all) : kNone;
  const float l0 = lane < parts ? load(ml + 2 * lane * all + 1) : 0.0f;
  const float m1 = far < parts ? load(ml + 2 * far * all) : kNone;
  const float l1 = far < parts ? load(ml + 2 * far * all + 1) : 0.0f;
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
    for (int j = 0; j < W; ++j) o[j] += load(from + k * all * D + j) * w;
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
  // heads side by side: the dies take workgroups in turn, and so get an equal
  // share of every sequence
  const int kh = blockIdx.x % c.kv_heads;
  Sequence q;
  int64_t tile;
  if (!find_sequence<false>(a, blockIdx.x / c.kv_heads, kRows, q, tile)) return;
  const int64_t rows = (int64_t)q.fresh * a.group;
  const int64_t row = tile * kRows + r;
  const bool live = row < rows;
  const int token = (int)((live ? row : rows - 1) / a.group);
  const int head = kh * a.group + (int)((live ? row : rows - 1) % a.group);
  half8_t query[D / 32];
  const float factor = load_query<D, 4>(
      a, a.q + (q.row0 + token) * a.q_token + head * a.q_head, g, query);
  int low, high;
  visible(a, q, token, low, high);
  // the keys that any row of the tile sees, and those that all see
  int from, to, all_from, all_to;
  visible(a, q, (int)(tile * kRows / a.group), from, all_to);
  visible(a, q, (int)((min(tile * kRows + kRows, rows) - 1) / a.group), all_from, to);
  const int c0 = from / kChunk, c1 = (to + kChunk - 1) / kChunk;
  const int parts = parts_of(a, c0, c1), part = blockIdx.y;
  if (part >= parts) return;
  const int begin = part_start(c0, c1, parts, part), stop = part_start(c0, c1, parts, part + 1);

  float m = kNone, l = 0.0f, vref = 0.0f;
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
  for (int ch = begin + wave; ch < stop; ch += NW) {
    const int t0 = ch * kChunk, vt = t0 + g * kKvTile;
    const bool more = ch + NW < stop;
    // (not zero, so that a hidden key's minus infinity stays one)
    const float f = fmaxf(kscale * factor, 1e-30f), vs = vscale;
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
    // weights are relative to the largest V scale so far
    float vmax = fmaxf(vs, __shfl_xor(vs, 16, kWave));
    vmax = fmaxf(fmaxf(vmax, other_half(vmax)), vref);
    const float inv = vmax > 0.0f ? __builtin_amdgcn_rcpf(vmax) : 0.0f;
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
    const float by = vref * (1.0f / kLift);
#pragma unroll
    for (int y = 0; y < D / 16; ++y) {
      const float4_t o = acc[y] * by;
      *reinterpret_cast<float4_t*>(&join_o[wave][r][y * 16 + g * 4]) = o;
    }
  }
  block_sync();
  // a wave joins every NW-th row, a lane its W channels of it
  const int64_t all = a.tokens * a.heads;
  for (int i = wave; i < kRows; i += NW) {
    const int64_t rr = tile * kRows + i;
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
    const int64_t tok = q.row0 + rr / a.group, hd = kh * a.group + rr % a.group;
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
    const int64_t rr = tile * kRows + i;
    if (rr >= rows) break;
    join_row<D, true>(a, q.row0 + rr / a.group, kh * a.group + rr % a.group, parts);
  }
}

// ---------------------------------------------------------------------------
// Many rows: tiles of NW * RT * 32 rows of one KV head.
//
// A wave holds RT * 32 rows (their queries and outputs in registers) and goes
// through the keys 32 at a time; the workgroup turns their codes into halves
// once and keeps them in LDS in operand order, so that every operand is one
// 16-byte LDS read without bank conflicts. As above, scores are taken as K q^T:
// a lane has the scores of one row (lane % 32) and, by the order in which keys
// are fed, of 16 consecutive keys, which the second product takes from
// registers.
//
// Three steps overlap, so that the matrix cores are fed while the vector units
// turn scores into weights: step j takes the scores of keys j + 1, the weights
// of keys j and the outputs of keys j - 1, which do not depend on each other.
// Codes are loaded four steps ahead and put into LDS two steps ahead.
constexpr int kWide = 32;  // rows of a matrix tile, and keys of a step
typedef float float16_t __attribute__((ext_vector_type(16)));

// The order of a step's instructions: every matrix instruction is followed by
// vector ones that run beside it, an operand read and an exponential.
template <int MATRIX, int VECTOR>
__device__ __forceinline__ void interleave() {
#pragma unroll
  for (int i = 0; i < MATRIX; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);       // matrix
    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);       // LDS reads
    __builtin_amdgcn_sched_group_barrier(0x002, VECTOR, 0);  // vector
    __builtin_amdgcn_sched_group_barrier(0x400, 1, 0);       // exponentials
  }
}

template <int D, int FMT, int NW, int RT>
__global__ __launch_bounds__(NW* kWave, NW / 4) void kv_attend_tile(KvAttendArgs a) {
  constexpr int NT = NW * kWave;
  constexpr int KS = D / 16;       // matrix steps of the score product
  constexpr int DY = D / 32;       // output tiles
  constexpr int UNITS = 4 * D;     // 16-byte units of a step's K and V
  constexpr int PER = UNITS > NT ? UNITS / NT : 1;  // of them per thread
  // Two waves per SIMD hold everything in vector registers; one has to keep
  // outputs and queries in the accumulation registers.
  constexpr bool PINNED = NW == 4;
  constexpr int ROWS = NW * RT * kWide;
  static_assert(NT * PER % UNITS == 0, "whole rounds of units");
  constexpr int KEYS = 2 * KS * kWave;      // [buffer][step][lane]
  constexpr int VALS = 4 * 2 * DY * kWave;  // [buffer][8 keys of either half][tile][lane]
  constexpr int PITCH = D / 8 + 1;          // of an output row at the end
  constexpr int OUTS = NW * kWide * PITCH;
  __shared__ half8_t pool[KEYS + VALS > OUTS ? KEYS + VALS : OUTS];
  half8_t* const keys = pool;
  half8_t* const vals = pool + KEYS;
  __shared__ float scales[4 * 4];               // [buffer][K tile 0, 1, V tile 0, 1]
  const KvView& c = a.c;
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int r = lane % kWide, h = lane / kWide;
  const int kh = blockIdx.x % c.kv_heads;
  Sequence q;
  int64_t tile;
  if (!find_sequence<true>(a, blockIdx.x / c.kv_heads, ROWS, q, tile)) return;
  const int64_t rows = (int64_t)q.fresh * a.group;
  // the keys that the workgroup's rows see
  int from, to, unused;
  visible(a, q, (int)(tile * ROWS / a.group), from, unused);
  visible(a, q, (int)((min(tile * ROWS + ROWS, rows) - 1) / a.group), unused, to);
  const int c0 = from / kChunk, c1 = (to + kChunk - 1) / kChunk;
  const int parts = parts_of(a, c0, c1), part = blockIdx.y;
  if (part >= parts) return;
  const int begin = 2 * part_start(c0, c1, parts, part);
  const int stop = 2 * part_start(c0, c1, parts, part + 1);

  const int64_t row0 = tile * ROWS + wave * (RT * kWide);
  half8_t query[RT][KS];
  float factor[RT];
  int low[RT], high[RT], token[RT], head[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const int64_t row = row0 + t * kWide + r;
    const bool live = row < rows;
    const int64_t at = live ? row : rows - 1;
    token[t] = (int)(at / a.group);
    head[t] = kh * a.group + (int)(at % a.group);
    factor[t] = load_query<D, 2>(
        a, a.q + (q.row0 + token[t]) * a.q_token + head[t] * a.q_head, h, query[t]);
    visible(a, q, token[t], low[t], high[t]);
    if (!live) {
      low[t] = 0;
      high[t] = 0;
      token[t] = -1;
    }
  }
  if (PINNED) {
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
      for (int k = 0; k < KS; ++k) asm volatile("" : "+a"(query[t][k]));
  }
  // the keys that all of this wave's rows see
  int all_from = 0, all_to = 0;
  if (row0 + RT * kWide <= rows) {
    visible(a, q, (int)(row0 / a.group), unused, all_to);
    visible(a, q, (int)((row0 + RT * kWide - 1) / a.group), all_from, unused);
    if (all_from >= all_to) all_to = 0;
  }

  const int64_t block_bytes = (int64_t)c.page_tokens * D;
  const int64_t k_off = ((int64_t)a.layer * 2 * c.kv_heads + kh) * block_bytes;
  const int64_t v_off = k_off + c.kv_heads * block_bytes;
  const int in_page = c.page_tokens - 1;
  const int last_block = (q.len - 1) >> c.page_shift;
  bool wrong = false;
  auto entry_of = [&](int t) __attribute__((always_inline)) {
    return q.table[min(t >> c.page_shift, last_block)];
  };
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
  uint4 raw[2][PER];
  float sraw[2] = {0.0f, 0.0f};
  int32_t page = 0;
  const float* const scale_at =
      c.scale + ((int64_t)a.layer * 2 + lane / 2 % 2) * c.kv_heads + kh;
  auto look_up = [&](int j) __attribute__((always_inline)) {
    page = entry_of(min(j, stop - 1) * kWide + lane % 2 * kKvTile);
  };
  // (all threads load and store one of the four scales: no branch)
  auto fetch = [&](int j, uint4 (&to)[PER], float& sc) __attribute__((always_inline)) {
    const int t0 = min(j, stop - 1) * kWide;
    const uint32_t mine = checked(page);
    const uint32_t both[2] = {(uint32_t)__builtin_amdgcn_readlane((int)mine, 0),
                              (uint32_t)__builtin_amdgcn_readlane((int)mine, 1)};
    // the next look-up goes first: loads return in order, and the next step
    // needs it before these
    look_up(j + 1);
    sc = scale_at[(int64_t)mine * c.page_scales];
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      const int t = t0 + unit_tile(k) * kKvTile;
      const uint8_t* p = c.data + (int64_t)both[unit_tile(k)] * c.page_bytes +
                         (t & in_page) * D + unit_off[k];
      to[k] = reinterpret_cast<const uint4*>(p)[lane];
    }
  };
  auto stage = [&](auto mask, int j, const uint4 (&from)[PER], float sc)
      __attribute__((always_inline)) {
    scales[(j & 3) * 4 + lane % 4] = sc;
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      uint4 w = from[k];
      // V codes beyond the length may be anything; K ones are hidden later
      if (decltype(mask)::value && !is_key(k)) {
        const int n = q.len - j * kWide - unit_tile(k) * kKvTile;
        w.x = keep_bytes(w.x, n);
        w.y = keep_bytes(w.y, n - 4);
        w.z = keep_bytes(w.z, n - 8);
        w.w = keep_bytes(w.w, n - 12);
      }
      half8_t lo, hi;
      codes_to_operands<FMT>(w, lo, hi);
      half8_t* to = is_key(k) ? keys + (j & 1) * (KS * kWave) : vals + (j & 3) * (2 * DY * kWave);
      to[unit_to[k]] = lo;
      to[unit_to[k] + (is_key(k) ? kWide : DY * kWave)] = hi;
    }
  };

  float m[RT], l[RT], vref = 0.0f;
  float16_t acc[RT][DY], s0[RT], s1[RT];
  half8_t w0[RT][2], w1[RT][2];
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    m[t] = kNone;
    l[t] = 0.0f;
#pragma unroll
    for (int y = 0; y < DY; ++y)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[t][y][i] = 0.0f;
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int i = 0; i < 8; ++i) w1[t][x][i] = (_Float16)0.0f;
  }
  auto score = [&](int j, float16_t (&s)[RT]) __attribute__((always_inline)) {
    const half8_t* from = keys + (j & 1) * (KS * kWave) + lane;
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[t][i] = 0.0f;
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      const half8_t kf = from[k * kWave];
#pragma unroll
      for (int t = 0; t < RT; ++t)
        s[t] = __builtin_amdgcn_mfma_f32_32x32x16_f16(kf, query[t][k], s[t], 0, 0, 0);
    }
  };
  auto output = [&](const half8_t (&vf)[2][DY], const half8_t (&w)[RT][2])
      __attribute__((always_inline)) {
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int y = 0; y < DY; ++y)
#pragma unroll
        for (int t = 0; t < RT; ++t)
          acc[t][y] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf[x][y], w[t][x], acc[t][y], 0, 0, 0);
  };
  auto read_vals = [&](int j, half8_t (&vf)[2][DY]) __attribute__((always_inline)) {
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int y = 0; y < DY; ++y)
        vf[x][y] = vals[(j & 3) * (2 * DY * kWave) + (x * DY + y) * kWave + lane];
  };
  // Scores of a row tile become weights; its outputs so far are to be multiplied
  // by `fade`.
  struct Scales {
    float ks, bias, unrel, older;
  };
  auto scales_of = [&](int j) __attribute__((always_inline)) {
    const float ks = scales[(j & 3) * 4 + h];
    const float vs0 = scales[(j & 3) * 4 + 2], vs1 = scales[(j & 3) * 4 + 3];
    // weights are relative to the largest V scale so far (the same in all lanes)
    const float vmax = fmaxf(fmaxf(vs0, vs1), vref);
    const float inv = vmax > 0.0f ? __builtin_amdgcn_rcpf(vmax) : 0.0f;
    const float older = vmax > vref ? vref * inv : 1.0f;
    vref = vmax;
    const float rel = fmaxf((h ? vs1 : vs0) * inv, 9.3e-10f) * kLift;  // (2^-30)
    return Scales{ks, __builtin_amdgcn_logf(rel), __builtin_amdgcn_rcpf(rel), older};
  };
  auto weigh = [&](int t, const Scales& z, const float16_t& s, half8_t (&w)[2], float& fade)
      __attribute__((always_inline)) {
    // (not zero, so that a hidden key's minus infinity stays one)
    const float f = fmaxf(z.ks * factor[t], 1e-30f);
    float top = s[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) top = __builtin_elementwise_maximum(top, s[i]);
    top *= f;
    top = __builtin_elementwise_maximum(top, other_half(top));
    const bool raise = top > m[t] + kSlack;
    const float next = raise ? top : m[t];
    const float shrink = raise ? __builtin_amdgcn_exp2f(m[t] - next) : 1.0f;
    m[t] = next;
    const float b = z.bias - (next == kNone ? 0.0f : next);
    float sum[2] = {0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], f, b));
      sum[i % 2] += p;
      w[i / 8][i % 8] = (_Float16)p;
    }
    l[t] = l[t] * shrink + (sum[0] + sum[1]) * z.unrel;
    fade = z.older * shrink;
    asm volatile("" : "+v"(w[0]), "+v"(w[1]));  // here, not where they are used
  };
  auto step = [&](auto mask, int j, float16_t (&cur)[RT], float16_t (&nxt)[RT],
                  const half8_t (&wp)[RT][2], half8_t (&wc)[RT][2], uint4 (&rw)[PER], float& sc)
      __attribute__((always_inline)) {
    if (decltype(mask)::value) {
      const int t0 = j * kWide + h * kKvTile;
#pragma unroll
      for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          cur[t][i] = t0 + i >= low[t] && t0 + i < high[t] ? cur[t][i] : kNone;
    }
    float fade[RT];
    half8_t vf[2][DY];
    __builtin_amdgcn_sched_barrier(0);
    const Scales z = scales_of(j);
    score(j + 1, nxt);
    weigh(0, z, cur[0], wc[0], fade[0]);
    read_vals(max(j - 1, begin), vf);
    __builtin_amdgcn_sched_group_barrier(0x100, 6, 0);
    interleave<RT * KS, 6>();
    __builtin_amdgcn_sched_barrier(0);
    output(vf, wp);
    if (RT > 1) weigh(RT - 1, z, cur[RT - 1], wc[RT - 1], fade[RT - 1]);
    stage(mask, j + 2, rw, sc);
    fetch(j + 4, rw, sc);
    interleave<RT * 2 * DY, 8>();
    __builtin_amdgcn_sched_barrier(0);
    bool any = false;
#pragma unroll
    for (int t = 0; t < RT; ++t) any |= fade[t] != 1.0f;
    if (__ballot(any)) {
#pragma unroll
      for (int t = 0; t < RT; ++t) {
#pragma unroll
        for (int y = 0; y < DY; ++y) {
          // one after the other: all of them at once in the vector registers
          // would push out other values
          if (PINNED) asm volatile("" : "+a"(acc[t][y]));
          acc[t][y] *= fade[t];
          if (PINNED) asm volatile("" : "+a"(acc[t][y]));
        }
      }
    }
    block_sync();
  };
  if (begin < stop) {
    constexpr std::false_type plain{};
    constexpr std::true_type masked{};
    look_up(begin);
    fetch(begin, raw[0], sraw[0]);
    fetch(begin + 1, raw[1], sraw[1]);
    stage(masked, begin, raw[0], sraw[0]);
    stage(masked, begin + 1, raw[1], sraw[1]);
    fetch(begin + 2, raw[0], sraw[0]);
    fetch(begin + 3, raw[1], sraw[1]);
    block_sync();
    score(begin, s0);
    block_sync();  // step `begin` puts keys begin + 2 where these were
    for (int j = begin; j < stop; j += 2) {
      // keys that all rows see, and codes that all are there
      if (j * kWide >= all_from && (j + 2) * kWide <= all_to && (j + 4) * kWide <= q.len) {
        step(plain, j, s0, s1, w1, w0, raw[0], sraw[0]);
        step(plain, j + 1, s1, s0, w0, w1, raw[1], sraw[1]);
      } else {
        step(masked, j, s0, s1, w1, w0, raw[0], sraw[0]);
        step(masked, j + 1, s1, s0, w0, w1, raw[1], sraw[1]);
      }
    }
    half8_t vf[2][DY];
    read_vals(stop - 1, vf);
    output(vf, w1);
  }
  block_sync();  // the buffers are free
  if (__ballot(wrong) && lane == 0) atomicOr(c.flags, kFlagInval);
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    l[t] += other_half(l[t]);
    if (parts > 1) {
      if (token[t] < 0) continue;
      const int64_t at = (q.row0 + token[t]) * a.heads + head[t];
      const int64_t slot = (int64_t)part * a.tokens * a.heads + at;
      const float by = vref * (1.0f / kLift);
      float* o = a.part_o + slot * D;
#pragma unroll
      for (int y = 0; y < DY; ++y)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float4_t x = {acc[t][y][4 * k] * by, acc[t][y][4 * k + 1] * by,
                              acc[t][y][4 * k + 2] * by, acc[t][y][4 * k + 3] * by};
          *reinterpret_cast<float4_t*>(o + y * 32 + k * 8 + h * 4) = x;
        }
      if (h == 0) {
        a.part_ml[2 * slot] = m[t];
        a.part_ml[2 * slot + 1] = l[t];
      }
      continue;
    }
    const bool some = l[t] > 0.0f || l[t] != l[t];
    const float inv = some ? vref * (1.0f / kLift) / l[t] : 0.0f;
    // through LDS, so that rows are written whole
    uint2* const row = reinterpret_cast<uint2*>(pool + (wave * kWide + r) * PITCH);
    if (a.bf16) {
#pragma unroll
      for (int y = 0; y < DY; ++y)
#pragma unroll
        for (int k = 0; k < 4; ++k)
          row[y * 8 + k * 2 + h] =
              make_uint2(pack_pair<true>(acc[t][y][4 * k] * inv, acc[t][y][4 * k + 1] * inv),
                         pack_pair<true>(acc[t][y][4 * k + 2] * inv, acc[t][y][4 * k + 3] * inv));
    } else {
#pragma unroll
      for (int y = 0; y < DY; ++y)
#pragma unroll
        for (int k = 0; k < 4; ++k)
          row[y * 8 + k * 2 + h] =
              make_uint2(pack_pair<false>(acc[t][y][4 * k] * inv, acc[t][y][4 * k + 1] * inv),
                         pack_pair<false>(acc[t][y][4 * k + 2] * inv, acc[t][y][4 * k + 3] * inv));
    }
    if (a.lse && h == 0 && token[t] >= 0)
      a.lse[(q.row0 + token[t]) * a.heads + head[t]] =
          some ? (m[t] + __builtin_amdgcn_logf(l[t])) * 0.6931471805599453f : kNone;
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // (a wave reads what it wrote)
    constexpr int LANES = D / 8;  // of a row
#pragma unroll 2
    for (int i = lane / LANES; i < kWide; i += kWave / LANES) {
      const int64_t rr = row0 + t * kWide + i;
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
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // before the next row tile's writes
  }
}

// Joins the parts of the key axis of the tile kernel: a wave per row.
constexpr int kJoinRows = 32;  // of a workgroup
template <int D>
__global__ __launch_bounds__(256) void kv_attend_join(KvAttendArgs a, int tile_rows) {
  Sequence q;
  int64_t tile;
  if (!find_sequence<false>(a, blockIdx.x / a.c.kv_heads, tile_rows, q, tile)) return;
  const int64_t rows = (int64_t)q.fresh * a.group;
  const int kh = blockIdx.x % a.c.kv_heads;
  int from, to, unused;
  visible(a, q, (int)(tile * tile_rows / a.group), from, unused);
  visible(a, q, (int)((min(tile * tile_rows + tile_rows, rows) - 1) / a.group), unused, to);
  const int parts = parts_of(a, from / kChunk, (to + kChunk - 1) / kChunk);
  if (parts == 1) return;
  const int64_t row0 = tile * tile_rows + (int64_t)blockIdx.y * kJoinRows;
  for (int i = threadIdx.x / kWave; i < kJoinRows && row0 + i < rows; i += 4) {
    const int64_t row = row0 + i;
    join_row<D, false>(a, q.row0 + row / a.group, kh * a.group + row % a.group, parts);
  }
}

// Waves of the tile kernel's workgroups, each with one tile of 32 rows.
template <int D>
constexpr int tile_waves() { return D > 128 ? 4 : 8; }
template <int D>
constexpr int tile_rows() { return tile_waves<D>() * kWide; }

template <int D, int FMT>
void launch_rows(const KvAttendArgs& a, dim3 grid, hipStream_t st) {
  if (D <= 128 && a.waves == 8)
    hipLaunchKernelGGL((kv_attend_rows<D, FMT, D <= 128 ? 8 : 4>), grid, dim3(8 * kWave), 0, st, a);
  else
    hipLaunchKernelGGL((kv_attend_rows<D, FMT, 4>), grid, dim3(4 * kWave), 0, st, a);
}

template <int D, int FMT>
hipError_t launch(const KvAttendArgs& a, hipStream_t st) {
  const int rows = a.tiled ? tile_rows<D>() : kRows;
  const int64_t tiles = a.cu ? a.tokens * a.group / rows + a.n
                             : a.n * ((a.group + rows - 1) / rows);
  const dim3 grid((unsigned)(tiles * a.c.kv_heads), (unsigned)a.parts);
  if (a.tiled)
    hipLaunchKernelGGL((kv_attend_tile<D, FMT, tile_waves<D>(), 1>), grid,
                       dim3(tile_waves<D>() * kWave), 0, st, a);
  else
    launch_rows<D, FMT>(a, grid, st);
  if (a.tiled && a.parts > 1)
    hipLaunchKernelGGL(kv_attend_join<D>,
                       dim3((unsigned)(tiles * a.c.kv_heads), (unsigned)(rows / kJoinRows)), dim3(256), 0, st,
                       a, rows);
  return hipGetLastError();
}

template <int D>
hipError_t launch_dim(const KvAttendArgs& a, hipStream_t st) {
  return a.c.format == SEM_KV_INT8 ? launch<D, SEM_KV_INT8>(a, st) : launch<D, SEM_KV_FP8>(a, st);
}

}  // namespace

KvSplit kv_attend_split(int dim, int64_t n, int64_t tokens, int heads, int kv_heads,
                        int64_t max_new, int64_t max_len) {
  KvSplit s = {};
  const int group = heads / kv_heads;
  s.tiled = max_new * group > 2 * kRows;
  const int rows = s.tiled ? (dim == 256 ? tile_rows<256>() : tile_rows<128>()) : kRows;
  const int64_t tiles = tokens == n ? n * ((group + rows - 1) / rows) : tokens * group / rows + n;
  const int64_t groups = std::max<int64_t>(tiles * kv_heads, 1);
  const int64_t chunks = std::max<int64_t>((max_len + kChunk - 1) / kChunk, 1);
  int64_t want = s.tiled ? 512 : 256;
  int64_t least = 32;  // chunks of a part
  if (!s.tiled) {
    s.waves = groups < 256 && dim <= 128 ? 8 : 4;
    least = 2 * s.waves;
    if (chunks <= 3 * s.waves) want = 1;
    // (their counters lie in the workspace's first bytes)
    static_assert(256 / 2 <= kKvCounts, "a counter for every tile with parts");
  }
  const int64_t parts = std::max<int64_t>(1, std::min<int64_t>(want / groups, kMostParts));
  s.part_chunks = (int)std::max<int64_t>(least, (chunks + parts - 1) / parts);
  s.parts = (int)((chunks + s.part_chunks - 1) / s.part_chunks);
  return s;
}

hipError_t launch_kv_attend(const KvAttendArgs& a, hipStream_t st) {
  if (a.n == 0 || a.tokens == 0) return hipSuccess;
  switch (a.c.head_dim) {
    case 64: return launch_dim<64>(a, st);
    case 128: return launch_dim<128>(a, st);
    default: return launch_dim<256>(a, st);
  }
}

}  // namespace semsched
