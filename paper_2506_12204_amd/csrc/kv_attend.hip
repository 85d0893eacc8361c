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

#include "device_common.h"
#include "kv.h"
#include "kv_codes.h"

namespace semsched {

namespace {

typedef float float4_t __attribute__((ext_vector_type(4)));

constexpr int kRows = 16;            // rows of a tile: a token and a head each
constexpr int kChunk = 64;           // keys a wave takes at a time
constexpr int kWaves = 4;
constexpr float kLift = 16384.0f;    // 2^14
constexpr float kNone = -__builtin_inff();

// Row tiles are numbered without reading the lengths: those of sequence i start
// at cu[i] * group / rows + i, which leaves room for a partly filled one.
__device__ __forceinline__ int64_t tile_start(const KvAttendArgs& a, int64_t i, int rows) {
  return ((int64_t)(a.cu ? a.cu[i] : (int32_t)i) * a.group) / rows + i;
}

struct Sequence {
  const int32_t* table;
  int64_t row0;     // first query token
  int fresh, len;   // query tokens, keys
};

// The sequence of row tile u and u's number in it; false if there is none.
__device__ __forceinline__ bool find_sequence(const KvAttendArgs& a, int64_t u, int rows,
                                              Sequence& q, int64_t& tile) {
  const KvView& c = a.c;
  int64_t i = 0, end = a.n;
  while (end - i > 1) {
    const int64_t mid = (i + end) / 2;
    if (tile_start(a, mid, rows) <= u) i = mid;
    else end = mid;
  }
  if (a.cu && u == 0 && (a.cu[0] != 0 || a.cu[a.n] != a.tokens) && threadIdx.x == 0)
    atomicOr(c.flags, kFlagInval);
  q.row0 = a.cu ? a.cu[i] : i;
  const int64_t fresh = a.cu ? (int64_t)a.cu[i + 1] - q.row0 : 1;
  if (fresh < 0 || q.row0 < 0 || q.row0 + fresh > a.tokens) {
    if (threadIdx.x == 0) atomicOr(c.flags, kFlagInval);
    return false;
  }
  tile = u - tile_start(a, i, rows);
  if (tile < 0 || tile * rows >= fresh * a.group) return false;
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

__device__ __forceinline__ uint16_t to16(float x, int bf16) {
  if (bf16) {
    const uint32_t u = __float_as_uint(x);
    if (x != x) return 0x7fc0;
    return (uint16_t)((u + 0x7fffu + ((u >> 16) & 1u)) >> 16);
  }
  return __builtin_bit_cast(uint16_t, (_Float16)x);
}

// A row's query in halves: lane group g holds channels (4 j + g) * 16 .. + 15
// for j < D / 64. Returns what the scores have to be multiplied by.
template <int D>
__device__ __forceinline__ float load_query(const KvAttendArgs& a, const uint16_t* row, bool live,
                                            int g, half8_t (&q)[D / 32]) {
  uint16_t e[D / 4];
#pragma unroll
  for (int j = 0; j < D / 64; ++j) {
    const uint16_t* p = row + (4 * j + g) * 16;
    if (!live) {
#pragma unroll
      for (int k = 0; k < 16; ++k) e[16 * j + k] = 0;
    } else if (a.wide) {
      *reinterpret_cast<uint4*>(e + 16 * j) = reinterpret_cast<const uint4*>(p)[0];
      *reinterpret_cast<uint4*>(e + 16 * j + 8) = reinterpret_cast<const uint4*>(p)[1];
    } else {
#pragma unroll
      for (int k = 0; k < 16; ++k) e[16 * j + k] = p[k];
    }
  }
  if (!a.bf16) {
#pragma unroll
    for (int k = 0; k < D / 4; ++k) q[k / 8][k % 8] = __builtin_bit_cast(_Float16, e[k]);
    return 1.0f;
  }
  float top = 0.0f;
#pragma unroll
  for (int k = 0; k < D / 4; ++k) top = fmaxf(top, fabsf(load16(e[k], 1)));
  top = fmaxf(top, __shfl_xor(top, 16, kWave));
  top = fmaxf(top, __shfl_xor(top, 32, kWave));
  // 2^(14 - exponent), between 2^-126 and 2^126; rows of zeros or with an
  // infinity stay as they are
  const int e2 = (int)(__float_as_uint(top) >> 23);
  const int shift = top > 0.0f && e2 < 255 ? min(max(14 - (e2 - 127), -126), 126) : 0;
  const float up = __uint_as_float((uint32_t)(127 + shift) << 23);
#pragma unroll
  for (int k = 0; k < D / 4; ++k) q[k / 8][k % 8] = (_Float16)(load16(e[k], 1) * up);
  return __uint_as_float((uint32_t)(127 - shift) << 23);
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

// One workgroup: a tile of 16 rows of one KV head over one part of the key
// axis; its four waves take chunks of 64 keys in turn and join at the end.
//
// The score product is taken as K q^T, so that a lane ends up with scores of
// one row (lane % 16) and of 16 consecutive keys (tile lane / 16 of the chunk),
// which is what the second product V^T P^T wants of it: weights go from one to
// the other in registers. The cache's tiles are laid out for these operands: a
// lane's 16-byte load is 16 channels of a key or 16 keys of a channel, and no
// LDS is used before the join. A lane's 16 keys lie in one page, so the scales
// are one number each per lane and chunk.
template <int D, int FMT>
__global__ __launch_bounds__(kWaves* kWave) void kv_attend_rows(KvAttendArgs a) {
  __shared__ float join_o[2][D][kRows];
  __shared__ float join_m[kWaves][kRows], join_l[kWaves][kRows];
  const KvView& c = a.c;
  const int lane = lane_id(), wave = threadIdx.x / kWave;
  const int r = lane % 16, g = lane / 16;
  const int kh = blockIdx.y;
  Sequence q;
  int64_t tile;
  if (!find_sequence(a, blockIdx.x, kRows, q, tile)) return;
  const int64_t rows = (int64_t)q.fresh * a.group;
  const int64_t row = tile * kRows + r;
  const bool live = row < rows;
  const int token = (int)((live ? row : rows - 1) / a.group);
  const int head = kh * a.group + (int)((live ? row : rows - 1) % a.group);
  half8_t query[D / 32];
  const float undo = load_query<D>(
      a, a.q + (q.row0 + token) * a.q_token + head * a.q_head, live, g, query);
  const float factor = undo * a.scale_log2;
  int low, high;
  visible(a, q, token, low, high);
  // the keys that any row of the tile sees
  int from, to, unused;
  visible(a, q, (int)(tile * kRows / a.group), from, unused);
  visible(a, q, (int)((min(tile * kRows + kRows, rows) - 1) / a.group), unused, to);
  const int c0 = from / kChunk, c1 = (to + kChunk - 1) / kChunk;
  const int per = (max(c1 - c0, 0) + a.splits - 1) / a.splits;
  const int begin = c0 + (int)blockIdx.z * per, stop = min(begin + per, c1);

  float m = kNone, l = 0.0f, vref = 0.0f;
  float4_t acc[D / 16];
#pragma unroll
  for (int y = 0; y < D / 16; ++y) acc[y] = float4_t{0.0f, 0.0f, 0.0f, 0.0f};
  const int64_t block_bytes = (int64_t)c.page_tokens * D;
  const int64_t k_off = (((int64_t)a.layer * 2) * c.kv_heads + kh) * block_bytes;
  const int64_t v_off = (((int64_t)a.layer * 2 + 1) * c.kv_heads + kh) * block_bytes;
  const int in_page = c.page_tokens - 1;
  const int last_block = (q.len - 1) >> c.page_shift;
  bool wrong = false;
  for (int ch = begin + wave; ch < stop; ch += kWaves) {
    const int t0 = ch * kChunk;
    // the pages of this lane's key rows and of its 16 keys
    const int kt = t0 + r / 4 * kKvTile, vt = t0 + g * kKvTile;
    int64_t kpage = q.table[min(kt >> c.page_shift, last_block)];
    int64_t vpage = q.table[min(vt >> c.page_shift, last_block)];
    if (kpage < 0 || kpage >= c.num_pages) {
      wrong = true;
      kpage = 0;
    }
    if (vpage < 0 || vpage >= c.num_pages) {
      wrong = true;
      vpage = 0;
    }
    const uint8_t* kp = c.data + kpage * c.page_bytes + k_off + (int64_t)(kt & in_page) * D +
                        (r % 4) * 16 + g * 256;
    const uint8_t* vp = c.data + vpage * c.page_bytes + v_off + (int64_t)(vt & in_page) * D + r * 16;
    const float* sp = c.scale + (vpage * c.layers + a.layer) * 2 * c.kv_heads + kh;
    const float ks = sp[0] * factor, vs = sp[c.kv_heads];
    uint4 kc[4][D / 64], vc[D / 16];
#pragma unroll
    for (int x = 0; x < 4; ++x)
#pragma unroll
      for (int j = 0; j < D / 64; ++j)
        kc[x][j] = *reinterpret_cast<const uint4*>(kp + x * 64 + j * 1024);
#pragma unroll
    for (int y = 0; y < D / 16; ++y) vc[y] = *reinterpret_cast<const uint4*>(vp + y * 256);
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
      for (int i = 0; i < 4; ++i) s[4 * x + i] = t[i] * ks;
    }
    // keys that this row does not see (whatever is held there)
#pragma unroll
    for (int k = 0; k < 16; ++k) s[k] = vt + k >= low && vt + k < high && live ? s[k] : kNone;
    if (t0 + kChunk > q.len) {
#pragma unroll
      for (int y = 0; y < D / 16; ++y) {
        const int n = q.len - vt;
        vc[y].x = keep_bytes(vc[y].x, n);
        vc[y].y = keep_bytes(vc[y].y, n - 4);
        vc[y].z = keep_bytes(vc[y].z, n - 8);
        vc[y].w = keep_bytes(vc[y].w, n - 12);
      }
    }
    float top = s[0];
#pragma unroll
    for (int k = 1; k < 16; ++k) top = fmaxf(top, s[k]);
    top = fmaxf(top, __shfl_xor(top, 16, kWave));
    top = fmaxf(top, __shfl_xor(top, 32, kWave));
    const float next = fmaxf(m, top);
    const float base = next == kNone ? 0.0f : next;  // no key so far: exp2(-inf) = 0
    float shrink = __builtin_amdgcn_exp2f(m - base);
    m = next;
    float sum = 0.0f;
    float p[16];
#pragma unroll
    for (int k = 0; k < 16; ++k) {
      p[k] = __builtin_amdgcn_exp2f(s[k] - base);
      sum += p[k];
    }
    l = l * shrink + sum;
    // weights relative to the largest V scale so far
    float vmax = fmaxf(vs, __shfl_xor(vs, 16, kWave));
    vmax = fmaxf(vmax, __shfl_xor(vmax, 32, kWave));
    if (vmax > vref) {
      shrink *= vref / vmax;
      vref = vmax;
    }
    const float rel = vref > 0.0f ? vs / vref * kLift : 0.0f;
    half8_t w0, w1;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      w0[k] = (_Float16)(p[k] * rel);
      w1[k] = (_Float16)(p[8 + k] * rel);
    }
#pragma unroll
    for (int y = 0; y < D / 16; ++y) {
      half8_t lo, hi;
      codes_to_operands<FMT>(vc[y], lo, hi);
      acc[y] *= shrink;
      acc[y] = __builtin_amdgcn_mfma_f32_16x16x32_f16(lo, w0, acc[y], 0, 0, 0);
      acc[y] = __builtin_amdgcn_mfma_f32_16x16x32_f16(hi, w1, acc[y], 0, 0, 0);
    }
  }
  if (__ballot(wrong) && lane == 0) atomicOr(c.flags, kFlagInval);
  // the four lane groups of a row each hold a quarter of its sum
  l += __shfl_xor(l, 16, kWave);
  l += __shfl_xor(l, 32, kWave);
  if (g == 0) {
    join_m[wave][r] = m;
    join_l[wave][r] = l;
  }
  block_sync();
  float most = kNone;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) most = fmaxf(most, join_m[w][r]);
  const float base = most == kNone ? 0.0f : most;
  float total = 0.0f;
#pragma unroll
  for (int w = 0; w < kWaves; ++w)
    total += join_l[w][r] * __builtin_amdgcn_exp2f(join_m[w][r] - base);
  const float mine = __builtin_amdgcn_exp2f(m - base) * (vref * (1.0f / kLift));
#pragma unroll
  for (int y = 0; y < D / 16; ++y) acc[y] *= mine;
#pragma unroll
  for (int half = kWaves / 2; half > 0; half /= 2) {
    if (wave >= half && wave < 2 * half) {
#pragma unroll
      for (int y = 0; y < D / 16; ++y)
#pragma unroll
        for (int i = 0; i < 4; ++i) join_o[wave - half][y * 16 + g * 4 + i][r] = acc[y][i];
    }
    block_sync();
    if (wave < half) {
#pragma unroll
      for (int y = 0; y < D / 16; ++y)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[y][i] += join_o[wave][y * 16 + g * 4 + i][r];
    }
    block_sync();
  }
  if (wave != 0 || !live) return;
  const int64_t at = (q.row0 + token) * a.heads + head;
  if (a.splits > 1) {
    const int64_t part = (int64_t)blockIdx.z * a.tokens * a.heads + at;
    float* o = a.part_o + part * D;
#pragma unroll
    for (int y = 0; y < D / 16; ++y)
      *reinterpret_cast<float4_t*>(o + y * 16 + g * 4) = acc[y];
    if (g == 0) {
      a.part_ml[2 * part] = most;
      a.part_ml[2 * part + 1] = total;
    }
    return;
  }
  const float inv = total > 0.0f || total != total ? 1.0f / total : 0.0f;
  uint16_t* o = a.out + (q.row0 + token) * a.out_token + head * a.out_head;
#pragma unroll
  for (int y = 0; y < D / 16; ++y)
#pragma unroll
    for (int i = 0; i < 4; ++i) o[y * 16 + g * 4 + i] = to16(acc[y][i] * inv, a.bf16);
  if (a.lse && g == 0)
    a.lse[at] = total > 0.0f || total != total
                    ? (most + __builtin_amdgcn_logf(total)) * 0.6931471805599453f
                    : kNone;
}

// Joins the parts of the key axis: one wave per row.
template <int D>
__global__ __launch_bounds__(256) void kv_attend_join(KvAttendArgs a) {
  const int64_t all = a.tokens * a.heads;
  const int64_t at = (int64_t)blockIdx.x * 4 + threadIdx.x / kWave;
  if (at >= all) return;
  const int lane = lane_id();
  float most = kNone;
  for (int k = 0; k < a.splits; ++k) most = fmaxf(most, a.part_ml[2 * (k * all + at)]);
  const float base = most == kNone ? 0.0f : most;
  float total = 0.0f, o[D / 64];
#pragma unroll
  for (int j = 0; j < D / 64; ++j) o[j] = 0.0f;
  for (int k = 0; k < a.splits; ++k) {
    const int64_t part = k * all + at;
    const float w = __builtin_amdgcn_exp2f(a.part_ml[2 * part] - base);
    total += a.part_ml[2 * part + 1] * w;
#pragma unroll
    for (int j = 0; j < D / 64; ++j) o[j] += a.part_o[part * D + j * 64 + lane] * w;
  }
  const float inv = total > 0.0f || total != total ? 1.0f / total : 0.0f;
  uint16_t* out = a.out + at / a.heads * a.out_token + at % a.heads * a.out_head;
#pragma unroll
  for (int j = 0; j < D / 64; ++j) out[j * 64 + lane] = to16(o[j] * inv, a.bf16);
  if (a.lse && lane == 0)
    a.lse[at] = total > 0.0f || total != total
                    ? (most + __builtin_amdgcn_logf(total)) * 0.6931471805599453f
                    : kNone;
}

template <int D, int FMT>
hipError_t launch(const KvAttendArgs& a, hipStream_t st) {
  const int64_t tiles = a.tokens * a.group / kRows + a.n;
  hipLaunchKernelGGL((kv_attend_rows<D, FMT>),
                     dim3((unsigned)tiles, (unsigned)a.c.kv_heads, (unsigned)a.splits),
                     dim3(kWaves * kWave), 0, st, a);
  if (a.splits > 1) {
    const int64_t all = a.tokens * a.heads;
    hipLaunchKernelGGL(kv_attend_join<D>, dim3((unsigned)((all + 3) / 4)), dim3(256), 0, st, a);
  }
  return hipGetLastError();
}

template <int D>
hipError_t launch_dim(const KvAttendArgs& a, hipStream_t st) {
  return a.c.format == SEM_KV_INT8 ? launch<D, SEM_KV_INT8>(a, st) : launch<D, SEM_KV_FP8>(a, st);
}

}  // namespace

int kv_attend_splits(int64_t n, int64_t tokens, int heads, int kv_heads, int64_t max_new,
                     int64_t max_len) {
  (void)max_new;
  const int64_t groups = (tokens * (heads / kv_heads) / kRows + n) * kv_heads;
  const int64_t most = (max_len + 4 * kChunk - 1) / (4 * kChunk);  // a chunk per wave at least
  return (int)std::max<int64_t>(1, std::min<int64_t>({most, 2048 / std::max<int64_t>(groups, 1),
                                                      128}));
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
