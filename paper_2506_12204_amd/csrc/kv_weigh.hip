// What the cached tokens weigh: the softmax weights that query rows give to every
// key, added up over rows and heads.
//
//   mass[j] += sum over rows r that see key j of exp(scale * ks_j (q_r . kc_j) - lse_r)
//
// with the logarithms of the sums that attention of the same rows returned, so one
// pass over the keys is enough and no values are read. The product runs on the matrix
// cores in the queries' own type, in which 8-bit codes are exact; sums and weights are
// in 32 bits. A key belongs to one workgroup, which adds its weights in an order that
// the call's sizes alone decide: results do not depend on the run.
//
// A wave has 64 keys of a head as operands in registers and goes through the row
// tiles. As in attention the product is K q^T: a lane ends up with the scores of one
// row (lane % 16) and 16 consecutive keys, whose weights it adds up in registers over
// all rows and heads that it takes.
#include <algorithm>

#include "device_common.h"
#include "kv.h"
#include "kv_codes.h"

namespace semsched {

namespace {

constexpr int WW = 8;       // waves of a workgroup
constexpr int kChunk = 64;  // keys of a wave
constexpr int kRows = 16;   // of a tile
typedef float float4_t __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));

// A listed sequence: its rows, keys, the chunks of keys that its rows see and the
// units (of several chunks) that they make.
struct Seen {
  int32_t row0, fresh, slot, len, c0, c1;
  uint32_t units;
};

__device__ __forceinline__ Seen seen_of(const KvWeighArgs& a, int64_t i) {
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
    if (blockIdx.x == 0) atomicOr(c.flags, kFlagInval);
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
  s.units = (uint32_t)((s.c1 - s.c0 + a.key_slots - 1) / a.key_slots);
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

template <int D, int FMT, bool BF16>
__global__ __launch_bounds__(WW* kWave) void kv_weigh(KvWeighArgs a) {
  using Operand = std::conditional_t<BF16, bf16x8_t, half8_t>;
  constexpr int N = D / 32;  // operands of a row or key
  __shared__ float sums[WW][kChunk];
  const KvView& c = a.c;
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int r = lane % 16, g = lane / 16;
  const int head_slots = WW / a.key_slots;
  const int key_slot = wave / head_slots, head_slot = wave % head_slots;
  if (a.cu && blockIdx.x == 0 && threadIdx.x == 0 && (a.cu[0] != 0 || a.cu[a.n] != a.tokens))
    atomicOr(c.flags, kFlagInval);
  // All units as one line, cut into equal pieces of neighbours.
  const Seen mine = seen_of(a, lane);
  uint64_t total = 0;
  for (int64_t at = 0; at < a.n; at += kWave) {
    const Seen s = at == 0 ? mine : seen_of(a, at + lane);
    total += last_lane_u64(wave_incl_scan_u64(s.units));
  }
  uint64_t u = total * blockIdx.x / gridDim.x;
  const uint64_t stop = total * (blockIdx.x + 1) / gridDim.x;
  if (u >= stop) return;
  Seen s = {};
  int64_t index = 0;
  uint32_t unit = 0;  // of the sequence
  uint64_t before = 0;
  for (int64_t at = 0; at < a.n; at += kWave) {
    const Seen x = at == 0 ? mine : seen_of(a, at + lane);
    const uint64_t upto = before + wave_incl_scan_u64(x.units);
    const uint64_t beyond = __ballot(upto > u);
    if (beyond) {
      const int first = __ffsll((unsigned long long)beyond) - 1;
      index = at + first;
      s = lane_seen(x, first);
      unit = (uint32_t)(u - (lane_u64(upto, first) - s.units));
      break;
    }
    before = last_lane_u64(upto);
  }
  const int64_t block_bytes = (int64_t)c.page_tokens * D;
  const int in_page = c.page_tokens - 1;
  bool wrong = false;
  for (; u < stop; ++u, ++unit) {
    while (unit >= s.units) {
      unit = 0;
      s = lane_seen(seen_of(a, ++index), 0);
    }
    const int chunk = s.c0 + (int)unit * a.key_slots + key_slot;
    float sum[16];
#pragma unroll
    for (int k = 0; k < 16; ++k) sum[k] = 0.0f;
    if (chunk < s.c1) {
      const int32_t* table = c.tables + (int64_t)s.slot * c.max_blocks;
      const int t0 = chunk * kChunk, vt = t0 + g * kKvTile;
      const uint32_t rows = (uint32_t)s.fresh * (uint32_t)a.group;
      const int last_block = (s.len - 1) >> c.page_shift;
      // the pages of this lane's K rows, and of its 16 keys
      const int32_t kentry = table[min((t0 + r / 4 * kKvTile) >> c.page_shift, last_block)];
      const int32_t ventry = table[min(vt >> c.page_shift, last_block)];
      const bool bad = (uint32_t)kentry >= (uint64_t)c.num_pages ||
                       (uint32_t)ventry >= (uint64_t)c.num_pages;
      wrong |= bad;
      const int64_t kpage = bad ? 0 : kentry, vpage = bad ? 0 : ventry;
      const float* scale = c.scale + (vpage * c.layers + a.layer) * 2 * c.kv_heads;
      const uint8_t* keys = c.data + kpage * c.page_bytes +
                            (int64_t)a.layer * 2 * c.kv_heads * block_bytes +
                            ((t0 + r / 4 * kKvTile) & in_page) * D + (r % 4) * 16 + g * 256;
      for (int kh = head_slot; kh < c.kv_heads; kh += head_slots) {
        Operand key[4][N];
#pragma unroll
        for (int x = 0; x < 4; ++x)
#pragma unroll
          for (int j = 0; j < D / 64; ++j)
            operands<FMT>(*reinterpret_cast<const uint4*>(keys + kh * block_bytes + x * 64 +
                                                          j * 1024),
                          key[x][2 * j], key[x][2 * j + 1]);
        const float f = scale[kh] * a.scale_log2;
        for (uint32_t row = r; row - r < rows; row += kRows) {
          const uint32_t at = min(row, rows - 1);
          const int token = (int)(at / (uint32_t)a.group);
          const int head = kh * a.group + (int)(at % (uint32_t)a.group);
          const uint16_t* q = a.q + (int64_t)(s.row0 + token) * a.q_token + head * a.q_head + g * 16;
          const float lse = a.lse[(int64_t)(s.row0 + token) * a.heads + head];
          Operand query[N];
#pragma unroll
          for (int j = 0; j < N; ++j) {
            const uint16_t* p = q + j / 2 * 64 + j % 2 * 8;
            uint4 w;
            if (a.wide) {
              w = *reinterpret_cast<const uint4*>(p);
            } else {
              w = make_uint4(p[0] | (uint32_t)p[1] << 16, p[2] | (uint32_t)p[3] << 16,
                             p[4] | (uint32_t)p[5] << 16, p[6] | (uint32_t)p[7] << 16);
            }
            query[j] = __builtin_bit_cast(Operand, w);
          }
          // Rows that see no key, are not numbers, or are not there weigh nothing.
          const bool live = row < rows && fabsf(lse) < __builtin_inff();
          if (__ballot(!live)) {
#pragma unroll
            for (int j = 0; j < N; ++j)
              query[j] = live ? query[j] : __builtin_bit_cast(Operand, make_uint4(0, 0, 0, 0));
          }
          const float base = live ? lse * 1.4426950408889634f : __builtin_inff();
          const int pos = s.len - s.fresh + token;
          const int high = a.causal ? min(pos + 1, s.len) : s.len;
          const int low = a.window > 0 && pos >= a.window ? pos + 1 - a.window : 0;
          const bool hides = __ballot(low > t0 || high < t0 + kChunk) != 0;
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            float4_t t = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int j = 0; j < N; ++j) t = product(key[x][j], query[j], t);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              float p = __builtin_amdgcn_exp2f(__builtin_fmaf(t[i], f, -base));
              if (hides) p = vt + 4 * x + i >= low && vt + 4 * x + i < high ? p : 0.0f;
              sum[4 * x + i] += p;
            }
          }
        }
      }
    }
    // the sixteen lanes of a group each hold other rows: lane r gets key r's sum
#pragma unroll
    for (int off = 8; off > 0; off /= 2) {
      const bool upper = (r & off) != 0;
#pragma unroll
      for (int k = 0; k < off; ++k) {
        const float give = upper ? sum[k] : sum[k + off];
        const float keep = upper ? sum[k + off] : sum[k];
        sum[k] = keep + __shfl_xor(give, off, kWave);
      }
    }
    if (head_slots > 1) {
      sums[wave][lane] = sum[0];
      block_sync();
    }
    const int key = chunk * kChunk + lane;
    if (head_slot == 0 && chunk < s.c1 && key < s.len) {
      float x = sum[0];
      for (int k = 1; k < head_slots; ++k) x += sums[wave + k][lane];
      a.mass[s.slot * a.mass_stride + key] += x;
    }
    if (head_slots > 1) block_sync();
  }
  if (__ballot(wrong) && lane == 0) atomicOr(c.flags, kFlagInval);
}

template <int D, int FMT>
void launch_type(const KvWeighArgs& a, unsigned grid, hipStream_t st) {
  if (a.bf16)
    hipLaunchKernelGGL((kv_weigh<D, FMT, true>), dim3(grid), dim3(WW * kWave), 0, st, a);
  else
    hipLaunchKernelGGL((kv_weigh<D, FMT, false>), dim3(grid), dim3(WW * kWave), 0, st, a);
}

template <int D>
void launch_dim(const KvWeighArgs& a, unsigned grid, hipStream_t st) {
  if (a.c.format == SEM_KV_INT8) launch_type<D, SEM_KV_INT8>(a, grid, st);
  else launch_type<D, SEM_KV_FP8>(a, grid, st);
}

}  // namespace

hipError_t launch_kv_weigh(const KvWeighArgs& args, int64_t max_len, hipStream_t st) {
  if (args.n == 0) return hipSuccess;  // (without tokens the offsets are looked at)
  KvWeighArgs a = args;
  // Waves that share 64 keys and deal out their heads, where there are too few keys
  // for a wave each.
  const int64_t chunks = std::max<int64_t>(1, a.n * ((max_len + kChunk - 1) / kChunk));
  int head_slots = 1;
  while (head_slots < WW && 2 * head_slots <= a.c.kv_heads && chunks * head_slots < 512 * WW)
    head_slots *= 2;
  a.key_slots = WW / head_slots;
  const unsigned grid =
      (unsigned)std::min<int64_t>(512, (chunks + a.key_slots - 1) / a.key_slots + a.n);
  switch (a.c.head_dim) {
    case 64: launch_dim<64>(a, grid, st); break;
    case 128: launch_dim<128>(a, grid, st); break;
    default: launch_dim<256>(a, grid, st);
  }
  return hipGetLastError();
}

}  // namespace semsched
