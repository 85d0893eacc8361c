// Appending to the KV cache: the new tokens' keys and values become 8-bit codes
// of their pages' blocks. A block (a page's K or V of one head) has one scale,
// the largest magnitude over its tokens over the largest code:
//
//   s' = max(s if the block holds older tokens else 0, max |x| * (1 / top))
//   older codes, if s' > s:  c <- round(c * s / s')
//   new codes:               c  = round(x / s')
//
// with quotients and products in 32 bits, each rounded once (the codes are the
// nearest to the quotients; a block of zeros has scale 0 and codes 0).
// Elements that are not finite count as 0 in the maximum, are stored as the
// largest code or 0 (NaN), and are reported as a range error.
//
// One wave per block. It holds up to 64 tokens of the block in registers, so
// that blocks of that size are read once; the loads are arranged so that a lane
// ends up with whole 16-byte units of the cache's layout, and no data passes
// through LDS. Bound by memory: prompts of 24 sequences (500 to 8192 tokens, 8 KV
// heads of 128 channels) are written at 4.7 TB/s of rows and codes (108 us), what
// a large copy reaches; one token for each of 256 sequences takes 8.2 us, the
// launch and the chain from the sequence to its page (13.8 us with offsets, whose
// search takes 64 at a time), for each of 4096 87 us (133 us with offsets: two units
// a sequence, each with a search of its own). Blocks of more than 64 tokens are read
// twice, for the maximum and for the codes: the same prompts on pages of 128 take
// 162 us, of 256 187 us, of 1024 327 us.
#include <algorithm>

#include "device_common.h"
#include "kv.h"
#include "kv_codes.h"

namespace semsched {

namespace {

constexpr int AW = 4;      // waves per workgroup, each on a block of its own
constexpr int kHeld = 64;  // tokens of a block that a wave holds at a time

// x / by for one `by`, rounded correctly from the reciprocal (rounded correctly,
// too) by one step with the remainder: Markstein's theorem, as long as nothing
// underflows, for which x and `by` are first brought to a middle range by the
// same power of two.
struct Quotient {
  float by, inv, lift;
  __device__ __forceinline__ explicit Quotient(float b) {
    lift = b < 0x1p-64f ? 0x1p64f : b > 0x1p64f ? 0x1p-64f : 1.0f;
    by = b * lift;
    inv = 1.0f / by;
  }
  __device__ __forceinline__ float of(float x) const {
    const float y = x * lift, q = y * inv;
    return __builtin_fmaf(__builtin_fmaf(-q, by, y), inv, q);
  }
};

// Four quotients as codes: ties to even, beyond the range the largest code. (NaN
// does not reach this.)
template <int FMT>
__device__ __forceinline__ uint32_t pack_codes(float a, float b, float c, float d) {
  const float top = code_max<FMT>();
  a = __builtin_amdgcn_fmed3f(a, -top, top);
  b = __builtin_amdgcn_fmed3f(b, -top, top);
  c = __builtin_amdgcn_fmed3f(c, -top, top);
  d = __builtin_amdgcn_fmed3f(d, -top, top);
  if (FMT == SEM_KV_INT8) {
    // 1.5 * 2^23 more: the sum's low byte is the nearest whole number
    const uint32_t x = __float_as_uint(a + 12582912.0f), y = __float_as_uint(b + 12582912.0f);
    const uint32_t z = __float_as_uint(c + 12582912.0f), w = __float_as_uint(d + 12582912.0f);
    return __builtin_amdgcn_perm(__builtin_amdgcn_perm(w, z, 0x0c0c0400u),
                                 __builtin_amdgcn_perm(y, x, 0x0c0c0400u), 0x05040100u);
  }
  int p = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, p, true);
}

template <int BF16>
__device__ __forceinline__ float low_half(uint32_t w) {
  return BF16 ? __uint_as_float(w << 16) : (float)__builtin_bit_cast(half2_t, w)[0];
}
template <int BF16>
__device__ __forceinline__ float high_half(uint32_t w) {
  return BF16 ? __uint_as_float(w & 0xffff0000u) : (float)__builtin_bit_cast(half2_t, w)[1];
}

// The larger of two pairs of 16-bit magnitudes: as numbers their order is that
// of the floats.
__device__ __forceinline__ uint32_t max_pairs(uint32_t a, uint32_t b) {
  typedef uint16_t pair_t __attribute__((ext_vector_type(2)));
  const pair_t x = __builtin_bit_cast(pair_t, a), y = __builtin_bit_cast(pair_t, b & 0x7fff7fffu);
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(x, y));
}

// A 16-bit element that is infinite becomes `top` with its sign, NaN becomes 0.
template <int BF16>
__device__ __forceinline__ uint32_t tame(uint32_t e, uint32_t top) {
  const uint32_t inf = BF16 ? 0x7f80u : 0x7c00u, m = e & 0x7fffu;
  return m < inf ? e : m == inf ? (e & 0x8000u) | top : 0u;
}

// Units of work: pages touched by new tokens, bounded and numbered without
// reading the lengths: sequence i starts at cu[i] / page_tokens + 2 i, which
// leaves room for a partly filled page at either end. Without offsets, one token
// each, unit i is sequence i's page.
__device__ __forceinline__ int64_t append_start(const KvAppendArgs& a, int64_t i) {
  return (a.cu[i] >> a.c.page_shift) + 2 * i;
}

// A block's new tokens [lo, hi), rows x + (token - lo) * stride.
//
// K: a lane takes the 16 channels of one unit, two 16-byte loads; the lanes of a
// load are 16 tokens of a tile times four units of 64 channels. V: a lane takes
// W = D / 64 channels (at least two) of the 16 tokens of a tile, whose codes are
// that many units side by side. Both hold 64 tokens in D / 2 registers.
template <int D, int FMT, int BF16, int WHICH, bool WIDE>
struct Block {
  static constexpr int W = D / 64 > 1 ? D / 64 : 2;    // V channels of a lane
  static constexpr int SIDE = kWave * W / D;           // V tiles that a wave's lanes cover
  static constexpr int TILES = kHeld / kKvTile;
  uint32_t x[D / 2];

  __device__ __forceinline__ static int v_tile(int i) {
    return i * SIDE + (SIDE > 1 ? lane_id() / (D / W) : 0);
  }
  __device__ __forceinline__ static int v_channel() { return lane_id() % (D / W) * W; }

  // Tokens [t0, t0 + 64) of the block; those outside [lo, hi) are zero.
  __device__ __forceinline__ void load(const uint16_t* rows, int64_t stride, int t0, int lo,
                                       int hi) {
    if (WHICH == 0) {
#pragma unroll
      for (int i = 0; i < TILES; ++i) {
        const int t = t0 + i * kKvTile + lane_id() % 16;
        const bool live = t >= lo && t < hi;
#pragma unroll
        for (int j = 0; j < D / 64; ++j) {
          uint32_t* to = x + (i * (D / 64) + j) * 8;
          const uint16_t* p = rows + (int64_t)(t - lo) * stride + (j * 4 + lane_id() / 16) * 16;
          if (!live) {
#pragma unroll
            for (int k = 0; k < 8; ++k) to[k] = 0;
          } else if (WIDE) {
            const uint4 a = reinterpret_cast<const uint4*>(p)[0];
            const uint4 b = reinterpret_cast<const uint4*>(p)[1];
            to[0] = a.x, to[1] = a.y, to[2] = a.z, to[3] = a.w;
            to[4] = b.x, to[5] = b.y, to[6] = b.z, to[7] = b.w;
          } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) to[k] = p[2 * k] | ((uint32_t)p[2 * k + 1] << 16);
          }
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < TILES / SIDE; ++i)
#pragma unroll
        for (int k = 0; k < 16; ++k) {
          const int t = t0 + v_tile(i) * kKvTile + k;
          uint32_t* to = x + (i * 16 + k) * (W / 2);
          const uint16_t* p = rows + (int64_t)(t - lo) * stride + v_channel();
          const bool live = t >= lo && t < hi;
#pragma unroll
          for (int w = 0; w < W / 2; ++w)
            to[w] = !live ? 0u
                    : WIDE ? reinterpret_cast<const uint32_t*>(p)[w]
                           : p[2 * w] | ((uint32_t)p[2 * w + 1] << 16);
        }
    }
  }

  __device__ __forceinline__ uint32_t largest() const {
    uint32_t top = 0;
#pragma unroll
    for (int k = 0; k < D / 2; ++k) top = max_pairs(top, x[k]);
    return max(top & 0xffffu, top >> 16);
  }

  __device__ __forceinline__ uint32_t largest_finite() const {
    const uint32_t inf = BF16 ? 0x7f80u : 0x7c00u;
    uint32_t top = 0;
#pragma unroll
    for (int k = 0; k < D / 2; ++k) {
      const uint32_t a = x[k] & 0x7fffu, b = x[k] >> 16 & 0x7fffu;
      if (a < inf) top = max(top, a);
      if (b < inf) top = max(top, b);
    }
    return top;
  }

  // Element (unit-relative) of the held tokens as a quotient.
  __device__ __forceinline__ uint32_t four(const uint32_t* p, int step, bool high,
                                           const Quotient& q) const {
    float f[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const uint32_t w = p[k * step];
      f[k] = q.of(high ? high_half<BF16>(w) : low_half<BF16>(w));
    }
    return pack_codes<FMT>(f[0], f[1], f[2], f[3]);
  }

  // Older codes of a unit on the new scale.
  __device__ __forceinline__ static uint32_t again(uint32_t codes, float was, const Quotient& q) {
    float f[4];
#pragma unroll
    for (int k = 0; k < 4; ++k)
      f[k] = q.of(code_to_float<FMT>(codes >> (8 * k) & 0xffu) * was);
    return pack_codes<FMT>(f[0], f[1], f[2], f[3]);
  }

  __device__ __forceinline__ void store(uint8_t* block, int t0, int lo, int hi, const Quotient& q) {
    if (WHICH == 0) {
#pragma unroll
      for (int i = 0; i < TILES; ++i) {
        const int tile = t0 / kKvTile + i, t = tile * kKvTile + lane_id() % 16;
        if (t < lo || t >= hi) continue;
#pragma unroll
        for (int j = 0; j < D / 64; ++j) {
          const uint32_t* p = x + (i * (D / 64) + j) * 8;
          uint32_t u[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const float e0 = q.of(low_half<BF16>(p[2 * k]));
            const float e1 = q.of(high_half<BF16>(p[2 * k]));
            const float e2 = q.of(low_half<BF16>(p[2 * k + 1]));
            const float e3 = q.of(high_half<BF16>(p[2 * k + 1]));
            u[k] = pack_codes<FMT>(e0, e1, e2, e3);
          }
          *reinterpret_cast<uint4*>(block + tile * (kKvTile * D) + (j * 4 + lane_id() / 16) * 256 +
                                    lane_id() % 16 * 16) = make_uint4(u[0], u[1], u[2], u[3]);
        }
      }
      return;
    }
#pragma unroll
    for (int i = 0; i < TILES / SIDE; ++i) {
      const int tile = t0 / kKvTile + v_tile(i), first = tile * kKvTile;
      const int k0 = max(lo - first, 0), k1 = min(hi - first, kKvTile);
      if (k1 <= k0) continue;
#pragma unroll
      for (int w = 0; w < W; ++w) {
        uint8_t* at = block + tile * (kKvTile * D) + (v_channel() + w) * 16;
        uint32_t u[4];
#pragma unroll
        for (int k = 0; k < 4; ++k)
          u[k] = four(x + (i * 16 + 4 * k) * (W / 2) + w / 2, W / 2, w % 2 != 0, q);
        if (k1 - k0 == kKvTile) {
          *reinterpret_cast<uint4*>(at) = make_uint4(u[0], u[1], u[2], u[3]);
        } else {  // the other tokens' codes stay
          for (int k = k0; k < k1; ++k) {
            const uint32_t word = k < 8 ? (k < 4 ? u[0] : u[1]) : (k < 12 ? u[2] : u[3]);
            at[k] = (uint8_t)(word >> (8 * (k & 3)));
          }
        }
      }
    }
  }

  // The codes of tokens [0, lo) on the new scale, before the new ones are stored.
  __device__ __forceinline__ static void rescale(uint8_t* block, int lo, float was,
                                                 const Quotient& q) {
    const int last = (lo + kKvTile - 1) / kKvTile * D;
    for (int u = lane_id(); u < last; u += kWave) {
      const int tile = u / D, in = u % D;
      if (WHICH == 0 && tile * kKvTile + in % 16 >= lo) continue;
      uint4* at = reinterpret_cast<uint4*>(block) + u;
      const uint4 old = *at;
      uint32_t w[4] = {old.x, old.y, old.z, old.w};
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint32_t now = again(w[k], was, q);
        const int n = WHICH == 0 ? 4 : lo - tile * kKvTile - 4 * k;  // older ones of these four
        const uint32_t keep = n >= 4 ? 0u : n <= 0 ? ~0u : ~0u << (8 * n);
        w[k] = (now & ~keep) | (w[k] & keep);
      }
      *at = make_uint4(w[0], w[1], w[2], w[3]);
    }
  }

  __device__ __forceinline__ void write(const uint16_t* rows, int64_t stride, uint8_t* block,
                                        int lo, int hi, float was, bool grown, bool wild,
                                        uint32_t top, const Quotient& q) {
    if (grown) {
      rescale(block, lo, was, q);
      wait_stores();  // (a unit may be shared by the two loops' lanes)
    }
    const int first = lo / kHeld * kHeld;
    const bool many = hi - first > kHeld;
    for (int t0 = first; t0 < hi; t0 += kHeld) {
      if (many) load(rows, stride, t0, lo, hi);
      if (wild) {
#pragma unroll
        for (int k = 0; k < D / 2; ++k)
          x[k] = tame<BF16>(x[k] & 0xffffu, top) | tame<BF16>(x[k] >> 16, top) << 16;
      }
      store(block, t0, lo, hi, q);
    }
  }

  __device__ __forceinline__ void run(const KvAppendArgs& a, const uint16_t* rows, int64_t stride,
                                      int lo, int hi, int64_t slot, int head) {
    const KvView& c = a.c;
    float* scale = c.scale + slot * c.kv_heads + head;
    uint8_t* block = c.data + (slot * c.kv_heads + head) * ((int64_t)c.page_tokens * D);
    const float was = lo > 0 ? *scale : 0.0f;
    const uint32_t inf = BF16 ? 0x7f80u : 0x7c00u;
    uint32_t top = 0;
    const int first = lo / kHeld * kHeld;
    bool wild = false;
    for (int t0 = first; t0 < hi; t0 += kHeld) {
      load(rows, stride, t0, lo, hi);
      uint32_t most = largest();
      if (most >= inf) {
        wild = true;
        most = largest_finite();
      }
      top = max(top, most);
    }
    top = wave_max_u32(top);
    wild = __ballot(wild) != 0;
    if (wild && lane_id() == 0) atomicOr(c.flags, kFlagRange);
    const float now = fmaxf(was, low_half<BF16>(top) * (1.0f / code_max<FMT>()));
    const bool grown = lo > 0 && now > was;
    if (lane_id() == 0 && (lo == 0 || grown)) *scale = now;
    const Quotient q(now > 0.0f ? now : 1.0f);
    // infinities: a little over the largest code, as far as the type reaches
    const float over = fminf(now * (code_max<FMT>() * 1.015625f), BF16 ? 0x1.fep127f : 65504.0f);
    const uint32_t huge = BF16 ? __float_as_uint(over) >> 16
                               : (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)over);
    write(rows, stride, block, lo, hi, was, grown, wild, huge, q);
  }
};

template <int D, int FMT, int BF16, bool WIDE>
__global__ __launch_bounds__(AW* kWave) void kv_append(KvAppendArgs a) {
  const KvView& c = a.c;
  const int64_t u = blockIdx.x;
  const int part = blockIdx.y * AW + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  // The columns behind the units look for offsets that fall, which the search below
  // need not come by. (Looked for by the units themselves, 4096 single tokens take
  // 140 us instead of 131.)
  if (blockIdx.x >= a.units) {
    const int64_t pair = (int64_t)(blockIdx.x - a.units) * (AW * kWave) + threadIdx.x;
    if (blockIdx.y == 0 && pair < a.n && a.cu[pair + 1] < a.cu[pair])
      atomicOr(c.flags, kFlagInval);
    return;
  }
  if (part >= 2 * c.kv_heads) return;
  int64_t i = u;
  if (a.cu) {  // the last sequence that starts at or before u, 64 at a time
    int64_t end = a.n;
    i = 0;
    while (end - i > 1) {
      const int64_t step = (end - i + kWave - 1) / kWave, mine = i + lane_id() * step;
      const int before = __popcll(__ballot(mine < end && append_start(a, mine) <= u));
      i += max(before - 1, 0) * step;
      end = min(i + step, end);
    }
  }
  const int64_t row = a.cu ? a.cu[i] : i;
  const int64_t fresh = a.cu ? (int64_t)a.cu[i + 1] - row : 1;
  const int32_t s = a.seqs[i];
  const bool leader = threadIdx.x == 0 && blockIdx.y == 0;
  if (a.cu && u == 0 && leader && (a.cu[0] != 0 || a.cu[a.n] != a.tokens))
    atomicOr(c.flags, kFlagInval);
  if (a.cu && u < append_start(a, i)) return;  // offsets that do not begin with 0
  if (fresh <= 0) {
    if (fresh < 0 && leader) atomicOr(c.flags, kFlagInval);
    return;
  }
  if ((uint32_t)s >= (uint32_t)c.slots || row < 0 || row + fresh > a.tokens) {
    if (leader) atomicOr(c.flags, kFlagInval);
    return;
  }
  const int64_t len = c.lens[s];
  const int64_t first = len - fresh;
  if (first < 0 || len > ((int64_t)c.max_blocks << c.page_shift)) {
    if (leader) atomicOr(c.flags, kFlagInval);
    return;
  }
  const int64_t b = (first >> c.page_shift) + (a.cu ? u - append_start(a, i) : 0);
  const int64_t b0 = b << c.page_shift;
  if (b0 >= len) return;
  const int64_t page = c.tables[(int64_t)s * c.max_blocks + b];
  if (page < 0 || page >= c.num_pages) {
    if (leader) atomicOr(c.flags, kFlagInval);
    return;
  }
  const int lo = (int)max(first - b0, (int64_t)0);
  const int hi = (int)min(len - b0, (int64_t)c.page_tokens);
  const int64_t row0 = row + (b0 + lo - first);
  const int64_t slot = (page * c.layers + a.layer) * 2;
  if (part < c.kv_heads) {
    Block<D, FMT, BF16, 0, WIDE> block;
    block.run(a, a.k + row0 * a.k_token + part * a.k_head, a.k_token, lo, hi, slot, part);
  } else {
    const int head = part - c.kv_heads;
    Block<D, FMT, BF16, 1, WIDE> block;
    block.run(a, a.v + row0 * a.v_token + head * a.v_head, a.v_token, lo, hi, slot + 1, head);
  }
}

template <int D, int FMT, int BF16>
void launch(const KvAppendArgs& a, dim3 grid, hipStream_t st) {
  if (a.wide) hipLaunchKernelGGL((kv_append<D, FMT, BF16, true>), grid, dim3(AW * kWave), 0, st, a);
  else hipLaunchKernelGGL((kv_append<D, FMT, BF16, false>), grid, dim3(AW * kWave), 0, st, a);
}

template <int D, int FMT>
void launch_type(const KvAppendArgs& a, dim3 grid, hipStream_t st) {
  if (a.bf16) launch<D, FMT, 1>(a, grid, st);
  else launch<D, FMT, 0>(a, grid, st);
}

template <int D>
void launch_format(const KvAppendArgs& a, dim3 grid, hipStream_t st) {
  if (a.c.format == SEM_KV_INT8) launch_type<D, SEM_KV_INT8>(a, grid, st);
  else launch_type<D, SEM_KV_FP8>(a, grid, st);
}

}  // namespace

hipError_t launch_kv_append(const KvAppendArgs& args, hipStream_t st) {
  if (args.n == 0) return hipSuccess;  // (without tokens the offsets are looked at)
  KvAppendArgs a = args;
  const int64_t units = a.cu ? (a.tokens >> a.c.page_shift) + 2 * a.n : a.n;
  const int64_t checks = a.cu ? (a.n + AW * kWave - 1) / (AW * kWave) : 0;
  if (!grid_fits(units + checks, AW * kWave)) return hipErrorInvalidConfiguration;
  a.units = (uint32_t)units;
  const dim3 grid((unsigned)(units + checks), (unsigned)((2 * a.c.kv_heads + AW - 1) / AW));
  switch (a.c.head_dim) {
    case 64: launch_format<64>(a, grid, st); break;
    case 128: launch_format<128>(a, grid, st); break;
    default: launch_format<256>(a, grid, st);
  }
  return hipGetLastError();
}

}  // namespace semsched
