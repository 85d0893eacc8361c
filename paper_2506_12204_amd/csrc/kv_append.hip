// Appending to the KV cache: the new tokens' keys and values become 8-bit codes
// of their pages' blocks. A block (a page's K or V of one head) has one scale,
// the largest magnitude over its tokens over the largest code:
//
//   s' = max(s if the block holds older tokens else 0, max |x| * (1 / top))
//   older codes, if s' > s:  c <- round(c * s / s')
//   new codes:               c  = round(x / s')
//
// with divisions and products in 32 bits, each rounded once (the codes are the
// nearest to the quotients; a block of zeros has scale 0 and codes 0).
// Elements that are not finite count as 0 in the maximum, are stored as the
// largest code or 0 (NaN), and are reported as a range error.
//
// One wave per block, so that a decode step of n sequences has 2 * n * kv_heads
// waves, and no two waves share a 16-byte unit. Bound by memory: a new token's
// K is whole 16-byte units of its block, its V one byte of each of head_dim
// units, written in place.
#include <algorithm>

#include "device_common.h"
#include "kv.h"
#include "kv_codes.h"

namespace semsched {

namespace {

constexpr int AW = 4;  // waves per workgroup, each on a block of its own

// Units of work: pages touched by new tokens, bounded and numbered without
// reading the lengths: sequence i starts at cu[i] / page_tokens + 2 i, which
// leaves room for a partly filled page at either end.
__device__ __forceinline__ int64_t append_start(const KvAppendArgs& a, int64_t i) {
  return ((a.cu ? a.cu[i] : (int32_t)i) >> a.c.page_shift) + 2 * i;
}

template <int FMT, int WHICH>
__device__ void append_block(const KvAppendArgs& a, int64_t row0, int lo, int hi, int64_t page,
                             int head) {
  const KvView& c = a.c;
  const int lane = lane_id();
  const int dim = c.head_dim;
  const uint16_t* x = (WHICH ? a.v : a.k) + head * (WHICH ? a.v_head : a.k_head);
  const int64_t stride = WHICH ? a.v_token : a.k_token;
  const int64_t slot = (page * c.layers + a.layer) * 2 + WHICH;
  uint8_t* block = c.data + (slot * c.kv_heads + head) * ((int64_t)c.page_tokens * dim);
  float* scale = c.scale + slot * c.kv_heads + head;
  x += row0 * stride;  // row `lo` of the page
  // the largest finite magnitude
  float top = 0.0f;
  bool wild = false;
  const int pieces = dim / 8;
  const int count = (hi - lo) * pieces;
  for (int i = lane; i < count; i += kWave) {
    const uint16_t* p = x + (int64_t)(i / pieces) * stride + (i % pieces) * 8;
    uint16_t e[8];
    if (a.wide) {
      *reinterpret_cast<uint4*>(e) = *reinterpret_cast<const uint4*>(p);
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k) e[k] = p[k];
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float m = fabsf(load16(e[k], a.bf16));
      const bool fine = m <= 3.4028235e38f;
      wild |= !fine;
      top = fine ? fmaxf(top, m) : top;
    }
  }
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor(top, off, kWave));
  if (__ballot(wild) && lane == 0) atomicOr(c.flags, kFlagRange);
  const float was = lo > 0 ? *scale : 0.0f;
  const float now = fmaxf(was, top * (1.0f / code_max<FMT>()));
  const bool grown = lo > 0 && now > was;
  if (lane == 0 && (lo == 0 || grown)) *scale = now;
  const float by = now > 0.0f ? now : 1.0f;
  // Units of 16 codes: K, 16 channels of one token; V, 16 tokens of one channel.
  const int first = grown ? 0 : (WHICH ? lo / kKvTile * dim : lo / kKvTile * dim);
  const int last = (hi + kKvTile - 1) / kKvTile * dim;
  for (int u = first + lane; u < last; u += kWave) {
    const int tile = u / dim, in = u % dim;
    union {
      uint4 v;
      uint8_t b[16];
      uint32_t w[4];
    } codes;
    uint4* at = reinterpret_cast<uint4*>(block) + u;
    if (WHICH == 0) {
      const int tok = tile * kKvTile + in % kKvTile, d0 = in / kKvTile * 16;
      if (tok >= hi || (tok < lo && !grown)) continue;
      if (tok < lo) {
        codes.v = *at;
#pragma unroll
        for (int k = 0; k < 16; ++k)
          codes.b[k] = (uint8_t)float_to_code<FMT>(code_to_float<FMT>(codes.b[k]) * was / by);
      } else {
        const uint16_t* p = x + (int64_t)(tok - lo) * stride + d0;
#pragma unroll
        for (int k = 0; k < 16; ++k)
          codes.b[k] = (uint8_t)float_to_code<FMT>(load16(p[k], a.bf16) / by);
      }
      *at = codes.v;
    } else {
      const int t0 = tile * kKvTile, d = in;
      if (t0 + kKvTile <= lo && !grown) continue;
      const int k0 = max(lo - t0, 0), k1 = min(hi - t0, kKvTile);
      // only the new tokens' bytes where the others stay as they are
      if (k1 - k0 < kKvTile && !grown) {
        for (int k = k0; k < k1; ++k)
          reinterpret_cast<uint8_t*>(at)[k] =
              (uint8_t)float_to_code<FMT>(load16(x[(int64_t)(t0 + k - lo) * stride + d], a.bf16) / by);
        continue;
      }
      codes.v = make_uint4(0, 0, 0, 0);
      if (grown) codes.v = *at;
#pragma unroll
      for (int k = 0; k < 16; ++k) {
        if (k < k0)
          codes.b[k] = (uint8_t)float_to_code<FMT>(code_to_float<FMT>(codes.b[k]) * was / by);
        else if (k < k1)
          codes.b[k] = (uint8_t)float_to_code<FMT>(
              load16(x[(int64_t)(t0 + k - lo) * stride + d], a.bf16) / by);
      }
      *at = codes.v;
    }
  }
}

template <int FMT>
__global__ __launch_bounds__(AW* kWave) void kv_append(KvAppendArgs a) {
  const KvView& c = a.c;
  const int64_t u = blockIdx.x;
  const int part = blockIdx.y * AW + threadIdx.x / kWave;  // (K or V, head)
  if (part >= 2 * c.kv_heads) return;
  // the last sequence that starts at or before u
  int64_t i = 0, end = a.n;
  while (end - i > 1) {
    const int64_t mid = (i + end) / 2;
    if (append_start(a, mid) <= u) i = mid;
    else end = mid;
  }
  const int64_t row = a.cu ? a.cu[i] : i;
  const int64_t fresh = a.cu ? (int64_t)a.cu[i + 1] - row : 1;
  const int32_t s = a.seqs[i];
  const bool leader = threadIdx.x == 0 && blockIdx.y == 0;
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
  const int64_t b = (first >> c.page_shift) + (u - append_start(a, i));
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
  if (part < c.kv_heads) append_block<FMT, 0>(a, row0, lo, hi, page, part);
  else append_block<FMT, 1>(a, row0, lo, hi, page, part - c.kv_heads);
}

}  // namespace

hipError_t launch_kv_append(const KvAppendArgs& a, hipStream_t st) {
  if (a.n == 0 || a.tokens == 0) return hipSuccess;
  const int64_t units = (a.tokens >> a.c.page_shift) + 2 * a.n;
  const dim3 grid((unsigned)units, (unsigned)((2 * a.c.kv_heads + AW - 1) / AW));
  if (a.c.format == SEM_KV_INT8)
    hipLaunchKernelGGL(kv_append<SEM_KV_INT8>, grid, dim3(AW * kWave), 0, st, a);
  else
    hipLaunchKernelGGL(kv_append<SEM_KV_FP8>, grid, dim3(AW * kWave), 0, st, a);
  return hipGetLastError();
}

}  // namespace semsched
