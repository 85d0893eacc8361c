// Norms of queries and keys and the rotation of their positions.
//
// For every row x (a token and a head) of head_dim channels:
//
//   y = x w / sqrt(mean(x^2) + eps)        (y = x where there are no weights)
//   (a, b) -> (a cos t - b sin t, b cos t + a sin t),  t = position * inv_freq[i]
//
// with a, b the channels i and i + rot_dim / 2, or 2 i and 2 i + 1, and the
// channels from rot_dim on as they are. Everything is in 32 bits and rounded once,
// at the end, but the angle: it is taken in turns, as the sum of two 64-bit numbers,
// less its whole turns, so that far positions are as exact as near ones.
//
// A lane holds 16 channels of a row, eight pairs whichever way they lie, so the
// rotation stays in the lane; D / 16 lanes make a row, a wave 1024 / D rows. The
// eight angles are the same for all heads of a token: a wave takes several steps
// of rows of one token with the sines and cosines of one.
//
// Bound by memory where there are many tokens: 16384 of 32 + 8 heads of 128 channels
// (335 MB read and written) take 68 us, 4.96 TB/s, a little over a large copy's rate.
// Few tokens are a launch: 8 us for one, as for 251.
#include <algorithm>

#include "device_common.h"
#include "kv.h"
#include "kv_codes.h"

namespace semsched {

namespace {

constexpr int RT = 256;  // threads of a workgroup, each wave on its own

// The sine and cosine of 2 pi r, |r| <= 1/2: r less the nearest quarter turn, the
// Taylor series there (|x| <= pi / 4: the first terms left out are below 2e-9 and
// 3e-8), and the quarter's symmetry.
__device__ __forceinline__ void sine_cosine(float r, float& s, float& c) {
  const float quarter = __builtin_rintf(4.0f * r);
  const float x = 6.283185307179586f * __builtin_fmaf(quarter, -0.25f, r), z = x * x;
  float p = __builtin_fmaf(z, 1.0f / 362880.0f, -1.0f / 5040.0f);
  p = __builtin_fmaf(p, z, 1.0f / 120.0f);
  p = __builtin_fmaf(p, z, -1.0f / 6.0f);
  p = __builtin_fmaf(p * z, x, x);
  float q = __builtin_fmaf(z, 1.0f / 40320.0f, -1.0f / 720.0f);
  q = __builtin_fmaf(q, z, 1.0f / 24.0f);
  q = __builtin_fmaf(q, z, -0.5f);
  q = __builtin_fmaf(q, z, 1.0f);
  const int turn = (int)quarter & 3;
  s = turn & 1 ? q : p;
  c = turn & 1 ? p : q;
  if (turn & 2) s = -s;
  if ((turn + 1) & 2) c = -c;
}

// The turns of the angle p f less the nearest whole number of them: the product has up to
// 55 bits and 1 / (2 pi) is taken to 107, so what 64-bit products round off is added once
// the whole turns are gone. (Left out, it is up to 3e-7 of the angle near position 2^31,
// three times the rounding of the result. With it 2000 tokens of 32 + 8 heads of 128
// channels take 10.4 us instead of 9.7, 16384 the same 64; one token is no slower.)
__device__ __forceinline__ float part_of_turn(double p, double f) {
  constexpr double kTurn = 0x1.45f306dc9c883p-3, kMore = -0x1.6b01ec5412aa7p-57;
  const double x = p * f;
  const double more = __builtin_fma(x, kMore, __builtin_fma(p, f, -x) * kTurn);
  const double r = __builtin_fma(x, kTurn, -__builtin_rint(x * kTurn)) + more;
  return (float)(r - __builtin_rint(r));  // (a little more than a half would lose a bit)
}

template <int D, bool BF16, bool PAIRS, bool WIDE>
__global__ __launch_bounds__(RT) void qk_rotate(QkRotateArgs a) {
  constexpr int LANES = D / 16;           // of a row
  constexpr int ROWS = kWave / LANES;     // of a step
  const int64_t wave = (int64_t)blockIdx.x * (RT / kWave) +
                       __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int64_t token = wave / a.parts;
  if (token >= a.tokens) return;
  const int part = (int)(wave % a.parts), piece = lane_id() % LANES;
  const int all = a.heads + a.kv_heads;
  const int begin = part * a.steps * ROWS + lane_id() / LANES;
  const int end = min(all, (part + 1) * a.steps * ROWS);
  // The lane's two runs of eight channels: two halves' where those are paired, side
  // by side where neighbours are and behind the rotated channels.
  const bool turns = piece * 16 < a.rot_dim;
  const bool split = !PAIRS && turns;
  const int c0 = split ? piece * 8 : piece * 16;
  const int c1 = split ? a.rot_dim / 2 + piece * 8 : c0 + 8;

  float cosine[8], sine[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    cosine[i] = 1.0f;
    sine[i] = 0.0f;
  }
  if (turns) {
    const double p = (double)a.positions[token];
#pragma unroll
    for (int i = 0; i < 8; ++i)
      sine_cosine(part_of_turn(p, (double)a.inv_freq[piece * 8 + i]), sine[i], cosine[i]);
  }
  const float* weights = nullptr;
  float w[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) w[i] = 1.0f;
  for (int row = begin; row < end; row += ROWS) {
    const bool key = row >= a.heads;
    const int head = key ? row - a.heads : row;
    const uint16_t* from = key ? a.k + token * a.k_token + head * a.k_head
                               : a.q + token * a.q_token + head * a.q_head;
    uint16_t* to = key ? a.k_out + token * a.ko_token + head * a.ko_head
                       : a.q_out + token * a.qo_token + head * a.qo_head;
    float x[16];
    if (WIDE) {
      const uint4 lo = *reinterpret_cast<const uint4*>(from + c0);
      const uint4 hi = *reinterpret_cast<const uint4*>(from + c1);
      const uint32_t u[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x[2 * i] = load16((uint16_t)u[i], BF16);
        x[2 * i + 1] = load16((uint16_t)(u[i] >> 16), BF16);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x[i] = load16(from[c0 + i], BF16);
        x[8 + i] = load16(from[c1 + i], BF16);
      }
    }
    const float* wanted = key ? a.k_weight : a.q_weight;
    if (wanted) {
      if (wanted != weights) {
        weights = wanted;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          w[i] = weights[c0 + i];
          w[8 + i] = weights[c1 + i];
        }
      }
      float sum = 0.0f;
#pragma unroll
      for (int i = 0; i < 16; ++i) sum = __builtin_fmaf(x[i], x[i], sum);
#pragma unroll
      for (int off = 1; off < LANES; off *= 2) sum += __shfl_xor(sum, off, kWave);
      const float inv = 1.0f / __builtin_sqrtf(__builtin_fmaf(sum, 1.0f / D, a.eps));
#pragma unroll
      for (int i = 0; i < 16; ++i) x[i] *= inv * w[i];
    }
    float y[16];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int p = PAIRS ? 2 * i : i, o = PAIRS ? 2 * i + 1 : 8 + i;
      y[p] = x[p] * cosine[i] - x[o] * sine[i];
      y[o] = x[o] * cosine[i] + x[p] * sine[i];
    }
    if (!turns) {  // (infinities times zero are not what they were)
#pragma unroll
      for (int i = 0; i < 16; ++i) y[i] = x[i];
    }
    uint32_t u[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) u[i] = pack_pair<BF16>(y[2 * i], y[2 * i + 1]);
    if (WIDE) {
      *reinterpret_cast<uint4*>(to + c0) = make_uint4(u[0], u[1], u[2], u[3]);
      *reinterpret_cast<uint4*>(to + c1) = make_uint4(u[4], u[5], u[6], u[7]);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        to[c0 + i] = (uint16_t)(u[i / 2] >> (16 * (i % 2)));
        to[c1 + i] = (uint16_t)(u[4 + i / 2] >> (16 * (i % 2)));
      }
    }
  }
}

template <int D, bool BF16, bool PAIRS>
void launch_width(const QkRotateArgs& a, unsigned grid, hipStream_t st) {
  if (a.wide)
    hipLaunchKernelGGL((qk_rotate<D, BF16, PAIRS, true>), dim3(grid), dim3(RT), 0, st, a);
  else
    hipLaunchKernelGGL((qk_rotate<D, BF16, PAIRS, false>), dim3(grid), dim3(RT), 0, st, a);
}

template <int D>
hipError_t launch_dim(QkRotateArgs a, hipStream_t st) {
  constexpr int ROWS = 1024 / D;
  // Steps of a wave: all of a token's where there are many tokens, one where there
  // are few. (The kernel alone, all or one: 16384 tokens 67 or 74 us, one 5.2 or 3.1.)
  const int64_t steps = (a.heads + a.kv_heads + ROWS - 1) / ROWS;
  constexpr int64_t kWaves = 4096;
  a.steps = (int32_t)std::min(steps, std::max<int64_t>(1, a.tokens * steps / kWaves));
  a.parts = (int32_t)((steps + a.steps - 1) / a.steps);
  const int64_t waves = a.tokens * a.parts, grid = (waves + RT / kWave - 1) / (RT / kWave);
  if (!grid_fits(grid, RT)) return hipErrorInvalidConfiguration;
  if (a.bf16) {
    if (a.pairs) launch_width<D, true, true>(a, (unsigned)grid, st);
    else launch_width<D, true, false>(a, (unsigned)grid, st);
  } else {
    if (a.pairs) launch_width<D, false, true>(a, (unsigned)grid, st);
    else launch_width<D, false, false>(a, (unsigned)grid, st);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_qk_rotate(const QkRotateArgs& a, int head_dim, hipStream_t st) {
  if (a.tokens == 0) return hipSuccess;
  switch (head_dim) {
    case 64: return launch_dim<64>(a, st);
    case 128: return launch_dim<128>(a, st);
    default: return launch_dim<256>(a, st);
  }
}

}  // namespace semsched
