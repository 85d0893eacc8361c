// The 8-bit numbers of the KV cache: int8 in [-127, 127] and e4m3 floats (four
// exponent and three mantissa bits, largest value 448, no infinities), both
// exact in half precision.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "semsched.h"

namespace semsched {

typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
typedef _Float16 half8_t __attribute__((ext_vector_type(8)));
typedef float float2_t __attribute__((ext_vector_type(2)));

template <int FMT>
__device__ __forceinline__ constexpr float code_max() {
  return FMT == SEM_KV_INT8 ? 127.0f : 448.0f;
}

// Four codes (one 32-bit word) as two pairs of halves.
template <int FMT>
__device__ __forceinline__ void codes_to_half(uint32_t w, half2_t& lo, half2_t& hi) {
  if (FMT == SEM_KV_INT8) {
    // x + 128 as the low mantissa bits of 1024 + x + 128, less 1152: exact
    const uint32_t u = w ^ 0x80808080u;
    const uint32_t a = __builtin_amdgcn_perm(0x64646464u, u, 0x07010700u);
    const uint32_t b = __builtin_amdgcn_perm(0x64646464u, u, 0x07030702u);
    const half2_t off = {(_Float16)1152.0f, (_Float16)1152.0f};
    lo = __builtin_bit_cast(half2_t, a) - off;
    hi = __builtin_bit_cast(half2_t, b) - off;
  } else {
    lo = __builtin_bit_cast(half2_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, false));
    hi = __builtin_bit_cast(half2_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, true));
  }
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

// Four codes as two pairs of bf16, exact too.
template <int FMT>
__device__ __forceinline__ void codes_to_bf16(uint32_t w, uint32_t& lo, uint32_t& hi) {
  if (FMT == SEM_KV_INT8) {
    // (whole numbers up to 128 have eight bits: a float's upper half holds them)
    const float a = (float)(int8_t)w, b = (float)(int8_t)(w >> 8);
    const float c = (float)(int8_t)(w >> 16), d = (float)(int8_t)(w >> 24);
    lo = __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
    hi = __builtin_amdgcn_perm(__float_as_uint(d), __float_as_uint(c), 0x07060302u);
  } else {
    lo = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, false));
    hi = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, true));
  }
}

// One code as a float.
template <int FMT>
__device__ __forceinline__ float code_to_float(uint32_t byte) {
  if (FMT == SEM_KV_INT8) return (float)(int8_t)byte;
  return __builtin_amdgcn_cvt_f32_fp8((int)byte, 0);
}

__device__ __forceinline__ float load16(uint16_t u, int bf16) {
  return bf16 ? __uint_as_float((uint32_t)u << 16) : (float)__builtin_bit_cast(_Float16, u);
}

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
  __device__ __forceinline__ float of(float x) const { return of_lifted(x * lift); }
  __device__ __forceinline__ float of_lifted(float y) const {
    const float q = y * inv;
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

}  // namespace semsched
