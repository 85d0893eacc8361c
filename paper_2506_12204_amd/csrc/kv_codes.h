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

// One code as a float.
template <int FMT>
__device__ __forceinline__ float code_to_float(uint32_t byte) {
  if (FMT == SEM_KV_INT8) return (float)(int8_t)byte;
  return __builtin_amdgcn_cvt_f32_fp8((int)byte, 0);
}

__device__ __forceinline__ float load16(uint16_t u, int bf16) {
  return bf16 ? __uint_as_float((uint32_t)u << 16) : (float)__builtin_bit_cast(_Float16, u);
}

}  // namespace semsched
