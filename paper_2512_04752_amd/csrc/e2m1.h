// Numbers in 4 bits: E2M1 codes times a power of two that a group shares.
#pragma once

#include "common.h"

namespace spec {

// e + 127 for a group whose largest magnitude has the fp32 bits `top`, `lowest` at
// least; 255 when the group holds an infinity or NaN.
__device__ __forceinline__ uint32_t scale_byte(uint32_t top, int lowest = 1) {
  if (top >= 0x7f800000u) return 255u;
  // top = 1.m 2^(E - 127) <= 6 2^e = 1.5 2^(e + 2)
  return (uint32_t)min(max(((int)top + 0x3fffff - (2 << 23)) >> 23, lowest), 252);
}

// N (4 or 8) E2M1 codes of f / 2^(byte - 127), dim n in bits 4n .. 4n + 3; 0 for a
// group without a scale, and 0 rather than -0.
template <int N>
__device__ __forceinline__ uint32_t pack_codes(const float* f, uint32_t byte) {
  const float s = __uint_as_float(byte << 23);
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[0], f[1], s, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[2], f[3], s, 1);
  if constexpr (N == 8) {
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[4], f[5], s, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[6], f[7], s, 3);
  }
  const uint32_t some = ((w & 0x77777777u) + 0x77777777u) & 0x88888888u;   // magnitude bits set
  w &= some | 0x77777777u;
  return byte == 255u ? 0u : w;
}

// Eight numbers of a word of codes, s a power of two, as bf16.
__device__ __forceinline__ i32x4 numbers(uint32_t w, float s) {
  return i32x4{__builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 0)),
               __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 1)),
               __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 2)),
               __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 3))};
}

}  // namespace spec
