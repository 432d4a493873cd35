// Conversions of the 4-bit latent cache (E2M1 codes, a power of two per 32 channels; the format is described in
// mx4_cache.hip).
#pragma once

#include "mlra_internal.h"

namespace mlra {
namespace mx4_tile {

typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) unsigned u32x4;

constexpr int kGroup = 32;             // channels that share a scale
constexpr unsigned kNaNScale = 255;

// A group's scale byte from the bits of its largest magnitude (0x200000: a quarter of the leading bit, which carries into
// the exponent from 1.75 on).
__device__ __forceinline__ unsigned scale_byte(unsigned top) {
  if (top >= 0x7f800000u) return kNaNScale;
  const int e = (int)((top + 0x200000u) >> 23) - 2;
  return (unsigned)min(max(e, 2), 252);
}

// 2^(byte - 127); the conversions below make NaN of the infinity that byte 255 is here
__device__ __forceinline__ float scale_of(unsigned byte) { return __uint_as_float(byte << 23); }

// Eight channels to codes, channel i in bits 4 i .. 4 i + 3 (the instruction rounds to nearest, ties to the even mantissa,
// and saturates).
__device__ __forceinline__ unsigned encode8(const float (&x)[8], unsigned byte) {
  const float scale = scale_of(byte);
  unsigned r = 0;
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[0], x[1], scale, 0);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[2], x[3], scale, 1);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[4], x[5], scale, 2);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[6], x[7], scale, 3);
  return r;
}

// Eight codes to bf16 (exact)
__device__ __forceinline__ u32x4 decode8(unsigned codes, float scale) {
  return u32x4{__builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0)),
               __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1)),
               __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2)),
               __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3))};
}

}  // namespace mx4_tile
}  // namespace mlra
