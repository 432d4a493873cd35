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

// 32 query channels, one group of the cache's side, as the sum of rows of E2M3 numbers (four significant bits, up to 7.5) with a
// power of two each for v_mfma_scale_f32_*_f8f6f4.  Two rows 2^-5 apart leave 2^-9 of the largest channel, 2^-8 where the second
// one is cut off (it holds 7.5 of the 8 units that the first can leave), and on normal channels less than bf16 leaves of a query
// in the mean (0.11 % against 0.165 %).  That is no longer so where a channel is far above the rest, which the two rows round as
// coarsely as it: if the largest is more than eight times the mean magnitude, three rows are wanted, of units 1, 2^-4 and 2^-9,
// none of which cuts off: 2^-13 of the largest is left, and nothing of a bf16 number down to 2^-6 of it.  all: every group wants
// them.  The first row takes the next power of two from 1.875 2^e on; a group with an infinity or a NaN is NaN.  Returns the
// scale bytes, first | second << 8 | third << 16.
typedef __attribute__((ext_vector_type(6))) unsigned u32x6;
typedef __attribute__((ext_vector_type(8))) int i32x8;
typedef __attribute__((ext_vector_type(32))) __bf16 bf16x32;
typedef __attribute__((ext_vector_type(32))) float f32x32;
constexpr unsigned kNotFinite = 0xffffff;     // ... NaN each
__device__ __forceinline__ u32x6 query_row(const f32x32& v, float scale) {
  bf16x32 x;
#pragma unroll
  for (int e = 0; e < 32; ++e) x[e] = (__bf16)v[e];
  return __builtin_amdgcn_cvt_scalef32_pk32_fp6_bf16(x, scale);
}
__device__ __forceinline__ unsigned split_query(f32x32 v, u32x6 (&rows)[3], bool& third,
                                                bool all = false) {
  float top = 0.f, sum = 0.f;      // (of 1/64 of the magnitudes, which no 32 finite ones overflow)
#pragma unroll
  for (int e = 0; e < 32; ++e) {
    top = fmaxf(top, fabsf(v[e]));
    sum = fmaf(fabsf(v[e]), 1.f / 64.f, sum);
  }
  const bool finite = sum < INFINITY;        // (a NaN is in the sum)
  // (from 0x1.ep127 on the first row is cut off, which one more cannot make good)
  const bool wanted = all || top * (1.f / 16.f) > sum || (finite && top >= 0x1.ep127f);
  third |= wanted;
  const int ex = min(max((int)((__float_as_uint(top) + 0x100000u) >> 23) - 2, 12), 252);
  const int ex1 = wanted ? ex - 4 : ex - 5, ex2 = ex - 9;
  auto scale = [&](int t) { return __uint_as_float((unsigned)(t == 0 ? ex : t == 1 ? ex1 : ex2) << 23); };
  rows[0] = query_row(v, scale(0));
  v -= __builtin_amdgcn_cvt_scalef32_pk32_f32_fp6(rows[0], scale(0));
  rows[1] = query_row(v, scale(1));
  rows[2] = u32x6{0u, 0u, 0u, 0u, 0u, 0u};
  if (__any(wanted)) {       // (a wave whose groups all do without skips it: a group that it may use has it or zeros)
    v -= __builtin_amdgcn_cvt_scalef32_pk32_f32_fp6(rows[1], scale(1));
    rows[2] = query_row(v, scale(2));
  }
  return finite ? (unsigned)ex | (unsigned)ex1 << 8 | (unsigned)ex2 << 16 : kNotFinite;
}

// Operands of the builtin, whose registers behind the format's are not read
__device__ __forceinline__ i32x8 operand(const u32x4& x) { return i32x8{(int)x[0], (int)x[1], (int)x[2], (int)x[3], 0, 0, 0, 0}; }
__device__ __forceinline__ i32x8 operand(const u32x6& x) {
  return i32x8{(int)x[0], (int)x[1], (int)x[2], (int)x[3], (int)x[4], (int)x[5], 0, 0};
}

}  // namespace mx4_tile
}  // namespace mlra
