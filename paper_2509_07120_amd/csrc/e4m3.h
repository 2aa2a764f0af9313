// Rows of 64 numbers held in 8 bits: e4m3 numbers (OCP: 4 exponent bits, 3 of the mantissa, up to 448, no infinities) and one exponent byte b for
// the row; a number c stands for c * 2^(b - 127).  The exponent is the least that keeps the row's largest finite number at or below 448, so that every
// rounding is at most half a step, 2^-4 of the number, down to 2^-15 of the largest.  A power of two and no factor of 32 bits: what a number
// stands for has four significant bits and is exact in bf16, and one byte of 65 is the scale, where a factor would take four of 68 and round again.
// Exponents stay in [-64, 80]: a scale times a weight of 2^-62 or more, which is all that counts, is no subnormal number, and keys of 448 * 2^80 whose weights add up to
// 2^26 (four lanes of 2^24 each, where a reference of the weights follows) add up to less than there is in 32 bits.  So numbers above 448 * 2^80 = 5.4e26 become that,
// and those below 2^-74 become zero.
#pragma once

#include <hip/hip_runtime.h>

#include "bf16_tile.h"

namespace bsga {
namespace {

struct E4m3 {};                     // as a type of a cache
constexpr int kLeastScale = 127 - 64, kMostScale = 127 + 80;

// The exponent byte of a row whose largest finite magnitude is `most`: 448 = 1.75 * 2^8.
__device__ __forceinline__ int scale_byte(float most) {
  return min(max(static_cast<int>((__float_as_uint(most) + 0x1fffffu) >> 23) - 8, kLeastScale), kMostScale);
}
__device__ __forceinline__ float scale_of(unsigned byte) { return __uint_as_float(byte << 23); }
__device__ __forceinline__ float inverse_scale(int byte) { return __uint_as_float(static_cast<unsigned>(254 - byte) << 23); }

// Four numbers, divided by the row's scale already, to the nearest e4m3 numbers; infinities and NaN become NaN.
__device__ __forceinline__ unsigned pack_e4m3(float a, float b, float c, float d) {
  const int half = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return static_cast<unsigned>(__builtin_amdgcn_cvt_pk_fp8_f32(c, d, half, true));
}

// Four numbers times a power of two, exactly.
__device__ __forceinline__ u32x2 unpack_bf16(unsigned four, float scale) {
  return u32x2{__builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(four, scale, false)),
               __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(four, scale, true))};
}
__device__ __forceinline__ f32x4 unpack_f32(unsigned four) {
  const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(four), false), b = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(four), true);
  return f32x4{a[0], a[1], b[0], b[1]};
}

}  // namespace
}  // namespace bsga
