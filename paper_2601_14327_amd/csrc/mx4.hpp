// Microscaled 4-bit values (MX4) on the device: steps 0, 1/2, 1, 3/2, 2, 3, 4, 6 with a
// sign, and per 32 consecutive columns of a row a power-of-two scale 2^(b - 127), kept
// as its biased exponent b.  Scales lie [C / 256, R, 8]: the eight of 256 columns
// together, so a matrix instruction's operand for four blocks is one dword of a row.
#pragma once

#include "common.hpp"

namespace laep {
namespace {

constexpr uint32_t kMx4Nan = 255;
constexpr int kMx4Block = 32, kMx4Group = 256;

inline int mx4_groups(int C) { return (C + kMx4Group - 1) / kMx4Group; }
inline size_t mx4_scale_bytes(int64_t R, int C) { return (size_t)R * mx4_groups(C) * 8; }

// biased exponent of a block's scale, from the bits of its largest magnitude (as
// unsigned integers, which order as the magnitudes do, NaNs above infinity)
__device__ __forceinline__ uint32_t mx4_exponent(uint32_t amax_bits) {
  const uint32_t e = amax_bits >> 23;
  return e == 255 ? kMx4Nan : (e > 2 ? e - 2 : 0);
}

// 2^(b - 127) as the conversions take it: 2^-127 is below float32's normal numbers
__device__ __forceinline__ float mx4_scale(uint32_t b) {
  return __uint_as_float(b == kMx4Nan ? 0x7FC00000u : (b == 0 ? 0x00400000u : b << 23));
}

__device__ __forceinline__ uint32_t mag_bits(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }
__device__ __forceinline__ uint32_t umax(uint32_t a, uint32_t b) { return a > b ? a : b; }

// Four values' codes (16 bits) at a scale.  The conversion divides by the scale (exact),
// rounds to the nearest step, ties to the even code, and takes 6 for what lies above.
__device__ __forceinline__ uint32_t mx4_codes4(float a, float b, float c, float d, float scale) {
  uint32_t w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, a, b, scale, 0);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, c, d, scale, 1);
}

// Eight values of one dword of codes, in bf16 (exact: steps have two significant bits)
__device__ __forceinline__ u32x4_t mx4_values8_bf16(uint32_t w, float scale) {
  return u32x4_t{
      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0)),
      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1)),
      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2)),
      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3))};
}

}  // namespace
}  // namespace laep
