// Reductions over lanes by register moves (no LDS).
#pragma once

#include "common.hpp"

namespace laep {

// Reductions over groups of NL neighbouring lanes (a power of two), the result in
// every lane: lane moves inside 16 lanes (quads, then mirrored halves and rows, whose
// lanes hold equal values by then), swaps of half rows and half waves beyond.  Every
// lane of the group must be active.
template <int NL, typename Op>
__device__ __forceinline__ float lanes_reduce(float v, Op op) {
  static_assert(NL >= 1 && NL <= kWave && (NL & (NL - 1)) == 0, "a power of two up to a wave");
  auto bits = [](float f) { return __builtin_bit_cast(int, f); };
  auto val = [](int i) { return __builtin_bit_cast(float, i); };
  if constexpr (NL >= 2) v = op(v, val(__builtin_amdgcn_mov_dpp(bits(v), 0xB1, 0xF, 0xF, true)));
  if constexpr (NL >= 4) v = op(v, val(__builtin_amdgcn_mov_dpp(bits(v), 0x4E, 0xF, 0xF, true)));
  if constexpr (NL >= 8) v = op(v, val(__builtin_amdgcn_mov_dpp(bits(v), 0x141, 0xF, 0xF, true)));
  if constexpr (NL >= 16) v = op(v, val(__builtin_amdgcn_mov_dpp(bits(v), 0x140, 0xF, 0xF, true)));
  if constexpr (NL >= 32) {
    const auto r = __builtin_amdgcn_permlane16_swap((unsigned)bits(v), (unsigned)bits(v), false, false);
    v = op(val((int)r[0]), val((int)r[1]));
  }
  if constexpr (NL >= 64) {
    const auto r = __builtin_amdgcn_permlane32_swap((unsigned)bits(v), (unsigned)bits(v), false, false);
    v = op(val((int)r[0]), val((int)r[1]));
  }
  return v;
}
template <int NL>
__device__ __forceinline__ float lanes_sum(float v) {
  return lanes_reduce<NL>(v, [](float a, float b) { return a + b; });
}
template <int NL>
__device__ __forceinline__ float lanes_max(float v) {
  return lanes_reduce<NL>(v, [](float a, float b) { return fmaxf(a, b); });
}

}  // namespace laep
