// A feature row held by a group of G neighbouring lanes in 16-byte chunks: chunk types, widening to fp32, and sums over the
// group (gate.hip, norm.hip).
#pragma once

#include "spa_common.h"

namespace spa {

template <typename T> struct Vec16;
template <> struct Vec16<float> {
  static constexpr int kElems = 4;
  // (for results that the path does not read again: non-temporal)
  __device__ static __forceinline__ void store(float* p, const float (&f)[4]) {
    floatx4 v = {f[0], f[1], f[2], f[3]};
    __builtin_nontemporal_store(v, reinterpret_cast<floatx4*>(p));
  }
};
template <> struct Vec16<__bf16> {
  static constexpr int kElems = 8;
  __device__ static __forceinline__ void store(__bf16* p, const float (&f)[8]) {
    floatx8 v;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = f[i];
    __builtin_nontemporal_store(float_to_bf16x8(v), reinterpret_cast<bf16x8*>(p));
  }
};

template <typename T> struct Raw16;
template <> struct Raw16<float> { using type = floatx4; };
template <> struct Raw16<__bf16> { using type = bf16x8; };
__device__ __forceinline__ void widen(floatx4 v, float (&f)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) f[i] = v[i];
}
__device__ __forceinline__ void widen(bf16x8 v, float (&f)[8]) {
  const floatx8 w = bf16x8_to_float(v);
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = w[i];
}

// Sum over groups of G neighbouring lanes, in every lane, in the order of exchanges with lane ^ G/2, ^ G/4, ... ^ 1, in the
// vector ALU: the two halves and the two 16-lane rows of a half by the lane swaps, ^ 8 as a rotation of the row by 8, ^ 4 as
// one by 4 once both halves of a row hold the same (groups of 8: as two shifts), ^ 2 and ^ 1 inside a quad.  An
// exchange through LDS takes 85 cycles, one of these 8 to 16, and the dot products wait for each of them.
__device__ __forceinline__ float add_lane_xor32(float v) {
  const unsigned u = __builtin_bit_cast(unsigned, v);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  const unsigned a = r[0], b = r[1];
  return __builtin_bit_cast(float, a) + __builtin_bit_cast(float, b);
}
__device__ __forceinline__ float add_lane_xor16(float v) {
  const unsigned u = __builtin_bit_cast(unsigned, v);
  const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  const unsigned a = r[0], b = r[1];
  return __builtin_bit_cast(float, a) + __builtin_bit_cast(float, b);
}
template <int G>
__device__ __forceinline__ float group_sum(float v) {
  constexpr int kRor = 0x120;
  if (G > 32) v = add_lane_xor32(v);
  if (G > 16) v = add_lane_xor16(v);
  if (G > 8) v += dpp_move<kRor + 8>(v);
  if (G > 8) v += dpp_move<kRor + 4>(v);
  else v += lane_xor<4>(v);
  v += lane_xor<2>(v);
  return v + lane_xor<1>(v);
}

}  // namespace spa
