// The products of an attention by type: a wave owns 32 rows, the others come in blocks of 32 (attn_bias.h, cross_attention.h).
#pragma once

#include "attn_tiles.h"
#include "spa_common.h"

namespace spa {

constexpr float kLog2e = 1.4426950408889634f;
// exp(s - m) as exp2(s log2 e - m2), m2 = m log2 e rounded, is off by what that rounding is: half a last place of m2, which at -1e10
// (a mask written into the table) is 2^9, and a row whose first keys are all masked ends as infinity times 0.  Rows whose maximum (lse) is
// this large or more take the difference before the factor, an instruction more a score; below it P is off by at most 2^-17 of itself.
constexpr float kFarScore = 128.f;

// ---- operands by type.  Row: the lane's share (half hh) of one row of a head as an operand of 32x32 products over the head dim.
template <typename T, int DH> struct Ops;
template <int DH> struct Ops<__bf16, DH> {
  static constexpr int RS = DH + 8, KK = DH / 16;             // elements from row to row of a tile in LDS
  struct Row {
    bf16x8 f[KK];
  };
  static __device__ __forceinline__ Row row(const __bf16* p, int hh) {
    Row r;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) r.f[kk] = *reinterpret_cast<const bf16x8*>(p + kk * 16 + hh * 8);
    return r;
  }
  static __device__ __forceinline__ void dot(floatx16& acc, const Row& a, const Row& b) {
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.f[kk], b.f[kk], acc, 0, 0, 0);
  }
  // acc += (rows sb 32 .. of the tile)^T p: p of a lane holds the 16 rows of acc_row of its column, P or dS, rounded here to bf16 as
  // operands of the product have to be (half a step each, 2^-8; the sums over them stay in fp32)
  static __device__ __forceinline__ void outer(floatx16 (&acc)[DH / 32], const __bf16* tile, int sb, const floatx16& p, int lane) {
#pragma unroll
    for (int mf = 0; mf < 2; ++mf) {
      floatx8 f;
#pragma unroll
      for (int j = 0; j < 8; ++j) f[j] = p[8 * mf + j];
      const bf16x8 b = float_to_bf16x8(f);
#pragma unroll
      for (int d = 0; d < DH / 32; ++d)
        acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(transposed_frag_rowmajor<RS>(tile, d, sb * 32, mf, lane), b, acc[d], 0, 0, 0);
    }
  }
  // this half's part of <a, b> and of sum |a|
  static __device__ __forceinline__ void sums(const Row& a, const Row& b, float& ab, float& a1) {
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      const floatx8 x = bf16x8_to_float(a.f[kk]), y = bf16x8_to_float(b.f[kk]);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        ab = fmaf(x[e], y[e], ab);
        a1 += fabsf(x[e]);
      }
    }
  }
  static __device__ __forceinline__ void store(const floatx16 (&acc)[DH / 32], float scale, __bf16* row, bool ok, int hh) {
    store_rows<DH>(acc, scale, row, ok, hh);
  }
};
// fp32: v_mfma_f32_32x32x2_f32.  The contraction order is free: a lane holds one half of the row.
template <int DH> struct Ops<float, DH> {
  static constexpr int RS = DH + 4, HD = DH / 2;
  struct Row {
    float f[HD];
  };
  static __device__ __forceinline__ Row row(const float* p, int hh) {
    Row r;
#pragma unroll
    for (int i = 0; i < HD; i += 4) {
      const floatx4 v = *reinterpret_cast<const floatx4*>(p + hh * HD + i);
#pragma unroll
      for (int e = 0; e < 4; ++e) r.f[i + e] = v[e];
    }
    return r;
  }
  static __device__ __forceinline__ void dot(floatx16& acc, const Row& a, const Row& b) {
#pragma unroll
    for (int i = 0; i < HD; ++i) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(a.f[i], b.f[i], acc, 0, 0, 0);
  }
  static __device__ __forceinline__ void outer(floatx16 (&acc)[DH / 32], const float* tile, int sb, const floatx16& p, int lane) {
#pragma unroll
    for (int r = 0; r < 16; ++r)
#pragma unroll
      for (int d = 0; d < DH / 32; ++d)
        acc[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(tile[(sb * 32 + acc_row(r, lane >> 5)) * RS + d * 32 + (lane & 31)], p[r], acc[d], 0, 0, 0);
  }
  static __device__ __forceinline__ void sums(const Row& a, const Row& b, float& ab, float& a1) {
#pragma unroll
    for (int i = 0; i < HD; ++i) {
      ab = fmaf(a.f[i], b.f[i], ab);
      a1 += fabsf(a.f[i]);
    }
  }
  static __device__ __forceinline__ void store(const floatx16 (&acc)[DH / 32], float scale, float* row, bool ok, int hh) {
    if (!ok) return;
#pragma unroll
    for (int d = 0; d < DH / 32; ++d)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *reinterpret_cast<floatx4*>(row + d * 32 + 8 * g + 4 * hh) =
            floatx4{acc[d][4 * g] * scale, acc[d][4 * g + 1] * scale, acc[d][4 * g + 2] * scale, acc[d][4 * g + 3] * scale};
  }
};

}  // namespace spa
