// Packed, per-image attention with a learned bias by the bucket of the relative position: the token of packed row j sits at
// n = gather_idx[j] mod (gh gw) of its image's map, row n / gw, column n mod gw, and
//   S_ij = scale q_i k_j + table[h, buckets[offset of i from j]],   O = softmax(S) V
// With p = row (2 gw - 1) + column the offset's index is p_i - p_j + (gh - 1)(2 gw - 1) + gw - 1: one subtraction.  A row whose
// scores are all -inf gives 0.
#include <algorithm>
#include <cmath>

#include "attn_bias.h"

namespace spa {

// As in the attention without a bias: one wave owns 32 queries and computes S^T = K Q^T, so that a lane holds 16 keys of one
// query a 32 x 32 block, and the probabilities (bf16: rounded) are the second product's operand in registers; K and V stream through LDS
// in tiles of 64.  fp32 takes the same steps on the fp32 matrix instructions.  Bound by the vector instructions: some 135 a 32 x 32
// block, 16 of them exponentials, of which the bias is a subtraction, a shift and a multiply-add each; at 8 images of 4200 tokens, 8 heads
// of 32, they fill 0.89 of the busy units' cycles.  us (the attention without a bias), medians of eight selections: 33 (24) at 16 images
// of 0.1 to 0.6 of 3136 tokens, 3 heads of 32; 18.3 (13.0) at 64 of 196, 12 heads of 64; 41 (25), 24 to 45 by the selection, at 8 of 4200.
template <typename T>
struct BiasFwd {
  const T *q, *k, *v;
  long qs, ks, vs;
  const int32_t* cu;
  BiasMap m;
  int H, B, nblk;
  float scale;
  T* out;
  float* lse;
  long lse_stride;
};

// SPLIT 2: the waves come twice, the second four take every other tile of 64 keys, and hand their sums to the first at the end.
template <typename T, int DH, int WIN, int SPLIT>
__global__ void __launch_bounds__(kBiasThreads * SPLIT) attn_bias_fwd_kernel(const BiasFwd<T> a) {
  using O = Ops<T, DH>;
  constexpr int DB = DH / 32;
  extern __shared__ __attribute__((aligned(16))) char win[];
  __shared__ QueryTiles<T, DH, SPLIT> l;
  const BiasBlock blk = bias_block(l.s_live, a.cu, a.H, a.B, a.nblk);
  if (!blk.valid) return;
  const int h = blk.h, n = blk.seg.nk, lane = threadIdx.x & 63, l32 = lane & 31, hh = lane >> 5, wv = (threadIdx.x >> 6) & 3;
  const int qi = blk.r0 + wv * 32 + l32;
  const bool wave_live = blk.r0 + wv * 32 < n, q_ok = qi < n;
  const long C = (long)a.H * DH, q_row = blk.seg.row0 + min(qi, n - 1);
  typename O::Row qf;
  floatx16 o[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[d][r] = 0.f;
  float m = -INFINITY, sum = 0.f;
  walk_keys<T, DH, WIN, SPLIT>(
      l, win, blk.seg, h, wave_live, a.k, a.ks, a.v, a.vs, a.m, a.cu, qi, [&] { qf = O::row(a.q + q_row * a.qs + h * DH, hh); },
      [] {}, [](const auto&) {},
      [&](const T* K, const T* V, const int* pos, int left, int own, int zero, bool in_window, auto whole) {
        floatx16 s[2];
        const int blocks = whole || left > 32 ? 2 : 1;        // of 32 keys that exist
#pragma unroll
        for (int sb = 0; sb < 2; ++sb)
          if (whole || sb < blocks)
            bias_scores<T, DH, WIN, 1>(s[sb], O::row(&K[(sb * 32 + l32) * O::RS], hh), qf, &pos[sb * 32], own, zero, in_window, a.m, h,
                                       a.scale, hh);
        if (!whole) {
#pragma unroll
          for (int sb = 0; sb < 2; ++sb)
#pragma unroll
            for (int r = 0; r < 16; ++r)
              if (sb * 32 + acc_row(r, hh) >= left) s[sb][r] = -INFINITY;
        }
        float mx = s[0][0];
#pragma unroll
        for (int sb = 0; sb < 2; ++sb)
#pragma unroll
          for (int r = 0; r < 16; ++r) mx = __builtin_elementwise_maximum(mx, s[sb][r]);
        const float m_new = __builtin_elementwise_maximum(m, max_across_halves(mx));
        if (__ballot(m_new != m) != 0) {
          const float f = m_new != m ? __builtin_amdgcn_exp2f((m - m_new) * kLog2e) : 1.f;
          sum *= f;
#pragma unroll
          for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[d][r] *= f;
          m = m_new;
        }
        if (__ballot(!(fabsf(m) < kFarScore)) == 0) {
          const float m2 = m * kLog2e;
#pragma unroll
          for (int sb = 0; sb < 2; ++sb)
#pragma unroll
            for (int r = 0; r < 16; ++r) s[sb][r] = __builtin_amdgcn_exp2f(fmaf(s[sb][r], kLog2e, -m2));
        } else {
          const float ref = m == -INFINITY ? 0.f : m;           // (no score yet: weights of 0)
#pragma unroll
          for (int sb = 0; sb < 2; ++sb)
#pragma unroll
            for (int r = 0; r < 16; ++r) s[sb][r] = __builtin_amdgcn_exp2f((s[sb][r] - ref) * kLog2e);
        }
#pragma unroll
        for (int sb = 0; sb < 2; ++sb) {
#pragma unroll
          for (int r = 0; r < 16; ++r) sum += s[sb][r];
          if (whole || sb < blocks) O::outer(o, V, sb, s[sb], lane);
        }
      });
  // (every wave is past its last read of the tiles)
  if constexpr (SPLIT > 1) {
    constexpr int W = DB * 16 + 2;
    static_assert(4 * W * kWave * sizeof(float) <= sizeof(l.K), "the sums of four waves");
    float* other = reinterpret_cast<float*>(&l.K[0][0]) + wv * W * kWave + lane;
    const int part = threadIdx.x >> 8;
    if (part == 1) {
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) other[(d * 16 + r) * kWave] = o[d][r];
      other[(W - 2) * kWave] = m;
      other[(W - 1) * kWave] = sum;
    }
    __syncthreads();
    if (part == 1) return;
    const float m1 = other[(W - 2) * kWave], both = __builtin_elementwise_maximum(m, m1);
    const float f0 = m == both ? 1.f : __builtin_amdgcn_exp2f((m - both) * kLog2e);
    const float f1 = m1 == both ? 1.f : __builtin_amdgcn_exp2f((m1 - both) * kLog2e);
    m = both;
    sum = sum * f0 + other[(W - 1) * kWave] * f1;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[d][r] = o[d][r] * f0 + other[(d * 16 + r) * kWave] * f1;
  }
  if (!wave_live) return;
  const float total = sum_across_halves(sum), inv = total == 0.f ? 0.f : 1.0f / total;      // (0: no key left, all weights 0)
  O::store(o, inv, a.out + q_row * C + h * DH, q_ok, hh);
  if (a.lse != nullptr && q_ok && hh == 0) a.lse[h * a.lse_stride + q_row] = total == 0.f ? -INFINITY : m + logf(total);
}

// Eight waves a block as well where the LDS of larger maps leaves few waves a unit otherwise: where that is twice the waves, or more
// waves and not too many blocks (of the longest possible segments, all that the host knows).  us four | eight waves, heads of 32: 50 x 84 map
// (8 | 16 waves a unit), 8 images 31.5 | 25.3, 32 images 132 | 117; 56 x 56 (12 | 16), 3 heads, 16 images 37.7 | 31.3, 20 (1500 blocks)
// 45.2 | 40.8, 24 (1800) 48.1 | 51.3, 32 55.2 | 57.3, 64 97 | 103, 8 heads, 8 (1600) 35.7 | 29.7, 12 (2400) 51.5 | 55.9; 28 x 28
// (16 | 16), 32 images 25.1 | 28.5.
template <typename T, int DH>
static bool fwd_eight(int offsets, int nblk, int H, int B) {
  if (few_blocks(nblk, H, B)) return true;
  constexpr int most = DH == 32 ? 16 : 12;                    // by registers
  const size_t win = window_bytes(offsets, sizeof(T));
  const int four = std::min<int>(most, 4 * (int)(kUnitLds / (sizeof(QueryTiles<T, DH, 1>) + win)));
  const int eight = std::min<int>(most, 8 * (int)(kUnitLds / (sizeof(QueryTiles<T, DH, 2>) + win)));
  return nblk >= 4 && (eight >= 2 * four || (eight > four && xcd_grid(nblk, H, B) <= 1700));
}

int bias_checks(const char* fn, const void* q, const void* k, const void* v, int64_t q_stride, int64_t k_stride, int64_t v_stride,
                const int32_t* cu, int B, int n_max, int H, int Dh, int dtype, float softmax_scale, const void* table,
                const int32_t* buckets, int n_buckets, const int32_t* gather_idx, int grid_h, int grid_w, BiasMap* m) {
  SPA_REFUSE_IN_GROUP(fn);
  SPA_REQUIRE(q && k && v && cu && table, SPA_ERR_INVALID_ARG, "%s: null pointer", fn);
  SPA_REQUIRE(B >= 1 && n_max >= 1 && H >= 1, SPA_ERR_INVALID_ARG, "%s: B, max_seqlen, H must be >= 1", fn);
  SPA_REQUIRE((long)B * n_max < 2147483647L, SPA_ERR_INVALID_ARG, "%s: B*max_seqlen must be < 2^31", fn);
  SPA_REQUIRE(B <= 65535 && H <= 65535, SPA_ERR_INVALID_ARG, "%s: B and H must be <= 65535", fn);
  SPA_REQUIRE(dtype == SPA_F32 || dtype == SPA_BF16, SPA_ERR_UNSUPPORTED, "%s: unknown dtype %d", fn, dtype);
  SPA_REQUIRE(Dh == 32 || Dh == 64, SPA_ERR_UNSUPPORTED, "%s: head dim %d not supported (32 or 64)", fn, Dh);
  const int64_t strides[3] = {q_stride, k_stride, v_stride};
  for (int64_t rs : strides) {
    SPA_REQUIRE(rs >= (int64_t)H * Dh, SPA_ERR_INVALID_ARG, "%s: row stride %ld < H*Dh", fn, (long)rs);
    SPA_REQUIRE(rs < (1 << 24), SPA_ERR_INVALID_ARG, "%s: row stride %ld must be < 2^24 elements", fn, (long)rs);
    SPA_REQUIRE((rs * elem_size(dtype)) % 16 == 0, SPA_ERR_INVALID_ARG, "%s: row stride is not a multiple of 16 bytes", fn);
  }
  SPA_REQUIRE(aligned16(q) && aligned16(k) && aligned16(v), SPA_ERR_INVALID_ARG, "%s: q/k/v not 16-byte aligned", fn);
  SPA_REQUIRE(aligned16(buckets), SPA_ERR_INVALID_ARG, "%s: buckets not 16-byte aligned", fn);
  SPA_REQUIRE(softmax_scale >= 0.f && std::isfinite(softmax_scale), SPA_ERR_INVALID_ARG,
              "%s: softmax_scale must be finite and >= 0 (0 = 1/sqrt(Dh))", fn);
  SPA_REQUIRE(grid_h >= 1 && grid_w >= 1 && (2 * (long)grid_h - 1) * (2 * (long)grid_w - 1) <= kMostOffsets, SPA_ERR_INVALID_ARG,
              "%s: grid_h, grid_w must be >= 1, with at most 2^26 offsets", fn);
  const long offsets = (2 * (long)grid_h - 1) * (2 * (long)grid_w - 1);
  SPA_REQUIRE(n_buckets >= 1 && n_buckets <= (1 << 26), SPA_ERR_INVALID_ARG, "%s: n_buckets must lie in 1 .. 2^26", fn);
  SPA_REQUIRE(buckets != nullptr || n_buckets == offsets, SPA_ERR_INVALID_ARG,
              "%s: without a bucket map there is a bucket per offset, %ld of them", fn, offsets);
  SPA_REQUIRE(n_max <= (long)grid_h * grid_w, SPA_ERR_INVALID_ARG, "%s: max_seqlen exceeds the %d x %d map", fn, grid_h, grid_w);
  *m = {table, buckets, gather_idx, n_buckets, grid_h * grid_w, (int)offsets, (grid_h - 1) * (2 * grid_w - 1) + grid_w - 1,
        divisor((uint32_t)grid_w), divisor((uint32_t)(grid_h * grid_w))};
  return SPA_OK;
}

}  // namespace spa

using namespace spa;

extern "C" int spa_packed_attention_bias(const void* q, const void* k, const void* v, int64_t q_row_stride, int64_t k_row_stride,
                                         int64_t v_row_stride, const int32_t* cu_seqlens, const int32_t* gather_idx, const void* table,
                                         const int32_t* buckets, int n_buckets, int grid_h, int grid_w, int B, int max_seqlen, int H,
                                         int Dh, int dtype, float softmax_scale, void* out, float* lse, void* stream) {
  const char* fn = "spa_packed_attention_bias";
  BiasMap m;
  if (int rc = bias_checks(fn, q, k, v, q_row_stride, k_row_stride, v_row_stride, cu_seqlens, B, max_seqlen, H, Dh, dtype, softmax_scale,
                           table, buckets, n_buckets, gather_idx, grid_h, grid_w, &m))
    return rc;
  SPA_REQUIRE(out != nullptr, SPA_ERR_INVALID_ARG, "%s: out is null", fn);
  SPA_REQUIRE(aligned16(out), SPA_ERR_INVALID_ARG, "%s: out not 16-byte aligned", fn);
  const int nblk = (max_seqlen + kBiasRows - 1) / kBiasRows;
  SPA_REQUIRE(((long)H * B + 8) * nblk < 2147483647L, SPA_ERR_INVALID_ARG, "%s: B*H*blocks must be < 2^31", fn);
  const float scale = softmax_scale > 0.f ? softmax_scale : 1.0f / std::sqrt((float)Dh);
  hipStream_t st = as_stream(stream);
#define SPA_FWD(T, D)                                                                                                         \
  do {                                                                                                                        \
    const BiasFwd<T> args = {(const T*)q, (const T*)k, (const T*)v, (long)q_row_stride, (long)k_row_stride, (long)v_row_stride, \
                             cu_seqlens, m, H, B, nblk, scale, (T*)out, lse, (long)B * max_seqlen};                           \
    SPA_QUERY_LAUNCH(attn_bias_fwd_kernel, T, D, (fwd_eight<T, D>(m.offsets, nblk, H, B)), args);                     \
  } while (0)
  if (dtype == SPA_F32) {
    if (Dh == 32) SPA_FWD(float, 32); else SPA_FWD(float, 64);
  } else {
    if (Dh == 32) SPA_FWD(__bf16, 32); else SPA_FWD(__bf16, 64);
  }
#undef SPA_FWD
  return check_launch(fn);
}
