// The gated feed-forward block on packed rows: both projections, the activation and their product in one kernel,
//   g_j = x_row(j) Wg^T + bg,  u_j = x_row(j) Wu^T + bu,  h_j = act(g_j) * u_j          (W [2F][K]: Wg's rows, then Wu's)
// and the step of its backward between the two products' gradients: with dh = dy W_down,
//   d_g = dh * u * act'(g),  d_u = dh * act(g)
// formed in the epilogue of that product, so that dh is never in memory.  The rest of the block are the projections of linear.hip and
// linear_bwd.hip: the way back onto the residual stream, and from d_pre = (d_g, d_u) the gradients of x, W and the biases.
//   act: SiLU g s(g), s = 1 / (1 + exp(-g)), slope s (1 + g (1 - s)); GELU g Phi(g), slope Phi(g) + g phi(g).
//
// Both are row GEMMs on the loop of gemm_async.h in the shapes of gemm_rows.h, chosen by its rules (2 F and F columns).  Forward, the rows
// of Wg and Wu lie in turns of one matrix tile in LDS, so that a wave has a column's gate and its factor in the same register of
// neighbouring accumulators.
// Rounded to bf16 are h and pre (from the same unrounded sums) and d_pre, the operands of the products that follow and what the backward
// keeps; act and its slope are formed from pre as kept. 6272 rows of 768 -> 2 x 2048 -> 768: forward 57 us (690 TFLOP/s; with 128 x 128
// tiles 68), 1.8 rounds of tiles and 77 MB on their way out; backward 45 (50), 20 GFLOP and 102 MB of pre and d_pre behind the loop, when
// all units store at once.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "f32_tiles.h"
#include "gemm_async.h"
#include "gemm_shape.h"
#include "spa_common.h"

namespace spa {

struct GatedArgs {
  const __bf16* a;               // row a_idx[j] (or j), stride lda
  const int32_t* a_idx;
  long lda;
  const int32_t* total;          // live rows on the device, or null (m_cap)
  int m_cap, kc, F;
  const __bf16 *w, *bias;        // forward: W [2F][kc], bias [2F] or null; backward: W_down [kc][F]
  __bf16* h;                     // forward: [M][F]; backward: d_pre [M][2F]
  __bf16* pre;                   // [M][2F]: forward: written, or null; backward: read
  LargeRule rule;
};

// Phi and phi of the normal distribution.  bf16: erfc(x) exp(x^2) = t P(t), t = 1 / (1 + x / 2), P of degree 6 fitted so that erfc is off
// by at most 1.5e-7 absolute and 2^-12 relative for every x >= 0 (0.5e-7 and 2^-12.6 reached), Phi by half of the first: far below 0, too,
// the rounding of the result to bf16 is what counts.  fp32: the library's.
struct Normal {
  float cdf, density;
};
template <bool EXACT>
__device__ __forceinline__ Normal normal_of(float g) {
  const float e = EXACT ? expf(-0.5f * g * g) : __expf(-0.5f * g * g), density = 0.3989422804014327f * e;
  if (EXACT) return {0.5f * erfcf(-0.7071067811865476f * g), density};
  const float t = __builtin_amdgcn_rcpf(fmaf(0.5f * 0.7071067811865476f, fabsf(g), 1.f));
  float p = fmaf(0.08170961f, t, -0.32737189f);
  p = fmaf(p, t, 0.33701283f);
  p = fmaf(p, t, 0.08411100f);
  p = fmaf(p, t, 0.26049545f);
  p = fmaf(p, t, 0.28199505f);
  p = fmaf(p, t, 0.28204799f);
  const float tail = 0.5f * p * t * e;
  return {g < 0.f ? tail : 1.f - tail, density};
}
template <bool EXACT>
__device__ __forceinline__ float sigmoid_of(float g) {
  if (EXACT) return 1.0f / (1.0f + expf(-g));
  return __builtin_amdgcn_rcpf(1.0f + __expf(-g));
}
struct Act {
  float value, slope;
};
template <int ACT, bool EXACT>
__device__ __forceinline__ Act act_of(float g) {
  if (ACT == SPA_ACT_SILU) {
    const float s = sigmoid_of<EXACT>(g);
    return {g * s, fmaf(g * s, 1.f - s, s)};
  }
  const Normal n = normal_of<EXACT>(g);
  return {g * n.cdf, fmaf(g, n.density, n.cdf)};
}

// Lanes of a wave hand each other values through its own part of LDS: nothing moves across this.
__device__ __forceinline__ void wave_exchange() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// Tile order, operands and loop as in gemm_rows_tiles of gemm_rows.h: live tiles m-major in eight ranges, one an XCD.
template <class MF, bool BACK, bool LOOP, int BM, int BN, int WGM, int WGN, int SA, int SB>
__device__ __forceinline__ void gated_tiles(const GatedArgs& p, int act, unsigned char* smem, unsigned block, unsigned blocks, int m_first, int M) {
  constexpr int E = MF::kEdge, THREADS = 64 * WGM * WGN, TM = BM / WGM / E, TN = BN / WGN / E;
  static_assert(BM == WGM * TM * E && BN == WGN * TN * E && (BACK || TN % 2 == 0), "whole matrix tiles, in pairs");
  using PA = RowsPieces<MF, BM, THREADS>;
  using PB = typename std::conditional<!BACK, RowsPieces<MF, BN, THREADS>,
                                       typename std::conditional<E == 16, DeepBlocks<BN, THREADS>, DeepPieces<BN, THREADS>>::type>::type;
  constexpr int COLS = BACK ? BN : BN / 2;                    // columns of h in a tile
  __bf16* lds = reinterpret_cast<__bf16*>(smem);
  __shared__ __attribute__((aligned(16))) float bias_s[BACK ? 1 : BN];
  const int n_tiles = (p.F + COLS - 1) / COLS, live_tiles = ((M - m_first + BM - 1) / BM) * n_tiles, per_xcd = (live_tiles + 7) >> 3;
  const int xcd = block & 7;
  for (int jx = block >> 3; jx < per_xcd && xcd * per_xcd + jx < live_tiles; jx += blocks >> 3) {
    const int tid = LOOP ? fresh_thread_id() : threadIdx.x, lane = tid & 63;
    const int wv = __builtin_amdgcn_readfirstlane(tid >> 6), tile_id = xcd * per_xcd + jx;
    const int mt = tile_id / n_tiles, nt = tile_id - mt * n_tiles;
    const int m0 = m_first + mt * BM, n0 = nt * COLS;
    const int wm = (wv / WGN) * TM * E, wn = (wv % WGN) * TN * E;
    // rows past the end fetch the last valid row and columns past the edge a valid column: they only reach outputs that are
    // never stored
    const __bf16* ap[PA::kCount];
    const __bf16* bp[PB::kCount];
    const int a_col = PA::col(tid, 0);
    int a_row[PA::kCount];
#pragma unroll
    for (int u = 0; u < PA::kCount; ++u) a_row[u] = min(m0 + PA::row(tid, u), M - 1);
    if (p.a_idx != nullptr) {
#pragma unroll
      for (int u = 0; u < PA::kCount; ++u) a_row[u] = p.a_idx[a_row[u]];
    }
#pragma unroll
    for (int u = 0; u < PA::kCount; ++u) ap[u] = p.a + (long)a_row[u] * p.lda + a_col;
    // row of W behind row r of the tile: matrix tiles of Wg and Wu in turn
    auto w_row = [&](int r) { return (long)(r / E & 1) * p.F + min(n0 + r / (2 * E) * E + r % E, p.F - 1); };
    __bf16 bias_v = static_cast<__bf16>(0.f);
    if (!BACK && p.bias != nullptr && tid < BN) bias_v = p.bias[w_row(tid)];
#pragma unroll
    for (int u = 0; u < PB::kCount; ++u) {
      const int r = PB::row(tid, u), b_col = PB::col(tid, u);
      bp[u] = BACK ? p.w + (long)r * p.F + (n0 + b_col < p.F ? n0 + b_col : n0) : p.w + w_row(r) * p.kc + b_col;
    }
    const int nk = (p.kc + kGaK - 1) / kGaK, k_tail = p.kc % kGaK;
    const __bf16* zeros = reinterpret_cast<const __bf16*>(gemm_zeros);
    const long b_step = BACK ? (long)kGaK * p.F : kGaK;
    // the last step may be partial: pieces past the contraction are zero in both operands
    auto next_a = [&](int u, int t, auto inside) {
      const __bf16* g = ap[u];
      ap[u] += kGaK;
      if (!inside && k_tail != 0 && t == nk - 1 && a_col >= k_tail) g = zeros;
      return g;
    };
    auto next_b = [&](int u, int t, auto inside) {
      const __bf16* g = bp[u];
      bp[u] += b_step;
      if (!inside && k_tail != 0 && t == nk - 1 && (BACK ? PB::row(tid, u) : PB::col(tid, u)) >= k_tail) g = zeros;
      return g;
    };
    auto frag_a = [&](const __bf16* tile, int i, int kk) { return rows_frag<MF>(tile, wm + i * E, kk, lane); };
    auto frag_b = [&](const __bf16* tile, int j, int kk) {
      if constexpr (BACK && E == 16) return deep_block_frag(tile, kk, wn + j * E, lane);
      else if constexpr (BACK) return deep_frag<BN>(tile, kk, wn + j * E, lane);
      else return rows_frag<MF>(tile, wn + j * E, kk, lane);
    };
    auto tables = [&] {
      if (!BACK && tid < BN) bias_s[tid] = static_cast<float>(bias_v);
    };
    static_assert(BACK || BN <= THREADS, "one a thread");
    typename MF::Acc acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int r = 0; r < 4 * MF::kGroups; ++r) acc[i][j][r] = 0.f;
    gemm_async_loop<MF, BM * kGaK, BN * kGaK, PA::kCount, PB::kCount, SA, SB, THREADS, TM, TN>(lds, nk, next_a, next_b, frag_a, frag_b, acc, tables);

    // EDGE rows of a row of matrix tiles at a time go through the wave's own part of LDS and leave as whole 16-byte pieces
    auto forward = [&](auto which) {
      constexpr int ACT = decltype(which)::value, NC = TN / 2 * E, ORS = NC + 8, PIECES = NC / 8, PER_LANE = (E * PIECES + 63) / 64;
      static_assert(WGM * WGN * 2 * E * ORS <= (SA * BM + SB * BN) * kGaK, "output staging fits in the operand buffers");
      const int first = n0 + wn / 2;
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        auto leave = [&](int turn, __bf16* to, long ld, auto value) {
          __bf16* tile = lds + (wv * 2 + (turn & 1)) * E * ORS;
#pragma unroll
          for (int j = 0; j < TN / 2; ++j)
#pragma unroll
            for (int g = 0; g < MF::kGroups; ++g) {
              const int n = MF::row(g, lane);               // 4 consecutive columns
              *reinterpret_cast<bf16x4*>(&tile[lane % E * ORS + j * E + n]) = __builtin_convertvector(value(j, g), bf16x4);
            }
          wave_exchange();
#pragma unroll
          for (int u = 0; u < PER_LANE; ++u) {
            const int c = lane + 64 * u, r = c / PIECES, ch = c % PIECES, row = m0 + wm + i * E + r, n = first + ch * 8;
            if (c < E * PIECES && row < M && n < p.F)
              *reinterpret_cast<bf16x8*>(to + (long)row * ld + n) = *reinterpret_cast<const bf16x8*>(&tile[r * ORS + ch * 8]);
          }
          wave_exchange();
        };
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
          for (int g = 0; g < MF::kGroups; ++g) {
            const floatx4 b = *reinterpret_cast<const floatx4*>(&bias_s[wn + j * E + MF::row(g, lane)]);
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[i][j][4 * g + e] += b[e];
          }
        auto part = [&](int j, int g) { return floatx4{acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]}; };
        const int turn = p.pre != nullptr ? 3 * i : i;
        leave(turn, p.h, p.F, [&](int j, int g) {             // (from the unrounded sums)
          const floatx4 a = part(2 * j, g), u = part(2 * j + 1, g);
          floatx4 v;
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = act_of<ACT, false>(a[e]).value * u[e];
          return v;
        });
        if (p.pre != nullptr) {
          leave(turn + 1, p.pre, 2L * p.F, [&](int j, int g) { return part(2 * j, g); });
          leave(turn + 2, p.pre + p.F, 2L * p.F, [&](int j, int g) { return part(2 * j + 1, g); });
        }
      }
    };
    // dh goes through LDS in fp32, so that d_pre is rounded once
    auto backward = [&](auto which) {
      constexpr int ACT = decltype(which)::value, NC = TN * E, ORS = NC + 4, PIECES = NC / 8, PER_LANE = E * PIECES / 64;
      static_assert(E * PIECES % 64 == 0 && WGM * WGN * E * ORS * 4 <= (SA * BM + SB * BN) * kGaK * 2, "output staging fits in the operand buffers");
      float* tile = reinterpret_cast<float*>(smem) + wv * E * ORS;
      const int first = n0 + wn;
      // (the pieces of g and u one ahead: all of a row of tiles at once spill beside the 128 accumulators of 256 x 256 tiles)
      bf16x8 gate[2], up[2];
      auto fetch = [&](int i, int u) {
        const int c = lane + 64 * u, row = min(m0 + wm + i * E + c / PIECES, M - 1), n = first + c % PIECES * 8;
        const __bf16* from = p.pre + (long)row * (2L * p.F) + (n < p.F ? n : n0);
        const int at = (i * PER_LANE + u) & 1;
        gate[at] = *reinterpret_cast<const bf16x8*>(from);
        up[at] = *reinterpret_cast<const bf16x8*>(from + p.F);
      };
      fetch(0, 0);
#pragma unroll
      for (int i = 0; i < TM; ++i) {
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
          for (int g = 0; g < MF::kGroups; ++g)
            *reinterpret_cast<floatx4*>(&tile[lane % E * ORS + j * E + MF::row(g, lane)]) =
                floatx4{acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]};
        wave_exchange();
#pragma unroll
        for (int u = 0; u < PER_LANE; ++u) {
          const int c = lane + 64 * u, r = c / PIECES, ch = c % PIECES, row = m0 + wm + i * E + r, n = first + ch * 8, at = (i * PER_LANE + u) & 1;
          if (u + 1 < PER_LANE) fetch(i, u + 1);
          else if (i + 1 < TM) fetch(i + 1, 0);
          const floatx4 lo = *reinterpret_cast<const floatx4*>(&tile[r * ORS + ch * 8]), hi = *reinterpret_cast<const floatx4*>(&tile[r * ORS + ch * 8 + 4]);
          const floatx8 gf = bf16x8_to_float(gate[at]), uf = bf16x8_to_float(up[at]);
          floatx8 dg, du;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float dh = e < 4 ? lo[e & 3] : hi[e & 3];
            const Act a = act_of<ACT, false>(gf[e]);
            dg[e] = dh * uf[e] * a.slope;
            du[e] = dh * a.value;
          }
          if (row < M && n < p.F) {
            __bf16* to = p.h + (long)row * (2L * p.F) + n;
            *reinterpret_cast<bf16x8*>(to) = float_to_bf16x8(dg);
            *reinterpret_cast<bf16x8*>(to + p.F) = float_to_bf16x8(du);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
        wave_exchange();
      }
    };
    using Silu = std::integral_constant<int, SPA_ACT_SILU>;
    using Gelu = std::integral_constant<int, SPA_ACT_GELU>;
    if constexpr (BACK) act == SPA_ACT_SILU ? backward(Silu{}) : backward(Gelu{});
    else act == SPA_ACT_SILU ? forward(Silu{}) : forward(Gelu{});
    if (!LOOP) break;
    __syncthreads();                 // the table and the buffers are read to the end
  }
}

__device__ __forceinline__ int gated_live_rows(const GatedArgs& p) { return p.total != nullptr ? min(p.total[0], p.m_cap) : p.m_cap; }

constexpr size_t kGatedSmallLds = (size_t)2 * (128 + 128) * kGaK * sizeof(__bf16), kGatedRingLds = 2 * kGatedSmallLds, kGatedTinyLds = kGatedRingLds / 2;
constexpr size_t kGatedBigLds = (size_t)std::max({3 * 192 + 3 * 192, 3 * 256 + 2 * 192, 2 * 256 + 2 * 256}) * kGaK * sizeof(__bf16);

// 128 x 128 tiles: four waves of 64 x 64, two workgroups a unit.
template <bool BACK>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2))) gated_small_kernel(const GatedArgs p, int act) {
  extern __shared__ __attribute__((aligned(16))) unsigned char gated_smem[];
  gated_tiles<Mfma32, BACK, false, 128, 128, 2, 2, 2, 2>(p, act, gated_smem, blockIdx.x, gridDim.x, 0, gated_live_rows(p));
}
// 128 x 128 tiles where a unit has one: eight waves and four steps in LDS (forward 32 x 64 a wave, which holds whole pairs).
template <bool BACK>
__global__ void __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(2))) gated_ring_kernel(const GatedArgs p, int act) {
  extern __shared__ __attribute__((aligned(16))) unsigned char gated_smem[];
  gated_tiles<Mfma32, BACK, false, 128, 128, BACK ? 2 : 4, BACK ? 4 : 2, 4, 4>(p, act, gated_smem, blockIdx.x, gridDim.x, 0, gated_live_rows(p));
}
// 64 x 64 tiles (32 columns of h) of few rows, as gemm_rows_tiny_kernel.
__global__ void __launch_bounds__(128) gated_tiny_kernel(const GatedArgs p, int act) {
  extern __shared__ __attribute__((aligned(16))) unsigned char gated_smem[];
  gated_tiles<Mfma32, false, false, 64, 64, 2, 1, 4, 4>(p, act, gated_smem, blockIdx.x, gridDim.x, 0, gated_live_rows(p));
}
// The large shapes, one resident workgroup a unit that walks the tiles of the plan for the live rows (gemm_shape.h).
template <bool BACK>
__global__ void __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(1))) gated_big_kernel(const GatedArgs p, int act) {
  extern __shared__ __attribute__((aligned(16))) unsigned char gated_smem[];
  const int M = gated_live_rows(p);
  const LargePlan plan = large_plan(M, BACK ? p.F : 2 * p.F, 0, p.rule);
  if (plan.medium) {
    gated_tiles<Mfma16, BACK, true, 192, 192, 4, 2, 3, 3>(p, act, gated_smem, blockIdx.x, gridDim.x, 0, M);
  } else {
    if (plan.wide_rows > 0) gated_tiles<Mfma32, BACK, true, 256, 256, 2, 4, 2, 2>(p, act, gated_smem, blockIdx.x, gridDim.x, 0, plan.wide_rows);
    if (plan.wide_rows < M) gated_tiles<Mfma16, BACK, true, 256, 192, 4, 2, 3, 2>(p, act, gated_smem, blockIdx.x, gridDim.x, plan.wide_rows, M);
  }
}

// ---- fp32 (tiny workload): f32_tiles.h, of W the rows of Wg and of Wu beside each other
struct GatedF32 {
  const float* a;
  const int32_t *a_idx, *total;
  long lda;
  int m_cap, kc, F;
  const float *w, *bias;
  float *h, *pre;
};
template <int ACT, bool BACK, int EDGE>
__global__ void __launch_bounds__(kF32Threads) gated_f32_kernel(const GatedF32 p) {
  using PA = F32Place<EDGE, true>;
  using PB = F32Place<EDGE, !BACK>;
  using Out = F32Quarter<EDGE>;
  constexpr int NB = BACK ? 1 : 2;
  __shared__ F32Lds<EDGE, NB> l;
  const int M = p.total != nullptr ? min(p.total[0], p.m_cap) : p.m_cap, n_tiles = (p.F + EDGE - 1) / EDGE;
  const long tiles = (long)((M + EDGE - 1) / EDGE) * n_tiles;
  for (long tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
    const int m0 = (int)(tile / n_tiles) * EDGE, n0 = (int)(tile % n_tiles) * EDGE;
    const float *ap[PA::kCount], *wp[PB::kCount];
#pragma unroll
    for (int i = 0; i < PA::kCount; ++i) {
      const int m = min(m0 + PA::line(i), M - 1);
      ap[i] = p.a + (p.a_idx != nullptr ? (long)p.a_idx[m] : (long)m) * p.lda;
    }
#pragma unroll
    for (int i = 0; i < PB::kCount; ++i) wp[i] = p.w + (long)min(n0 + PB::line(i), p.F - 1) * (BACK ? 1 : p.kc);
    typename Out::Acc acc[NB] = {};
    f32_tile_sums<EDGE, NB, true, !BACK, 2>(l, p.kc, [&](int i, int k) { return ap[i][k]; },
                                         [&](int q, int i, int k) { return BACK ? wp[i][(long)k * p.F] : wp[i][(long)q * p.F * p.kc + k]; }, F32AsIs{}, F32AsIs{},
                                         acc, [](const auto&, int) {});
    __syncthreads();                 // (the next tile's first step goes where this one's last may be read)
#pragma unroll
    for (int e = 0; e < Out::kCount; ++e) {
        const int m = m0 + Out::row(e), n = n0 + Out::col();
        if (m >= M || n >= p.F) continue;
        const long at = (long)m * 2 * p.F + n;
        if constexpr (BACK) {
          const Act a = act_of<ACT, true>(p.pre[at]);
          p.h[at] = acc[0][e] * p.pre[at + p.F] * a.slope;
          p.h[at + p.F] = acc[0][e] * a.value;
        } else {
          const float g = acc[0][e] + (p.bias != nullptr ? p.bias[n] : 0.f), u = acc[NB - 1][e] + (p.bias != nullptr ? p.bias[p.F + n] : 0.f);
          p.h[(long)m * p.F + n] = act_of<ACT, true>(g).value * u;
          if (p.pre != nullptr) {
            p.pre[at] = g;
            p.pre[at + p.F] = u;
          }
        }
      }
  }
}

// ------------------------------------------------------------------------------- host
template <bool BACK>
static int launch_gated(const char* fn, GatedArgs args, int act, hipStream_t st) {
  const int ncols = BACK ? args.F : 2 * args.F;
  const bool counted = args.total != nullptr;
  const int cfg = options().gemm_tm;
  const bool big = cfg != 0 ? cfg >= 6 : large_tiles(args.m_cap, counted, ncols, args.kc), ring = !big && ring_tiles(args.m_cap, counted, ncols);
  const bool tiny = !BACK && !big && cfg == 0 && tiny_tiles(args.m_cap, counted, ncols);
  args.rule = large_rule(ncols, args.kc, false);
  const size_t smem = big ? kGatedBigLds : tiny ? kGatedTinyLds : ring ? kGatedRingLds : kGatedSmallLds;
  const long tiles = gemm_tiles<long>(args.m_cap, ncols, big ? 192 : tiny ? 64 : 128);          // (no less than with 256)
  SPA_REQUIRE(big || tiles + 8 < 4294967296L / 512, SPA_ERR_INVALID_ARG, "%s: too many tiles (a launch has fewer than 2^32 threads)", fn);
  const long tiles8 = (tiles + 7) / 8 * 8;
  const auto kernel = big ? gated_big_kernel<BACK> : tiny ? gated_tiny_kernel : ring ? gated_ring_kernel<BACK> : gated_small_kernel<BACK>;
  const hipError_t attr = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  SPA_REQUIRE(attr == hipSuccess, SPA_ERR_HIP, "%s: cannot reserve %zu bytes of LDS", fn, smem);
  hipLaunchKernelGGL(kernel, dim3((unsigned)(big ? std::min(tiles8, 256L) : tiles8)), dim3(tiny ? 128 : big || ring ? 512 : 256), smem, st, args, act);
  return check_launch(fn);
}

template <bool BACK>
static int launch_gated_f32(const char* fn, const GatedF32& a, int act, hipStream_t st) {
  const bool wide = f32_wide(a.m_cap, a.F);
  const auto kernel = act == SPA_ACT_SILU ? (wide ? gated_f32_kernel<SPA_ACT_SILU, BACK, 64> : gated_f32_kernel<SPA_ACT_SILU, BACK, 32>)
                                          : (wide ? gated_f32_kernel<SPA_ACT_GELU, BACK, 64> : gated_f32_kernel<SPA_ACT_GELU, BACK, 32>);
  hipLaunchKernelGGL(kernel, dim3((unsigned)std::min(f32_tiles(a.m_cap, a.F, wide ? 64 : 32), 8192L)), dim3(kF32Threads), 0, st, a);
  return check_launch(fn);
}

static int gated_checks(const char* fn, int M_cap, int K, int F, int act, int dtype) {
  SPA_REFUSE_IN_GROUP(fn);
  SPA_REQUIRE(M_cap >= 1 && K >= 1 && F >= 1, SPA_ERR_INVALID_ARG, "%s: M_cap, the contraction and F must be >= 1", fn);
  SPA_REQUIRE(M_cap < 2147483647 - 512 && F < (1 << 30), SPA_ERR_INVALID_ARG, "%s: M_cap must be < 2^31 - 513 and F < 2^30", fn);
  SPA_REQUIRE(dtype == SPA_F32 || dtype == SPA_BF16, SPA_ERR_UNSUPPORTED, "%s: unknown dtype %d", fn, dtype);
  SPA_REQUIRE(act == SPA_ACT_SILU || act == SPA_ACT_GELU, SPA_ERR_INVALID_ARG, "%s: unknown activation %d", fn, act);
  return SPA_OK;
}

}  // namespace spa

using namespace spa;

extern "C" int spa_gated_linear_packed(const void* x, const int32_t* gather_idx, const int32_t* total, const void* W, const void* bias, int M_cap, int K,
                                       int F, int act, int dtype, void* h, void* pre, void* stream) {
  const char* fn = "spa_gated_linear_packed";
  if (int rc = gated_checks(fn, M_cap, K, F, act, dtype)) return rc;
  SPA_REQUIRE(x && W && h, SPA_ERR_INVALID_ARG, "%s: null pointer", fn);
  hipStream_t st = as_stream(stream);
  if (dtype == SPA_F32) {
    const GatedF32 a = {(const float*)x, gather_idx, total, (long)K, M_cap, K, F, (const float*)W, (const float*)bias, (float*)h, (float*)pre};
    return launch_gated_f32<false>(fn, a, act, st);
  }
  SPA_REQUIRE(K % 8 == 0 && F % 8 == 0, SPA_ERR_UNSUPPORTED, "%s: K and F must be multiples of 8 for bf16", fn);
  SPA_REQUIRE(K <= kMostContraction, SPA_ERR_INVALID_ARG, "%s: K must be < 2^31 - 64 for bf16", fn);
  SPA_REQUIRE(aligned16(x) && aligned16(W) && aligned16(h) && aligned16(pre), SPA_ERR_INVALID_ARG, "%s: x / W / h / pre not 16-byte aligned", fn);
  GatedArgs a = {(const __bf16*)x, gather_idx, (long)K, total, M_cap, K, F, (const __bf16*)W, (const __bf16*)bias, (__bf16*)h, (__bf16*)pre, {}};
  return launch_gated<false>(fn, a, act, st);
}

extern "C" int spa_gated_linear_packed_bwd(const void* dy, const int32_t* dy_idx, int64_t dy_row_stride, const int32_t* total, const void* W_down,
                                           const void* pre, int M_cap, int N_out, int F, int act, int dtype, void* d_pre, void* stream) {
  const char* fn = "spa_gated_linear_packed_bwd";
  if (int rc = gated_checks(fn, M_cap, N_out, F, act, dtype)) return rc;
  SPA_REQUIRE(dy && W_down && pre && d_pre, SPA_ERR_INVALID_ARG, "%s: null pointer", fn);
  SPA_REQUIRE(dy_row_stride >= N_out && dy_row_stride < (1LL << 31), SPA_ERR_INVALID_ARG, "%s: dy_row_stride out of range", fn);
  hipStream_t st = as_stream(stream);
  if (dtype == SPA_F32) {
    const GatedF32 a = {(const float*)dy, dy_idx, total, (long)dy_row_stride, M_cap, N_out, F, (const float*)W_down, nullptr, (float*)d_pre, (float*)pre};
    return launch_gated_f32<true>(fn, a, act, st);
  }
  SPA_REQUIRE(N_out % 8 == 0 && F % 8 == 0 && dy_row_stride % 8 == 0, SPA_ERR_UNSUPPORTED, "%s: N_out, F and dy_row_stride must be multiples of 8 for bf16",
              fn);
  SPA_REQUIRE(N_out <= kMostContraction, SPA_ERR_INVALID_ARG, "%s: N_out must be < 2^31 - 64 for bf16", fn);
  SPA_REQUIRE(aligned16(dy) && aligned16(W_down) && aligned16(pre) && aligned16(d_pre), SPA_ERR_INVALID_ARG,
              "%s: dy / W_down / pre / d_pre not 16-byte aligned", fn);
  GatedArgs a = {(const __bf16*)dy, dy_idx, (long)dy_row_stride, total, M_cap, N_out, F, (const __bf16*)W_down, nullptr, (__bf16*)d_pre, (__bf16*)pre, {}};
  return launch_gated<true>(fn, a, act, st);
}
