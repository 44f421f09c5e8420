// Backward of the attention to another sequence (cross_attention.hip): with P = exp(S - lse), dP = dO V^T, D_r = <dO_r, O_r>, dS = P (dP -
// D)
//   dQ = scale dS K,   dK = scale dS^T Q,   dV = P^T dO        (sums over the tokens and the heads that share the key head)
// Two launches.  The dq launch walks the keys for 32 rows a wave as the forward does and leaves D; the dk / dv launch walks the rows for 32
// keys a wave, S and dP un-transposed (a lane is a key), so that P and dS are operands in registers again.  D is formed from the rounded
// result.  Few owned rows: the four waves share them.  Few units and many rows on the other side: those are split over workgroups, whose
// fp32 sums a further launch adds in the order of the splits.  Everything is added in a fixed order.  Units of few rows and keys take one
// launch (cross_bwd_short_kernel).
// Bound by the order within a wave, products, exponentials, products, at two (dk / dv) and three waves a SIMD: of the busy cycles the
// matrix pipe has 0.38 and 0.42, the vector instructions 0.43 and 0.54, LDS 0.44 (half of that conflicts of banks in dk / dv); S and dP are
// formed in both launches, seven products where five would do.  8 x 1568 to 3136 tokens, 410 to 1024 states, 12 and 4 heads of 64: dq 89
// us, dk / dv 137 and 10 for the splits' sums.
#include <algorithm>
#include <cmath>

#include "cross_attention.h"

namespace spa {

template <typename T>
struct CrossBwd {
  const T *q, *k, *v, *out, *dout;
  long qs, ks, vs;
  CrossShape s;
  const float* lse;
  float* D;                      // [H][stat_stride]
  T *dq, *dk, *dv;
  long dqs, dks, dvs;
  float* part;                   // [unit][split][owned row][DH], of dk / dv [..][2][DH]; or null
  long part_rows;
};

template <typename T, int DH, int KW>
struct CrossDqTiles {
  static constexpr int STEP = CrossSteps<KW>::STEP, RS = Ops<T, DH>::RS;
  __attribute__((aligned(16))) T K[2][STEP * RS];
  __attribute__((aligned(16))) T V[2][STEP * RS];
};

template <typename T, int DH, int KW>
__global__ void __launch_bounds__(kCrossThreads, sizeof(T) == 4 ? 1 : 2) cross_dq_kernel(const CrossBwd<T> a) {
  using O = Ops<T, DH>;
  using W = CrossSteps<KW>;
  constexpr int DB = DH / 32, NB = W::TILE / 32;
  extern __shared__ __attribute__((aligned(16))) unsigned char cross_smem[];
  CrossDqTiles<T, DH, KW>& l = *reinterpret_cast<CrossDqTiles<T, DH, KW>*>(cross_smem);
  const CrossUnit u = cross_unit(a.s);
  const int r0 = u.block * W::ROWS;
  if (!u.valid || r0 >= u.nq) return;
  const int lane = threadIdx.x & 63, l32 = lane & 31, hh = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int rw = wave / KW, part = wave % KW, r = r0 + rw * 32 + l32;
  const bool ok = r < u.nq, wave_live = r0 + rw * 32 < u.nq;
  const int rc = min(r, u.nq - 1), G = (int)a.s.G.d;
  const Share sh = share_of<W::STEP>(u.nk, a.s.splits, u.split);
  if (sh.n <= 0 && u.split > 0) return;
  const int n = sh.n, nt = (n + W::STEP - 1) / W::STEP;
  const long first = u.k0 + sh.from, C = (long)a.s.H * DH;
  floatx16 acc[DB], negD;
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[d][i] = 0.f;
  CrossStage<T, DH, W::STEP, false> st(a.k + first * a.ks + u.hk * DH, a.ks, a.v + first * a.vs + u.hk * DH, a.vs, a.s.G, n - 1);
  if (nt > 0) st.load(0);
  const uint32_t token = quotient((uint32_t)rc, a.s.G);
  const long stat = (u.hk * G + (rc - (int)(token * G))) * a.s.stat_stride + u.q0 + token;
  const long dense = u.q0 * C + (long)u.hk * G * DH + group_row<DH>(a.s.G, rc, C);
  const float lse = a.lse[stat];
  const typename O::Row qf = O::row(a.q + u.q0 * a.qs + (long)u.hk * G * DH + group_row<DH>(a.s.G, rc, a.qs), hh);
  const typename O::Row gf = O::row(a.dout + dense, hh);
  {
    const typename O::Row of = O::row(a.out + dense, hh);
    float D = 0.f, unused = 0.f;
    O::sums(gf, of, D, unused);
    D = sum_across_halves(D);
#pragma unroll
    for (int i = 0; i < 16; ++i) negD[i] = -D;
    if (u.split == 0 && part == 0 && ok && hh == 0) a.D[stat] = D;
  }
  const bool none = lse == -INFINITY || !ok, far = __ballot(!none && fabsf(lse) >= kFarScore) != 0;
  const float ref = none ? INFINITY : lse, lse2 = ref * kLog2e;
  if (nt > 0) st.template store<true>(l.K[0], l.V[0]);
  __syncthreads();
  walk_tiles(nt, [&](int t, auto at) {
    constexpr bool end = decltype(at)::value == kTileLast;
    const int buf = t & 1, left = n - t * W::STEP - part * W::TILE;
    if (!end) st.load(t * W::STEP + W::STEP);
    if (wave_live) {
      const T *K = &l.K[buf][part * W::TILE * O::RS], *V = &l.V[buf][part * W::TILE * O::RS];
#pragma unroll
      for (int sb = 0; sb < NB; ++sb) {
        if (end && sb * 32 >= left) break;
        floatx16 s, dp = negD;
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = 0.f;
        O::dot(s, O::row(&K[(sb * 32 + l32) * O::RS], hh), qf);
        O::dot(dp, O::row(&V[(sb * 32 + l32) * O::RS], hh), gf);
        if (end) {
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (sb * 32 + acc_row(i, hh) >= left) s[i] = -INFINITY;
        }
        if (!far) {
#pragma unroll
          for (int i = 0; i < 16; ++i) s[i] = __builtin_amdgcn_exp2f(fmaf(s[i], a.s.c, -lse2));
        } else {
#pragma unroll
          for (int i = 0; i < 16; ++i) s[i] = __builtin_amdgcn_exp2f(fmaf(s[i], a.s.scale, -ref) * kLog2e);
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) dp[i] *= s[i];
        O::outer(acc, K, sb, dp, lane);
      }
    }
    if (!end) st.template store<decltype(at)::value == kTileBeforeLast>(l.K[buf ^ 1], l.V[buf ^ 1]);
    __syncthreads();
  });
  if constexpr (KW > 1) {
    constexpr int N = DB * 16;
    static_assert((KW - 1) * W::RW * N * kWave * sizeof(float) <= sizeof(l), "the sums of the other waves");
    float* const sums = reinterpret_cast<float*>(cross_smem) + lane;
    if (part > 0) {
      float* mine = sums + ((part - 1) * W::RW + rw) * N * kWave;
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) mine[(d * 16 + i) * kWave] = acc[d][i];
    }
    __syncthreads();
    if (part > 0) return;
#pragma unroll
    for (int p = 0; p < KW - 1; ++p) {
      const float* other = sums + (p * W::RW + rw) * N * kWave;
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[d][i] += other[(d * 16 + i) * kWave];
    }
  }
  if (!wave_live) return;
  if (a.part != nullptr) {
    if (!ok) return;
    float* row = a.part + ((((long)u.b * a.s.Hk + u.hk) * a.s.splits + u.split) * a.part_rows + rc) * DH;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *reinterpret_cast<floatx4*>(row + d * 32 + 8 * g + 4 * hh) = floatx4{acc[d][4 * g], acc[d][4 * g + 1], acc[d][4 * g + 2], acc[d][4 * g + 3]};
    return;
  }
  O::store(acc, a.s.scale, a.dq + u.q0 * a.dqs + (long)u.hk * G * DH + group_row<DH>(a.s.G, rc, a.dqs), ok, hh);
}

template <typename T, int DH, int KW>
struct CrossKeyTiles {
  static constexpr int STEP = CrossSteps<KW>::STEP, RS = Ops<T, DH>::RS;
  __attribute__((aligned(16))) T Q[2][STEP * RS];
  __attribute__((aligned(16))) T G[2][STEP * RS];             // dO
  __attribute__((aligned(16))) float lse[2][STEP];            // +inf: no key, or no row (probability 0)
  __attribute__((aligned(16))) float lse2[2][STEP];           // times log2 e
  __attribute__((aligned(16))) float negD[2][STEP];
  int far[2][STEP / 64];
};

template <typename T, int DH, int KW>
__global__ void __launch_bounds__(kCrossThreads, sizeof(T) == 4 ? 1 : 2) cross_dkdv_kernel(const CrossBwd<T> a) {
  using O = Ops<T, DH>;
  using W = CrossSteps<KW>;
  constexpr int DB = DH / 32, NB = W::TILE / 32;
  extern __shared__ __attribute__((aligned(16))) unsigned char cross_smem[];
  CrossKeyTiles<T, DH, KW>& l = *reinterpret_cast<CrossKeyTiles<T, DH, KW>*>(cross_smem);
  const CrossUnit u = cross_unit(a.s);
  const int k0 = u.block * W::ROWS;
  if (!u.valid || k0 >= u.held) return;
  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, hh = lane >> 5, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rw = wave / KW, part = wave % KW, ki = k0 + rw * 32 + l32, G = (int)a.s.G.d;
  const bool wave_live = k0 + rw * 32 < u.nk;
  const Share sh = share_of<W::STEP>(u.nq, a.s.splits, u.split);
  if (sh.n <= 0 && u.split > 0) return;
  if (a.part != nullptr && k0 >= u.nk) return;                // (rows behind the keys: the launch that adds clears them)
  const int n = k0 < u.nk ? sh.n : 0, nt = (n + W::STEP - 1) / W::STEP;
  const long C = (long)a.s.H * DH, head = (long)u.hk * G * DH, k_row = u.k0 + min(ki, max(u.nk - 1, 0));
  floatx16 dka[DB], dva[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) dka[d][i] = dva[d][i] = 0.f;
  if (nt > 0) {
    CrossStage<T, DH, W::STEP, true> st(a.q + u.q0 * a.qs + head, a.qs, a.dout + u.q0 * C + head, C, a.s.G, sh.from + n - 1);      // (rows of the unit)
    float lse_t = 0.f, d_t = 0.f;
    const long stat0 = (long)u.hk * G * a.s.stat_stride + u.q0;
    auto load = [&](int t0) {
      st.load(sh.from + t0);
      const int r = sh.from + min(t0 + (tid & (W::STEP - 1)), n - 1);
      const uint32_t i = quotient((uint32_t)r, a.s.G);
      const long stat = stat0 + (long)((uint64_t)(uint32_t)(r - (int)(i * G)) * (uint32_t)a.s.stat_stride) + i;
      lse_t = a.lse[stat];
      d_t = a.D[stat];
    };
    auto store = [&](int buf, int t0, auto clear) {
      st.template store<clear>(l.Q[buf], l.G[buf]);
      if (tid < W::STEP) {
        const bool none = lse_t == -INFINITY || t0 + tid >= n;
        const bool any = __ballot(!none && fabsf(lse_t) >= kFarScore) != 0;
        l.lse[buf][tid] = none ? INFINITY : lse_t;
        l.lse2[buf][tid] = none ? INFINITY : lse_t * kLog2e;
        l.negD[buf][tid] = -d_t;
        if (lane == 0) l.far[buf][tid >> 6] = any;
      }
    };
    load(0);
    const typename O::Row kf = O::row(a.k + k_row * a.ks + u.hk * DH, hh), vf = O::row(a.v + k_row * a.vs + u.hk * DH, hh);
    store(0, 0, std::true_type{});
    __syncthreads();
    walk_tiles(nt, [&](int t, auto at) {
      constexpr bool end = decltype(at)::value == kTileLast;
      const int buf = t & 1, left = n - t * W::STEP - part * W::TILE;
      if (!end) load(t * W::STEP + W::STEP);
      if (wave_live) {
#pragma unroll
        for (int sb = 0; sb < NB; ++sb) {
          if (end && sb * 32 >= left) break;
          const int at0 = part * W::TILE + sb * 32;
          floatx16 s, dp;
#pragma unroll
          for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            const floatx4 d4 = *reinterpret_cast<const floatx4*>(&l.negD[buf][at0 + 8 * g + 4 * hh]);
#pragma unroll
            for (int i = 0; i < 4; ++i) dp[4 * g + i] = d4[i];
          }
          O::dot(s, O::row(&l.Q[buf][(at0 + l32) * O::RS], hh), kf);
          O::dot(dp, O::row(&l.G[buf][(at0 + l32) * O::RS], hh), vf);
          if (__builtin_amdgcn_readfirstlane(l.far[buf][at0 >> 6]) == 0) {
#pragma unroll
            for (int g = 0; g < 4; ++g) {
              const floatx4 l4 = *reinterpret_cast<const floatx4*>(&l.lse2[buf][at0 + 8 * g + 4 * hh]);
#pragma unroll
              for (int i = 0; i < 4; ++i) s[4 * g + i] = __builtin_amdgcn_exp2f(fmaf(s[4 * g + i], a.s.c, -l4[i]));
            }
          } else {
#pragma unroll
            for (int g = 0; g < 4; ++g) {
              const floatx4 l4 = *reinterpret_cast<const floatx4*>(&l.lse[buf][at0 + 8 * g + 4 * hh]);
#pragma unroll
              for (int i = 0; i < 4; ++i) s[4 * g + i] = __builtin_amdgcn_exp2f(fmaf(s[4 * g + i], a.s.scale, -l4[i]) * kLog2e);
            }
          }
#pragma unroll
          for (int i = 0; i < 16; ++i) dp[i] *= s[i];
          O::outer(dva, &l.G[buf][0], at0 / 32, s, lane);
          O::outer(dka, &l.Q[buf][0], at0 / 32, dp, lane);
        }
      }
      if (!end) store(buf ^ 1, t * W::STEP + W::STEP, std::bool_constant<decltype(at)::value == kTileBeforeLast>{});
      __syncthreads();
    });
  }
  if constexpr (KW > 1) {
    constexpr int N = 2 * DB * 16;
    static_assert((KW - 1) * W::RW * N * kWave * sizeof(float) <= sizeof(l), "the sums of the other waves");
    float* const sums = reinterpret_cast<float*>(cross_smem) + lane;
    if (part > 0) {
      float* mine = sums + ((part - 1) * W::RW + rw) * N * kWave;
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          mine[(d * 16 + i) * kWave] = dka[d][i];
          mine[((DB + d) * 16 + i) * kWave] = dva[d][i];
        }
    }
    __syncthreads();
    if (part > 0) return;
#pragma unroll
    for (int p = 0; p < KW - 1; ++p) {
      const float* other = sums + (p * W::RW + rw) * N * kWave;
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          dka[d][i] += other[(d * 16 + i) * kWave];
          dva[d][i] += other[((DB + d) * 16 + i) * kWave];
        }
    }
  }
  if (a.part != nullptr) {
    if (ki >= u.nk) return;
    float* row = a.part + ((((long)u.b * a.s.Hk + u.hk) * a.s.splits + u.split) * a.part_rows + ki) * 2 * DH;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        float* to = row + d * 32 + 8 * g + 4 * hh;
        *reinterpret_cast<floatx4*>(to) = floatx4{dka[d][4 * g], dka[d][4 * g + 1], dka[d][4 * g + 2], dka[d][4 * g + 3]};
        *reinterpret_cast<floatx4*>(to + DH) = floatx4{dva[d][4 * g], dva[d][4 * g + 1], dva[d][4 * g + 2], dva[d][4 * g + 3]};
      }
    return;
  }
  if (ki >= u.nk) {                                           // places without a key: no gradient
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) dka[d][i] = dva[d][i] = 0.f;
  }
  const bool ok = ki < u.held;
  const long row = u.k0 + min(ki, u.held - 1);
  O::store(dka, a.s.scale, a.dk + row * a.dks + u.hk * DH, ok, hh);
  O::store(dva, 1.0f, a.dv + row * a.dvs + u.hk * DH, ok, hh);
}

// Adds the splits' sums of an owned row in their order: DH / 4 lanes a row of dq (WHICH 1), twice as many a row of dk and dv (WHICH 2).
template <typename T, int DH, int STEP, int WHICH>
__global__ void __launch_bounds__(kCrossThreads) cross_sum_kernel(const CrossBwd<T> a) {
  constexpr int LANES = WHICH * DH / 4, ROWS = kCrossThreads / LANES, U = 8;
  const int G = (int)a.s.G.d, c = threadIdx.x % LANES * 4;
  const long per = (a.part_rows + ROWS - 1) / ROWS, unit = blockIdx.x / per;
  const int r = (int)(blockIdx.x % per) * ROWS + threadIdx.x / LANES, b = (int)(unit / a.s.Hk), hk = (int)(unit % a.s.Hk);
  const int q0 = a.s.cu_q[b], k0 = a.s.cu_k[b];
  int nq, nk, held;
  cross_lengths(a.s, b, q0, k0, nq, nk, held);
  if (r >= (WHICH == 1 ? nq : held)) return;
  const int live = WHICH == 2 && r >= nk ? 0 : share_of<STEP>(WHICH == 1 ? nk : nq, a.s.splits, 0).live;
  const float* p = a.part + (unit * a.s.splits * a.part_rows + r) * WHICH * DH + c;
  floatx4 sum = {0.f, 0.f, 0.f, 0.f};
  for (int s0 = 0; s0 < live; s0 += U) {
    floatx4 v[U];
#pragma unroll
    for (int i = 0; i < U; ++i) v[i] = *reinterpret_cast<const floatx4*>(p + (long)min(s0 + i, live - 1) * a.part_rows * WHICH * DH);
#pragma unroll
    for (int i = 0; i < U; ++i)
      if (s0 + i < live) sum += v[i];
  }
  T* to;
  if (WHICH == 1) {
    to = a.dq + (long)q0 * a.dqs + (long)hk * G * DH + group_row<DH>(a.s.G, r, a.dqs) + c;
    sum *= a.s.scale;
  } else if (c < DH) {
    to = a.dk + ((long)k0 + r) * a.dks + hk * DH + c;
    sum *= a.s.scale;
  } else {
    to = a.dv + ((long)k0 + r) * a.dvs + hk * DH + c - DH;
  }
  if constexpr (sizeof(T) == 2) *reinterpret_cast<bf16x4*>(to) = __builtin_convertvector(sum, bf16x4);
  else *reinterpret_cast<floatx4*>(to) = sum;
}

// Few rows and keys in a unit (bf16): all of it in one workgroup, whose rows, keys and gradients are fetched once and whose scores are
// formed again instead of exchanged.  First the waves take 32 rows each (then the second half of the rows): K and V in LDS, Q and dO in
// registers, which then go to LDS in their place, 128 rows at a time.  64 x 196 tokens to captions of up to 77, 12 heads of 64: 23.1 us (dq
// and dk / dv one by one 18.0 + 16.8), 19 of them without any products: the memory phases of one round of workgroups.  With those the waves
// take 32 keys each, two or four waves to a block of keys where there are fewer blocks, whose sums the first adds in order.
constexpr int kShortRows = 256, kShortKeys = 128;
template <int DH>
struct CrossShort {
  static constexpr int RS = Ops<__bf16, DH>::RS, N = (DH / 32) * 16;                           // N: sums of a lane of one gradient
  static __host__ __device__ constexpr int tiles(int rows) { return rows >= 128 ? 4 : (rows + 31) / 32; }
  static constexpr size_t bytes(int rows, int keys) {
    const size_t held = (size_t)2 * 32 * std::max(tiles(rows), tiles(keys)) * RS * sizeof(__bf16);
    // waves that hand over their sums: of two blocks of keys one each, of one up to three
    const int others = tiles(rows) == 1 ? 0 : tiles(rows) <= 3 ? 2 : 3;
    const size_t sums = (size_t)others * N * kWave * sizeof(float);
    return std::max(held, sums);
  }
};

template <int DH>
__global__ void __launch_bounds__(kCrossThreads) __attribute__((amdgpu_waves_per_eu(3))) cross_bwd_short_kernel(const CrossBwd<__bf16> a) {
  using T = __bf16;
  using O = Ops<T, DH>;
  using S = CrossShort<DH>;
  constexpr int DB = DH / 32, KK = DH / 16, CPR = DH / 8, RPP = kCrossThreads / CPR, CPT = kShortKeys / RPP;
  extern __shared__ __attribute__((aligned(16))) unsigned char cross_smem[];
  __shared__ __attribute__((aligned(16))) float lse_s[kShortRows], lse2_s[kShortRows], negD_s[kShortRows];
  __shared__ int far_s[kShortRows / 32];
  const CrossUnit u = cross_unit(a.s);
  if (!u.valid || (u.nq <= 0 && u.held <= 0)) return;
  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, hh = lane >> 5, wave = __builtin_amdgcn_readfirstlane(tid >> 6), G = (int)a.s.G.d;
  const int nq = u.nq, nk = u.nk, row_tiles = (nq + 31) >> 5, key_tiles = (nk + 31) >> 5;
  const long C = (long)a.s.H * DH, head = (long)u.hk * G * DH;
  T* const first = reinterpret_cast<T*>(cross_smem);
  T* const second = first + 32 * max(S::tiles(a.s.most_q * G), S::tiles(a.s.most_k)) * S::RS;
  // ---- K, V on their way to LDS; every wave's rows
  uintx4 kv[2][CPT];
  if (nk > 0) {
#pragma unroll
    for (int t = 0; t < CPT; ++t) {
      const long row = u.k0 + min(tid / CPR + t * RPP, nk - 1);
      const int c = u.hk * DH + tid % CPR * 8;
      kv[0][t] = *reinterpret_cast<const uintx4*>(a.k + row * a.ks + c);
      kv[1][t] = *reinterpret_cast<const uintx4*>(a.v + row * a.vs + c);
    }
  }
  typename O::Row qf, gf;
  float lse = 0.f;
  auto load_rows = [&](int tile) {
    const int rc = min(tile * 32 + l32, nq - 1);
    const uint32_t token = quotient((uint32_t)rc, a.s.G);
    qf = O::row(a.q + u.q0 * a.qs + head + group_row<DH>(a.s.G, rc, a.qs), hh);
    gf = O::row(a.dout + u.q0 * C + head + group_row<DH>(a.s.G, rc, C), hh);
    lse = a.lse[(u.hk * G + (rc - (int)(token * G))) * a.s.stat_stride + u.q0 + token];
  };
  if (wave < row_tiles) load_rows(wave);
  // (places behind the last block of keys: no gradient; while the loads are under way)
  for (int r = key_tiles * 32 + tid / CPR; r < u.held; r += RPP) {
    const int c = u.hk * DH + tid % CPR * 8;
    *reinterpret_cast<bf16x8*>(a.dk + (u.k0 + r) * a.dks + c) = zero_bf16x8();
    *reinterpret_cast<bf16x8*>(a.dv + (u.k0 + r) * a.dvs + c) = zero_bf16x8();
  }
  if (nk > 0) {
#pragma unroll
    for (int t = 0; t < CPT; ++t) {
      const int r = tid / CPR + t * RPP, o = r * S::RS + tid % CPR * 8;
      if (r >= key_tiles * 32) break;
      const bool ok = r < nk;
      *reinterpret_cast<uintx4*>(first + o) = ok ? kv[0][t] : uintx4{0, 0, 0, 0};
      *reinterpret_cast<uintx4*>(second + o) = ok ? kv[1][t] : uintx4{0, 0, 0, 0};
    }
  }
  __syncthreads();
  // ---- as rows
  for (int tile = wave; tile < row_tiles; tile += 4) {
    if (tile != wave) load_rows(tile);
    const int r = tile * 32 + l32;
    const bool ok = r < nq, none = lse == -INFINITY || !ok, far = __ballot(!none && fabsf(lse) >= kFarScore) != 0;
    const float ref = none ? INFINITY : lse, lse2 = ref * kLog2e;
    floatx16 acc[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[d][e] = 0.f;
    // (P of a block of keys, and dP - D on top of what dP starts from)
    auto scores = [&](int kb, float start, floatx16& s, floatx16& dp) {
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        s[e] = 0.f;
        dp[e] = start;
      }
      O::dot(s, O::row(&first[(kb * 32 + l32) * S::RS], hh), qf);
      O::dot(dp, O::row(&second[(kb * 32 + l32) * S::RS], hh), gf);
      if (kb * 32 + 32 > nk) {
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (kb * 32 + acc_row(e, hh) >= nk) s[e] = -INFINITY;
      }
      if (!far) {
#pragma unroll
        for (int e = 0; e < 16; ++e) s[e] = __builtin_amdgcn_exp2f(fmaf(s[e], a.s.c, -lse2));
      } else {
#pragma unroll
        for (int e = 0; e < 16; ++e) s[e] = __builtin_amdgcn_exp2f(fmaf(s[e], a.s.scale, -ref) * kLog2e);
      }
    };
    floatx16 s, dp;
    float D = 0.f;
    for (int kb = 0; kb < key_tiles; ++kb) {
      scores(kb, 0.f, s, dp);
#pragma unroll
      for (int e = 0; e < 16; ++e) D = fmaf(s[e], dp[e], D);
    }
    D = sum_across_halves(D);
    for (int kb = 0; kb < key_tiles; ++kb) {
      scores(kb, -D, s, dp);
#pragma unroll
      for (int e = 0; e < 16; ++e) dp[e] *= s[e];
      O::outer(acc, first, kb, dp, lane);
    }
    O::store(acc, a.s.scale, a.dq + u.q0 * a.dqs + head + group_row<DH>(a.s.G, min(r, nq - 1), a.dqs), ok, hh);
    if (hh == 0) {
      lse_s[r] = ref;
      lse2_s[r] = lse2;
      negD_s[r] = -D;
    }
    if (lane == 0) far_s[tile] = far;
  }
  if (u.held <= 0) return;
  // ---- as keys: parts waves a block of keys
  const int share = key_tiles <= 1 ? 1 : key_tiles == 2 ? 2 : 4, parts = min(4 / share, max(row_tiles, 1)), kb = wave % share, part = wave / share;
  const bool key_live = kb < key_tiles && part < parts;
  typename O::Row kf, vf;
  if (key_live) {
    kf = O::row(&first[(kb * 32 + l32) * S::RS], hh);
    vf = O::row(&second[(kb * 32 + l32) * S::RS], hh);
  }
  floatx16 dka[DB], dva[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int e = 0; e < 16; ++e) dka[d][e] = dva[d][e] = 0.f;
  // (a wave has the rows of one tile in registers: 168 do not hold two beside the rest)
  if (row_tiles > 4) load_rows(wave);
  auto keys_pass = [&](int i) {
    __syncthreads();
    if (wave + 4 * i < row_tiles) {
      const int r = wave * 32 + l32;
      const bool ok = i * 128 + r < nq;
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) {
        *reinterpret_cast<bf16x8*>(&first[r * S::RS + kk * 16 + hh * 8]) = ok ? qf.f[kk] : zero_bf16x8();
        *reinterpret_cast<bf16x8*>(&second[r * S::RS + kk * 16 + hh * 8]) = ok ? gf.f[kk] : zero_bf16x8();
      }
    }
    __syncthreads();
    if (key_live)
      for (int t = 4 * i + part; t < min(4 * i + 4, row_tiles); t += parts) {
        floatx16 s, dp;
#pragma unroll
        for (int e = 0; e < 16; ++e) s[e] = 0.f;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const floatx4 d4 = *reinterpret_cast<const floatx4*>(&negD_s[t * 32 + 8 * g + 4 * hh]);
#pragma unroll
          for (int e = 0; e < 4; ++e) dp[4 * g + e] = d4[e];
        }
        O::dot(s, O::row(&first[((t & 3) * 32 + l32) * S::RS], hh), kf);
        O::dot(dp, O::row(&second[((t & 3) * 32 + l32) * S::RS], hh), vf);
        if (__builtin_amdgcn_readfirstlane(far_s[t]) == 0) {
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            const floatx4 l4 = *reinterpret_cast<const floatx4*>(&lse2_s[t * 32 + 8 * g + 4 * hh]);
#pragma unroll
            for (int e = 0; e < 4; ++e) s[4 * g + e] = __builtin_amdgcn_exp2f(fmaf(s[4 * g + e], a.s.c, -l4[e]));
          }
        } else {
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            const floatx4 l4 = *reinterpret_cast<const floatx4*>(&lse_s[t * 32 + 8 * g + 4 * hh]);
#pragma unroll
            for (int e = 0; e < 4; ++e) s[4 * g + e] = __builtin_amdgcn_exp2f(fmaf(s[4 * g + e], a.s.scale, -l4[e]) * kLog2e);
          }
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) dp[e] *= s[e];
        O::outer(dva, second, t & 3, s, lane);
        O::outer(dka, first, t & 3, dp, lane);
      }
  };
  keys_pass(0);
  if (row_tiles > 4) {
    load_rows(wave + 4);
    keys_pass(1);
  }
  if (parts > 1) {
    float* const sums = reinterpret_cast<float*>(cross_smem) + lane;
    auto join = [&](floatx16 (&x)[DB]) {
      __syncthreads();
      if (key_live && part > 0) {
        float* mine = sums + ((part - 1) * share + kb) * S::N * kWave;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
          for (int e = 0; e < 16; ++e) mine[(d * 16 + e) * kWave] = x[d][e];
      }
      __syncthreads();
      if (key_live && part == 0)
        for (int p = 0; p < parts - 1; ++p) {
          const float* other = sums + (p * share + kb) * S::N * kWave;
#pragma unroll
          for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int e = 0; e < 16; ++e) x[d][e] += other[(d * 16 + e) * kWave];
        }
    };
    join(dka);
    join(dva);
  }
  if (key_live && part == 0) {
    const int ki = kb * 32 + l32;
    if (ki >= nk) {                                             // places without a key: no gradient
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e) dka[d][e] = dva[d][e] = 0.f;
    }
    const long row = u.k0 + min(ki, u.held - 1);
    O::store(dka, a.s.scale, a.dk + row * a.dks + u.hk * DH, ki < u.held, hh);
    O::store(dva, 1.0f, a.dv + row * a.dvs + u.hk * DH, ki < u.held, hh);
  }
}

// ------------------------------------------------------------------------------- host
static CrossPlan dq_plan(int B, int max_q, int max_k, int H, int Hk, int dtype) { return cross_plan((long)B * Hk, (long)max_q * (H / Hk), max_k, dtype); }
static CrossPlan dkdv_plan(int B, int max_q, int max_k, int H, int Hk, int dtype) { return cross_plan((long)B * Hk, max_k, (long)max_q * (H / Hk), dtype); }

template <typename T, int DH, int KW, bool KEYS>
static int launch_bwd(const char* fn, const CrossBwd<T>& a, hipStream_t st) {
  constexpr size_t lds = KEYS ? sizeof(CrossKeyTiles<T, DH, KW>) : sizeof(CrossDqTiles<T, DH, KW>);
  const auto kernel = KEYS ? cross_dkdv_kernel<T, DH, KW> : cross_dq_kernel<T, DH, KW>;
  const hipError_t attr = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
  SPA_REQUIRE(attr == hipSuccess, SPA_ERR_HIP, "%s: cannot reserve %zu bytes of LDS", fn, lds);
  hipLaunchKernelGGL(kernel, dim3((unsigned)cross_grid(a.s)), dim3(kCrossThreads), lds, st, a);
  if (a.part != nullptr) {
    constexpr int which = KEYS ? 2 : 1, rows = kCrossThreads / (which * DH / 4);
    const long blocks = (long)a.s.B * a.s.Hk * ((a.part_rows + rows - 1) / rows);
    hipLaunchKernelGGL((cross_sum_kernel<T, DH, CrossSteps<KW>::STEP, which>), dim3((unsigned)blocks), dim3(kCrossThreads), 0, st, a);
  }
  return check_launch(fn);
}

// A unit's rows and keys fit one workgroup, and there are units for every compute unit, or few products in each: else dq and dk / dv are
// sooner formed beside each other by more workgroups.  us, one workgroup a unit | two launches, heads of 64: 6 units of 196 rows and 77
// keys 16.8 | 14.7, 96 15.6 | 14.9, 160 to 256 17.0 to 17.5 | 17.0 to 17.4 (a tie, 192 17.3 | 17.1), 288 18.4 | 20.3, 384 21.1 | 24.5, 768
// 26.3 | 39.3; 96 of 256 and 128 20.5 | 17.7, 192 21.3 | 20.6, 256 21.9 | 21.6, 288 22.2 | 26.0, 1536 56.2 | 78.9; 12 of 30 and 20 6.2 |
// 11.3, 768 of 60 and 77 14.4 | 23.9.
// Units of up to 128 rows and more than 8192 products are faster in one workgroup below 256 units, too (64 of 128 and 128 12.2 | 15.2); the
// rule, which decides how D is formed and with it the bits, leaves them.
static bool cross_short(long units, int max_q, int max_k, int G, int dtype) {
  const long rows = (long)max_q * G;
  return dtype == SPA_BF16 && rows <= kShortRows && max_k <= kShortKeys && (units >= 256 || rows * max_k <= 8192);
}

template <int DH>
static int launch_short(const char* fn, const CrossBwd<__bf16>& a, hipStream_t st) {
  const size_t lds = CrossShort<DH>::bytes(a.s.most_q * (int)a.s.G.d, a.s.most_k);
  const auto kernel = cross_bwd_short_kernel<DH>;
  const hipError_t attr = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize,
                                              (int)CrossShort<DH>::bytes(kShortRows, kShortKeys));
  SPA_REQUIRE(attr == hipSuccess, SPA_ERR_HIP, "%s: cannot reserve %zu bytes of LDS", fn, lds);
  hipLaunchKernelGGL(kernel, dim3((unsigned)cross_grid(a.s)), dim3(kCrossThreads), lds, st, a);
  return check_launch(fn);
}

struct CrossGrads {
  const void *out, *dout;
  const float* lse;
  void *dq, *dk, *dv;
  int64_t dqs, dks, dvs;
};

template <typename T>
static int run_bwd(const char* fn, const CrossCall& c, const CrossGrads& g, void* ws, hipStream_t st) {
  if constexpr (sizeof(T) == 2)
    if (cross_short((long)c.B * c.Hk, c.max_q, c.max_k, c.H / c.Hk, c.dtype)) {
      const CrossBwd<T> a = {(const T*)c.q, (const T*)c.k, (const T*)c.v, (const T*)g.out, (const T*)g.dout, (long)c.qs, (long)c.ks, (long)c.vs,
                             cross_shape(c, {1, 1, 1}), g.lse, nullptr, (T*)g.dq, (T*)g.dk, (T*)g.dv, (long)g.dqs, (long)g.dks, (long)g.dvs, nullptr, 0};
      return c.Dh == 32 ? launch_short<32>(fn, a, st) : launch_short<64>(fn, a, st);
    }
  const CrossPlan plans[2] = {dq_plan(c.B, c.max_q, c.max_k, c.H, c.Hk, c.dtype), dkdv_plan(c.B, c.max_q, c.max_k, c.H, c.Hk, c.dtype)};
  float* D = (float*)ws;
  float* part = (float*)((char*)ws + cross_up((size_t)c.H * c.B * c.max_q * sizeof(float)));
  for (int keys = 0; keys < 2; ++keys) {
    const CrossPlan& p = plans[keys];
    CrossBwd<T> a = {(const T*)c.q, (const T*)c.k, (const T*)c.v, (const T*)g.out, (const T*)g.dout, (long)c.qs, (long)c.ks, (long)c.vs,
                     cross_shape(c, p), g.lse, D, (T*)g.dq, (T*)g.dk, (T*)g.dv, (long)g.dqs, (long)g.dks, (long)g.dvs, nullptr, 0};
    if (p.splits > 1) {
      a.part = part;                                          // (dq's are added before dk's and dv's are written)
      a.part_rows = keys ? c.max_k : (long)c.max_q * (c.H / c.Hk);
    }
#define SPA_KW(D_, K_) \
  p.kw == 1 ? launch_bwd<T, D_, 1, K_>(fn, a, st) : p.kw == 2 ? launch_bwd<T, D_, 2, K_>(fn, a, st) : launch_bwd<T, D_, 4, K_>(fn, a, st)
    const int rc = c.Dh == 32 ? (keys ? SPA_KW(32, true) : SPA_KW(32, false)) : (keys ? SPA_KW(64, true) : SPA_KW(64, false));
#undef SPA_KW
    if (rc != SPA_OK) return rc;
  }
  return SPA_OK;
}

}  // namespace spa

using namespace spa;

extern "C" size_t spa_cross_attention_bwd_workspace_bytes(int B, int max_q, int max_k, int H, int Hk, int Dh, int dtype) {
  if (!cross_sizes_ok(B, max_q, max_k, H, Hk, Dh, dtype)) return 0;
  const CrossPlan q = dq_plan(B, max_q, max_k, H, Hk, dtype), k = dkdv_plan(B, max_q, max_k, H, Hk, dtype);
  const size_t rows_q = q.splits > 1 ? (size_t)B * max_q * H * q.splits : 0, rows_k = k.splits > 1 ? (size_t)B * max_k * Hk * k.splits * 2 : 0;
  return cross_up((size_t)H * B * max_q * sizeof(float)) + cross_up(std::max(rows_q, rows_k) * Dh * sizeof(float));
}

extern "C" int spa_cross_attention_bwd(const void* q, const void* k, const void* v, int64_t q_row_stride, int64_t k_row_stride,
                                       int64_t v_row_stride, const void* out, const void* dout, const float* lse, const int32_t* cu_seqlens_q,
                                       const int32_t* cu_seqlens_k, const int32_t* key_lens, int B, int max_q, int max_k, int H, int Hk, int Dh,
                                       int dtype, float softmax_scale, void* dq, void* dk, void* dv, int64_t dq_row_stride,
                                       int64_t dk_row_stride, int64_t dv_row_stride, void* workspace, size_t workspace_bytes, void* stream) {
  const char* fn = "spa_cross_attention_bwd";
  const CrossCall c = {q, k, v, q_row_stride, k_row_stride, v_row_stride, cu_seqlens_q, cu_seqlens_k, key_lens, B, max_q, max_k, H, Hk, Dh, dtype,
                       softmax_scale};
  if (int rc = cross_checks(fn, c)) return rc;
  SPA_REQUIRE(out && dout && lse && dq && dk && dv, SPA_ERR_INVALID_ARG, "%s: null pointer", fn);
  const int64_t strides[3] = {dq_row_stride, dk_row_stride, dv_row_stride};
  for (int i = 0; i < 3; ++i) {
    SPA_REQUIRE(strides[i] >= (int64_t)(i == 0 ? H : Hk) * Dh && strides[i] < (1LL << 31), SPA_ERR_INVALID_ARG, "%s: row stride %ld out of range", fn,
                (long)strides[i]);
    SPA_REQUIRE(strides[i] * elem_size(dtype) % 16 == 0, SPA_ERR_INVALID_ARG, "%s: row stride is not a multiple of 16 bytes", fn);
  }
  SPA_REQUIRE(aligned16(out) && aligned16(dout) && aligned16(dq) && aligned16(dk) && aligned16(dv), SPA_ERR_INVALID_ARG,
              "%s: tensors not 16-byte aligned", fn);
  for (const CrossPlan& p : {dq_plan(B, max_q, max_k, H, Hk, dtype), dkdv_plan(B, max_q, max_k, H, Hk, dtype)})
    SPA_REQUIRE(((long)Hk * B + 8) * p.blocks * p.splits < 4294967296L / kCrossThreads, SPA_ERR_INVALID_ARG,
                "%s: too many workgroups (B*max_q*H must be < about 2^31)", fn);
  const size_t need = spa_cross_attention_bwd_workspace_bytes(B, max_q, max_k, H, Hk, Dh, dtype);
  SPA_REQUIRE(workspace != nullptr && workspace_bytes >= need, SPA_ERR_WORKSPACE, "%s: workspace of %zu bytes needed, %zu given", fn, need,
              workspace_bytes);
  SPA_REQUIRE((reinterpret_cast<uintptr_t>(workspace) & 255u) == 0, SPA_ERR_INVALID_ARG, "%s: workspace not 256-byte aligned", fn);
  const CrossGrads g = {out, dout, lse, dq, dk, dv, dq_row_stride, dk_row_stride, dv_row_stride};
  return dtype == SPA_F32 ? run_bwd<float>(fn, c, g, workspace, as_stream(stream)) : run_bwd<__bf16>(fn, c, g, workspace, as_stream(stream));
}
