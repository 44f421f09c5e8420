// Backward of the packed attention with a relative position bias (attention_bias.hip): beside dQ, dK, dV of the attention without one
//   dtable[h, b] = sum over the pairs of bucket b of dS_ij,  dS = P (dP - D)
// D from the rounded out is off by a share of that rounding; sum_j dS_ij = sum_j P_ij dP_ij - D_i is what it is off by, and is added to
// the D that dK and dtable are formed with.  dQ is formed while that sum is and keeps the first D, as in the attention without a bias;
// rows of one block of 32 keys have the sum in time.  The order in which the many dS of an offset are added would be the launch's, so
// they are added as integers: dS is rounded to a multiple of 2^-40 (kDsBits) of a power of two above every |dS| of the head.  Sums are then
// the same in any order, and finer than fp32 ones.
// P = exp(S - lse) adds up to 1 as long as lse holds its own logarithm beside the maximum.  Beside a mask it does not (at -1e9 its last place
// is 64, and a row of n such keys has log n to add): for rows of |lse| >= kFarScore the dq launch adds up exp(S - lse), at most e^17
// either way, divides by the sum at its end and leaves the logarithm of it for the other launch's exponent.
//
// Two launches and the sums behind them.  The dq launch walks the keys for 128 queries a workgroup, as the forward does, and leaves
// what the second launch needs: the corrected D of every row, and for every block of queries a number that no |dS| of its
// rows exceeds in that launch.  The dk / dv launch walks the queries for 128 (or 192) keys, S and dP un-transposed (a lane is a key), so that P
// and dS are operands in registers again.  There dS goes into a histogram over the offsets in LDS, 64-bit integers: 32 lanes
// hold 32 keys against one query, so that the lanes of an instruction have offsets of their own.  A workgroup keeps its
// histogram over all the blocks it takes, of one head, and writes it once, as fp32; the sum over the workgroups has a fixed order.
// Maps with more offsets than LDS has room for are taken in slices: the first pass over the blocks does everything but the offsets of
// later slices, the others only go over the tiles that have offsets in theirs.
#include <algorithm>
#include <cfloat>
#include <cmath>

#include "attn_bias.h"

namespace spa {

// Bits of an integer dS below the power of two that is above twice every |dS|: one is below 2^(bits - 1), and as many as a workgroup can
// meet at one offset (rows at the same place all meet at the middle one: its rows of keys times the longest segment) stay inside
// 64 bits.  40 for up to 2^24 pairs, a bit less for every doubling beyond.
constexpr int kDsBits = 40;
inline int ds_bits(double pairs) { return std::min(kDsBits, 63 - std::ilogb(pairs)); }
__device__ __forceinline__ double power_of_two(int e) { return __builtin_bit_cast(double, (uint64_t)(e + 1023) << 52); }
// x factor, a power of two, rounded to an integer: the low bits of the sum with 1.5 2^52, whose own bits are taken off again
__device__ __forceinline__ unsigned long long ds_integer(float x, double factor) {
  const double magic = 6755399441055744.0;
  return __builtin_bit_cast(uint64_t, fma((double)x, factor, magic)) - __builtin_bit_cast(uint64_t, magic);
}

template <typename T>
struct BiasBwd {
  const T *q, *k, *v, *out, *dout;
  long qs, ks, vs;
  const float* lse;
  floatx2* dvec;                  // [H][lse_stride]: D, log2 of what exp(S - lse) of the row adds up to (far rows, else 0)
  long lse_stride;
  const int32_t* cu;
  BiasMap m;
  int H, B, nblk;                 // nblk: blocks of kBiasRows rows of the longest possible segment
  float scale;
  T *dq, *dk, *dv;
  long dqs, dks, dvs;
  uint32_t* most;                 // [H][B * nblk]: what no |dS| of a block of queries exceeds
  float* partial;                 // [H][groups][offsets] or null
  int key_blocks, groups, slice;  // dk / dv: blocks of keys of the longest possible segment, workgroups a head, offsets of a histogram
  int bits;                       // of an integer dS
};

// The dq launch: bound by the vector instructions like the forward (0.63 of the busy units' cycles at 16 images of 0.1 to 0.6 of 3136
// tokens, 3 heads of 32, three waves a SIMD by registers and LDS), 49 us there; 27 at 64 images of 196, 12 heads of 64.  A block of eight
// waves holds no more waves a unit, so only few blocks get it.  (Two waves a SIMD at least are named for heads of 32, which their registers
// allow in any case: left to itself the compiler orders the same loop so that it takes 58 us.)
template <typename T, int DH, int WIN, int SPLIT>
__global__ void __launch_bounds__(kBiasThreads * SPLIT, DH == 32 ? 2 : 1) attn_bias_dq_kernel(const BiasBwd<T> a) {
  using O = Ops<T, DH>;
  constexpr int DB = DH / 32, WAVES = 4 * SPLIT;
  extern __shared__ __attribute__((aligned(16))) char win[];
  __shared__ QueryTiles<T, DH, SPLIT> l;
  __shared__ float s_most[2][WAVES];
  const BiasBlock blk = bias_block(l.s_live, a.cu, a.H, a.B, a.nblk);
  if (!blk.valid) return;
  const int h = blk.h, n = blk.seg.nk, lane = threadIdx.x & 63, l32 = lane & 31, hh = lane >> 5, wv = (threadIdx.x >> 6) & 3;
  const int part = SPLIT > 1 ? threadIdx.x >> 8 : 0, qi = blk.r0 + wv * 32 + l32;
  const bool wave_live = blk.r0 + wv * 32 < n, q_ok = qi < n;
  const long C = (long)a.H * DH, q_row = blk.seg.row0 + min(qi, n - 1);
  typename O::Row qf, gf, of;
  float D = 0.f, l1 = 0.f;                                    // <dO, out> and sum |dO| of the lane's row
  floatx16 acc[DB], negD;
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[d][r] = 0.f;
  const float lse = a.lse[h * a.lse_stride + q_row];
  const bool none = lse == -INFINITY || !q_ok;                // no score, or no row: probability 0
  const bool far_row = !none && fabsf(lse) >= kFarScore, far = __ballot(far_row) != 0;
  const float lse2 = none ? INFINITY : lse * kLog2e;
  float left = 0.f, most = 0.f, v_most = 0.f, all = 0.f;      // sum and largest magnitude of the row's dS; largest |V|; sum of P
  walk_keys<T, DH, WIN, SPLIT>(
      l, win, blk.seg, h, wave_live, a.k, a.ks, a.v, a.vs, a.m, a.cu, qi,
      [&] {
        qf = O::row(a.q + q_row * a.qs + h * DH, hh);
        gf = O::row(a.dout + q_row * C + h * DH, hh);
        of = O::row(a.out + q_row * C + h * DH, hh);
      },
      [&] {
        O::sums(gf, of, D, l1);
        D = sum_across_halves(D);
        l1 = sum_across_halves(l1);
#pragma unroll
        for (int r = 0; r < 16; ++r) negD[r] = -D;
      },
      [&](const auto& st) { v_most = st.most(v_most); },
      [&](const T* K, const T* V, const int* pos, int rows, int own, int zero, bool in_window, auto whole) {
#pragma unroll
        for (int sb = 0; sb < 2; ++sb) {
          if (!whole && sb * 32 >= rows) break;
          floatx16 s, dp = negD;
          const typename O::Row kr = O::row(&K[(sb * 32 + l32) * O::RS], hh), vr = O::row(&V[(sb * 32 + l32) * O::RS], hh);
          bias_scores<T, DH, WIN, 1>(s, kr, qf, &pos[sb * 32], own, zero, in_window, a.m, h, a.scale, hh);
          O::dot(dp, vr, gf);
          if (!whole) {
#pragma unroll
            for (int r = 0; r < 16; ++r)
              if (sb * 32 + acc_row(r, hh) >= rows) s[r] = -INFINITY;
          }
          if (!far) {
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], kLog2e, -lse2));
          } else {
            const float ref = none ? INFINITY : lse;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
              s[r] = __builtin_amdgcn_exp2f((s[r] - ref) * kLog2e);
              all += s[r];
            }
          }
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            dp[r] *= s[r];
            left += dp[r];
            most = __builtin_elementwise_maximum(most, fabsf(dp[r]));
          }
          if (!whole && n <= 32) {                            // the whole row is here: what its dS add up to off them as well
            float off = sum_across_halves(left);
            if (far) off = far_row ? off / sum_across_halves(all) : off;
#pragma unroll
            for (int r = 0; r < 16; ++r) dp[r] = fmaf(-off, s[r], dp[r]);
          }
          O::outer(acc, K, sb, dp, lane);
        }
      });
  v_most = __builtin_bit_cast(float, wave_pick<true>((int)(__builtin_bit_cast(uint32_t, v_most) & 0x7fffffffu)));
  if (lane == 0) s_most[0][threadIdx.x >> 6] = v_most;
  __syncthreads();
  if constexpr (SPLIT > 1) {
    constexpr int W = DB * 16 + 3;
    static_assert(4 * W * kWave * sizeof(float) <= sizeof(l.K), "the sums of four waves");
    float* other = reinterpret_cast<float*>(&l.K[0][0]) + wv * W * kWave + lane;
    if (part == 1) {
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) other[(d * 16 + r) * kWave] = acc[d][r];
      other[(W - 3) * kWave] = left;
      other[(W - 2) * kWave] = most;
      other[(W - 1) * kWave] = all;
    }
    __syncthreads();
    if (part == 0) {
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[d][r] += other[(d * 16 + r) * kWave];
      left += other[(W - 3) * kWave];
      most = __builtin_elementwise_maximum(most, other[(W - 2) * kWave]);
      all += other[(W - 1) * kWave];
    }
  }
  all = sum_across_halves(all);
  const float inv = far_row ? 1.0f / all : 1.f;
  left = sum_across_halves(left) * inv;
  most *= inv;
  if (part == 0) {
    O::store(acc, a.scale * inv, a.dq + q_row * a.dqs + h * DH, q_ok, hh);
    if (q_ok && hh == 0) a.dvec[h * a.lse_stride + q_row] = floatx2{D + left, far_row ? log2f(all) : 0.f};
  }
  // |dS| of the other launch: of this one, plus what D moves by, plus what the order of Dh products in dP can make (at most
  // Dh U sum|dO V| in either launch)
#pragma unroll
  for (int w = 0; w < WAVES; ++w) v_most = __builtin_elementwise_maximum(v_most, s_most[0][w]);
  const float more = fabsf(left) + l1 * 0x1p-16f * v_most;
  float bound = q_ok && part == 0 ? most + more : 0.f;
  if (bound == INFINITY && most < INFINITY && more < INFINITY) bound = FLT_MAX;               // (every |dS| is a finite number)
  const int bits = wave_pick<true>((int)(__builtin_bit_cast(uint32_t, bound) & 0x7fffffffu));      // (a NaN above all)
  if (lane == 0) s_most[1][threadIdx.x >> 6] = __builtin_bit_cast(float, bits);
  __syncthreads();
  if (threadIdx.x == 0) {
    uint32_t all = 0;
#pragma unroll
    for (int w = 0; w < 4; ++w) all = max(all, __builtin_bit_cast(uint32_t, s_most[1][w]));
    a.most[((long)h * a.B + blk.img) * a.nblk + blk.r0 / kBiasRows] = all;
  }
}

// What becomes of dS by offset: nothing, a histogram of all offsets of the map in LDS, or one slice of them after the other.
enum HistMode { kHistNone, kHistWhole, kHistSlices };

// The head's blocks of keys in the order in which the workgroups take them: up to 256 segments by length, longest first,
// blocks that exist numbered through; more segments in index order, with blocks of the longest possible one each.
struct KeyBlocks {
  int from[kLptMaxB], len[kLptMaxB], upto[kLptMaxB];          // by rank: first row, rows, blocks up to and including the rank's
  int all;
};
template <int THREADS>
__device__ __forceinline__ void list_key_blocks(KeyBlocks& k, const int32_t* cu, int B, int rows, int kblk) {
  if (B > kLptMaxB) {
    if (threadIdx.x == 0) k.all = B * kblk;
    __syncthreads();
    return;
  }
  for (int b = threadIdx.x; b < B; b += THREADS) k.upto[b] = max(cu[b + 1] - cu[b], 0);
  __syncthreads();
  for (int b = threadIdx.x; b < B; b += THREADS) {
    const int mine = k.upto[b];
    int rank = 0;
#pragma unroll 8
    for (int i = 0; i < B; ++i) {
      const int other = k.upto[i];
      rank += (other > mine) | ((other == mine) & (i < b));
    }
    k.from[rank] = cu[b];
    k.len[rank] = mine;
  }
  __syncthreads();
  if (threadIdx.x < kWave) {
    int before = 0;
    for (int r0 = 0; r0 < B; r0 += kWave) {
      const int r = r0 + threadIdx.x, nb = r < B ? min((k.len[r] + rows - 1) / rows, kblk) : 0, to = before + wave_scan(nb);
      if (r < B) k.upto[r] = to;
      before = __builtin_amdgcn_readlane(to, 63);
    }
    if (threadIdx.x == 0) k.all = before;
  }
  __syncthreads();
}
struct KeyBlock {
  long row0;
  int n, k0;
};
__device__ __forceinline__ KeyBlock key_block(const KeyBlocks& k, const int32_t* cu, int B, int rows, int kblk, int i) {
  if (B > kLptMaxB) {
    const int img = i / kblk, from = cu[img];
    return {from, cu[img + 1] - from, i % kblk * rows};
  }
  int rank = 0, at = i;                                       // the first rank with upto > i
  for (int r0 = 0; r0 < B; r0 += kWave) {
    const int r = r0 + (threadIdx.x & (kWave - 1)), upto = r < B ? k.upto[r] : 0x7fffffff;
    const int before = __popcll(__ballot(upto <= i));
    if (before > 0) at = i - __builtin_amdgcn_readlane(upto, before - 1);
    rank += before;
    if (before < kWave) break;
  }
  return {__builtin_amdgcn_readfirstlane(k.from[rank]), __builtin_amdgcn_readfirstlane(k.len[rank]), at * rows};
}

// The scale of a head's integers: 2^e is above twice what the dq launch found (its blocks that exist); `unit` NaN: some dS of
// the head is not a finite number.  All threads call it.
struct DsScale {
  double quantum, factor;         // what an integer stands for, and its reciprocal (0: see unit)
  float unit;
};
template <int THREADS>
__device__ __forceinline__ DsScale ds_scale(const uint32_t* most_h, const int32_t* cu, int B, int nblk, int bits, uint32_t* s_most) {
  uint32_t most = 0;
  for (int i = threadIdx.x; i < B * nblk; i += THREADS) {
    const int img = i / nblk, n = cu[img + 1] - cu[img];
    const uint32_t its = most_h[i];
    if ((i - img * nblk) * kBiasRows < n) most = max(most, its);
  }
  most = (uint32_t)wave_pick<true>((int)most);
  if ((threadIdx.x & 63) == 0) s_most[threadIdx.x >> 6] = most;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < THREADS / kWave; ++w) most = max(most, s_most[w]);
  const int e = __builtin_amdgcn_readfirstlane((int)(most >> 23) - 126 + 1);
  const bool bad = most >= 0x7f800000u;
  return {power_of_two(e - bits), bad ? 0. : power_of_two(bits - e), bad ? NAN : 0.f};
}
// A workgroup's histogram of `size` offsets of its head from `from` on, around the end, as fp32; all threads call it, behind the last add.
template <int THREADS>
__device__ __forceinline__ void write_partial(const unsigned long long* hist, const DsScale& s, int size, int from, int offsets, float* out) {
  __syncthreads();
  for (int i = threadIdx.x; i < size; i += THREADS)
    out[from + i - (from + i < offsets ? 0 : offsets)] = s.unit + (float)((double)(long long)hist[i] * s.quantum);
  __syncthreads();
}

constexpr int kLaterBlocks = 32;                // blocks of a workgroup whose tiles the later slices need are kept
template <typename T, int DH, int RW, int SPLIT>
struct KeyTiles {
  static constexpr int RS = Ops<T, DH>::RS;
  __attribute__((aligned(16))) T Q[2][kBiasBN * RS];
  __attribute__((aligned(16))) T G[2][kBiasBN * RS];          // dO
  __attribute__((aligned(16))) float lse[2][kBiasBN];         // +inf: no score, or no row (probability 0)
  __attribute__((aligned(16))) float lse2[2][kBiasBN];        // times log2 e; of a tile with far rows: log2 of the sums of their P
  __attribute__((aligned(16))) float negD[2][kBiasBN];
  __attribute__((aligned(16))) int pos[2][kBiasBN];
  int range[2][1][2], far[2];
  int own[RW][2];
  uint32_t most[RW * SPLIT];
  typename WindowFill<T, kBiasThreads>::Raw row[kTableLds];
  unsigned long long later[kLaterBlocks];
  KeyBlocks blocks;
};

// RW waves own 32 keys each.  SPLIT 2: the waves come twice, the second ones take the second half of every tile of 64 queries, and hand
// their sums to the first at the end of a block.  Bound by latency and LDS together: a block's chain (look-ups, products, exponentials,
// products, 16 atomic adds) runs on two or three waves a SIMD, LDS is busy 0.54 of the time (half of it the adds, for the offsets of
// a wave's keys meet in banks).  us: 75 at 16 images of 0.1 to 0.6 of 3136 tokens, 3 heads of 32; 31 at 64 of 196, 12 heads of 64.
template <typename T, int DH, int WIN, int RW, int SPLIT, int HIST>
__global__ void __launch_bounds__(kWave * RW * SPLIT) attn_bias_dkdv_kernel(const BiasBwd<T> a) {
  using O = Ops<T, DH>;
  constexpr int RS = O::RS, DB = DH / 32, BN = kBiasBN, THREADS = kWave * RW * SPLIT, ROWS = 32 * RW, WB = sizeof(T);
  constexpr bool RANGES = WIN == kWinMoving || HIST == kHistSlices;                // the offsets of a tile lie where?
  extern __shared__ __attribute__((aligned(16))) unsigned long long hist[];        // [slice], then the window
  __shared__ KeyTiles<T, DH, RW, SPLIT> l;
  const int h = blockIdx.x % a.H, group = blockIdx.x / a.H;
  const int tid = threadIdx.x, lane = tid & 63, wv = (tid >> 6) % RW, l32 = lane & 31, hh = lane >> 5;
  const int part = SPLIT > 1 ? __builtin_amdgcn_readfirstlane(tid / (kWave * RW)) : 0;
  const bool stages = tid < kBiasThreads;                     // (the first four waves)
  const long C = (long)a.H * DH;
  void* win = hist + (HIST != kHistNone ? a.slice : 0);
  const float* lse_h = a.lse + h * a.lse_stride;
  const floatx2* d_h = a.dvec + h * a.lse_stride;

  WindowFill<T, THREADS> fill(a.m, h);
  if (WIN == kWinWhole) fill.start(0, a.m.offsets);
  list_key_blocks<THREADS>(l.blocks, a.cu, a.B, ROWS, a.key_blocks);
  DsScale scale = {0., 0., 0.f};
  if (HIST != kHistNone) scale = ds_scale<THREADS>(a.most + (long)h * a.B * a.nblk, a.cu, a.B, a.nblk, a.bits, l.most);
  int zero = 0;
  if (WIN == kWinWhole) zero = fill.finish(win, l.row);

  const int passes = HIST == kHistSlices ? (a.m.offsets + a.slice - 1) / a.slice : 1;
  for (int pass = 0; pass < passes; ++pass) {
    // slices: the first around the middle, where most pairs are, the others go on from there and around the end
    const int E = a.m.offsets, size = HIST == kHistSlices ? min(a.slice, E - pass * a.slice) : E;
    const int start = (E - a.slice) / 2 + pass * a.slice, from = HIST == kHistSlices ? (start < E ? start : start - E) : 0;
    if (HIST != kHistNone) {
      for (int i = tid; i < a.slice; i += THREADS) hist[i] = 0;
      // (in front of the first add there is the barrier behind a block's first tile)
    }
    for (int round = 0;; ++round) {
      // there and back, so that every workgroup has long and short blocks
      const int item = round * a.groups + (round & 1 ? a.groups - 1 - group : group);
      if (item >= l.blocks.all) break;
      const KeyBlock kb = key_block(l.blocks, a.cu, a.B, ROWS, a.key_blocks, item);
      if (kb.k0 >= kb.n) continue;
      const int n = kb.n, last = n - 1, ki = kb.k0 + wv * 32 + l32, nt = (n + BN - 1) / BN;
      const bool wave_live = kb.k0 + wv * 32 < n, k_ok = ki < n;
      // which tiles the first pass left something of (one bit each; longer segments and later blocks: any)
      const bool listed = HIST == kHistSlices && nt <= 64 && round < kLaterBlocks;
      unsigned long long todo = ~0ull;
      if (listed && pass > 0) {
        todo = l.later[round];
        todo = (unsigned long long)(uint32_t)__builtin_amdgcn_readfirstlane((int)(todo >> 32)) << 32 |
               (uint32_t)__builtin_amdgcn_readfirstlane((int)todo);
        if (todo == 0) continue;
      }
      auto next_tile = [&](int t) -> int {
        if (HIST != kHistSlices || !listed || pass == 0) return t + 1;
        const unsigned long long rest = t < 0 ? todo : todo & ~((2ull << t) - 1);
        return rest != 0 ? __builtin_ctzll(rest) : nt;
      };
      unsigned long long left_over = 0;
      const long k_row = kb.row0 + min(ki, last);
      RowPair<T, DH, kBiasThreads, BN> st(tid, a.q + h * DH, a.qs, a.dout + h * DH, C, kb.row0, last);
      const BiasTokens tokens(a.m, a.cu, kb.row0);
      int token = 0, token_j = 0;
      float lse_t = 0.f;
      floatx2 d_t = {0.f, 0.f};
      auto load_tile = [&](int qt) {
        if (stages) st.load(qt);
        token_j = min(qt + lane, last);
        token = tokens.load(token_j);
        lse_t = lse_h[kb.row0 + token_j];
        d_t = d_h[kb.row0 + token_j];
      };
      auto store_tile = [&](int buf, int qt, auto clear) {
        if (stages) st.template store<clear>(l.Q[buf], l.G[buf]);
        if (tid < BN) {
          const bool none = lse_t == -INFINITY || qt + tid >= n;
          const bool any = __ballot(!none && fabsf(lse_t) >= kFarScore) != 0;
          l.lse[buf][tid] = none ? INFINITY : lse_t;
          l.lse2[buf][tid] = any ? d_t[1] : none ? INFINITY : lse_t * kLog2e;
          l.negD[buf][tid] = -d_t[0];
          const int p = tokens.position(a.m, token, token_j) + a.m.centre;
          l.pos[buf][tid] = WB * p;
          if (RANGES) put_range(l.range[buf][0], p);
          if (tid == 0) l.far[buf] = any;
        }
      };
      const int own_token = tokens.load(min(ki, last));
      int t = next_tile(-1);
      load_tile(t * BN);
      const typename O::Row kf = O::row(a.k + k_row * a.ks + h * DH, hh), vf = O::row(a.v + k_row * a.vs + h * DH, hh);
      const int own = tokens.position(a.m, own_token, min(ki, last));
      __syncthreads();                                        // every wave is past its last read of the tiles before
      if (RANGES && part == 0) put_range(l.own[wv], own);
      floatx16 dka[DB], dva[DB];
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) dka[d][r] = dva[d][r] = 0.f;
      store_tile(0, t * BN, std::true_type{});
      __syncthreads();
      const Range mine = RANGES ? whole_range(l.own) : Range{0, 0};
      int base = -0x40000000;
      for (int step = 0; t < nt; ++step) {
        const int buf = (HIST == kHistSlices ? step : t) & 1, qt = t * BN, next = next_tile(t);
        const bool end = next >= nt;
        if (!end) load_tile(next * BN);
        bool in_window = true, adds = HIST != kHistNone, inside = true;
        int wrap = 0;                                         // of the tile's offsets, where they are inside around the end
        if (RANGES) {
          const Range tile = whole_range(l.range[buf]);
          const int lo = tile.lo - mine.hi, hi = tile.hi - mine.lo;
          if (WIN == kWinMoving) {
            in_window = hi - lo < kWindow - 3;
            if (in_window && (lo < base || hi >= base + kWindow)) {   // the queries' positions grow, so do the offsets
              base = lo & ~3;
              fill.start(base, min(kWindow, a.m.offsets - base));
              zero = fill.finish(win, l.row);
              __syncthreads();
            }
          }
          if (HIST == kHistSlices) {
            wrap = hi + E < from + size ? E : 0;
            inside = wrap != 0 || (lo >= from && hi < from + size);
            adds = (hi >= from && lo < from + size) || lo + E < from + size;
            if (!inside && t < 64) left_over |= 1ull << t;
          }
        }
        if (wave_live && (pass == 0 || adds)) {
          const bool far = __builtin_amdgcn_readfirstlane(l.far[buf]) != 0;
#pragma unroll
          for (int half = 0; half < 2 / SPLIT; ++half) {
            const int sb = SPLIT > 1 ? part : half;
            if (qt + sb * 32 >= n) break;
            const int* pos = &l.pos[buf][sb * 32];
            const typename O::Row qr = O::row(&l.Q[buf][(sb * 32 + l32) * RS], hh), gr = O::row(&l.G[buf][(sb * 32 + l32) * RS], hh);
            floatx16 s, dp;
            bias_scores<T, DH, WIN, -1>(s, qr, kf, pos, own, zero, in_window, a.m, h, a.scale, hh);
#pragma unroll
            for (int g = 0; g < 4; ++g) {
              const floatx4 d4 = *reinterpret_cast<const floatx4*>(&l.negD[buf][sb * 32 + 8 * g + 4 * hh]);
#pragma unroll
              for (int i = 0; i < 4; ++i) dp[4 * g + i] = d4[i];
            }
            O::dot(dp, gr, vf);
            if (!far) {
#pragma unroll
              for (int g = 0; g < 4; ++g) {
                const floatx4 l4 = *reinterpret_cast<const floatx4*>(&l.lse2[buf][sb * 32 + 8 * g + 4 * hh]);
#pragma unroll
                for (int i = 0; i < 4; ++i) s[4 * g + i] = __builtin_amdgcn_exp2f(fmaf(s[4 * g + i], kLog2e, -l4[i]));
              }
            } else {
#pragma unroll
              for (int g = 0; g < 4; ++g) {
                const floatx4 l4 = *reinterpret_cast<const floatx4*>(&l.lse[buf][sb * 32 + 8 * g + 4 * hh]);
                const floatx4 a4 = *reinterpret_cast<const floatx4*>(&l.lse2[buf][sb * 32 + 8 * g + 4 * hh]);
#pragma unroll
                for (int i = 0; i < 4; ++i) s[4 * g + i] = __builtin_amdgcn_exp2f(fmaf(s[4 * g + i] - l4[i], kLog2e, -a4[i]));
              }
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) dp[r] *= s[r];
            if (pass == 0) {
              O::outer(dva, l.G[buf], sb, s, lane);
              O::outer(dka, l.Q[buf], sb, dp, lane);
            }
            if (HIST != kHistNone && adds && k_ok) {
              const int to = lds_address(hist) - 8 * (own + from - wrap);
#pragma unroll
              for (int g = 0; g < 4; ++g) {
                const intx4 p = *reinterpret_cast<const intx4*>(&pos[8 * g + 4 * hh]);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                  const unsigned long long v = ds_integer(dp[4 * g + i], scale.factor);
                  if (HIST == kHistWhole || inside) lds_add(p[i] * (8 / WB) + to, v);
                  else if (const int off = p[i] / WB - own - from, at = off + (off < 0 ? E : 0); at < size) lds_add(lds_address(hist) + 8 * at, v);
                }
              }
            }
          }
        }
        if (!end) {
          if (next + 1 == nt) store_tile(buf ^ 1, next * BN, std::true_type{});
          else store_tile(buf ^ 1, next * BN, std::false_type{});
          __syncthreads();
        }
        t = next;
      }
      if (listed && pass == 0 && tid == 0) l.later[round] = left_over;
      if (pass == 0) {
        if constexpr (SPLIT > 1) {
          static_assert(RW * DB * 8 * kWave * sizeof(float) <= sizeof(l.Q) + sizeof(l.G), "half a sum of the waves");
          float* other = reinterpret_cast<float*>(&l.Q[0][0]) + wv * DB * 8 * kWave + lane;
#pragma unroll
          for (int which = 0; which < 4; ++which) {
            floatx16(&sum)[DB] = which < 2 ? dka : dva;
            const int r0 = which & 1 ? 8 : 0;
            __syncthreads();                                  // every wave is past its last read of the tiles, or of the sums before
            if (part == 1) {
#pragma unroll
              for (int d = 0; d < DB; ++d)
#pragma unroll
                for (int r = 0; r < 8; ++r) other[(d * 8 + r) * kWave] = sum[d][r0 + r];
            }
            __syncthreads();
            if (part == 0) {
#pragma unroll
              for (int d = 0; d < DB; ++d)
#pragma unroll
                for (int r = 0; r < 8; ++r) sum[d][r0 + r] += other[(d * 8 + r) * kWave];
            }
          }
        }
        if (part == 0) {
          O::store(dka, a.scale, a.dk + k_row * a.dks + h * DH, k_ok, hh);
          O::store(dva, 1.0f, a.dv + k_row * a.dvs + h * DH, k_ok, hh);
        }
      }
    }
    if (HIST != kHistNone) write_partial<THREADS>(hist, scale, size, from, E, a.partial + ((long)h * a.groups + group) * a.m.offsets);
  }
}

// The sums over the workgroups, in their order: 32 offsets a workgroup, eight slices of the rows beside each other, each with eight
// loads in flight (85 workgroups x 12321 offsets x 3 heads, 12.6 MB: 6.2 us; a row at a time 8.3).
struct BiasSum {
  const float* partial;
  int groups, offsets;
  float* sums;                    // [H][offsets]
};
__global__ void __launch_bounds__(256) attn_bias_sum_kernel(const BiasSum a) {
  constexpr int SL = 8, U = 8;
  __shared__ double s[SL][32];
  const int h = blockIdx.y, c = threadIdx.x & 31, sl = threadIdx.x >> 5, o = blockIdx.x * 32 + c;
  double v = 0.;
  if (o < a.offsets) {
    const float* p = a.partial + (long)h * a.groups * a.offsets + o;
    for (int g0 = sl; g0 < a.groups; g0 += SL * U) {
      float f[U];
#pragma unroll
      for (int u = 0; u < U; ++u) f[u] = g0 + SL * u < a.groups ? p[(long)(g0 + SL * u) * a.offsets] : 0.f;
#pragma unroll
      for (int u = 0; u < U; ++u) v += (double)f[u];
    }
  }
  s[sl][c] = v;
  __syncthreads();
  if (sl == 0 && o < a.offsets) {
    for (int i = 1; i < SL; ++i) v += s[i][c];
    a.sums[(long)h * a.offsets + o] = (float)v;
  }
}

// The sums of the offsets into those of their buckets, with integers again, of 2^-40 of the power of two above the largest: a
// workgroup has kTableBuckets buckets of a head in LDS and goes over all offsets.  Few workgroups on a small map: it
// adds up their sums as well, a launch less (us backward, two launches | one: 2 images of 62 tokens, fp32, 14 x 14 map, 2
// workgroups a head 29.4 | 28.3; 64 images, 42 workgroups a head 62 | 62).
constexpr int kTableBuckets = 2048, kTableSums = 2048;
struct BiasTable {
  const float* sums;              // [H][offsets], or the workgroups' [H][groups][offsets]
  const int32_t* buckets;
  int nb, offsets, groups;
  float* d_table;
};
template <bool ADDS>
__global__ void __launch_bounds__(1024) attn_bias_table_kernel(const BiasTable a) {
  constexpr int U = 8, UG = 16;
  __shared__ unsigned long long s[kTableBuckets];
  __shared__ uint32_t s_most[16];
  __shared__ float s_sums[ADDS ? kTableSums : 1];
  const int h = blockIdx.y, b0 = blockIdx.x * kTableBuckets, nb = min(kTableBuckets, a.nb - b0);
  const float* sums = ADDS ? s_sums : a.sums + (long)h * a.offsets;
  if (ADDS) {
    for (int o = threadIdx.x; o < a.offsets; o += 1024) {
      const float* p = a.sums + (long)h * a.groups * a.offsets + o;
      double v = 0.;
      for (int g0 = 0; g0 < a.groups; g0 += UG) {
        float f[UG];
#pragma unroll
        for (int u = 0; u < UG; ++u) f[u] = p[(long)min(g0 + u, a.groups - 1) * a.offsets];
#pragma unroll
        for (int u = 0; u < UG; ++u) v += g0 + u < a.groups ? (double)f[u] : 0.;
      }
      s_sums[o] = (float)v;
    }
    __syncthreads();
  }
  uint32_t most = 0;
  for (int i0 = threadIdx.x; i0 < a.offsets; i0 += U * 1024) {
    float v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = sums[min(i0 + u * 1024, a.offsets - 1)];
#pragma unroll
    for (int u = 0; u < U; ++u) most = max(most, __builtin_bit_cast(uint32_t, v[u]) & 0x7fffffffu);
  }
  most = (uint32_t)wave_pick<true>((int)most);
  if ((threadIdx.x & 63) == 0) s_most[threadIdx.x >> 6] = most;
  for (int i = threadIdx.x; i < nb; i += 1024) s[i] = 0;
  __syncthreads();
  for (int w = 0; w < 16; ++w) most = max(most, s_most[w]);
  const bool bad = most >= 0x7f800000u;
  const int bits = min(40, 62 - (32 - __builtin_clz(a.offsets))), e = (int)(most >> 23) - 126;
  if (!bad)
    for (int i0 = threadIdx.x; i0 < a.offsets; i0 += U * 1024) {
      int b[U];
      float v[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        b[u] = a.buckets[min(i0 + u * 1024, a.offsets - 1)] - b0;
        v[u] = sums[min(i0 + u * 1024, a.offsets - 1)];
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (i0 + u * 1024 < a.offsets && (unsigned)b[u] < (unsigned)nb && v[u] != 0.f) atomicAdd(&s[b[u]], ds_integer(v[u], power_of_two(bits - e)));
    }
  __syncthreads();
  for (int i = threadIdx.x; i < nb; i += 1024)
    a.d_table[(long)h * a.nb + b0 + i] = bad ? NAN : (float)((double)(long long)s[i] * power_of_two(e - bits));
}

// ------------------------------------------------------------------------------- host
static size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }

// The dk / dv launch.  Two workgroups a unit where that leaves each room for the whole map in LDS; else one, of eight waves in
// bf16, with as much of the histogram as fits.  Few blocks take eight waves there too (us backward, four | eight waves, heads of 32,
// 28 x 28 map: one image of 700 tokens, 8 heads, 47.8 | 41.1, four 50.6 | 43.5).  As many workgroups a head as are resident
// together, no more than there are blocks of keys, and no more than 256 MB of partial sums.
struct BiasPlan {
  bool whole;                     // the window
  int rows, split, key_blocks, slice, groups, bits;   // rows: waves that own keys
  size_t window, lds;
};
// Twelve waves for 192 keys where registers allow and there may be many blocks (of the longest possible segments, all that the host
// knows): us backward, eight | twelve waves, heads of 32, 56 x 56 map, images of 0.1 to 0.6 of 3136 tokens: 3 heads, 8 images (600 blocks)
// 91 | 102, 14 (1050) 106 | 115, 16 (1200) 115.3 | 114.9, 20 151 | 144, 64 350 | 326; 8 heads, 5 images (1000) 72 | 80, 8 (1600) 111 | 106.
template <int DH>
constexpr int kSplitRows = DH == 32 ? 6 : 4;
template <typename T, int DH>
static BiasPlan bias_plan_of(int H, int B, int n_max, long offsets) {
  BiasPlan p = {};
  const size_t most = kUnitLds;
  const long all = (offsets + 63) & ~63L;
  p.whole = offsets <= kWholeBytes / (long)sizeof(T);
  p.window = window_bytes(p.whole ? (int)offsets : kWindow, sizeof(T));
  size_t tiles = sizeof(KeyTiles<T, DH, 4, 1>);
  const bool two = p.whole && tiles + p.window + all * 8 <= most / 2;
  const int nblk = (n_max + kBiasRows - 1) / kBiasRows;
  p.split = sizeof(T) == 2 && p.whole && (!two || few_blocks(nblk, H, B)) ? 2 : 1;
  if (p.split == 2) tiles = sizeof(KeyTiles<T, DH, kSplitRows<DH>, 2>);
  p.slice = (int)std::min<long>(all, (long)(most - tiles - p.window) / 8 / 64 * 64);
  p.lds = p.window + (size_t)p.slice * 8;
  p.rows = p.split == 2 && p.slice == all && (long)H * B * nblk >= 1200 ? kSplitRows<DH> : 4;
  p.key_blocks = (n_max + 32 * p.rows - 1) / (32 * p.rows);
  const long fit = std::max<long>(1, (256L << 20) / (4 * H * offsets));
  p.groups = (int)std::max<long>(1, std::min<long>(std::min<long>((two ? 512 : 256) / H, (long)B * p.key_blocks), fit));
  const long turns = ((long)B * p.key_blocks + p.groups - 1) / p.groups;                 // blocks of keys of a workgroup
  p.bits = ds_bits((double)std::min(turns * 32 * p.rows, (long)B * n_max) * n_max);
  return p;
}
static BiasPlan bias_plan(int H, int B, int n_max, int Dh, long offsets, int dtype) {
  if (dtype == SPA_F32) return Dh == 32 ? bias_plan_of<float, 32>(H, B, n_max, offsets) : bias_plan_of<float, 64>(H, B, n_max, offsets);
  return Dh == 32 ? bias_plan_of<__bf16, 32>(H, B, n_max, offsets) : bias_plan_of<__bf16, 64>(H, B, n_max, offsets);
}

template <typename T, int D>
static int launch_bias_bwd(const char* fn, const BiasBwd<T>& args, const BiasPlan& plan, bool hist, hipStream_t st) {
  const BiasMap& m = args.m;
  const int H = args.H, B = args.B, nblk = args.nblk;
  SPA_QUERY_LAUNCH(attn_bias_dq_kernel, T, D, few_blocks(nblk, H, B), args);
#define SPA_DKDV(WIN, RW, SPLIT, MODE)                                                                                          \
  SPA_BIAS_LAUNCH((attn_bias_dkdv_kernel<T, D, WIN, RW, SPLIT, MODE>), (sizeof(KeyTiles<T, D, RW, SPLIT>)), H * plan.groups,      \
                  SPLIT * RW * kWave, hist ? plan.lds : plan.window, args)
  const bool slices = plan.slice < m.offsets;
  if (!plan.whole) {
    if (!hist) SPA_DKDV(kWinMoving, 4, 1, kHistNone);
    else SPA_DKDV(kWinMoving, 4, 1, kHistSlices);
  } else if (plan.split == 1) {
    if (!hist) SPA_DKDV(kWinWhole, 4, 1, kHistNone);
    else if (!slices) SPA_DKDV(kWinWhole, 4, 1, kHistWhole);
    else if constexpr (sizeof(T) == 4) SPA_DKDV(kWinWhole, 4, 1, kHistSlices);
  } else if constexpr (sizeof(T) == 2) {
    if (hist && slices) SPA_DKDV(kWinWhole, 4, 2, kHistSlices);
    else if (hist && plan.rows == 4) SPA_DKDV(kWinWhole, 4, 2, kHistWhole);
    else if (plan.rows == 4) SPA_DKDV(kWinWhole, 4, 2, kHistNone);
    else if (hist) SPA_DKDV(kWinWhole, kSplitRows<D>, 2, kHistWhole);
    else SPA_DKDV(kWinWhole, kSplitRows<D>, 2, kHistNone);
  }
#undef SPA_DKDV
  return SPA_OK;
}

}  // namespace spa

using namespace spa;

extern "C" size_t spa_attention_bias_bwd_workspace_bytes(int B, int max_seqlen, int H, int Dh, int grid_h, int grid_w, int dtype) {
  if (B < 1 || max_seqlen < 1 || H < 1 || grid_h < 1 || grid_w < 1 || (2 * (long)grid_h - 1) * (2 * (long)grid_w - 1) > kMostOffsets) return 0;
  const long offsets = (2 * (long)grid_h - 1) * (2 * (long)grid_w - 1);
  const int nblk = (max_seqlen + kBiasRows - 1) / kBiasRows;
  const BiasPlan p = bias_plan(H, B, max_seqlen, Dh, offsets, dtype);
  return up256((size_t)H * B * max_seqlen * 8) + up256((size_t)H * B * nblk * 4) + up256((size_t)H * p.groups * offsets * 4) +
         up256((size_t)H * offsets * 4);
}

extern "C" int spa_packed_attention_bias_bwd(const void* q, const void* k, const void* v, int64_t q_row_stride, int64_t k_row_stride,
                                             int64_t v_row_stride, const void* out, const void* dout,
                                             const float* lse, const int32_t* cu_seqlens, const int32_t* gather_idx, const void* table,
                                             const int32_t* buckets, int n_buckets, int grid_h, int grid_w, int B, int max_seqlen,
                                             int H, int Dh, int dtype, float softmax_scale, void* dq, void* dk, void* dv,
                                             int64_t dq_row_stride, int64_t dk_row_stride, int64_t dv_row_stride, float* d_table,
                                             void* workspace, size_t workspace_bytes, void* stream) {
  const char* fn = "spa_packed_attention_bias_bwd";
  BiasMap m;
  if (int rc = bias_checks(fn, q, k, v, q_row_stride, k_row_stride, v_row_stride, cu_seqlens, B, max_seqlen, H, Dh, dtype, softmax_scale,
                           table, buckets, n_buckets, gather_idx, grid_h, grid_w, &m))
    return rc;
  SPA_REQUIRE(out && dout && lse && dq && dk && dv, SPA_ERR_INVALID_ARG, "%s: null pointer", fn);
  const int64_t strides[3] = {dq_row_stride, dk_row_stride, dv_row_stride};
  for (int64_t rs : strides) {
    SPA_REQUIRE(rs >= (int64_t)H * Dh, SPA_ERR_INVALID_ARG, "%s: row stride %ld < H*Dh", fn, (long)rs);
    SPA_REQUIRE((rs * elem_size(dtype)) % 16 == 0, SPA_ERR_INVALID_ARG, "%s: row stride is not a multiple of 16 bytes", fn);
  }
  SPA_REQUIRE(aligned16(out) && aligned16(dout) && aligned16(dq) && aligned16(dk) && aligned16(dv),
              SPA_ERR_INVALID_ARG, "%s: tensors not 16-byte aligned", fn);
  const size_t need = spa_attention_bias_bwd_workspace_bytes(B, max_seqlen, H, Dh, grid_h, grid_w, dtype);
  SPA_REQUIRE(workspace != nullptr && workspace_bytes >= need, SPA_ERR_WORKSPACE, "%s: workspace of %zu bytes needed, %zu given", fn,
              need, workspace_bytes);
  SPA_REQUIRE((reinterpret_cast<uintptr_t>(workspace) & 255u) == 0, SPA_ERR_INVALID_ARG, "%s: workspace not 256-byte aligned", fn);
  const float scale = softmax_scale > 0.f ? softmax_scale : 1.0f / std::sqrt((float)Dh);
  const long ls = (long)B * max_seqlen;
  const int nblk = (max_seqlen + kBiasRows - 1) / kBiasRows;
  SPA_REQUIRE(((long)H * B + 8) * nblk < 2147483647L, SPA_ERR_INVALID_ARG, "%s: B*H*blocks must be < 2^31", fn);
  const BiasPlan plan = bias_plan(H, B, max_seqlen, Dh, m.offsets, dtype);
  char* ws = static_cast<char*>(workspace);
  auto take = [&](size_t bytes) {
    char* at = ws;
    ws += up256(bytes);
    return at;
  };
  floatx2* dvec = reinterpret_cast<floatx2*>(take((size_t)H * ls * 8));
  uint32_t* most = reinterpret_cast<uint32_t*>(take((size_t)H * B * nblk * 4));
  float* partial = reinterpret_cast<float*>(take((size_t)H * plan.groups * m.offsets * 4));
  float* sums = buckets != nullptr ? reinterpret_cast<float*>(take((size_t)H * m.offsets * 4)) : d_table;
  hipStream_t st = as_stream(stream);
  const bool hist = d_table != nullptr;
#define SPA_BWD(T, D)                                                                                                        \
  do {                                                                                                                       \
    const BiasBwd<T> args = {(const T*)q, (const T*)k, (const T*)v, (const T*)out, (const T*)dout, (long)q_row_stride,       \
                             (long)k_row_stride, (long)v_row_stride, lse, dvec, ls, cu_seqlens, m, H, B, nblk, scale, (T*)dq, \
                             (T*)dk, (T*)dv, (long)dq_row_stride, (long)dk_row_stride, (long)dv_row_stride, most, partial,   \
                             plan.key_blocks, plan.groups, plan.slice, plan.bits};                                                            \
    if (int rc = launch_bias_bwd<T, D>(fn, args, plan, hist, st)) return rc;                                                 \
  } while (0)
  if (dtype == SPA_F32) {
    if (Dh == 32) SPA_BWD(float, 32); else SPA_BWD(float, 64);
  } else {
    if (Dh == 32) SPA_BWD(__bf16, 32); else SPA_BWD(__bf16, 64);
  }
#undef SPA_BWD
  if (hist) {
    const bool one = buckets != nullptr && m.offsets <= kTableSums && (m.offsets + 1023) / 1024 * plan.groups <= 32;
    const dim3 grid((n_buckets + kTableBuckets - 1) / kTableBuckets, H);
    const BiasTable to_buckets = {one ? partial : sums, buckets, n_buckets, m.offsets, plan.groups, d_table};
    if (one) {
      hipLaunchKernelGGL(attn_bias_table_kernel<true>, grid, dim3(1024), 0, st, to_buckets);
    } else {
      const BiasSum sum = {partial, plan.groups, m.offsets, sums};
      hipLaunchKernelGGL(attn_bias_sum_kernel, dim3((m.offsets + 31) / 32, H), dim3(256), 0, st, sum);
      if (buckets != nullptr) hipLaunchKernelGGL(attn_bias_table_kernel<false>, grid, dim3(1024), 0, st, to_buckets);
    }
  }
  return check_launch(fn);
}
