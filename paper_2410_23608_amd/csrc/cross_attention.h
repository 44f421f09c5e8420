// What the forward and the backward of the attention to another sequence share (cross_attention.hip, cross_attention_bwd.hip).
//
// The rows of a unit (segment b, key head hk) are the nq tokens of the segment times the G = H / Hk query heads that share the key
// head: row r is token r / G, head hk G + r % G.  So keys and values are fetched once for all of them, a few tokens fill a wave's 32
// rows, and the sums over the heads of a group are the sums over rows of the backward.
#pragma once

#include <type_traits>

#include "attn_ops.h"
#include "attn_tiles.h"
#include "divisor.h"
#include "share.h"
#include "spa_common.h"

namespace spa {

constexpr int kCrossThreads = 256;

struct CrossShape {
  const int32_t *cu_q, *cu_k, *key_lens;
  int B, H, Hk;
  Divisor G;                     // query heads a key head
  int blocks;                    // workgroups along the owned rows of the longest possible segment
  int splits;                    // and along the others
  float scale, c;                // c = scale log2 e: exponents of 2
  long stat_stride;              // of lse and D: entry (h, row)
  int most_q, most_k;            // tokens and keys of the longest possible segment (longer ones are cut)
};

// A workgroup's unit: (segment, key head, block of owned rows, split of the others)
struct CrossUnit {
  int b, hk, block, split;
  bool valid;
  long q0, k0;                   // the segment's first rows
  int nq, nk, held;              // rows (tokens times heads), keys, keys the segment has places for
};
// What of a segment is looked at: no more tokens and keys than the longest may have, no token from the B max_q-th on (lse and D have no
// place for it), nothing of one that starts below 0.
__device__ __forceinline__ void cross_lengths(const CrossShape& s, int b, int q0, int k0, int& nq, int& nk, int& held) {
  const int room = q0 < 0 ? 0 : (int)max(s.stat_stride - q0, 0L);
  nq = min(min(max(s.cu_q[b + 1] - q0, 0), s.most_q), room) * (int)s.G.d;
  held = k0 < 0 ? 0 : min(max(s.cu_k[b + 1] - k0, 0), s.most_k);
  nk = s.key_lens != nullptr ? min(max(s.key_lens[b], 0), held) : held;
}
// Blocks and splits of a pair (segment, key head) next to each other on one XCD, whose L2 then holds what they share, pairs dealt to the
// XCDs there and back.  So fewer than eight pairs leave XCDs without work, however many blocks each has (one image of 3136 tokens and keys,
// 8 heads of 64 on 1 | 2 | 4 | 8 key heads: forward 205 | 121 | 75 | 51 us, backward 624 | 337 | 204 | 138), nine to fifteen give some two
// of them.
// Up to kRankedB segments come by their products, most first; ranking more costs every workgroup more than it gives (8 segments of 1568 to
// 3136 tokens and 410 to 1024 keys, 12 and 4 heads of 64, dk / dv in index order 171 us, ranked 158).
constexpr int kRankedB = 16;
__device__ __forceinline__ CrossUnit cross_unit(const CrossShape& s) {
  const int per = s.blocks * s.splits, xcd = blockIdx.x & 7, j = blockIdx.x >> 3, pl = j / per, qb = j - pl * per;
  const int pair = pl * 8 + (pl & 1 ? 7 - xcd : xcd);
  CrossUnit u = {};
  u.valid = pair < s.Hk * s.B;
  if (!u.valid) return u;
  u.b = pair / s.Hk;
  u.hk = pair - u.b * s.Hk;
  u.block = qb / s.splits;
  u.split = qb - u.block * s.splits;
  int q0, k0;
  if (s.B > 1 && s.B <= kRankedB) {
    const int lane = threadIdx.x & 63, b = min(lane, s.B - 1);
    q0 = s.cu_q[b];
    k0 = s.cu_k[b];
    cross_lengths(s, b, q0, k0, u.nq, u.nk, u.held);
    const float cost = (float)u.nq * (float)u.nk;
    int rank = 0;
    for (int o = 0; o < s.B; ++o) {
      const float other = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, cost), o));
      rank += (other > cost) | ((other == cost) & (o < lane));
    }
    const int at = __builtin_ctzll(__ballot(lane < s.B && rank == u.b));
    u.b = at;
    q0 = __builtin_amdgcn_readlane(q0, at);
    k0 = __builtin_amdgcn_readlane(k0, at);
    u.nq = __builtin_amdgcn_readlane(u.nq, at);
    u.nk = __builtin_amdgcn_readlane(u.nk, at);
    u.held = __builtin_amdgcn_readlane(u.held, at);
  } else {
    q0 = s.cu_q[u.b];
    k0 = s.cu_k[u.b];
    cross_lengths(s, u.b, q0, k0, u.nq, u.nk, u.held);
  }
  u.q0 = q0;
  u.k0 = k0;
  return u;
}

// Offset of row r (token r / G, head r % G of the group) of a tensor of `stride` elements a token (below 2^31)
template <int DH>
__device__ __forceinline__ long group_row(const Divisor& G, int r, long stride) {
  const uint32_t i = quotient((uint32_t)r, G);
  return (long)((uint64_t)i * (uint32_t)stride) + (r - (int)(i * G.d)) * DH;
}

// BT rows of two operands on their way to LDS, in 16-byte pieces.  Nothing here waits for a load or branches on one between load() and
// store(); rows past the end are loaded as the last one, and store<true>() clears operand 1's (the caller gives such rows probability 0,
// and 0 times an infinity of the last row would be NaN).  GROUPED: rows of a unit's tokens and heads (group_row), else of one head.
// (Addresses of whole steps from the first step's by a scalar's distance, without the multiplications: registers for them cost dq a wave a
// SIMD, 91 -> 100 us at 8 segments of 1568 to 3136 tokens and 410 to 1024 keys, 12 and 4 heads of 64; forward 78 -> 77, dk / dv 141 ->
// 148.)
template <typename T, int DH, int BT, bool GROUPED>
struct CrossStage {
  static constexpr int RS = Ops<T, DH>::RS, VE = 16 / sizeof(T), CPR = DH / VE, CPT = BT * CPR / kCrossThreads, RPP = kCrossThreads / CPR;
  static_assert(BT * CPR % kCrossThreads == 0, "whole passes");
  const T *a, *b;                // the thread's column of the first row
  long as, bs;
  const Divisor& G;
  int tid, last, from;
  uintx4 v[2][CPT];
  __device__ __forceinline__ CrossStage(const T* a_, long as_, const T* b_, long bs_, const Divisor& G_, int last_)
      : a(a_ + threadIdx.x % CPR * VE), b(b_ + threadIdx.x % CPR * VE), as(as_), bs(bs_), G(G_), tid(threadIdx.x), last(last_), from(0) {}
  __device__ __forceinline__ int row(int t) const { return tid / CPR + t * RPP; }
  __device__ __forceinline__ long offset(int r, long stride) const {
    return GROUPED ? group_row<DH>(G, r, stride) : (long)((uint64_t)(uint32_t)r * (uint32_t)stride);
  }
  __device__ __forceinline__ void load(int t0) {
    from = t0;
#pragma unroll
    for (int t = 0; t < CPT; ++t) {
      const int r = min(t0 + row(t), last);
      v[0][t] = *reinterpret_cast<const uintx4*>(a + offset(r, as));
      v[1][t] = *reinterpret_cast<const uintx4*>(b + offset(r, bs));
    }
  }
  template <bool LAST>
  __device__ __forceinline__ void store(T* ta, T* tb) {
#pragma unroll
    for (int t = 0; t < CPT; ++t) {
      if (LAST && from + row(t) > last) v[1][t] = uintx4{0, 0, 0, 0};
      const int o = row(t) * RS + tid % CPR * VE;
      *reinterpret_cast<uintx4*>(ta + o) = v[0][t];
      *reinterpret_cast<uintx4*>(tb + o) = v[1][t];
    }
  }
};

// KW waves of the four share 32 owned rows, each takes a part of every step of the others.
template <int KW>
struct CrossSteps {
  static constexpr int RW = 4 / KW, STEP = KW == 1 ? 64 : 128, TILE = STEP / KW, ROWS = 32 * RW;
};

// ---- host
struct CrossPlan {
  int kw, blocks, splits;
};
size_t cross_up(size_t n);
// What the entry points of both directions check and have in common.
struct CrossCall {
  const void *q, *k, *v;
  int64_t qs, ks, vs;
  const int32_t *cu_q, *cu_k, *key_lens;
  int B, max_q, max_k, H, Hk, Dh, dtype;
  float softmax_scale;
};
int cross_checks(const char* fn, const CrossCall& c);
bool cross_sizes_ok(int B, int max_q, int max_k, int H, int Hk, int Dh, int dtype);
// Blocks of owned rows and splits of the others for `owned` and `others` rows of the longest segment in `units` units
CrossPlan cross_plan(long units, long owned, long others, int dtype);
CrossShape cross_shape(const CrossCall& c, const CrossPlan& p);
inline long cross_grid(const CrossShape& s) { return ((long)s.Hk * s.B + 7) / 8 * 8 * s.blocks * s.splits; }

}  // namespace spa
