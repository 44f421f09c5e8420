// Packed, per-image attention with a learned bias by the bucket of the relative position: the token of packed row j sits at
// n = gather_idx[j] mod (gh gw) of its image's map, row n / gw, column n mod gw, and
//   S_ij = scale q_i k_j + table[h, buckets[offset of i from j]],   O = softmax(S) V
// With p = row (2 gw - 1) + column the offset's index is p_i - p_j + (gh - 1)(2 gw - 1) + gw - 1: one subtraction.  A row whose
// scores are all -inf gives 0.  Backward, beside dQ, dK, dV of the attention without a bias,
//   dtable[h, b] = sum over the pairs of bucket b of dS_ij,  dS = P (dP - D)
// The order in which the many dS of an offset are added would be the launch's, so they are added as integers: dS is rounded
// to a multiple of 2^(e - shift), where 2^e is above every |dS| the head can have (|dS| <= |dP| + |D| <= 2 Dh max|dO| max|V|) and
// shift (40 for up to 4 million rows) leaves a 64-bit sum no way to overflow.  Sums are then the same in any order, and finer than fp32 ones.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "attn_tiles.h"
#include "spa_common.h"

namespace spa {

// x / d for 0 <= x < 2^31 by one high product: with 2^s >= d > 2^(s-1), M = floor(2^(31+s) / d) + 1 < 2^32 is at most 2^s / d too
// large in units of its last place, which times x is below 2^(31+s) / d: the quotient is exact.  (d = 1: M = 0.)
struct Divisor {
  uint32_t d, M, shift;
};
static Divisor divisor(uint32_t d) {
  uint32_t s = 0;
  while ((1ull << s) < d) ++s;
  return d == 1 ? Divisor{1, 0, 0} : Divisor{d, (uint32_t)((1ull << (31 + s)) / d + 1), s - 1};
}
__device__ __forceinline__ uint32_t quotient(uint32_t x, const Divisor& d) { return d.M == 0 ? x : __umulhi(x, d.M) >> d.shift; }

struct BiasMap {
  const void* table;             // [H, nb]
  const int32_t *buckets, *gather_idx;
  int nb, tokens, offsets, centre;          // tokens = gh gw
  Divisor gw, per_image;
};

// What says where packed row `row` sits, number j of its segment; the position index it gives.
__device__ __forceinline__ int bias_token(const BiasMap& m, long row, int j) {
  return m.gather_idx != nullptr ? m.gather_idx[row] & 0x7fffffff : min(j, m.tokens - 1);
}
__device__ __forceinline__ int bias_position(const BiasMap& m, int token) {
  const uint32_t n = (uint32_t)token - quotient((uint32_t)token, m.per_image) * m.per_image.d, r = quotient(n, m.gw);
  return (int)(n + r * (m.gw.d - 1));                         // r (2 gw - 1) + n - r gw
}
__device__ __forceinline__ int bias_position(const BiasMap& m, long row, int j) { return bias_position(m, bias_token(m, row, j)); }
template <typename T>
__device__ __forceinline__ float bias_at(const BiasMap& m, int h, int offset) {
  const int b = m.buckets != nullptr ? m.buckets[offset] : offset;
  return (unsigned)b < (unsigned)m.nb ? (float)static_cast<const T*>(m.table)[(long)h * m.nb + b] : 0.f;
}

constexpr int kRowThreads = 128, kRowTile = 32;

// Rows [t, t + 32) of one head of two operands as fp32 in LDS; rows past the segment read as zero.
template <typename T, int DH>
__device__ __forceinline__ void stage_rows(const T* a, long as, const T* b, long bs, long row0, int t, int n, float* As, float* Bs) {
  for (int i = threadIdx.x; i < kRowTile * DH; i += kRowThreads) {
    const int r = i / DH, c = i % DH;
    const bool in = t + r < n;
    As[i] = in ? (float)a[(row0 + t + r) * as + c] : 0.f;
    Bs[i] = in ? (float)b[(row0 + t + r) * bs + c] : 0.f;
  }
}

// One thread per query, the keys streaming through LDS.
template <typename T, int DH>
__global__ void __launch_bounds__(kRowThreads)
attn_bias_rows_kernel(const T* __restrict__ q, const T* __restrict__ k, const T* __restrict__ v, long qs, long ks, long vs,
                      const int32_t* __restrict__ cu, BiasMap m, int H, float scale, T* __restrict__ out,
                      float* __restrict__ lse, long lse_stride) {
  __shared__ float Ks[kRowTile * DH], Vs[kRowTile * DH];
  __shared__ int pos[kRowTile];
  const int h = blockIdx.y, q0 = blockIdx.x * kRowThreads;
  const long row0 = cu[blockIdx.z];
  const int n = (int)(cu[blockIdx.z + 1] - row0);
  if (q0 >= n) return;
  const int qi = q0 + threadIdx.x;
  const bool ok = qi < n;
  const long row = row0 + (ok ? qi : 0), C = (long)H * DH;
  float qf[DH], o[DH];
#pragma unroll
  for (int d = 0; d < DH; ++d) {
    qf[d] = (float)q[row * qs + h * DH + d] * scale;
    o[d] = 0.f;
  }
  const int p = bias_position(m, row, ok ? qi : 0) + m.centre;
  float mx = -INFINITY, l = 0.f;
  for (int t = 0; t < n; t += kRowTile) {
    __syncthreads();
    stage_rows<T, DH>(k + h * DH, ks, v + h * DH, vs, row0, t, n, Ks, Vs);
    if (threadIdx.x < kRowTile && t + threadIdx.x < n) pos[threadIdx.x] = bias_position(m, row0 + t + threadIdx.x, t + threadIdx.x);
    __syncthreads();
    const int tn = min(kRowTile, n - t);
    for (int j = 0; j < tn; ++j) {
      float s = bias_at<T>(m, h, p - pos[j]);
#pragma unroll
      for (int d = 0; d < DH; ++d) s = fmaf(qf[d], Ks[j * DH + d], s);
      const float m_new = __builtin_elementwise_maximum(mx, s);
      const float ref = m_new == -INFINITY ? 0.f : m_new;            // no score yet: weights of 0
      const float a = expf(mx - ref), e = expf(s - ref);
      mx = m_new;
      l = fmaf(l, a, e);
#pragma unroll
      for (int d = 0; d < DH; ++d) o[d] = fmaf(o[d], a, e * Vs[j * DH + d]);
    }
  }
  if (!ok) return;
  const bool some = mx != -INFINITY;
  const float inv = some ? 1.0f / l : 0.f;
#pragma unroll
  for (int d = 0; d < DH; ++d) {
    out[row * C + h * DH + d] = (T)(some ? o[d] * inv : 0.f);
  }
  if (lse != nullptr) lse[h * lse_stride + row] = some ? mx + logf(l) : -INFINITY;
}

// ------------------------------------------------------------------------- bf16 / MFMA
// As in the attention without a bias: one wave owns 32 queries and computes S^T = K Q^T, so that a lane holds 16 keys of one
// query a 32 x 32 block, and the rounded P is the second product's operand in registers; K and V stream through LDS in tiles of
// 64.  The bias of a score is one LDS read at (p_i - p_j): the keys' positions of a tile lie beside it, and `win` holds the
// biases, as bf16 like the table, of all offsets of the map (WHOLE: up to kWholeMost), or of kWindow neighbouring ones.  On
// larger maps the offsets between the workgroup's queries and a tile's keys are a narrow range that moves steadily with the tiles,
// as packed rows are in the order of their positions: the window is loaded anew where a tile leaves it.  A tile whose
// offsets exceed the window (few tokens far apart, rows in another order) looks each bias up in memory.
constexpr float kLog2e = 1.4426950408889634f;
// Beyond this a score times log2 e is no fp32 number any more (table entries of the type's lowest value, or -inf): such rows take
// the difference to their maximum before the factor.
constexpr float kFarScore = 2e38f;
constexpr int kBiasBN = 64, kBiasThreads = 256, kBiasRows = 128;
constexpr int kWholeMost = 32768, kWindow = 8192;

template <bool MAX>
__device__ __forceinline__ int pick(int a, int b) { return MAX ? max(a, b) : min(a, b); }
template <int CTRL, bool MAX>
__device__ __forceinline__ int pick_dpp(int v) { return pick<MAX>(v, __builtin_amdgcn_update_dpp(v, v, CTRL, 0xF, 0xF, false)); }
// The largest (smallest) value of the wave, in every lane
template <bool MAX>
__device__ __forceinline__ int wave_pick(int v) {
  const auto h = __builtin_amdgcn_permlane32_swap((unsigned)v, (unsigned)v, false, false);
  const unsigned a = h[0], b = h[1];
  v = pick<MAX>((int)a, (int)b);
  const auto q = __builtin_amdgcn_permlane16_swap((unsigned)v, (unsigned)v, false, false);
  const unsigned c = q[0], d = q[1];
  v = pick<MAX>((int)c, (int)d);
  return pick_dpp<0xB1, MAX>(pick_dpp<0x4E, MAX>(pick_dpp<0x124, MAX>(pick_dpp<0x128, MAX>(v))));
}

// The biases of offsets [base, base + n) of head h to win[shift ..]; returns shift.  Without a bucket map the table's row is
// copied as it lies in memory, 16 bytes at a time (shift: where it starts in its first 16); through one, a row of up to
// kTableLds entries is brought to LDS first, and the map comes in 16-byte pieces too where `base` allows.
constexpr int kTableLds = 1024;
__device__ __forceinline__ int load_window(const BiasMap& m, int h, int base, int n, uint16_t* win, uint16_t* row_lds) {
  const uint16_t* row = static_cast<const uint16_t*>(m.table) + (long)h * m.nb;
  n = min(n, m.offsets - base);
  const int tid = threadIdx.x;
  if (m.buckets == nullptr) {
    const uintptr_t at = reinterpret_cast<uintptr_t>(row + base);
    const int shift = (int)(at & 15) / 2, first = (8 - shift) & 7;              // entries in front of the first whole piece
    const int whole = n > first ? (n - first) / 8 : 0;
    constexpr int U = 8;
    for (int i0 = tid; i0 < whole; i0 += U * kBiasThreads) {
      uintx4 v[U];
#pragma unroll
      for (int u = 0; u < U; ++u)
        v[u] = *reinterpret_cast<const uintx4*>(row + base + first + 8 * min(i0 + u * kBiasThreads, whole - 1));
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (i0 + u * kBiasThreads < whole) *reinterpret_cast<uintx4*>(win + shift + first + 8 * (i0 + u * kBiasThreads)) = v[u];
    }
    if (tid < min(first, n)) win[shift + tid] = row[base + tid];
    const int rest = first + 8 * whole + tid;                                   // behind the last whole piece
    if (tid < 8 && rest < n) win[shift + rest] = row[base + rest];
    return shift;
  }
  const bool in_lds = m.nb <= kTableLds;
  if (in_lds) {
    for (int i = tid; i < m.nb; i += kBiasThreads) row_lds[i] = row[i];
    __syncthreads();
  }
  const uint16_t* from = in_lds ? row_lds : row;
  auto entry = [&](int b) -> uint16_t { return (unsigned)b < (unsigned)m.nb ? from[b] : (uint16_t)0; };
  typedef int intx4 __attribute__((ext_vector_type(4)));
  const int quads = (base & 3) == 0 ? n / 4 : 0;
  constexpr int U = 8;
  for (int i0 = tid; i0 < quads; i0 += U * kBiasThreads) {
    intx4 b[U];
#pragma unroll
    for (int u = 0; u < U; ++u) b[u] = *reinterpret_cast<const intx4*>(m.buckets + base + 4 * min(i0 + u * kBiasThreads, quads - 1));
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uintx2 w = {(uint32_t)entry(b[u][0]) | (uint32_t)entry(b[u][1]) << 16, (uint32_t)entry(b[u][2]) | (uint32_t)entry(b[u][3]) << 16};
      if (i0 + u * kBiasThreads < quads) *reinterpret_cast<uintx2*>(win + 4 * (i0 + u * kBiasThreads)) = w;
    }
  }
  for (int i = 4 * quads + tid; i < n; i += kBiasThreads) win[i] = entry(m.buckets[base + i]);
  return 0;
}

// Positions of the streamed rows of a tile and their range, and the range of the workgroup's own rows.
struct BiasPos {
  __attribute__((aligned(16))) int pos[2][kBiasBN];
  int range[2][2];
  int own[kBiasThreads / kWave][2];
};
// The first wave's 64 lanes: the tile's positions, and their smallest and largest.
__device__ __forceinline__ void put_positions(BiasPos& l, int buf, const BiasMap& m, int token, bool ranges) {
  if (threadIdx.x < kBiasBN) {
    const int p = bias_position(m, token);
    l.pos[buf][threadIdx.x] = p;
    if (ranges) {
      const int lo = wave_pick<false>(p), hi = wave_pick<true>(p);
      if (threadIdx.x == 0) {
        l.range[buf][0] = lo;
        l.range[buf][1] = hi;
      }
    }
  }
}
struct Range {
  int lo, hi;
};
__device__ __forceinline__ Range own_range(const BiasPos& l) {
  Range r = {l.own[0][0], l.own[0][1]};
#pragma unroll
  for (int w = 1; w < kBiasThreads / kWave; ++w) r = {min(r.lo, l.own[w][0]), max(r.hi, l.own[w][1])};
  return {__builtin_amdgcn_readfirstlane(r.lo), __builtin_amdgcn_readfirstlane(r.hi)};
}

template <int DH>
struct BiasTiles {
  static constexpr int RS = DH + 8;
  __attribute__((aligned(16))) __bf16 A[2][kBiasBN * RS];     // K (forward, dq) | Q (dk, dv)
  __attribute__((aligned(16))) __bf16 B[2][kBiasBN * RS];     // V | dO
  BiasPos p;
  uint16_t row[kTableLds];
  int s_live[sizeof(LiveTile) / sizeof(int)];
};

// The workgroup's block: (segment, head, rows from r0), longest segments first where they can be ranked.
struct BiasBlock {
  Segment seg;
  int h, r0;
  bool valid;
};
template <int DH>
__device__ __forceinline__ BiasBlock bias_block(BiasTiles<DH>& l, const int32_t* cu, int H, int B, int nblk) {
  const int xcd = blockIdx.x & 7, j = blockIdx.x >> 3;
  if (B <= kLptMaxB) {
    LiveTile* slot = reinterpret_cast<LiveTile*>(l.s_live);
    const LiveTile t = live_tiles_apply(H, B) ? live_tile_block<1>(xcd, j, H, B, cu, kBiasRows, nblk, slot)
                                              : class_tile_block<1>(xcd, j, H, B, cu, kBiasRows, nblk, slot);
    return {{t.row0, t.len, t.len}, t.h, t.qb * kBiasRows, t.valid};
  }
  const TileId t = xcd_tile_at(xcd, j, nblk, H, B);
  if (!t.valid) return {{0, 0, 0}, 0, 0, false};
  const Segment seg = segment_of(t.rank, cu, nullptr, 0);
  return {seg, t.h, t.qb * kBiasRows, t.qb * kBiasRows < seg.nq};
}

struct BiasFwd {
  const __bf16 *q, *k, *v;
  long qs, ks, vs;
  const int32_t* cu;
  BiasMap m;
  int H, B, nblk;
  float scale;
  __bf16* out;
  float* lse;
  long lse_stride;
};

// Scores of the wave's 32 rows against a tile's 64 with their biases: s scale + bias.  pos: positions of the tile's rows, own:
// that of this lane's row (with the centre), SIGN: 1 if the offset is own - pos, else pos - own.  win: where offset 0 would lie.
template <int SIGN>
__device__ __forceinline__ void add_bias(floatx16 (&s)[2], const int* pos, int own, bool in_window, const BiasMap& m, int h,
                                         const uint16_t* win, float scale, int hh) {
  typedef int intx4 __attribute__((ext_vector_type(4)));
#pragma unroll
  for (int sb = 0; sb < 2; ++sb) {
    float b[16];
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const intx4 p = *reinterpret_cast<const intx4*>(&pos[sb * 32 + 8 * g + 4 * hh]);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int o = SIGN > 0 ? own - p[e] : p[e] - own;
        b[4 * g + e] = in_window ? __builtin_bit_cast(float, (uint32_t)win[o] << 16) : bias_at<__bf16>(m, h, o);
      }
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) s[sb][r] = fmaf(s[sb][r], scale, b[r]);
  }
}

template <int DH, bool WHOLE>
__global__ void __launch_bounds__(kBiasThreads) attn_bias_fwd_kernel(const BiasFwd a) {
  constexpr int RS = DH + 8, KK = DH / 16, DB = DH / 32, BN = kBiasBN;
  extern __shared__ __attribute__((aligned(16))) uint16_t win[];
  __shared__ BiasTiles<DH> l;
  const BiasBlock blk = bias_block<DH>(l, a.cu, a.H, a.B, a.nblk);
  if (!blk.valid) return;
  const Segment seg = blk.seg;
  const int h = blk.h, n = seg.nk, lane = threadIdx.x & 63, wv = threadIdx.x >> 6, l32 = lane & 31, hh = lane >> 5;
  const int qi = blk.r0 + wv * 32 + l32, last = n - 1;
  const bool wave_live = blk.r0 + wv * 32 < n, q_ok = qi < n;
  const long C = (long)a.H * DH, q_row = seg.row0 + min(qi, last);

  PairStage<DH, kBiasThreads, BN, false, false> st(threadIdx.x);
  st.gi = nullptr;
  st.last = last;
  st.source(0, a.k + h * DH, a.ks, seg.row0);
  st.source(1, a.v + h * DH, a.vs, seg.row0);
  int token = 0;
  auto load_tile = [&](int kt) {
    st.load(kt);
    const int j = min(kt + lane, last);
    if (threadIdx.x < BN) token = bias_token(a.m, seg.row0 + j, j);
  };
  auto store_tile = [&](int buf, auto clear) {
    st.template store<clear>(l.A[buf], l.B[buf]);
    put_positions(l.p, buf, a.m, token, !WHOLE);
  };
  load_tile(0);
  bf16x8 qf[KK];
#pragma unroll
  for (int kk = 0; kk < KK; ++kk) qf[kk] = *reinterpret_cast<const bf16x8*>(a.q + q_row * a.qs + h * DH + kk * 16 + hh * 8);
  const int own = bias_position(a.m, q_row, min(qi, last)) + a.m.centre;
  const uint16_t* at0 = win;                                  // where offset 0 would lie
  if (!WHOLE) {
    const int lo = wave_pick<false>(own), hi = wave_pick<true>(own);
    if (lane == 0) {
      l.p.own[wv][0] = lo;
      l.p.own[wv][1] = hi;
    }
  } else {
    at0 = win + load_window(a.m, h, 0, a.m.offsets, win, l.row);
  }
  floatx16 o[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[d][r] = 0.f;
  float m = -INFINITY, sum = 0.f;
  store_tile(0, std::true_type{});
  __syncthreads();
  const Range mine = WHOLE ? Range{0, 0} : own_range(l.p);
  int base = -0x40000000;                                     // (no window yet)
  const int nt = (n + BN - 1) / BN;
  walk_tiles(nt, [&](int t, auto at) {
    constexpr bool end = decltype(at)::value == kTileLast;
    const int buf = t & 1, kt = t * BN;
    if (!end) load_tile(kt + BN);
    bool in_window = true;
    if (!WHOLE) {
      const int lo = mine.lo - l.p.range[buf][1], hi = mine.hi - l.p.range[buf][0];
      in_window = hi - lo < kWindow - 3;
      if (in_window && (lo < base || hi >= base + kWindow)) {  // the keys' positions grow, so the next offsets are lower
        base = max(hi - kWindow + 4, 0) & ~3;                 // (16-byte pieces of the map)
        at0 = win + load_window(a.m, h, base, kWindow, win, l.row) - base;
        __syncthreads();
      }
    }
    if (wave_live) {
      floatx16 s[2];
#pragma unroll
      for (int sb = 0; sb < 2; ++sb) {
#pragma unroll
        for (int r = 0; r < 16; ++r) s[sb][r] = 0.f;
#pragma unroll
        for (int kk = 0; kk < KK; ++kk)
          s[sb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8*>(&l.A[buf][(sb * 32 + l32) * RS + kk * 16 + hh * 8]),
                                                          qf[kk], s[sb], 0, 0, 0);
      }
      if (WHOLE || in_window) add_bias<1>(s, l.p.pos[buf], own, true, a.m, h, at0, a.scale, hh);
      else add_bias<1>(s, l.p.pos[buf], own, false, a.m, h, at0, a.scale, hh);
      if (end) {
#pragma unroll
        for (int sb = 0; sb < 2; ++sb)
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if (kt + sb * 32 + acc_row(r, hh) >= n) s[sb][r] = -INFINITY;
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
        const float ref = m == -INFINITY ? 0.f : m;             // (no score yet: weights of 0)
#pragma unroll
        for (int sb = 0; sb < 2; ++sb)
#pragma unroll
          for (int r = 0; r < 16; ++r) s[sb][r] = __builtin_amdgcn_exp2f((s[sb][r] - ref) * kLog2e);
      }
#pragma unroll
      for (int sb = 0; sb < 2; ++sb)
#pragma unroll
        for (int mf = 0; mf < 2; ++mf) {
          floatx8 f;
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            f[j] = s[sb][8 * mf + j];
            sum += f[j];
          }
          const bf16x8 pb = float_to_bf16x8(f);
#pragma unroll
          for (int d = 0; d < DB; ++d)
            o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(transposed_frag_rowmajor<RS>(l.B[buf], d, sb * 32, mf, lane), pb, o[d], 0, 0, 0);
        }
    }
    if (!end) store_tile(buf ^ 1, std::bool_constant<decltype(at)::value == kTileBeforeLast>{});
    __syncthreads();
  });
  const float total = sum_across_halves(sum), inv = total == 0.f ? 0.f : 1.0f / total;
  __bf16* parked = &l.A[0][0] + wv * 32 * RS;                 // (every wave is past its last read of the tiles)
  if (wave_live) {
    park_tile<DH, RS>(o, inv, parked, l32, hh);
    if (a.lse != nullptr && q_ok && hh == 0)
      a.lse[h * a.lse_stride + q_row] = total == 0.f ? -INFINITY : m + __logf(total);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    flush_tile<DH, RS>(parked, a.out + (seg.row0 + blk.r0 + wv * 32) * C + h * DH, C, min(32, n - blk.r0 - wv * 32), lane);
  }
}

// ------------------------------------------------------------------------------- backward
constexpr int kBiasParts = 32;                 // shares of the rows whose largest |dO| and |V| are found apart

// The largest |dO| and |V| of every head and share of the rows (as bits, which order like the magnitudes, a NaN above all; a
// row whose lse or D is not a number counts as one), and the cleared sums.
struct BiasPrep {
  const void *out, *dout, *v;
  long vs;
  const float* lse;
  long lse_stride;
  const int32_t* cu;
  int B, H;
  uint32_t* largest;              // [H][kBiasParts][2]
  unsigned long long* sums;       // [H][offsets]
  long nsums;
};
template <typename T, int DH>
__global__ void __launch_bounds__(256) attn_bias_prep_kernel(const BiasPrep a) {
  const long T_rows = a.cu[a.B], C = (long)a.H * DH;
  const int h = blockIdx.y;
  const long threads = (long)gridDim.x * gridDim.y * 256;
  for (long i = ((long)blockIdx.y * gridDim.x + blockIdx.x) * 256 + threadIdx.x; i < a.nsums; i += threads) a.sums[i] = 0;
  uint32_t mo = 0, mv = 0;
  for (long row = (long)blockIdx.x * 256 + threadIdx.x; row < T_rows; row += (long)gridDim.x * 256) {
    float D = 0.f;
    for (int d = 0; d < DH; ++d) {
      const float g = (float)static_cast<const T*>(a.dout)[row * C + h * DH + d];
      D = fmaf(g, (float)static_cast<const T*>(a.out)[row * C + h * DH + d], D);
      mo = max(mo, __builtin_bit_cast(uint32_t, g) & 0x7fffffffu);
      mv = max(mv, __builtin_bit_cast(uint32_t, (float)static_cast<const T*>(a.v)[row * a.vs + h * DH + d]) & 0x7fffffffu);
    }
    const float l = a.lse[h * a.lse_stride + row];
    if (!(l < INFINITY) || !(fabsf(D) < INFINITY)) mo = 0x7fffffffu;
  }
  __shared__ uint32_t s[2];
  if (threadIdx.x < 2) s[threadIdx.x] = 0;
  __syncthreads();
  atomicMax(&s[0], mo);
  atomicMax(&s[1], mv);
  __syncthreads();
  if (threadIdx.x < 2) a.largest[(h * kBiasParts + blockIdx.x) * 2 + threadIdx.x] = s[threadIdx.x];
}

// The power of two above every |dS| of a head; `bad`: a gradient or a value of it is not finite, or the bound is beyond fp32.
struct DsBound {
  int e;
  bool bad;
};
template <int DH>
__device__ __forceinline__ DsBound ds_bound(const uint32_t* largest, int h) {
  uint32_t mo = 0, mv = 0;
  for (int i = 0; i < kBiasParts; ++i) {
    mo = max(mo, largest[(h * kBiasParts + i) * 2]);
    mv = max(mv, largest[(h * kBiasParts + i) * 2 + 1]);
  }
  // |x| < 2^(exponent + 1), exponent = (bits >> 23) - 127 (subnormals: below 2^-126); Dh products, dP and D
  const int e = (int)(mo >> 23) - 126 + (int)(mv >> 23) - 126 + (DH == 32 ? 5 : 6) + 2;
  return {e, mo >= 0x7f800000u || mv >= 0x7f800000u || e > 126};
}
__device__ __forceinline__ double power_of_two(int e) { return __builtin_bit_cast(double, (uint64_t)(e + 1023) << 52); }
// x / 2^(e - shift) rounded to an integer: the low bits of the sum with 1.5 2^52, whose own bits are taken off again
__device__ __forceinline__ unsigned long long ds_integer(float x, double factor) {
  const double magic = 6755399441055744.0;
  return __builtin_bit_cast(uint64_t, fma((double)x, factor, magic)) - __builtin_bit_cast(uint64_t, magic);
}

struct BiasBwd {
  const void *q, *k, *v, *out, *dout;
  long qs, ks, vs;
  const float* lse;
  float* dvec;                    // D of every (head, row): the query side writes it, the key side reads it
  long lse_stride;
  const int32_t* cu;
  int H;
  float scale;
  BiasMap m;
  void *dq, *dk, *dv;
  long dqs, dks, dvs;
  const uint32_t* largest;
  unsigned long long* sums;
  int shift;
};

// One thread per row: a query (dq, and D), or a key (dk, dv, and dS into the sums); the other side streams through LDS.
// D from the rounded out is off by a share of that rounding.  sum_j dS_ij = sum_j P_ij dP_ij - D_i is what it is off by: the query
// side adds it to the D that the key side takes.
template <typename T, int DH, bool kKeySide>
__global__ void __launch_bounds__(kRowThreads) attn_bias_bwd_rows_kernel(const BiasBwd a) {
  __shared__ float As[kRowTile * DH], Bs[kRowTile * DH], lses[kRowTile], Ds[kRowTile];
  __shared__ int pos[kRowTile];
  const int h = blockIdx.y, r0 = blockIdx.x * kRowThreads;
  const long row0 = a.cu[blockIdx.z], C = (long)a.H * DH;
  const int n = (int)(a.cu[blockIdx.z + 1] - row0);
  if (r0 >= n) return;
  const int ri = r0 + threadIdx.x;
  const bool ok = ri < n;
  const long row = row0 + (ok ? ri : 0);
  const T *q = static_cast<const T*>(a.q) + h * DH, *k = static_cast<const T*>(a.k) + h * DH, *v = static_cast<const T*>(a.v) + h * DH,
          *dout = static_cast<const T*>(a.dout) + h * DH;
  float x[DH], y[DH], acc0[DH], acc1[DH];
#pragma unroll
  for (int d = 0; d < DH; ++d) {
    x[d] = (float)(kKeySide ? k[row * a.ks + d] : q[row * a.qs + d]);
    y[d] = (float)(kKeySide ? v[row * a.vs + d] : dout[row * C + d]);
    acc0[d] = acc1[d] = 0.f;
  }
  const int p = bias_position(a.m, row, ok ? ri : 0);
  const float my_lse = a.lse[h * a.lse_stride + row];
  float my_d = 0.f, left = 0.f;
  if (!kKeySide)
    for (int d = 0; d < DH; ++d) my_d = fmaf(y[d], (float)static_cast<const T*>(a.out)[row * C + h * DH + d], my_d);
  double factor = 0.;
  if (kKeySide && a.sums != nullptr) {
    const DsBound b = ds_bound<DH>(a.largest, h);
    if (!b.bad) factor = power_of_two(a.shift - b.e);
  }
  for (int t = 0; t < n; t += kRowTile) {
    __syncthreads();
    if (kKeySide) stage_rows<T, DH>(q, a.qs, dout, C, row0, t, n, As, Bs);
    else stage_rows<T, DH>(k, a.ks, v, a.vs, row0, t, n, As, Bs);
    if (threadIdx.x < kRowTile && t + threadIdx.x < n) {
      const long r = row0 + t + threadIdx.x;
      pos[threadIdx.x] = bias_position(a.m, r, t + threadIdx.x);
      lses[threadIdx.x] = a.lse[h * a.lse_stride + r];
      if (kKeySide) Ds[threadIdx.x] = a.dvec[h * a.lse_stride + r];
    }
    __syncthreads();
    const int tn = min(kRowTile, n - t);
    for (int j = 0; j < tn; ++j) {
      float s = 0.f, dp = 0.f;
#pragma unroll
      for (int d = 0; d < DH; ++d) {
        s = fmaf(x[d], As[j * DH + d], s);
        dp = fmaf(y[d], Bs[j * DH + d], dp);
      }
      const int offset = (kKeySide ? pos[j] - p : p - pos[j]) + a.m.centre;
      const float l = kKeySide ? lses[j] : my_lse, D = kKeySide ? Ds[j] : my_d;
      const float pr = l == -INFINITY ? 0.f : expf(fmaf(s, a.scale, bias_at<T>(a.m, h, offset)) - l);   // (a row without a score)
      const float ds = pr * (dp - D);
      left += ds;
      if (kKeySide && factor != 0. && ok) atomicAdd(&a.sums[(long)h * a.m.offsets + offset], ds_integer(ds, factor));
#pragma unroll
      for (int d = 0; d < DH; ++d) {
        acc0[d] = fmaf(ds, As[j * DH + d], acc0[d]);
        if (kKeySide) acc1[d] = fmaf(pr, Bs[j * DH + d], acc1[d]);
      }
    }
  }
  if (!ok) return;
  if (!kKeySide) a.dvec[h * a.lse_stride + row] = my_d + left;
#pragma unroll
  for (int d = 0; d < DH; ++d) {
    if (kKeySide) {
      static_cast<T*>(a.dk)[row * a.dks + h * DH + d] = (T)(acc0[d] * a.scale);
      static_cast<T*>(a.dv)[row * a.dvs + h * DH + d] = (T)acc1[d];
    } else {
      static_cast<T*>(a.dq)[row * a.dqs + h * DH + d] = (T)(acc0[d] * a.scale);
    }
  }
}

// The sums of the offsets into those of their buckets.  A workgroup has kTableBuckets buckets of a head in LDS and goes over
// all offsets, again with integers.
constexpr int kTableBuckets = 4096;
struct BiasTable {
  const unsigned long long* sums;
  const int32_t* buckets;
  const uint32_t* largest;
  int nb, offsets, shift;
  float* d_table;
};
template <int DH>
__global__ void __launch_bounds__(1024) attn_bias_table_kernel(const BiasTable a) {
  __shared__ unsigned long long s[kTableBuckets];
  const int h = blockIdx.y, b0 = blockIdx.x * kTableBuckets, nb = min(kTableBuckets, a.nb - b0);
  const unsigned long long* sums = a.sums + (long)h * a.offsets;
  if (a.buckets != nullptr) {
    for (int i = threadIdx.x; i < nb; i += 1024) s[i] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < a.offsets; i += 1024) {
      const int b = a.buckets[i] - b0;
      const unsigned long long v = sums[i];
      if ((unsigned)b < (unsigned)nb && v != 0) atomicAdd(&s[b], v);
    }
    __syncthreads();
  }
  const DsBound e = ds_bound<DH>(a.largest, h);
  const double unit = power_of_two(e.bad ? 0 : e.e - a.shift);
  for (int i = threadIdx.x; i < nb; i += 1024) {
    const long long v = (long long)(a.buckets != nullptr ? s[i] : sums[b0 + i]);
    a.d_table[(long)h * a.nb + b0 + i] = e.bad ? NAN : (float)((double)v * unit);
  }
}

// ------------------------------------------------------------------------------- host
static int bias_checks(const char* fn, const void* q, const void* k, const void* v, int64_t q_stride, int64_t k_stride, int64_t v_stride,
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
  SPA_REQUIRE(grid_h >= 1 && grid_w >= 1 && (2 * (long)grid_h - 1) * (2 * (long)grid_w - 1) <= (1L << 26), SPA_ERR_INVALID_ARG,
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

// Bits below the bound that a sum of that many values leaves: 62 less those of their number, at most 40.
static int ds_shift(long rows) {
  int bits = 0;
  while ((1L << bits) < rows) ++bits;
  return std::min(40, 62 - bits);
}
// LDS of a window of that many offsets: it may start up to 7 entries into its first 16 bytes
static size_t window_bytes(int offsets) { return ((size_t)offsets + 7 + 7) / 8 * 16; }
#define SPA_BIAS_LAUNCH(KERNEL, GRID, LDS, ARGS)                                                                              \
  do {                                                                                                                        \
    const hipError_t attr = hipFuncSetAttribute((const void*)KERNEL, hipFuncAttributeMaxDynamicSharedMemorySize, (int)(LDS)); \
    SPA_REQUIRE(attr == hipSuccess, SPA_ERR_HIP, "%s: cannot reserve %zu bytes of LDS", fn, (size_t)(LDS));                   \
    hipLaunchKernelGGL(KERNEL, dim3(GRID), dim3(kBiasThreads), LDS, st, ARGS);                                                \
  } while (0)
static size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }

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
  const float scale = softmax_scale > 0.f ? softmax_scale : 1.0f / std::sqrt((float)Dh);
  const long ls = (long)B * max_seqlen;
  hipStream_t st = as_stream(stream);
  if (dtype == SPA_BF16) {
    const int nblk = (max_seqlen + kBiasRows - 1) / kBiasRows;
    SPA_REQUIRE(((long)H * B + 8) * nblk < 2147483647L, SPA_ERR_INVALID_ARG, "%s: B*H*blocks must be < 2^31", fn);
    const BiasFwd args = {(const __bf16*)q, (const __bf16*)k, (const __bf16*)v, (long)q_row_stride, (long)k_row_stride, (long)v_row_stride,
                          cu_seqlens, m, H, B, nblk, scale, (__bf16*)out, lse, ls};
    const dim3 blocks(xcd_grid(nblk, H, B));
#define SPA_BIAS(D)                                                                                                        \
  do {                                                                                                                     \
    if (m.offsets <= kWholeMost) SPA_BIAS_LAUNCH((attn_bias_fwd_kernel<D, true>), blocks, window_bytes(m.offsets), args);  \
    else SPA_BIAS_LAUNCH((attn_bias_fwd_kernel<D, false>), blocks, window_bytes(kWindow), args);                           \
  } while (0)
    if (Dh == 32) SPA_BIAS(32); else SPA_BIAS(64);
#undef SPA_BIAS
    return check_launch(fn);
  }
  const dim3 grid((max_seqlen + kRowThreads - 1) / kRowThreads, H, B);
#define SPA_BIAS(T, D)                                                                                                         \
  hipLaunchKernelGGL((attn_bias_rows_kernel<T, D>), grid, dim3(kRowThreads), 0, st, (const T*)q, (const T*)k, (const T*)v,       \
                     (long)q_row_stride, (long)k_row_stride, (long)v_row_stride, cu_seqlens, m, H, scale, (T*)out, lse, ls)
  if (Dh == 32) SPA_BIAS(float, 32); else SPA_BIAS(float, 64);
#undef SPA_BIAS
  return check_launch(fn);
}

extern "C" size_t spa_attention_bias_bwd_workspace_bytes(int B, int max_seqlen, int H, int Dh, int grid_h, int grid_w, int dtype) {
  (void)Dh; (void)dtype;
  if (B < 1 || max_seqlen < 1 || H < 1 || grid_h < 1 || grid_w < 1) return 0;
  const size_t offsets = (2 * (size_t)grid_h - 1) * (2 * (size_t)grid_w - 1);
  return up256((size_t)H * B * max_seqlen * sizeof(float)) + up256((size_t)H * kBiasParts * 2 * sizeof(uint32_t)) +
         (size_t)H * offsets * sizeof(unsigned long long);
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
  char* ws = static_cast<char*>(workspace);
  float* dvec = reinterpret_cast<float*>(ws);
  ws += up256((size_t)H * ls * sizeof(float));
  uint32_t* largest = reinterpret_cast<uint32_t*>(ws);
  ws += up256((size_t)H * kBiasParts * 2 * sizeof(uint32_t));
  unsigned long long* sums = d_table != nullptr ? reinterpret_cast<unsigned long long*>(ws) : nullptr;
  hipStream_t st = as_stream(stream);
  const BiasPrep prep = {out, dout, v, (long)v_row_stride, lse, ls, cu_seqlens, B, H, largest, sums, (long)H * m.offsets};
  const BiasBwd args = {q, k, v, out, dout, (long)q_row_stride, (long)k_row_stride, (long)v_row_stride, lse, dvec, ls, cu_seqlens, H, scale, m,
                        dq, dk, dv, (long)dq_row_stride, (long)dk_row_stride, (long)dv_row_stride, largest, sums, ds_shift(ls)};
  const BiasTable table_args = {sums, buckets, largest, n_buckets, m.offsets, ds_shift(ls), d_table};
  const dim3 grid((max_seqlen + kRowThreads - 1) / kRowThreads, H, B);
#define SPA_BIAS(T, D)                                                                                                        \
  do {                                                                                                                        \
    if (d_table != nullptr) hipLaunchKernelGGL((attn_bias_prep_kernel<T, D>), dim3(kBiasParts, H), dim3(256), 0, st, prep);   \
    hipLaunchKernelGGL((attn_bias_bwd_rows_kernel<T, D, false>), grid, dim3(kRowThreads), 0, st, args);                       \
    hipLaunchKernelGGL((attn_bias_bwd_rows_kernel<T, D, true>), grid, dim3(kRowThreads), 0, st, args);                        \
    if (d_table != nullptr)                                                                                                   \
      hipLaunchKernelGGL(attn_bias_table_kernel<D>, dim3((n_buckets + kTableBuckets - 1) / kTableBuckets, H), dim3(1024), 0, st, \
                         table_args);                                                                                         \
  } while (0)
  if (dtype == SPA_F32) {
    if (Dh == 32) SPA_BIAS(float, 32); else SPA_BIAS(float, 64);
  } else {
    if (Dh == 32) SPA_BIAS(__bf16, 32); else SPA_BIAS(__bf16, 64);
  }
#undef SPA_BIAS
  return check_launch(fn);
}
