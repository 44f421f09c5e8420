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

// Where the rows of the segment from packed row row0 sit: entry j of the index, in flight from load() on (nothing here may ask for
// its value before it is wanted; without an index some word is loaded and not used), and the position index it gives.
struct BiasTokens {
  const int32_t* at;
  int step;
  __device__ __forceinline__ BiasTokens(const BiasMap& m, const int32_t* any, long row0)
      : at(m.gather_idx != nullptr ? m.gather_idx + row0 : any), step(m.gather_idx != nullptr) {}
  __device__ __forceinline__ int load(int j) const { return at[j * step]; }
  __device__ __forceinline__ int position(const BiasMap& m, int loaded, int j) const {
    const uint32_t t = step != 0 ? (uint32_t)loaded & 0x7fffffffu : (uint32_t)min(j, m.tokens - 1);
    const uint32_t n = t - quotient(t, m.per_image) * m.per_image.d, r = quotient(n, m.gw);
    return (int)(n + r * (m.gw.d - 1));                       // r (2 gw - 1) + n - r gw
  }
  __device__ __forceinline__ int position(const BiasMap& m, int j) const { return position(m, load(j), j); }
};
typedef int intx4 __attribute__((ext_vector_type(4)));
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
  const BiasTokens tokens(m, cu, row0);
  const int p = tokens.position(m, ok ? qi : 0) + m.centre;
  float mx = -INFINITY, l = 0.f;
  for (int t = 0; t < n; t += kRowTile) {
    __syncthreads();
    stage_rows<T, DH>(k + h * DH, ks, v + h * DH, vs, row0, t, n, Ks, Vs);
    if (threadIdx.x < kRowTile && t + threadIdx.x < n) pos[threadIdx.x] = tokens.position(m, t + threadIdx.x);
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

// LDS by byte address: what a look-up costs in vector instructions is then the one subtraction of two positions.
typedef __attribute__((address_space(3))) uint16_t* lds_u16_ptr;
typedef __attribute__((address_space(3))) unsigned long long* lds_u64_ptr;
__device__ __forceinline__ int lds_address(const void* p) { return (int)(uintptr_t)(__attribute__((address_space(3))) const char*)p; }
__device__ __forceinline__ void lds_add(int address, unsigned long long v) {
  __hip_atomic_fetch_add((lds_u64_ptr)(uint32_t)address, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
}

// The biases of offsets [base, base + n) of head h to win[shift ..]; returns shift.  Without a bucket map the table's row is
// copied as it lies in memory, 16 bytes at a time (shift: where it starts in its first 16); through one, a row of up to
// kTableLds entries is brought to LDS first, and the map comes in 16-byte pieces too where `base` allows.
constexpr int kTableLds = 1024;
template <int THREADS = kBiasThreads>
__device__ __forceinline__ int load_window(const BiasMap& m, int h, int base, int n, uint16_t* win, uint16_t* row_lds) {
  const uint16_t* row = static_cast<const uint16_t*>(m.table) + (long)h * m.nb;
  n = min(n, m.offsets - base);
  const int tid = threadIdx.x;
  if (m.buckets == nullptr) {
    const uintptr_t at = reinterpret_cast<uintptr_t>(row + base);
    const int shift = (int)(at & 15) / 2, first = (8 - shift) & 7;              // entries in front of the first whole piece
    const int whole = n > first ? (n - first) / 8 : 0;
    constexpr int U = 8;
    for (int i0 = tid; i0 < whole; i0 += U * THREADS) {
      uintx4 v[U];
#pragma unroll
      for (int u = 0; u < U; ++u)
        v[u] = *reinterpret_cast<const uintx4*>(row + base + first + 8 * min(i0 + u * THREADS, whole - 1));
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (i0 + u * THREADS < whole) *reinterpret_cast<uintx4*>(win + shift + first + 8 * (i0 + u * THREADS)) = v[u];
    }
    if (tid < min(first, n)) win[shift + tid] = row[base + tid];
    const int rest = first + 8 * whole + tid;                                   // behind the last whole piece
    if (tid < 8 && rest < n) win[shift + rest] = row[base + rest];
    return shift;
  }
  const int quads = (base & 3) == 0 ? n / 4 : 0;
  auto fill = [&](auto from) {                                                  // (all of a thread's look-ups in flight)
    auto entry = [&](int b) -> uint32_t {
      const uint32_t v = from[min((uint32_t)b, (uint32_t)m.nb - 1)];
      return (uint32_t)b < (uint32_t)m.nb ? v : 0u;
    };
    constexpr int U = 4;
    for (int i0 = tid; i0 < quads; i0 += U * THREADS) {
      intx4 b[U];
#pragma unroll
      for (int u = 0; u < U; ++u) b[u] = *reinterpret_cast<const intx4*>(m.buckets + base + 4 * min(i0 + u * THREADS, quads - 1));
      uint32_t v[U][4];
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) v[u][i] = entry(b[u][i]);
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (i0 + u * THREADS < quads) *reinterpret_cast<uintx2*>(win + 4 * (i0 + u * THREADS)) = uintx2{v[u][0] | v[u][1] << 16, v[u][2] | v[u][3] << 16};
    }
    for (int i = 4 * quads + tid; i < n; i += THREADS) win[i] = (uint16_t)entry(m.buckets[base + i]);
  };
  if (m.nb <= kTableLds) {
    for (int i = tid; i < m.nb; i += THREADS) row_lds[i] = row[i];
    __syncthreads();
    fill(row_lds);
  } else {
    fill(row);
  }
  return 0;
}

// Positions of the streamed rows of a step (SPLIT tiles) and the range of each tile's, and the range of the workgroup's own rows.
template <int SPLIT>
struct BiasPos {
  __attribute__((aligned(16))) int pos[2][kBiasBN * SPLIT];   // twice the position: bytes of a window
  int range[2][SPLIT][2];
  int own[4 * SPLIT][2];
};
// A wave a tile: its positions, and their smallest and largest.
template <int SPLIT>
__device__ __forceinline__ void put_positions(BiasPos<SPLIT>& l, int buf, const BiasMap& m, const BiasTokens& tokens, int loaded, int j, bool ranges) {
  if (threadIdx.x < kBiasBN * SPLIT) {
    const int p = tokens.position(m, loaded, j);
    l.pos[buf][threadIdx.x] = 2 * p;
    if (ranges) {
      const int lo = wave_pick<false>(p), hi = wave_pick<true>(p);
      if ((threadIdx.x & 63) == 0) {
        l.range[buf][threadIdx.x >> 6][0] = lo;
        l.range[buf][threadIdx.x >> 6][1] = hi;
      }
    }
  }
}
struct Range {
  int lo, hi;
};
template <int N>
__device__ __forceinline__ Range whole_range(const int (&of)[N][2]) {
  Range r = {of[0][0], of[0][1]};
#pragma unroll
  for (int i = 1; i < N; ++i) r = {min(r.lo, of[i][0]), max(r.hi, of[i][1])};
  return {__builtin_amdgcn_readfirstlane(r.lo), __builtin_amdgcn_readfirstlane(r.hi)};
}

template <int DH, int SPLIT>
struct BiasTiles {
  static constexpr int RS = DH + 8, STEP = kBiasBN * SPLIT;
  __attribute__((aligned(16))) __bf16 A[2][STEP * RS];        // K
  __attribute__((aligned(16))) __bf16 B[2][STEP * RS];        // V
  BiasPos<SPLIT> p;
  uint16_t row[kTableLds];
  int s_live[sizeof(LiveTile) / sizeof(int)];
};

// The workgroup's block: (segment, head, rows from r0), longest segments first where they can be ranked.
struct BiasBlock {
  Segment seg;
  int img, h, r0;
  bool valid;
};
__device__ __forceinline__ BiasBlock bias_block(int* s_live, const int32_t* cu, int H, int B, int nblk) {
  const int xcd = blockIdx.x & 7, j = blockIdx.x >> 3;
  if (B <= kLptMaxB) {
    LiveTile* slot = reinterpret_cast<LiveTile*>(s_live);
    const LiveTile t = live_tiles_apply(H, B) ? live_tile_block<1>(xcd, j, H, B, cu, kBiasRows, nblk, slot)
                                              : class_tile_block<1>(xcd, j, H, B, cu, kBiasRows, nblk, slot);
    return {{t.row0, t.len, t.len}, t.img, t.h, t.qb * kBiasRows, t.valid};
  }
  const TileId t = xcd_tile_at(xcd, j, nblk, H, B);
  if (!t.valid) return {{0, 0, 0}, 0, 0, 0, false};
  const Segment seg = segment_of(t.rank, cu, nullptr, 0);
  return {seg, t.rank, t.h, t.qb * kBiasRows, t.qb * kBiasRows < seg.nq};
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

// The biases (upper halves of fp32) of a lane's row against the 16 of a 32-row block that it holds scores of: LDS reads, in flight
// from here on.  pos2: twice the positions of the block's rows, own: that of the lane's row, one of the two with the centre;
// SIGN: 1 if the offset is own - pos, else pos - own.  win0: the LDS address that offset 0 would have.
template <int SIGN>
__device__ __forceinline__ void read_bias(uint32_t (&raw)[16], const int* pos2, int own, int win0, bool in_window, const BiasMap& m, int h,
                                          int hh) {
  const int from = SIGN > 0 ? 2 * own + win0 : win0 - 2 * own;
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    const intx4 p2 = *reinterpret_cast<const intx4*>(&pos2[8 * g + 4 * hh]);
#pragma unroll
    for (int e = 0; e < 4; ++e)
      raw[4 * g + e] = in_window ? *(lds_u16_ptr)(uint32_t)(SIGN > 0 ? from - p2[e] : from + p2[e])
                                 : __builtin_bit_cast(uint32_t, bias_at<__bf16>(m, h, SIGN * (own - (p2[e] >> 1)))) >> 16;
  }
}
__device__ __forceinline__ void add_bias(floatx16& s, const uint32_t (&raw)[16], float scale) {
#pragma unroll
  for (int r = 0; r < 16; ++r) s[r] = fmaf(s[r], scale, __builtin_bit_cast(float, raw[r] << 16));
}

// SPLIT 2: the waves come twice, the second four take every other tile of 64 keys, and hand their sums to the first at the end.
template <int DH, bool WHOLE, int SPLIT>
__global__ void __launch_bounds__(kBiasThreads * SPLIT) attn_bias_fwd_kernel(const BiasFwd a) {
  constexpr int RS = DH + 8, KK = DH / 16, DB = DH / 32, THREADS = kBiasThreads * SPLIT, STEP = kBiasBN * SPLIT;
  extern __shared__ __attribute__((aligned(16))) uint16_t win[];
  __shared__ BiasTiles<DH, SPLIT> l;
  const BiasBlock blk = bias_block(l.s_live, a.cu, a.H, a.B, a.nblk);
  if (!blk.valid) return;
  const Segment seg = blk.seg;
  const int h = blk.h, n = seg.nk, lane = threadIdx.x & 63, l32 = lane & 31, hh = lane >> 5;
  const int wv = (threadIdx.x >> 6) & 3, part = SPLIT > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 8) : 0;
  const int qi = blk.r0 + wv * 32 + l32, last = n - 1;
  const bool wave_live = blk.r0 + wv * 32 < n, q_ok = qi < n;
  const long C = (long)a.H * DH, q_row = seg.row0 + min(qi, last);

  PairStage<DH, THREADS, STEP, false, false> st(threadIdx.x);
  st.gi = nullptr;
  st.last = last;
  st.source(0, a.k + h * DH, a.ks, seg.row0);
  st.source(1, a.v + h * DH, a.vs, seg.row0);
  const BiasTokens tokens(a.m, a.cu, seg.row0);
  int token = 0, token_j = 0;
  auto load_tile = [&](int kt) {
    st.load(kt);
    token_j = min(kt + (int)(threadIdx.x & (STEP - 1)), last);
    token = tokens.load(token_j);
  };
  auto store_tile = [&](int buf, auto clear) {
    st.template store<clear>(l.A[buf], l.B[buf]);
    put_positions(l.p, buf, a.m, tokens, token, token_j, !WHOLE);
  };
  load_tile(0);
  bf16x8 qf[KK];
#pragma unroll
  for (int kk = 0; kk < KK; ++kk) qf[kk] = *reinterpret_cast<const bf16x8*>(a.q + q_row * a.qs + h * DH + kk * 16 + hh * 8);
  const int own = tokens.position(a.m, min(qi, last)) + a.m.centre;
  int win0 = lds_address(win);                                // where offset 0 would lie
  if (!WHOLE) {
    const int lo = wave_pick<false>(own), hi = wave_pick<true>(own);
    if (lane == 0) {
      l.p.own[threadIdx.x >> 6][0] = lo;
      l.p.own[threadIdx.x >> 6][1] = hi;
    }
  } else {
    win0 += 2 * load_window<THREADS>(a.m, h, 0, a.m.offsets, win, l.row);
  }
  floatx16 o[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[d][r] = 0.f;
  float m = -INFINITY, sum = 0.f;
  store_tile(0, std::true_type{});
  __syncthreads();
  const Range mine = WHOLE ? Range{0, 0} : whole_range(l.p.own);
  int base = -0x40000000;                                     // (no window yet)
  const int nt = (n + STEP - 1) / STEP;
  walk_tiles(nt, [&](int t, auto at) {
    constexpr bool end = decltype(at)::value == kTileLast;
    const int buf = t & 1, kt = t * STEP + part * kBiasBN;      // (the wave's tile)
    if (!end) load_tile(t * STEP + STEP);
    bool in_window = true;
    if (!WHOLE) {
      const Range tile = whole_range(l.p.range[buf]);
      const int lo = mine.lo - tile.hi, hi = mine.hi - tile.lo;
      in_window = hi - lo < kWindow - 3;
      if (in_window && (lo < base || hi >= base + kWindow)) {  // the keys' positions grow, so the next offsets are lower
        base = max(hi - kWindow + 4, 0) & ~3;                 // (16-byte pieces of the map)
        win0 = lds_address(win) + 2 * (load_window<THREADS>(a.m, h, base, kWindow, win, l.row) - base);
        __syncthreads();
      }
    }
    if (wave_live && (SPLIT == 1 || !end || kt < n)) {
      const __bf16 *A = &l.A[buf][part * kBiasBN * RS], *B = &l.B[buf][part * kBiasBN * RS];
      const int* pos = &l.p.pos[buf][part * kBiasBN];
      // LDS answers in order: the operands of the first products, then the biases, which arrive during them
      bf16x8 kf[2][KK];
#pragma unroll
      for (int sb = 0; sb < 2; ++sb)
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) kf[sb][kk] = *reinterpret_cast<const bf16x8*>(&A[(sb * 32 + l32) * RS + kk * 16 + hh * 8]);
      __builtin_amdgcn_sched_barrier(0);
      uint32_t raw[2][16];
#pragma unroll
      for (int sb = 0; sb < 2; ++sb) read_bias<1>(raw[sb], &pos[sb * 32], own, win0, WHOLE || in_window, a.m, h, hh);
      __builtin_amdgcn_sched_barrier(0);
      floatx16 s[2];
#pragma unroll
      for (int sb = 0; sb < 2; ++sb) {
#pragma unroll
        for (int r = 0; r < 16; ++r) s[sb][r] = 0.f;
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) s[sb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[sb][kk], qf[kk], s[sb], 0, 0, 0);
        add_bias(s[sb], raw[sb], a.scale);
      }
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
            o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(transposed_frag_rowmajor<RS>(B, d, sb * 32, mf, lane), pb, o[d], 0, 0, 0);
        }
    }
    if (!end) store_tile(buf ^ 1, std::bool_constant<decltype(at)::value == kTileBeforeLast>{});
    __syncthreads();
  });
  // (every wave is past its last read of the tiles)
  if constexpr (SPLIT > 1) {
    constexpr int W = DB * 16 + 2;
    static_assert(4 * W * kWave * sizeof(float) <= sizeof(l.B), "the sums of four waves");
    float* other = reinterpret_cast<float*>(&l.B[0][0]) + wv * W * kWave + lane;
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
  const float total = sum_across_halves(sum), inv = total == 0.f ? 0.f : 1.0f / total;
  __bf16* parked = &l.A[0][0] + wv * 32 * RS;
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
// Bits of an integer dS below the power of two above every |dS|: the sum of a workgroup's, one per offset and row it goes over,
// stays inside 64 bits for up to 2^22 rows (and |dS| cannot add up to more than its rows' |dP|).
constexpr int kDsBits = 40;
__device__ __forceinline__ double power_of_two(int e) { return __builtin_bit_cast(double, (uint64_t)(e + 1023) << 52); }
// x factor, a power of two, rounded to an integer: the low bits of the sum with 1.5 2^52, whose own bits are taken off again
__device__ __forceinline__ unsigned long long ds_integer(float x, double factor) {
  const double magic = 6755399441055744.0;
  return __builtin_bit_cast(uint64_t, fma((double)x, factor, magic)) - __builtin_bit_cast(uint64_t, magic);
}

// ------------------------------------------------------------------------- bf16 backward
// Two launches and the sums behind them (fp32: one thread per row in each, below).  The dq launch walks the keys for 128 queries a workgroup, as the forward does, with D
// from the rounded out, and leaves what the second launch needs: the corrected D of every row, and for every
// block of queries a number that no |dS| of its rows exceeds in that launch.  The dk / dv launch walks the queries for the
// keys of a workgroup, S and dP un-transposed (a lane is a key), so that P and dS are operands in registers again.
// There dS goes into a histogram over the offsets in LDS, 64-bit integers: 32 lanes hold 32 keys against one query, so
// that the lanes of an instruction have offsets of their own.  A workgroup keeps its histogram over all the blocks it
// takes, of one head, and writes it once, as fp32; the sum over the workgroups has a fixed order.  Maps with more offsets than LDS
// has room for are taken in slices: the first pass over the blocks does everything but the offsets of later slices, the
// others only go over the tiles that have offsets in theirs.
template <typename T>
struct BiasBwd {
  const T *q, *k, *v, *out, *dout;
  long qs, ks, vs;
  const float* lse;
  float* dvec;
  long lse_stride;
  const int32_t* cu;
  BiasMap m;
  int H, B, nblk;                 // nblk: blocks of kBiasRows rows of the longest possible segment
  float scale;
  T *dq, *dk, *dv;
  long dqs, dks, dvs;
  uint32_t* most;                 // [H][B * nblk]: what no |dS| of a block of queries exceeds
  float* partial;                 // [H][groups][offsets] or null
  int groups, slice;              // dk / dv: workgroups a head; offsets of a histogram
  int kblk;                       // dk / dv: blocks of 32 NW keys of the longest possible segment
};

template <int DH, bool WHOLE, int SPLIT>
__global__ void __launch_bounds__(kBiasThreads * SPLIT) attn_bias_dq_kernel(const BiasBwd<__bf16> a) {
  constexpr int RS = DH + 8, KK = DH / 16, DB = DH / 32, THREADS = kBiasThreads * SPLIT, STEP = kBiasBN * SPLIT;
  extern __shared__ __attribute__((aligned(16))) uint16_t win[];
  __shared__ BiasTiles<DH, SPLIT> l;
  __shared__ float s_most[2][THREADS / kWave];
  const BiasBlock blk = bias_block(l.s_live, a.cu, a.H, a.B, a.nblk);
  if (!blk.valid) return;
  const Segment seg = blk.seg;
  const int h = blk.h, n = seg.nk, lane = threadIdx.x & 63, l32 = lane & 31, hh = lane >> 5;
  const int wv = (threadIdx.x >> 6) & 3, part = SPLIT > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 8) : 0;
  const int qi = blk.r0 + wv * 32 + l32, last = n - 1;
  const bool wave_live = blk.r0 + wv * 32 < n, q_ok = qi < n;
  const long C = (long)a.H * DH, q_row = seg.row0 + min(qi, last);

  PairStage<DH, THREADS, STEP, false, false> st(threadIdx.x);
  st.gi = nullptr;
  st.last = last;
  st.source(0, a.k + h * DH, a.ks, seg.row0);
  st.source(1, a.v + h * DH, a.vs, seg.row0);
  const BiasTokens tokens(a.m, a.cu, seg.row0);
  int token = 0, token_j = 0;
  auto load_tile = [&](int kt) {
    st.load(kt);
    token_j = min(kt + (int)(threadIdx.x & (STEP - 1)), last);
    token = tokens.load(token_j);
  };
  float v_most = 0.f;                                         // of |V|, of the rows this thread stages
  auto store_tile = [&](int buf, auto clear) {
    st.template store<clear>(l.A[buf], l.B[buf]);
    put_positions(l.p, buf, a.m, tokens, token, token_j, !WHOLE);
#pragma unroll
    for (int t = 0; t < decltype(st)::CPT; ++t) {
      const floatx8 f = bf16x8_to_float(st.v[1][t]);
#pragma unroll
      for (int e = 0; e < 8; ++e) v_most = __builtin_elementwise_maximum(v_most, fabsf(f[e]));
    }
  };
  load_tile(0);
  bf16x8 qf[KK], dof[KK];
  float D = 0.f, l1 = 0.f;                                    // <dO, out> and sum |dO| of the lane's row
#pragma unroll
  for (int kk = 0; kk < KK; ++kk) {
    const int col = h * DH + kk * 16 + hh * 8;
    qf[kk] = *reinterpret_cast<const bf16x8*>(a.q + q_row * a.qs + col);
    dof[kk] = *reinterpret_cast<const bf16x8*>(a.dout + q_row * C + col);
    const floatx8 g = bf16x8_to_float(dof[kk]), o = bf16x8_to_float(*reinterpret_cast<const bf16x8*>(a.out + q_row * C + col));
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      D = fmaf(g[e], o[e], D);
      l1 += fabsf(g[e]);
    }
  }
  D = sum_across_halves(D);
  l1 = sum_across_halves(l1);
  const float lse = a.lse[h * a.lse_stride + q_row];
  const bool far = __ballot(fabsf(lse) >= kFarScore && lse != -INFINITY) != 0;
  const float lse2 = lse == -INFINITY || !q_ok ? INFINITY : lse * kLog2e;      // (no score, or no row: probability 0)
  const int own = tokens.position(a.m, min(qi, last)) + a.m.centre;
  int win0 = lds_address(win);
  if (!WHOLE) {
    const int lo = wave_pick<false>(own), hi = wave_pick<true>(own);
    if (lane == 0) {
      l.p.own[threadIdx.x >> 6][0] = lo;
      l.p.own[threadIdx.x >> 6][1] = hi;
    }
  } else {
    win0 += 2 * load_window<THREADS>(a.m, h, 0, a.m.offsets, win, l.row);
  }
  floatx16 acc[DB], negD;
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    negD[r] = -D;
#pragma unroll
    for (int d = 0; d < DB; ++d) acc[d][r] = 0.f;
  }
  float left = 0.f, most = 0.f;
  store_tile(0, std::true_type{});
  __syncthreads();
  const Range mine = WHOLE ? Range{0, 0} : whole_range(l.p.own);
  int base = -0x40000000;
  const int nt = (n + STEP - 1) / STEP;
  walk_tiles(nt, [&](int t, auto at) {
    constexpr bool end = decltype(at)::value == kTileLast;
    const int buf = t & 1, kt = t * STEP + part * kBiasBN;      // (the wave's tile)
    if (!end) load_tile(t * STEP + STEP);
    bool in_window = true;
    if (!WHOLE) {
      const Range tile = whole_range(l.p.range[buf]);
      const int lo = mine.lo - tile.hi, hi = mine.hi - tile.lo;
      in_window = hi - lo < kWindow - 3;
      if (in_window && (lo < base || hi >= base + kWindow)) {
        base = max(hi - kWindow + 4, 0) & ~3;
        win0 = lds_address(win) + 2 * (load_window<THREADS>(a.m, h, base, kWindow, win, l.row) - base);
        __syncthreads();
      }
    }
    if (wave_live && (SPLIT == 1 || !end || kt < n)) {
      const __bf16 *A = &l.A[buf][part * kBiasBN * RS], *B = &l.B[buf][part * kBiasBN * RS];
      const int* pos = &l.p.pos[buf][part * kBiasBN];
#pragma unroll
      for (int sb = 0; sb < 2; ++sb) {
        bf16x8 kf[KK], vf[KK];
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) {
          const int at_row = (sb * 32 + l32) * RS + kk * 16 + hh * 8;
          kf[kk] = *reinterpret_cast<const bf16x8*>(&A[at_row]);
          vf[kk] = *reinterpret_cast<const bf16x8*>(&B[at_row]);
        }
        uint32_t raw[16];
        read_bias<1>(raw, &pos[sb * 32], own, win0, WHOLE || in_window, a.m, h, hh);
        floatx16 s, dp = negD;
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = 0.f;
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) {
          s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[kk], qf[kk], s, 0, 0, 0);
          dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[kk], dof[kk], dp, 0, 0, 0);
        }
        add_bias(s, raw, a.scale);
        if (end) {
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if (kt + sb * 32 + acc_row(r, hh) >= n) s[r] = -INFINITY;
        }
        if (!far) {
#pragma unroll
          for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], kLog2e, -lse2));
        } else {
          const float ref = lse2 == INFINITY ? INFINITY : lse;
#pragma unroll
          for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f((s[r] - ref) * kLog2e);
        }
#pragma unroll
        for (int mf = 0; mf < 2; ++mf) {
          floatx8 f;
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            f[j] = s[8 * mf + j] * dp[8 * mf + j];
            left += f[j];
            most = __builtin_elementwise_maximum(most, fabsf(f[j]));
          }
          const bf16x8 dsb = float_to_bf16x8(f);
#pragma unroll
          for (int d = 0; d < DB; ++d)
            acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(transposed_frag_rowmajor<RS>(A, d, sb * 32, mf, lane), dsb, acc[d], 0, 0, 0);
        }
      }
    }
    if (!end) {
      store_tile(buf ^ 1, std::bool_constant<decltype(at)::value == kTileBeforeLast>{});
      __syncthreads();
    }
  });
  v_most = __builtin_bit_cast(float, wave_pick<true>((int)(__builtin_bit_cast(uint32_t, v_most) & 0x7fffffffu)));
  if (lane == 0) s_most[0][threadIdx.x >> 6] = v_most;
  __syncthreads();                                            // (and every wave is past its last read of the tiles)
  if constexpr (SPLIT > 1) {
    constexpr int W = DB * 16 + 2;
    static_assert(4 * W * kWave * sizeof(float) <= sizeof(l.B), "the sums of four waves");
    float* other = reinterpret_cast<float*>(&l.B[0][0]) + wv * W * kWave + lane;
    if (part == 1) {
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) other[(d * 16 + r) * kWave] = acc[d][r];
      other[(W - 2) * kWave] = left;
      other[(W - 1) * kWave] = most;
    }
    __syncthreads();
    if (part == 0) {
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[d][r] += other[(d * 16 + r) * kWave];
      left += other[(W - 2) * kWave];
      most = __builtin_elementwise_maximum(most, other[(W - 1) * kWave]);
    }
  }
  left = sum_across_halves(left);
  if (part == 0) {
    store_rows<DH>(acc, a.scale, a.dq + q_row * a.dqs + h * DH, q_ok, hh);
    if (q_ok && hh == 0) a.dvec[h * a.lse_stride + q_row] = D + left;
  }
  // |dS| of the other launch: of this one, plus what D moves by, plus what the order of Dh products in dP can make (at most
  // Dh U sum|dO V| in either launch)
#pragma unroll
  for (int w = 0; w < THREADS / kWave; ++w) v_most = __builtin_elementwise_maximum(v_most, s_most[0][w]);
  const float bound = q_ok && part == 0 ? most + fabsf(left) + l1 * v_most * 0x1p-16f : 0.f;
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
  int img[kLptMaxB], len[kLptMaxB], upto[kLptMaxB];           // by rank; blocks up to and including the rank's
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
    for (int i = 0; i < B; ++i) rank += k.upto[i] > mine || (k.upto[i] == mine && i < b);
    k.img[rank] = b;
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
  int img, at;
  if (B > kLptMaxB) {
    img = i / kblk;
    at = i % kblk;
  } else {
    int lo = 0, hi = B - 1;                                   // the first rank with upto > i
    while (lo < hi) {
      const int mid = (lo + hi) / 2;
      if (k.upto[mid] > i) hi = mid;
      else lo = mid + 1;
    }
    img = k.img[lo];
    at = i - (lo > 0 ? k.upto[lo - 1] : 0);
  }
  img = __builtin_amdgcn_readfirstlane(img);
  const int from = cu[img];
  return {from, cu[img + 1] - from, __builtin_amdgcn_readfirstlane(at) * rows};
}

// The scale of a head's integers: 2^e is above twice what the dq launch found (its blocks that exist); `unit` NaN: some dS of
// the head is not a finite number.  All threads call it.
struct DsScale {
  int e;
  double factor;
  float unit;
};
template <int THREADS>
__device__ __forceinline__ DsScale ds_scale(const uint32_t* most_h, const int32_t* cu, int B, int nblk, uint32_t* s_most) {
  uint32_t most = 0;
  for (int i = threadIdx.x; i < B * nblk; i += THREADS) {
    const int img = i / nblk;
    if ((i - img * nblk) * kBiasRows < cu[img + 1] - cu[img]) most = max(most, most_h[i]);
  }
  most = (uint32_t)wave_pick<true>((int)most);
  if ((threadIdx.x & 63) == 0) s_most[threadIdx.x >> 6] = most;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < THREADS / kWave; ++w) most = max(most, s_most[w]);
  const int e = __builtin_amdgcn_readfirstlane((int)(most >> 23) - 126 + 1);
  const bool bad = most >= 0x7f800000u || e > 126;
  return {e, bad ? 0. : power_of_two(kDsBits - e), bad ? NAN : 0.f};
}
// A workgroup's histogram of offsets from .. from + slice of its head, as fp32; all threads call it, behind the last add.
template <int THREADS>
__device__ __forceinline__ void write_partial(const unsigned long long* hist, const DsScale& s, int slice, int from, int offsets, float* out) {
  __syncthreads();
  const double quantum = power_of_two(s.e - kDsBits);
  for (int i = threadIdx.x; i < min(slice, offsets - from); i += THREADS) out[from + i] = s.unit + (float)((double)(long long)hist[i] * quantum);
  __syncthreads();
}

template <int DH, int SPLIT>
struct DkdvTiles {
  static constexpr int RS = DH + 8;
  __attribute__((aligned(16))) __bf16 Q[2][kBiasBN * RS];
  __attribute__((aligned(16))) __bf16 G[2][kBiasBN * RS];     // dO
  __attribute__((aligned(16))) float lse[2][kBiasBN];         // +inf: no score, or no row (probability 0)
  __attribute__((aligned(16))) float lse2[2][kBiasBN];        // times log2 e
  __attribute__((aligned(16))) float negD[2][kBiasBN];
  __attribute__((aligned(16))) int pos[2][kBiasBN];
  int range[2][2], far[2];
  int own[4][2];
  uint32_t most[4 * SPLIT];
  uint16_t row[kTableLds];
  KeyBlocks blocks;
};

// SPLIT 2: the waves come twice, the second four take the second half of every tile of 64 queries, and hand their sums to the
// first at the end of a block.
template <int DH, int SPLIT, bool WHOLE, int HIST>
__global__ void __launch_bounds__(kBiasThreads * SPLIT) attn_bias_dkdv_kernel(const BiasBwd<__bf16> a) {
  constexpr int RS = DH + 8, KK = DH / 16, DB = DH / 32, BN = kBiasBN, THREADS = kBiasThreads * SPLIT, ROWS = kBiasRows;
  constexpr bool RANGES = !WHOLE || HIST == kHistSlices;      // the offsets of a tile lie where?
  extern __shared__ __attribute__((aligned(16))) unsigned long long hist[];       // [slice], then the window of biases
  __shared__ DkdvTiles<DH, SPLIT> l;
  const int h = blockIdx.x % a.H, group = blockIdx.x / a.H;
  const int tid = threadIdx.x, lane = tid & 63, wv = (tid >> 6) & 3, l32 = lane & 31, hh = lane >> 5;
  const int part = SPLIT > 1 ? __builtin_amdgcn_readfirstlane(tid >> 8) : 0;
  const bool stages = part == 0;                              // (the first four waves)
  const long C = (long)a.H * DH;
  uint16_t* win = reinterpret_cast<uint16_t*>(hist + (HIST != kHistNone ? a.slice : 0));
  const float* lse_h = a.lse + h * a.lse_stride;
  const float* d_h = a.dvec + h * a.lse_stride;

  list_key_blocks<THREADS>(l.blocks, a.cu, a.B, ROWS, a.kblk);
  DsScale scale = {0, 0., 0.f};
  if (HIST != kHistNone) scale = ds_scale<THREADS>(a.most + (long)h * a.B * a.nblk, a.cu, a.B, a.nblk, l.most);
  int win0 = lds_address(win);                                // where offset 0 would lie
  if (WHOLE) win0 += 2 * load_window<THREADS>(a.m, h, 0, a.m.offsets, win, l.row);

  const int passes = HIST == kHistSlices ? (a.m.offsets + a.slice - 1) / a.slice : 1;
  for (int pass = 0; pass < passes; ++pass) {
    const int from = HIST == kHistSlices ? pass * a.slice : 0;
    if (HIST != kHistNone) {
      for (int i = tid; i < a.slice; i += THREADS) hist[i] = 0;
      // (in front of the first add there is the barrier behind a block's first tile)
    }
    for (int round = 0;; ++round) {
      const int item = round * a.groups + (round & 1 ? a.groups - 1 - group : group);
      if (item >= l.blocks.all) break;
      const KeyBlock kb = key_block(l.blocks, a.cu, a.B, ROWS, a.kblk, item);
      if (kb.k0 >= kb.n) continue;
      const int n = kb.n, last = n - 1, ki = kb.k0 + wv * 32 + l32;
      const bool wave_live = kb.k0 + wv * 32 < n, k_ok = ki < n;
      const long k_row = kb.row0 + min(ki, last);
      PairStage<DH, kBiasThreads, BN, false, false> st(tid);
      st.gi = nullptr;
      st.last = last;
      st.source(0, a.q + h * DH, a.qs, kb.row0);
      st.source(1, a.dout + h * DH, C, kb.row0);
      const BiasTokens tokens(a.m, a.cu, kb.row0);
      int token = 0, token_j = 0;
      float lse_t = 0.f, d_t = 0.f;
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
          l.lse[buf][tid] = none ? INFINITY : lse_t;
          l.lse2[buf][tid] = none ? INFINITY : lse_t * kLog2e;
          l.negD[buf][tid] = -d_t;
          const int p = tokens.position(a.m, token, token_j) + a.m.centre;
          l.pos[buf][tid] = 2 * p;
          const bool any = __ballot(!none && fabsf(lse_t) >= kFarScore) != 0;
          const int lo = RANGES ? wave_pick<false>(p) : 0, hi = RANGES ? wave_pick<true>(p) : 0;
          if (tid == 0) {
            l.range[buf][0] = lo;
            l.range[buf][1] = hi;
            l.far[buf] = any;
          }
        }
      };
      load_tile(0);
      bf16x8 kf[KK], vf[KK];
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) {
        const int col = h * DH + kk * 16 + hh * 8;
        kf[kk] = *reinterpret_cast<const bf16x8*>(a.k + k_row * a.ks + col);
        vf[kk] = *reinterpret_cast<const bf16x8*>(a.v + k_row * a.vs + col);
      }
      const int own = tokens.position(a.m, min(ki, last));
      __syncthreads();                                        // every wave is past its last read of the tiles before
      if (RANGES) {
        const int lo = wave_pick<false>(own), hi = wave_pick<true>(own);
        if (lane == 0 && part == 0) {
          l.own[wv][0] = lo;
          l.own[wv][1] = hi;
        }
      }
      floatx16 dka[DB], dva[DB];
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) dka[d][r] = dva[d][r] = 0.f;
      store_tile(0, 0, std::true_type{});
      __syncthreads();
      Range mine = {0, 0};
      if (RANGES) {
        mine = whole_range(l.own);
      }
      int base = -0x40000000;
      const int nt = (n + BN - 1) / BN;
      for (int t = 0; t < nt; ++t) {
        const int buf = t & 1, qt = t * BN;
        const bool end = t + 1 == nt;
        if (!end) load_tile(qt + BN);
        bool in_window = true, adds = HIST != kHistNone, inside = true;
        if (RANGES) {
          const int lo = __builtin_amdgcn_readfirstlane(l.range[buf][0] - mine.hi);
          const int hi = __builtin_amdgcn_readfirstlane(l.range[buf][1] - mine.lo);
          if (!WHOLE) {
            in_window = hi - lo < kWindow - 3;
            if (in_window && (lo < base || hi >= base + kWindow)) {   // the queries' positions grow, so do the offsets
              base = lo & ~3;
              win0 = lds_address(win) + 2 * (load_window<THREADS>(a.m, h, base, kWindow, win, l.row) - base);
              __syncthreads();
            }
          }
          if (HIST == kHistSlices) {
            adds = hi >= from && lo < from + a.slice;
            inside = lo >= from && hi < from + a.slice;
          }
        }
        if (wave_live && (pass == 0 || adds)) {
          const bool far = __builtin_amdgcn_readfirstlane(l.far[buf]) != 0;
#pragma unroll
          for (int half = 0; half < 2 / SPLIT; ++half) {
            const int sb = SPLIT > 1 ? part : half;
            bf16x8 qf[KK], gf[KK];
#pragma unroll
            for (int kk = 0; kk < KK; ++kk) {
              const int at_row = (sb * 32 + l32) * RS + kk * 16 + hh * 8;
              qf[kk] = *reinterpret_cast<const bf16x8*>(&l.Q[buf][at_row]);
              gf[kk] = *reinterpret_cast<const bf16x8*>(&l.G[buf][at_row]);
            }
            const int* pos2 = &l.pos[buf][sb * 32];
            uint32_t raw[16];
            read_bias<-1>(raw, pos2, own, win0, WHOLE || in_window, a.m, h, hh);
            floatx16 s, dp;
#pragma unroll
            for (int g = 0; g < 4; ++g) {
              const floatx4 d4 = *reinterpret_cast<const floatx4*>(&l.negD[buf][sb * 32 + 8 * g + 4 * hh]);
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                dp[4 * g + i] = d4[i];
                s[4 * g + i] = 0.f;
              }
            }
#pragma unroll
            for (int kk = 0; kk < KK; ++kk) {
              s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qf[kk], kf[kk], s, 0, 0, 0);
              dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(gf[kk], vf[kk], dp, 0, 0, 0);
            }
            add_bias(s, raw, a.scale);
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
#pragma unroll
                for (int i = 0; i < 4; ++i) s[4 * g + i] = __builtin_amdgcn_exp2f((s[4 * g + i] - l4[i]) * kLog2e);
              }
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) dp[r] *= s[r];
            if (pass == 0) {
#pragma unroll
              for (int mf = 0; mf < 2; ++mf) {
                floatx8 fp, fd;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                  fp[j] = s[8 * mf + j];
                  fd[j] = dp[8 * mf + j];
                }
                const bf16x8 pb = float_to_bf16x8(fp), dsb = float_to_bf16x8(fd);
#pragma unroll
                for (int d = 0; d < DB; ++d) {
                  dva[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(transposed_frag_rowmajor<RS>(l.G[buf], d, sb * 32, mf, lane), pb, dva[d], 0, 0, 0);
                  dka[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(transposed_frag_rowmajor<RS>(l.Q[buf], d, sb * 32, mf, lane), dsb, dka[d], 0, 0, 0);
                }
              }
            }
            if (HIST != kHistNone && adds && k_ok) {
              const int to = lds_address(hist) - 8 * (own + from);          // (four times twice a position: 8 bytes an offset)
#pragma unroll
              for (int g = 0; g < 4; ++g) {
                const intx4 p2 = *reinterpret_cast<const intx4*>(&pos2[8 * g + 4 * hh]);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                  const unsigned long long v = ds_integer(dp[4 * g + i], scale.factor);
                  if (HIST == kHistWhole || inside) lds_add(p2[i] * 4 + to, v);
                  else if ((unsigned)((p2[i] >> 1) - own - from) < (unsigned)a.slice) lds_add(p2[i] * 4 + to, v);
                }
              }
            }
          }
        }
        if (!end) {
          if (t + 2 == nt) store_tile(buf ^ 1, qt + BN, std::true_type{});
          else store_tile(buf ^ 1, qt + BN, std::false_type{});
          __syncthreads();
        }
      }
      if (pass == 0) {
        if constexpr (SPLIT > 1) {
          static_assert(4 * DB * 16 * kWave * sizeof(float) <= sizeof(l.Q) + sizeof(l.G), "one sum of four waves");
          float* other = reinterpret_cast<float*>(&l.Q[0][0]) + wv * DB * 16 * kWave + lane;
#pragma unroll
          for (int which = 0; which < 2; ++which) {
            floatx16(&sum)[DB] = which == 0 ? dka : dva;
            __syncthreads();                                  // every wave is past its last read of the tiles, or of the sums before
            if (part == 1) {
#pragma unroll
              for (int d = 0; d < DB; ++d)
#pragma unroll
                for (int r = 0; r < 16; ++r) other[(d * 16 + r) * kWave] = sum[d][r];
            }
            __syncthreads();
            if (part == 0) {
#pragma unroll
              for (int d = 0; d < DB; ++d)
#pragma unroll
                for (int r = 0; r < 16; ++r) sum[d][r] += other[(d * 16 + r) * kWave];
            }
          }
        }
        if (part == 0) {
          store_rows<DH>(dka, a.scale, a.dk + k_row * a.dks + h * DH, k_ok, hh);
          store_rows<DH>(dva, 1.0f, a.dv + k_row * a.dvs + h * DH, k_ok, hh);
        }
      }
    }
    if (HIST != kHistNone) write_partial<THREADS>(hist, scale, a.slice, from, a.m.offsets, a.partial + ((long)h * a.groups + group) * a.m.offsets);
  }
}

// The sums over the workgroups, in their order: 64 offsets a workgroup, four slices of the rows beside each other.
struct BiasSum {
  const float* partial;
  int groups, offsets;
  float* sums;                    // [H][offsets]
};
__global__ void __launch_bounds__(256) attn_bias_sum_kernel(const BiasSum a) {
  __shared__ double s[4][64];
  const int h = blockIdx.y, c = threadIdx.x & 63, sl = threadIdx.x >> 6, o = blockIdx.x * 64 + c;
  double v = 0.;
  if (o < a.offsets) {
    const float* p = a.partial + (long)h * a.groups * a.offsets + o;
    constexpr int U = 8;
    for (int g0 = sl; g0 < a.groups; g0 += 4 * U) {
      float f[U];
#pragma unroll
      for (int u = 0; u < U; ++u) f[u] = g0 + 4 * u < a.groups ? p[(long)(g0 + 4 * u) * a.offsets] : 0.f;
#pragma unroll
      for (int u = 0; u < U; ++u) v += (double)f[u];
    }
  }
  s[sl][c] = v;
  __syncthreads();
  if (sl == 0 && o < a.offsets) a.sums[(long)h * a.offsets + o] = (float)((s[0][c] + s[1][c]) + (s[2][c] + s[3][c]));
}

// The sums of the offsets into those of their buckets, with integers again, of 2^-40 of the power of two above the largest: a
// workgroup has kTableBuckets buckets of a head in LDS and goes over all offsets.
constexpr int kTableBuckets = 4096;
struct BiasTable {
  const float* sums;
  const int32_t* buckets;
  int nb, offsets;
  float* d_table;
};
__global__ void __launch_bounds__(1024) attn_bias_table_kernel(const BiasTable a) {
  __shared__ unsigned long long s[kTableBuckets];
  __shared__ uint32_t s_most[16];
  const int h = blockIdx.y, b0 = blockIdx.x * kTableBuckets, nb = min(kTableBuckets, a.nb - b0);
  const float* sums = a.sums + (long)h * a.offsets;
  uint32_t most = 0;
  for (int i = threadIdx.x; i < a.offsets; i += 1024) most = max(most, __builtin_bit_cast(uint32_t, sums[i]) & 0x7fffffffu);
  most = (uint32_t)wave_pick<true>((int)most);
  if ((threadIdx.x & 63) == 0) s_most[threadIdx.x >> 6] = most;
  for (int i = threadIdx.x; i < nb; i += 1024) s[i] = 0;
  __syncthreads();
  for (int w = 0; w < 16; ++w) most = max(most, s_most[w]);
  const bool bad = most >= 0x7f800000u;
  const int bits = min(40, 62 - (32 - __builtin_clz(a.offsets))), e = (int)(most >> 23) - 126;
  if (!bad)
    for (int i = threadIdx.x; i < a.offsets; i += 1024) {
      const int b = a.buckets[i] - b0;
      const float v = sums[i];
      if ((unsigned)b < (unsigned)nb && v != 0.f) atomicAdd(&s[b], ds_integer(v, power_of_two(bits - e)));
    }
  __syncthreads();
  for (int i = threadIdx.x; i < nb; i += 1024)
    a.d_table[(long)h * a.nb + b0 + i] = bad ? NAN : (float)((double)(long long)s[i] * power_of_two(e - bits));
}

// ------------------------------------------------------------------------------- fp32 backward
// One thread per row, the other side streaming through LDS: the queries (dq, D, and what no |dS| exceeds), then the keys.
__device__ __forceinline__ float block_most(float v, float* s) {           // largest of the 128 threads' (a NaN above all)
  const int b = wave_pick<true>((int)(__builtin_bit_cast(uint32_t, v) & 0x7fffffffu));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = __builtin_bit_cast(float, b);
  __syncthreads();
  return __builtin_elementwise_maximum(s[0], s[1]);
}
template <int DH>
__global__ void __launch_bounds__(kRowThreads) attn_bias_dq_rows_kernel(const BiasBwd<float> a) {
  __shared__ float Ks[kRowTile * DH], Vs[kRowTile * DH], s_most[2];
  __shared__ int pos[kRowTile];
  const int h = blockIdx.y, r0 = blockIdx.x * kRowThreads;
  const long row0 = a.cu[blockIdx.z], C = (long)a.H * DH;
  const int n = (int)(a.cu[blockIdx.z + 1] - row0);
  if (r0 >= n) return;
  const int ri = r0 + threadIdx.x;
  const bool ok = ri < n;
  const long row = row0 + (ok ? ri : 0);
  float q[DH], g[DH], acc[DH], D = 0.f, l1 = 0.f;
#pragma unroll
  for (int d = 0; d < DH; ++d) {
    q[d] = a.q[row * a.qs + h * DH + d];
    g[d] = a.dout[row * C + h * DH + d];
    D = fmaf(g[d], a.out[row * C + h * DH + d], D);
    l1 += fabsf(g[d]);
    acc[d] = 0.f;
  }
  const BiasTokens tokens(a.m, a.cu, row0);
  const int p = tokens.position(a.m, ok ? ri : 0) + a.m.centre;
  const float l = a.lse[h * a.lse_stride + row];
  float left = 0.f, most = 0.f, v_most = 0.f;
  for (int t = 0; t < n; t += kRowTile) {
    __syncthreads();
    stage_rows<float, DH>(a.k + h * DH, a.ks, a.v + h * DH, a.vs, row0, t, n, Ks, Vs);
    if (threadIdx.x < kRowTile && t + threadIdx.x < n) pos[threadIdx.x] = tokens.position(a.m, t + threadIdx.x);
    __syncthreads();
    for (int i = threadIdx.x; i < kRowTile * DH; i += kRowThreads) v_most = __builtin_elementwise_maximum(v_most, fabsf(Vs[i]));
    const int tn = min(kRowTile, n - t);
    for (int j = 0; j < tn; ++j) {
      float s = 0.f, dp = 0.f;
#pragma unroll
      for (int d = 0; d < DH; ++d) {
        s = fmaf(q[d], Ks[j * DH + d], s);
        dp = fmaf(g[d], Vs[j * DH + d], dp);
      }
      const float pr = l == -INFINITY ? 0.f : expf(fmaf(s, a.scale, bias_at<float>(a.m, h, p - pos[j])) - l);   // (a row without a score)
      const float ds = pr * (dp - D);
      left += ds;
      most = __builtin_elementwise_maximum(most, fabsf(ds));
#pragma unroll
      for (int d = 0; d < DH; ++d) acc[d] = fmaf(ds, Ks[j * DH + d], acc[d]);
    }
  }
  v_most = block_most(v_most, s_most);
  most = block_most(ok ? most + fabsf(left) + l1 * v_most * 0x1p-16f : 0.f, s_most);
  if (threadIdx.x == 0)
    a.most[((long)h * a.B + blockIdx.z) * a.nblk + blockIdx.x] = __builtin_bit_cast(uint32_t, most) & 0x7fffffffu;
  if (!ok) return;
  a.dvec[h * a.lse_stride + row] = D + left;
#pragma unroll
  for (int d = 0; d < DH; ++d) a.dq[row * a.dqs + h * DH + d] = acc[d] * a.scale;
}

template <int DH, bool HIST>
__global__ void __launch_bounds__(kRowThreads) attn_bias_dkdv_rows_kernel(const BiasBwd<float> a) {
  extern __shared__ __attribute__((aligned(16))) unsigned long long hist[];
  __shared__ float Qs[kRowTile * DH], Gs[kRowTile * DH], lses[kRowTile], Ds[kRowTile];
  __shared__ int pos[kRowTile];
  __shared__ uint32_t s_most[kRowThreads / kWave];
  __shared__ KeyBlocks blocks;
  const int h = blockIdx.x % a.H, group = blockIdx.x / a.H;
  const long C = (long)a.H * DH;
  list_key_blocks<kRowThreads>(blocks, a.cu, a.B, kRowThreads, a.kblk);
  DsScale scale = {0, 0., 0.f};
  if (HIST) scale = ds_scale<kRowThreads>(a.most + (long)h * a.B * a.nblk, a.cu, a.B, a.nblk, s_most);
  const int passes = HIST ? (a.m.offsets + a.slice - 1) / a.slice : 1;
  for (int pass = 0; pass < passes; ++pass) {
    const int from = pass * a.slice;
    if (HIST)
      for (int i = threadIdx.x; i < a.slice; i += kRowThreads) hist[i] = 0;
    for (int round = 0;; ++round) {
      const int item = round * a.groups + (round & 1 ? a.groups - 1 - group : group);
      if (item >= blocks.all) break;
      const KeyBlock kb = key_block(blocks, a.cu, a.B, kRowThreads, a.kblk, item);
      if (kb.k0 >= kb.n) continue;
      const int ki = kb.k0 + threadIdx.x;
      const bool ok = ki < kb.n;
      const long row = kb.row0 + (ok ? ki : 0);
      float k[DH], v[DH], dk[DH], dv[DH];
#pragma unroll
      for (int d = 0; d < DH; ++d) {
        k[d] = a.k[row * a.ks + h * DH + d];
        v[d] = a.v[row * a.vs + h * DH + d];
        dk[d] = dv[d] = 0.f;
      }
      const BiasTokens tokens(a.m, a.cu, kb.row0);
      const int p = tokens.position(a.m, ok ? ki : 0) - a.m.centre;
      for (int t = 0; t < kb.n; t += kRowTile) {
        __syncthreads();
        stage_rows<float, DH>(a.q + h * DH, a.qs, a.dout + h * DH, C, kb.row0, t, kb.n, Qs, Gs);
        if (threadIdx.x < kRowTile && t + threadIdx.x < kb.n) {
          const long r = kb.row0 + t + threadIdx.x;
          pos[threadIdx.x] = tokens.position(a.m, t + threadIdx.x);
          lses[threadIdx.x] = a.lse[h * a.lse_stride + r];
          Ds[threadIdx.x] = a.dvec[h * a.lse_stride + r];
        }
        __syncthreads();
        const int tn = min(kRowTile, kb.n - t);
        for (int j = 0; j < tn; ++j) {
          const int o = pos[j] - p;
          const bool adds = HIST && ok && (unsigned)(o - from) < (unsigned)a.slice;
          if (pass > 0 && __ballot(adds) == 0) continue;
          float s = 0.f, dp = 0.f;
#pragma unroll
          for (int d = 0; d < DH; ++d) {
            s = fmaf(k[d], Qs[j * DH + d], s);
            dp = fmaf(v[d], Gs[j * DH + d], dp);
          }
          const float pr = lses[j] == -INFINITY ? 0.f : expf(fmaf(s, a.scale, bias_at<float>(a.m, h, o)) - lses[j]);
          const float ds = pr * (dp - Ds[j]);
          if (adds) lds_add(lds_address(hist) + 8 * (o - from), ds_integer(ds, scale.factor));
          if (pass > 0) continue;
#pragma unroll
          for (int d = 0; d < DH; ++d) {
            dk[d] = fmaf(ds, Qs[j * DH + d], dk[d]);
            dv[d] = fmaf(pr, Gs[j * DH + d], dv[d]);
          }
        }
      }
      if (pass > 0 || !ok) continue;
#pragma unroll
      for (int d = 0; d < DH; ++d) {
        a.dk[row * a.dks + h * DH + d] = dk[d] * a.scale;
        a.dv[row * a.dvs + h * DH + d] = dv[d];
      }
    }
    if (HIST) write_partial<kRowThreads>(hist, scale, a.slice, from, a.m.offsets, a.partial + ((long)h * a.groups + group) * a.m.offsets);
  }
}

// ------------------------------------------------------------------------------- host
constexpr long kMostOffsets = 1L << 26;
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

// LDS of a window of that many offsets: it may start up to 7 entries into its first 16 bytes
static size_t window_bytes(int offsets) { return ((size_t)offsets + 7 + 7) / 8 * 16; }
#define SPA_BIAS_LAUNCH(KERNEL, GRID, THREADS, LDS, ARGS)                                                                              \
  do {                                                                                                                        \
    const hipError_t attr = hipFuncSetAttribute((const void*)KERNEL, hipFuncAttributeMaxDynamicSharedMemorySize, (int)(LDS)); \
    SPA_REQUIRE(attr == hipSuccess, SPA_ERR_HIP, "%s: cannot reserve %zu bytes of LDS", fn, (size_t)(LDS));                   \
    hipLaunchKernelGGL(KERNEL, dim3(GRID), dim3(THREADS), LDS, st, ARGS);                                                     \
  } while (0)
static size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }

// Forward and dq: eight waves a block (SPLIT) where a unit has one block at most and segments may have several tiles; a block is
// then a chain of half the steps.  us forward, four | eight waves, 3 heads of 32, 56 x 56 map: one image of 1792 tokens
// 33.6 | 26.0, 512 12.3 | 10.6; 16 images of 1792 63 | 77, of 512 13.8 | 13.9.
static bool few_blocks(int nblk, int H, int B) { return nblk >= 4 && xcd_grid(nblk, H, B) <= 256; }

// The dk / dv launch of the backward.  Two workgroups a unit where that leaves each room for the whole map in LDS (10 bytes an
// offset); else one, with as much of the histogram as fits.  As many workgroups a head as are resident together, no more than
// there are blocks of keys, and no more than 256 MB of partial sums.
struct BiasPlan {
  int split, slice, groups, kblk;
  size_t lds;
};
static BiasPlan bias_plan(int H, int B, int n_max, int Dh, long offsets, int dtype) {
  BiasPlan p = {};
  const bool whole = offsets <= kWholeMost;
  const size_t window = window_bytes((int)(whole ? offsets : kWindow)), most = 160 * 1024;
  const size_t tiles = Dh == 32 ? sizeof(DkdvTiles<32, 2>) : sizeof(DkdvTiles<64, 2>);
  const auto up64 = [](long n) { return (n + 63) & ~63L; };
  int a_unit = 2;
  p.split = 1;
  if (dtype == SPA_F32) {
    p.slice = (int)std::min<long>(up64(offsets), 4096);
    p.lds = (size_t)p.slice * 8;
  } else if (tiles + window + up64(offsets) * 8 <= most / 2) {
    p.slice = (int)up64(offsets);
    p.lds = window + (size_t)p.slice * 8;
  } else {
    a_unit = 1;
    p.split = whole ? 2 : 1;                                    // (eight waves with look-ups in memory: too few registers)
    p.slice = (int)std::min<long>(up64(offsets), (long)(most - tiles - window) / 8 / 64 * 64);
    p.lds = window + (size_t)p.slice * 8;
  }
  p.kblk = (n_max + kBiasRows - 1) / kBiasRows;
  const long fit = std::max<long>(1, (256L << 20) / (4 * H * offsets));
  p.groups = (int)std::max<long>(1, std::min<long>(std::min<long>(256 * a_unit / H, (long)B * p.kblk), fit));
  return p;
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
  const float scale = softmax_scale > 0.f ? softmax_scale : 1.0f / std::sqrt((float)Dh);
  const long ls = (long)B * max_seqlen;
  hipStream_t st = as_stream(stream);
  if (dtype == SPA_BF16) {
    const int nblk = (max_seqlen + kBiasRows - 1) / kBiasRows;
    SPA_REQUIRE(((long)H * B + 8) * nblk < 2147483647L, SPA_ERR_INVALID_ARG, "%s: B*H*blocks must be < 2^31", fn);
    const BiasFwd args = {(const __bf16*)q, (const __bf16*)k, (const __bf16*)v, (long)q_row_stride, (long)k_row_stride, (long)v_row_stride,
                          cu_seqlens, m, H, B, nblk, scale, (__bf16*)out, lse, ls};
    const dim3 blocks(xcd_grid(nblk, H, B));
    const bool split = few_blocks(nblk, H, B);
#define SPA_BIAS(D)                                                                                                        \
  do {                                                                                                                     \
    const size_t window = window_bytes(m.offsets <= kWholeMost ? m.offsets : kWindow);                                     \
    if (m.offsets > kWholeMost) SPA_BIAS_LAUNCH((attn_bias_fwd_kernel<D, false, 1>), blocks, kBiasThreads, window, args);  \
    else if (split) SPA_BIAS_LAUNCH((attn_bias_fwd_kernel<D, true, 2>), blocks, 2 * kBiasThreads, window, args);           \
    else SPA_BIAS_LAUNCH((attn_bias_fwd_kernel<D, true, 1>), blocks, kBiasThreads, window, args);                          \
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
  if (B < 1 || max_seqlen < 1 || H < 1 || grid_h < 1 || grid_w < 1 || (2 * (long)grid_h - 1) * (2 * (long)grid_w - 1) > kMostOffsets) return 0;
  const long offsets = (2 * (long)grid_h - 1) * (2 * (long)grid_w - 1);
  const BiasPlan p = bias_plan(H, B, max_seqlen, Dh, offsets, dtype);
  const size_t nblk = (max_seqlen + kBiasRows - 1) / kBiasRows;
  return up256((size_t)H * B * max_seqlen * 4) + up256((size_t)H * B * nblk * 4) + up256((size_t)H * p.groups * offsets * 4) +
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
  const BiasPlan plan = bias_plan(H, B, max_seqlen, Dh, m.offsets, dtype);
  const int nblk = (max_seqlen + kBiasRows - 1) / kBiasRows;
  SPA_REQUIRE(((long)H * B + 8) * nblk < 2147483647L, SPA_ERR_INVALID_ARG, "%s: B*H*blocks must be < 2^31", fn);
  char* ws = static_cast<char*>(workspace);
  auto take = [&](size_t bytes) {
    char* at = ws;
    ws += up256(bytes);
    return at;
  };
  float* dvec = reinterpret_cast<float*>(take((size_t)H * ls * 4));
  uint32_t* most = reinterpret_cast<uint32_t*>(take((size_t)H * B * nblk * 4));
  float* partial = reinterpret_cast<float*>(take((size_t)H * plan.groups * m.offsets * 4));
  float* sums = buckets != nullptr ? reinterpret_cast<float*>(take((size_t)H * m.offsets * 4)) : d_table;
  hipStream_t st = as_stream(stream);
  const bool hist = d_table != nullptr, whole = m.offsets <= kWholeMost;
  const size_t window = window_bytes(whole ? m.offsets : kWindow);
#define SPA_ARGS(T)                                                                                                          \
  {(const T*)q, (const T*)k, (const T*)v, (const T*)out, (const T*)dout, (long)q_row_stride, (long)k_row_stride, (long)v_row_stride, lse, \
   dvec, ls, cu_seqlens, m, H, B, nblk, scale, (T*)dq, (T*)dk, (T*)dv, (long)dq_row_stride, (long)dk_row_stride, (long)dv_row_stride,     \
   most, partial, plan.groups, plan.slice, plan.kblk}
  const bool split = few_blocks(nblk, H, B);
#define SPA_DKDV(D, SPLIT, W, MODE) \
  SPA_BIAS_LAUNCH((attn_bias_dkdv_kernel<D, SPLIT, W, MODE>), H * plan.groups, SPLIT * kBiasThreads, hist ? plan.lds : window, args)
#define SPA_BIAS16(D)                                                                                                        \
  do {                                                                                                                       \
    const unsigned blocks = xcd_grid(nblk, H, B);                                                                            \
    if (!whole) SPA_BIAS_LAUNCH((attn_bias_dq_kernel<D, false, 1>), blocks, kBiasThreads, window, args);                     \
    else if (split) SPA_BIAS_LAUNCH((attn_bias_dq_kernel<D, true, 2>), blocks, 2 * kBiasThreads, window, args);              \
    else SPA_BIAS_LAUNCH((attn_bias_dq_kernel<D, true, 1>), blocks, kBiasThreads, window, args);                             \
    if (!whole && hist) SPA_DKDV(D, 1, false, kHistSlices);                                                                  \
    else if (!whole) SPA_DKDV(D, 1, false, kHistNone);                                                                       \
    else if (!hist && plan.split == 2) SPA_DKDV(D, 2, true, kHistNone);                                                      \
    else if (!hist) SPA_DKDV(D, 1, true, kHistNone);                                                                         \
    else if (plan.slice < m.offsets) SPA_DKDV(D, 2, true, kHistSlices);                                                      \
    else if (plan.split == 2) SPA_DKDV(D, 2, true, kHistWhole);                                                              \
    else SPA_DKDV(D, 1, true, kHistWhole);                                                                                   \
  } while (0)
#define SPA_BIAS32(D)                                                                                                        \
  do {                                                                                                                       \
    hipLaunchKernelGGL(attn_bias_dq_rows_kernel<D>, dim3(nblk, H, B), dim3(kRowThreads), 0, st, args);                       \
    if (hist) SPA_BIAS_LAUNCH((attn_bias_dkdv_rows_kernel<D, true>), H * plan.groups, kRowThreads, plan.lds, args);          \
    else hipLaunchKernelGGL((attn_bias_dkdv_rows_kernel<D, false>), dim3(H * plan.groups), dim3(kRowThreads), 0, st, args);  \
  } while (0)
  if (dtype == SPA_F32) {
    const BiasBwd<float> args = SPA_ARGS(float);
    if (Dh == 32) SPA_BIAS32(32); else SPA_BIAS32(64);
  } else {
    const BiasBwd<__bf16> args = SPA_ARGS(__bf16);
    if (Dh == 32) SPA_BIAS16(32); else SPA_BIAS16(64);
  }
#undef SPA_ARGS
#undef SPA_DKDV
#undef SPA_BIAS16
#undef SPA_BIAS32
  if (hist) {
    const BiasSum sum = {partial, plan.groups, m.offsets, sums};
    hipLaunchKernelGGL(attn_bias_sum_kernel, dim3((m.offsets + 63) / 64, H), dim3(256), 0, st, sum);
    if (buckets != nullptr) {
      const BiasTable table_args = {sums, buckets, n_buckets, m.offsets, d_table};
      hipLaunchKernelGGL(attn_bias_table_kernel, dim3((n_buckets + kTableBuckets - 1) / kTableBuckets, H), dim3(1024), 0, st, table_args);
    }
  }
  return check_launch(fn);
}
