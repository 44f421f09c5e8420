// What the attention with a relative position bias shares between its forward and its backward (attention_bias.hip,
// attention_bias_bwd.hip).
#pragma once

#include <type_traits>

#include "attn_tiles.h"
#include "spa_common.h"

namespace spa {

constexpr float kLog2e = 1.4426950408889634f;
// exp(s - m) as exp2(s log2 e - m2), m2 = m log2 e rounded, is off by what that rounding is: half a last place of m2, which at -1e10
// (a mask written into the table) is 2^9, and a row whose first keys are all masked ends as infinity times 0.  Rows whose maximum (lse) is
// this large or more take the difference before the factor, an instruction more a score; below it P is off by at most 2^-17 of itself.
constexpr float kFarScore = 128.f;
// A wave owns 32 rows and a workgroup 128 (eight waves: each row twice, SPLIT 2), the others stream through LDS in tiles of 64.
constexpr int kBiasBN = 64, kBiasThreads = 256, kBiasRows = 128;

// x / d for 0 <= x < 2^31 by one high product: with 2^s >= d > 2^(s-1), M = floor(2^(31+s) / d) + 1 < 2^32 is at most 2^s / d too
// large in units of its last place, which times x is below 2^(31+s) / d: the quotient is exact.  (d = 1: M = 0.)
struct Divisor {
  uint32_t d, M, shift;
};
inline Divisor divisor(uint32_t d) {
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
typedef __attribute__((address_space(3))) float* lds_f32_ptr;
typedef __attribute__((address_space(3))) unsigned long long* lds_u64_ptr;
__device__ __forceinline__ int lds_address(const void* p) { return (int)(uintptr_t)(__attribute__((address_space(3))) const char*)p; }
__device__ __forceinline__ void lds_add(int address, unsigned long long v) {
  __hip_atomic_fetch_add((lds_u64_ptr)(uint32_t)address, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
}

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

// BT rows of one head of two operands on their way to LDS, in 16-byte pieces.  Nothing here waits for a load or branches on one between
// load() and store(); rows past the segment's end are loaded as its last row, and store<true>() clears operand 1's (the caller
// gives such rows probability 0, and 0 times an infinity of the last row would be NaN).
template <typename T, int DH, int THREADS, int BT>
struct RowPair {
  static constexpr int RS = Ops<T, DH>::RS, VE = 16 / sizeof(T), CPR = DH / VE, CPT = BT * CPR / THREADS, RPP = THREADS / CPR;
  static_assert(BT * CPR % THREADS == 0, "whole passes");
  const int tid;
  uintx4 v[2][CPT];
  const char* base[2];
  uint32_t stride[2];            // bytes
  int last, from;
  __device__ __forceinline__ RowPair(int tid_, const T* a, long as, const T* b, long bs, long row0, int last_) : tid(tid_), last(last_), from(0) {
    base[0] = reinterpret_cast<const char*>(a + row0 * as + tid % CPR * VE);
    base[1] = reinterpret_cast<const char*>(b + row0 * bs + tid % CPR * VE);
    stride[0] = (uint32_t)as * (uint32_t)sizeof(T);
    stride[1] = (uint32_t)bs * (uint32_t)sizeof(T);
  }
  __device__ __forceinline__ int row(int t) const { return tid / CPR + t * RPP; }
  __device__ __forceinline__ void load(int t0) {
    from = t0;
#pragma unroll
    for (int t = 0; t < CPT; ++t) {
      const uint64_t r = (uint32_t)min(t0 + row(t), last);
      v[0][t] = *reinterpret_cast<const uintx4*>(base[0] + r * stride[0]);
      v[1][t] = *reinterpret_cast<const uintx4*>(base[1] + r * stride[1]);
    }
  }
  template <bool LAST>
  __device__ __forceinline__ void store(T* a, T* b) {
#pragma unroll
    for (int t = 0; t < CPT; ++t) {
      if (LAST && from + row(t) > last) v[1][t] = uintx4{0, 0, 0, 0};
      const int o = row(t) * RS + tid % CPR * VE;
      *reinterpret_cast<uintx4*>(a + o) = v[0][t];
      *reinterpret_cast<uintx4*>(b + o) = v[1][t];
    }
  }
  // the largest magnitude of operand 1's pieces (a NaN stays one)
  __device__ __forceinline__ float most(float m) const {
#pragma unroll
    for (int t = 0; t < CPT; ++t) {
      float f[VE];
      if constexpr (VE == 8) {
        const floatx8 w = bf16x8_to_float(__builtin_bit_cast(bf16x8, v[1][t]));
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = w[e];
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) f[e] = __builtin_bit_cast(float, v[1][t][e]);
      }
#pragma unroll
      for (int e = 0; e < VE; ++e) m = __builtin_elementwise_maximum(m, fabsf(f[e]));
    }
    return m;
  }
};

// ---- the window of biases in LDS, in the table's type, and how a score's bias is found.
//   kWinWhole: all offsets of the map.
//   kWinMoving: kWindow neighbouring offsets.  The offsets between the workgroup's rows and a tile's are a narrow range that
//     moves steadily with the tiles, as packed rows are in the order of their positions: the window is loaded anew where a tile
//     leaves it.  A tile whose offsets exceed the window (few tokens far apart, rows in another order) looks each bias up in memory.
enum WinMode { kWinWhole, kWinMoving };
constexpr int kWholeBytes = 65536, kWindow = 8192;

constexpr int kTableLds = 1024;                // a table row of up to so many entries is brought to LDS where a map picks from it

// The entries of offsets [base, base + n) on their way to the window, 16 bytes of the map (four entries; base must be a
// multiple of 4 then) or, without a map, of the table's row a time.  start() asks for a thread's first pieces and, of a short row
// that a map picks from, its part of the row; nothing waits for them before finish(), which all threads call; a barrier follows
// before the window is read.  (Asked for where the window is filled instead, behind the first rows: forward of 64 images of 196 tokens,
// 12 heads of 64, 18.6 -> 20.2 us.)
template <typename T, int THREADS>
struct WindowFill {
  using Raw = std::conditional_t<sizeof(T) == 4, uint32_t, uint16_t>;
  static constexpr int VE = 16 / sizeof(T), U = 4, PART = (kTableLds + THREADS - 1) / THREADS;
  const BiasMap& m;
  const Raw* row;
  const int tid;
  int base, n, shift, first, pieces;         // shift: where the row starts in its first 16 bytes, first: entries in front of the next
  intx4 v[U];
  Raw part[PART];
  uintx2 ends;                                // what is in front of the first whole piece and behind the last, of the thread
  __device__ __forceinline__ WindowFill(const BiasMap& m_, int h)
      : m(m_), row(static_cast<const Raw*>(m_.table) + (long)h * m_.nb), tid(threadIdx.x), base(0), n(0), shift(0), first(0), pieces(0) {}
  __device__ __forceinline__ void load(int p0) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int p = min(p0 + tid + u * THREADS, pieces - 1);
      v[u] = m.buckets == nullptr ? *reinterpret_cast<const intx4*>(row + base + first + VE * p)
                                  : *reinterpret_cast<const intx4*>(m.buckets + base + 4 * p);
    }
  }
  __device__ __forceinline__ int behind() const { return first + (m.buckets == nullptr ? VE : 4) * pieces + tid; }      // the last whole piece
  __device__ __forceinline__ void start(int base_, int n_) {
    base = base_;
    n = n_;
    if (m.buckets == nullptr) {
      shift = (int)(reinterpret_cast<uintptr_t>(row + base) & 15) / (int)sizeof(T);
      first = (VE - shift) & (VE - 1);
      pieces = n > first ? (n - first) / VE : 0;
      ends[0] = row[base + min(tid, n - 1)];
      ends[1] = row[base + min(behind(), n - 1)];
    } else {
      pieces = n / 4;
      ends[1] = (uint32_t)m.buckets[base + min(behind(), n - 1)];
      if (m.nb <= kTableLds) {
#pragma unroll
        for (int i = 0; i < PART; ++i) part[i] = row[min(tid + i * THREADS, m.nb - 1)];
      }
    }
    if (pieces > 0) load(0);
  }
  // the LDS address that offset 0 would have
  __device__ __forceinline__ int finish(void* window, Raw* row_lds) {
    Raw* win = static_cast<Raw*>(window);
    auto each = [&](auto put) {
      for (int p0 = 0; p0 < pieces; p0 += U * THREADS) {
        if (p0 > 0) load(p0);
        put(p0);
      }
    };
    if (m.buckets == nullptr) {
      each([&](int p0) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int p = p0 + tid + u * THREADS;
          if (p < pieces) *reinterpret_cast<intx4*>(win + shift + first + VE * p) = v[u];
        }
      });
      if (tid < min(first, n)) win[shift + tid] = (Raw)ends[0];
      if (tid < VE && behind() < n) win[shift + behind()] = (Raw)ends[1];
    } else {
      auto pick = [&](const Raw* from) {                      // (all of a thread's look-ups in flight)
        auto entry = [&](int b) -> uint32_t {
          const uint32_t e = from[min((uint32_t)b, (uint32_t)m.nb - 1)];
          return (uint32_t)b < (uint32_t)m.nb ? e : 0u;
        };
        each([&](int p0) {
          uint32_t e[U][4];
#pragma unroll
          for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i) e[u][i] = entry(v[u][i]);
#pragma unroll
          for (int u = 0; u < U; ++u) {
            const int p = p0 + tid + u * THREADS;
            if (p >= pieces) continue;
            if constexpr (sizeof(T) == 4) *reinterpret_cast<uintx4*>(win + 4 * p) = uintx4{e[u][0], e[u][1], e[u][2], e[u][3]};
            else *reinterpret_cast<uintx2*>(win + 4 * p) = uintx2{e[u][0] | e[u][1] << 16, e[u][2] | e[u][3] << 16};
          }
        });
        if (tid < 4 && behind() < n) win[behind()] = (Raw)entry((int)ends[1]);
      };
      if (m.nb <= kTableLds) {
#pragma unroll
        for (int i = 0; i < PART; ++i)
          if (tid + i * THREADS < m.nb) row_lds[tid + i * THREADS] = part[i];
        __syncthreads();
        pick(row_lds);
      } else {
        pick(row);
      }
    }
    return lds_address(win) + (int)sizeof(T) * (shift - base);
  }
};

// Scores of a lane's row against the 16 of a 32-row block that it holds, biases included.  pos: positions of the block's rows
// in bytes of the window, own: position of the lane's row, one of the two with the centre; SIGN: 1 if the offset is own - pos,
// else pos - own.  a, b: the rows of the block and the lane's row.
template <typename T, int DH, int WIN, int SIGN>
__device__ __forceinline__ void bias_scores(floatx16& s, const typename Ops<T, DH>::Row& a, const typename Ops<T, DH>::Row& b, const int* pos,
                                            int own, int zero, bool in_window, const BiasMap& m, int h, float scale, int hh) {
  constexpr int WB = sizeof(T);
  const int from = zero + SIGN * WB * own;
  float bias[16];
  auto each = [&](auto entry) {
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const intx4 p = *reinterpret_cast<const intx4*>(&pos[8 * g + 4 * hh]);
#pragma unroll
      for (int e = 0; e < 4; ++e) bias[4 * g + e] = entry(p[e]);
    }
  };
  if (WIN == kWinWhole || in_window)
    each([&](int p) {
      const uint32_t at = (uint32_t)(from - SIGN * p);
      if constexpr (WB == 4) return *(lds_f32_ptr)at;
      else return __builtin_bit_cast(float, (uint32_t)*(lds_u16_ptr)at << 16);
    });
  else
    each([&](int p) { return bias_at<T>(m, h, SIGN * (own - p / WB)); });
#pragma unroll
  for (int r = 0; r < 16; ++r) s[r] = 0.f;
  Ops<T, DH>::dot(s, a, b);
#pragma unroll
  for (int r = 0; r < 16; ++r) s[r] = fmaf(s[r], scale, bias[r]);
}

// ---- positions of the streamed rows
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
// A wave's smallest and largest position
__device__ __forceinline__ void put_range(int (&to)[2], int p) {
  const int lo = wave_pick<false>(p), hi = wave_pick<true>(p);
  if ((threadIdx.x & 63) == 0) {
    to[0] = lo;
    to[1] = hi;
  }
}

// The workgroup's block: (segment, head, rows from r0), longest segments first where they can be ranked.
struct BiasBlock {
  Segment seg;
  int img, h, r0;
  bool valid;
};
__device__ __forceinline__ BiasBlock bias_block(int* s_live, const int32_t* cu, int H, int B, int nblk) {
  // there and back: a unit that got a long block in one turn of the XCD's 32 units gets a short one in the next (us forward,
  // four waves a block, there alone | there and back: 16 images of 0.1 - 0.6 of 3136 tokens, 3 heads of 32, 38.9 | 37.2; 8 of 0.05 - 0.4 of 4200,
  // 8 heads, 32.7 | 31.2)
  const int xcd = blockIdx.x & 7, turn = blockIdx.x >> 3 & ~31, width = min(32, (int)(gridDim.x >> 3) - turn);
  const int at = blockIdx.x >> 3 & 31, j = turn + (turn & 32 ? width - 1 - at : at);
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

// What a workgroup that owns 128 queries and walks the keys has in LDS (beside the window).
template <typename T, int DH, int SPLIT>
struct QueryTiles {
  static constexpr int RS = Ops<T, DH>::RS, STEP = kBiasBN * SPLIT;
  __attribute__((aligned(16))) T K[2][STEP * RS];
  __attribute__((aligned(16))) T V[2][STEP * RS];
  __attribute__((aligned(16))) int pos[2][STEP];
  int range[2][SPLIT][2], own[4 * SPLIT][2];
  typename WindowFill<T, kBiasThreads>::Raw row[kTableLds];
  int s_live[sizeof(LiveTile) / sizeof(int)];
};

// The walk of such a workgroup over the keys of its segment, SPLIT tiles of 64 a step: staging, positions, the window.
// asked(): the workgroup's own loads; arrived(): what is made of them in front of the first tile; work(K, V, pos,
// rows left in the wave's tile, own position, window, in_window, whole): the wave's tile; whole: all of its 64 keys exist.
template <typename T, int DH, int WIN, int SPLIT, class Asked, class Arrived, class Staged, class Work>
__device__ __forceinline__ void walk_keys(QueryTiles<T, DH, SPLIT>& l, void* win, const Segment& seg, int h, bool wave_live,
                                          const T* k, long ks, const T* v, long vs, const BiasMap& m, const int32_t* cu, int row, Asked asked, Arrived arrived,
                                          Staged staged, Work work) {
  constexpr int RS = Ops<T, DH>::RS, THREADS = kBiasThreads * SPLIT, STEP = kBiasBN * SPLIT, WB = sizeof(T);
  const int tid = threadIdx.x, n = seg.nk, last = n - 1, part = SPLIT > 1 ? __builtin_amdgcn_readfirstlane(tid >> 8) : 0;
  RowPair<T, DH, THREADS, STEP> st(tid, k + h * DH, ks, v + h * DH, vs, seg.row0, last);
  const BiasTokens tokens(m, cu, seg.row0);
  int token = 0, token_j = 0;
  auto load = [&](int t0) {
    st.load(t0);
    token_j = min(t0 + (tid & (STEP - 1)), last);
    token = tokens.load(token_j);
  };
  auto store = [&](int buf, auto clear) {
    st.template store<clear>(l.K[buf], l.V[buf]);
    staged(st);
    if (tid < STEP) {
      const int p = tokens.position(m, token, token_j);
      l.pos[buf][tid] = WB * p;
      if (WIN == kWinMoving) put_range(l.range[buf][(tid >> 6) & (SPLIT - 1)], p);
    }
  };
  WindowFill<T, THREADS> fill(m, h);
  if (WIN == kWinWhole) fill.start(0, m.offsets);             // (what the longer chains of loads begin with, first)
  const int own_token = tokens.load(min(row, last));
  load(0);
  asked();
  const int own = tokens.position(m, own_token, min(row, last)) + m.centre;
  int zero = 0;
  if (WIN == kWinWhole) zero = fill.finish(win, l.row);
  else put_range(l.own[tid >> 6], own);
  arrived();
  store(0, std::true_type{});
  __syncthreads();
  const Range mine = WIN == kWinMoving ? whole_range(l.own) : Range{0, 0};
  int base = -0x40000000;                                     // (no window yet)
  walk_tiles((n + STEP - 1) / STEP, [&](int t, auto at) {
    constexpr bool end = decltype(at)::value == kTileLast;
    const int buf = t & 1, left = n - t * STEP - part * kBiasBN;
    if (!end) load(t * STEP + STEP);
    bool in_window = true;
    if (WIN == kWinMoving) {
      const Range tile = whole_range(l.range[buf]);
      const int lo = mine.lo - tile.hi, hi = mine.hi - tile.lo;
      in_window = hi - lo < kWindow - 3;
      if (in_window && (lo < base || hi >= base + kWindow)) {  // the keys' positions grow, so the next offsets are lower
        base = max(hi - kWindow + 4, 0) & ~3;                 // (16-byte pieces of the map)
        fill.start(base, min(kWindow, m.offsets - base));
        zero = fill.finish(win, l.row);
        __syncthreads();
      }
    }
    if (wave_live && (SPLIT == 1 || !end || left > 0))
      work(&l.K[buf][part * kBiasBN * RS], &l.V[buf][part * kBiasBN * RS], &l.pos[buf][part * kBiasBN], left, own, zero, in_window,
           std::bool_constant<!end>{});
    if (!end) store(buf ^ 1, std::bool_constant<decltype(at)::value == kTileBeforeLast>{});
    __syncthreads();
  });
}

// ---- host
int bias_checks(const char* fn, const void* q, const void* k, const void* v, int64_t q_stride, int64_t k_stride, int64_t v_stride,
                const int32_t* cu, int B, int n_max, int H, int Dh, int dtype, float softmax_scale, const void* table,
                const int32_t* buckets, int n_buckets, const int32_t* gather_idx, int grid_h, int grid_w, BiasMap* m);
constexpr long kMostOffsets = 1L << 26;
// LDS of a window of that many offsets: a bf16 one may start up to 7 entries into its first 16 bytes
inline size_t window_bytes(int offsets, int each) { return ((size_t)offsets + 7 + 7) / 8 * 8 * each; }
// Eight waves a block (SPLIT) where a unit has one block at most and segments may have several tiles; a block is then a chain of half
// the steps.  us forward / backward, four | eight waves, 3 heads of 32, 56 x 56 map: one image of 1792 tokens 37.0 / 110 | 26.4 / 100, of 512
// 13.4 / 44.7 | 11.2 / 42.5; 64 images of 196 19.5 / 57.5 | 26.5 / 83.0.
inline bool few_blocks(int nblk, int H, int B) { return nblk >= 4 && xcd_grid(nblk, H, B) <= 256; }
// The kernel's limit of LDS is all that its own arrays (OWN bytes) leave, one value whatever the call: threads that launch with other maps set
// it too, and a launch must not find a smaller one.
constexpr size_t kUnitLds = 160 * 1024;
#define SPA_BIAS_LAUNCH(KERNEL, OWN, GRID, THREADS, LDS, ARGS)                                                                 \
  do {                                                                                                                        \
    constexpr size_t room = kUnitLds - (OWN);                                                                                 \
    const hipError_t attr = hipFuncSetAttribute((const void*)KERNEL, hipFuncAttributeMaxDynamicSharedMemorySize, (int)room);  \
    SPA_REQUIRE(attr == hipSuccess && (LDS) <= room, SPA_ERR_HIP, "%s: cannot reserve %zu bytes of LDS", fn, (size_t)(LDS));  \
    hipLaunchKernelGGL(KERNEL, dim3(GRID), dim3(THREADS), LDS, st, ARGS);                                                     \
  } while (0)
// KERNEL<type, head dim, window, SPLIT> of a launch whose workgroups own queries; EIGHT: whether a block has eight waves
template <typename T, int DH, int SPLIT>
constexpr size_t kQueryLds = sizeof(QueryTiles<T, DH, SPLIT>) + 256;             // (what a kernel has beside the tiles is less)
#define SPA_QUERY_LAUNCH(KERNEL, T, D, EIGHT, ARGS)                                                                           \
  do {                                                                                                                        \
    const bool whole = m.offsets <= kWholeBytes / (int)sizeof(T);                                                             \
    const size_t lds = window_bytes(whole ? m.offsets : kWindow, sizeof(T));                                                  \
    const unsigned blocks = xcd_grid(nblk, H, B);                                                                             \
    if (!whole) {                                                                                                             \
      SPA_BIAS_LAUNCH((KERNEL<T, D, kWinMoving, 1>), (kQueryLds<T, D, 1>), blocks, kBiasThreads, lds, ARGS);                  \
    } else {                                                                                                                  \
      if constexpr (sizeof(T) == 2)                                                                                           \
        if (EIGHT) {                                                                                                          \
          SPA_BIAS_LAUNCH((KERNEL<T, D, kWinWhole, 2>), (kQueryLds<T, D, 2>), blocks, 2 * kBiasThreads, lds, ARGS);           \
          break;                                                                                                              \
        }                                                                                                                     \
      SPA_BIAS_LAUNCH((KERNEL<T, D, kWinWhole, 1>), (kQueryLds<T, D, 1>), blocks, kBiasThreads, lds, ARGS);                   \
    }                                                                                                                         \
  } while (0)

}  // namespace spa
