// Tiles of fp32 products for the projections of small fp32 workloads (linear.hip, linear_bwd.hip, gated_linear.hip): every element is one chain of fused multiply-adds in
// the order of the contraction, whatever the tile, so that neither its size nor the rest of the call touches an element's bits.
// 256 threads have EDGE x EDGE elements; both operands of a step of the contraction are in LDS, the next step's on their way in registers, eight loads of each operand a thread
// (with steps of 16 a step of a small tile waits 0.8 us for its loads).
#pragma once

#include <type_traits>

#include "spa_common.h"

namespace spa {

constexpr int kF32Threads = 256;
template <int EDGE> constexpr int kF32Step = 2048 / EDGE;       // contraction elements of a step

// Which element of an operand's step thread t fetches as its i-th: LINES: the contraction runs along the operand's rows in memory
// (a step's neighbouring elements for neighbouring lanes), else down them (EDGE neighbouring lanes take EDGE of a row).
template <int EDGE, bool LINES>
struct F32Place {
  static constexpr int STEP = kF32Step<EDGE>, kCount = EDGE * STEP / kF32Threads;
  static __device__ __forceinline__ int line(int i) { return LINES ? threadIdx.x / STEP + kF32Threads / STEP * i : threadIdx.x & (EDGE - 1); }
  static __device__ __forceinline__ int k(int i) { return LINES ? threadIdx.x & (STEP - 1) : threadIdx.x / EDGE + kF32Threads / EDGE * i; }
};
// (a thread's TM neighbours are one read: 8 bytes of 32-element tiles, 16 of 64; writes of neighbouring steps fall on few banks twice)
template <int EDGE> constexpr int kF32Row = EDGE + EDGE / 16;
template <int EDGE, int NB>
struct F32Lds {
  __attribute__((aligned(16))) float a[2][kF32Step<EDGE>][kF32Row<EDGE>];
  __attribute__((aligned(16))) float b[2][NB][kF32Step<EDGE>][kF32Row<EDGE>];
};

template <int N>
__device__ __forceinline__ void read_floats(const float* p, float (&v)[N]) {
  static_assert(N == 2 || N == 4, "one read");
  if constexpr (N == 2) {
    const floatx2 w = *reinterpret_cast<const floatx2*>(p);
    v[0] = w[0], v[1] = w[1];
  } else {
    const floatx4 w = *reinterpret_cast<const floatx4*>(p);
    v[0] = w[0], v[1] = w[1], v[2] = w[2], v[3] = w[3];
  }
}
struct F32Nothing {
  __device__ __forceinline__ void operator()(int) const {}
};
// acc[q][r][c] += sum over k in order of A(ty TM + r, k) B_q(tx TM + c, k).  fetch_a(i, k), fetch_b(q, i, k): the thread's i-th element of the step as it lies
// in memory, at contraction index k < kc (clamped; what is past kc is replaced by 0); done_a(i, v), done_b(q, i, v): what is made of it, when it is there (nothing may
// ask for a value before, or it waits in front of the products: the weight side of 1750 rows 135 us instead of 106, and 64 with its indices ahead).  beside(a): the step's A in LDS, behind its products.  ahead(k0): called a
// step before the fetches from k0 on, for what these need of memory themselves.
template <int EDGE, int NB, bool A_LINES, bool B_LINES, class FA, class FB, class DA, class DB, class BS, class AH = F32Nothing>
__device__ __forceinline__ void f32_tile_sums(F32Lds<EDGE, NB>& l, int kc, FA&& fetch_a, FB&& fetch_b, DA&& done_a, DB&& done_b,
                                              float (&acc)[NB][EDGE / 16][EDGE / 16], BS&& beside, AH&& ahead = AH{}) {
  using PA = F32Place<EDGE, A_LINES>;
  using PB = F32Place<EDGE, B_LINES>;
  constexpr int TM = EDGE / 16, STEP = kF32Step<EDGE>;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4, steps = (kc + STEP - 1) / STEP;
  float ra[PA::kCount], rb[NB][PB::kCount];
  auto load = [&](int k0) {
#pragma unroll
    for (int i = 0; i < PA::kCount; ++i) ra[i] = fetch_a(i, min(k0 + PA::k(i), kc - 1));
#pragma unroll
    for (int q = 0; q < NB; ++q)
#pragma unroll
      for (int i = 0; i < PB::kCount; ++i) rb[q][i] = fetch_b(q, i, min(k0 + PB::k(i), kc - 1));
  };
  if (steps > 0) {
    ahead(0);
    load(0);
    ahead(STEP);
  }
  for (int s = 0; s < steps; ++s) {
    const int buf = s & 1;
#pragma unroll
    for (int i = 0; i < PA::kCount; ++i) l.a[buf][PA::k(i)][PA::line(i)] = s * STEP + PA::k(i) < kc ? done_a(i, ra[i]) : 0.f;
#pragma unroll
    for (int q = 0; q < NB; ++q)
#pragma unroll
      for (int i = 0; i < PB::kCount; ++i) l.b[buf][q][PB::k(i)][PB::line(i)] = s * STEP + PB::k(i) < kc ? done_b(q, i, rb[q][i]) : 0.f;
    __syncthreads();                                          // (a buffer is written again two steps on, behind the barrier between)
    if (s + 1 < steps) {
      load((s + 1) * STEP);
      ahead((s + 2) * STEP);
    }
    const int ks = min(STEP, kc - s * STEP);
    // G contraction elements at a time, the reads of the next ones in front of the products of these (left to itself the compiler reads, waits
    // and multiplies in turn: twice the time)
    constexpr int G = 16 / TM / NB;
    struct Operands {
      float a[G][TM], b[G][NB][TM];
    };
    auto read = [&](Operands& o, int kk) {
#pragma unroll
      for (int j = 0; j < G; ++j) {
        read_floats<TM>(&l.a[buf][kk + j][ty * TM], o.a[j]);
#pragma unroll
        for (int q = 0; q < NB; ++q) read_floats<TM>(&l.b[buf][q][kk + j][tx * TM], o.b[j][q]);
      }
    };
    auto products = [&](const Operands& o, int n) {
#pragma unroll
      for (int j = 0; j < G; ++j)
        if (j < n) {                                          // (a product of zeros would make -0 of a sum 0)
#pragma unroll
          for (int q = 0; q < NB; ++q)
#pragma unroll
            for (int r = 0; r < TM; ++r)
#pragma unroll
              for (int c = 0; c < TM; ++c) acc[q][r][c] = fmaf(o.a[j][r], o.b[j][q][c], acc[q][r][c]);
        }
    };
    Operands o[2];
    read(o[0], 0);
    if (ks == STEP) {
#pragma unroll
      for (int g = 0; g < STEP / G; ++g) {
        if (g + 1 < STEP / G) read(o[(g + 1) & 1], (g + 1) * G);
        __builtin_amdgcn_sched_barrier(0);
        products(o[g & 1], G);
        __builtin_amdgcn_sched_barrier(0);
      }
    } else {
      for (int kk = 0; kk < ks; kk += G) {
        if (kk > 0) read(o[0], kk);
        if (kk + G <= ks) products(o[0], G);
        else products(o[0], ks - kk);
      }
    }
    beside(l.a[buf], ks);
  }
}
struct F32AsIs {
  __device__ __forceinline__ float operator()(int, float v) const { return v; }
  __device__ __forceinline__ float operator()(int, int, float v) const { return v; }
};
// The larger tiles where there are enough of them for all units.
inline bool f32_wide(long rows, long cols) { return ((rows + 63) / 64) * ((cols + 63) / 64) >= 512; }
inline long f32_tiles(long rows, long cols, int edge) { return ((rows + edge - 1) / edge) * ((cols + edge - 1) / edge); }

}  // namespace spa
