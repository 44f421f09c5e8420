// Tiles of fp32 products for the projections of small fp32 workloads (linear.hip, linear_bwd.hip, gated_linear.hip): every element is one
// chain of fused multiply-adds in the order of the contraction, whatever the tile, so that neither its size nor the rest of the call
// touches an element's bits (the weight side adds up chains of 1024 rows).
// Four waves have a quarter each of EDGE x EDGE elements, in fp32 matrix instructions, whose products are that chain (checked bit for bit,
// with denormals, infinities and zeros of either sign; 1000 rows of 1400 -> 1000 108 us in vector instructions, 53 so).  Both operands of a
// step of the contraction are in LDS, those of the next steps on their way in registers, eight loads of each operand a thread.
#pragma once

#include <type_traits>

#include "f32_shape.h"
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
template <int EDGE> constexpr int kF32Row = EDGE + EDGE / 16;
template <int EDGE, int NB>
struct F32Lds {
  __attribute__((aligned(16))) float a[2][kF32Step<EDGE>][kF32Row<EDGE>];
  __attribute__((aligned(16))) float b[2][NB][kF32Step<EDGE>][kF32Row<EDGE>];
};

// The quarter of a tile that a wave has, of one fp32 matrix instruction (16x16x4 or 32x32x2): element e of a lane, and which of KD
// neighbouring contraction elements a lane hands to it.  The instruction is a chain of fused multiply-adds in the order of its contraction
// elements.
template <int EDGE>
struct F32Quarter {
  static constexpr int Q = EDGE / 2, KD = Q == 16 ? 4 : 2, kCount = Q * Q / 64;
  typedef float Acc __attribute__((ext_vector_type(kCount)));
  static __device__ __forceinline__ int lane() { return threadIdx.x & 63; }
  static __device__ __forceinline__ int line_a() { return (threadIdx.x >> 7) * Q + lane() % Q; }
  static __device__ __forceinline__ int line_b() { return (threadIdx.x >> 6 & 1) * Q + lane() % Q; }
  static __device__ __forceinline__ int k() { return lane() / Q; }
  static __device__ __forceinline__ int row(int e) { return (threadIdx.x >> 7) * Q + (Q == 16 ? 4 * k() + e : e / 4 * 8 + 4 * k() + e % 4); }
  static __device__ __forceinline__ int col() { return line_b(); }
  static __device__ __forceinline__ Acc mul(float a, float b, const Acc& c) {
    if constexpr (Q == 16) return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0);
  }
};
struct F32Nothing {
  __device__ __forceinline__ void operator()(int) const {}
};
// acc[q] of row m and column n += sum over k in order of A(m, k) B_q(n, k).  fetch_a(i, k), fetch_b(q, i, k): the thread's i-th element of
// the step as it lies in memory, at contraction index k < kc (clamped; what is past kc is replaced by zeros whose product is -0, which
// leaves any sum as it is); done_a(i, v), done_b(q, i, v): what is made of it, when it is there (nothing may ask for a value before, or it
// waits in front of the products).  beside(a): the step's A in LDS, behind its products.  ahead(k0): called a step before the fetches from
// k0 on, for what these need of memory themselves.  DEPTH: steps whose loads are under way.
template <int EDGE, int NB, bool A_LINES, bool B_LINES, int DEPTH, class FA, class FB, class DA, class DB, class BS, class AH = F32Nothing>
__device__ __forceinline__ void f32_tile_sums(F32Lds<EDGE, NB>& l, int kc, FA&& fetch_a, FB&& fetch_b, DA&& done_a, DB&& done_b,
                                              typename F32Quarter<EDGE>::Acc (&acc)[NB], BS&& beside, AH&& ahead = AH{}) {
  using PA = F32Place<EDGE, A_LINES>;
  using PB = F32Place<EDGE, B_LINES>;
  using W = F32Quarter<EDGE>;
  constexpr int STEP = kF32Step<EDGE>, G = 4, GROUPS = STEP / (G * W::KD);
  const int steps = f32_steps(kc, STEP), la = W::line_a(), lb = W::line_b(), lk = W::k();
  float ra[DEPTH][PA::kCount], rb[DEPTH][NB][PB::kCount];
  auto load = [&](float (&a)[PA::kCount], float (&b)[NB][PB::kCount], int k0) {
#pragma unroll
    for (int i = 0; i < PA::kCount; ++i) a[i] = fetch_a(i, f32_at(k0, PA::k(i), kc));
#pragma unroll
    for (int q = 0; q < NB; ++q)
#pragma unroll
      for (int i = 0; i < PB::kCount; ++i) b[q][i] = fetch_b(q, i, f32_at(k0, PB::k(i), kc));
  };
  if (steps > 0) {
    ahead(0);
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) {
      load(ra[d], rb[d], min(d, steps - 1) * STEP);
      ahead(min(d + 1, steps - 1) * STEP);
    }
  }
  // left: contraction elements from the step's first on; in the last turn possibly none
  auto step = [&](int s, int left, int buf, float (&fa)[PA::kCount], float (&fb)[NB][PB::kCount]) {
#pragma unroll
    for (int i = 0; i < PA::kCount; ++i) l.a[buf][PA::k(i)][PA::line(i)] = PA::k(i) < left ? done_a(i, fa[i]) : 0.f;
#pragma unroll
    for (int q = 0; q < NB; ++q)
#pragma unroll
      for (int i = 0; i < PB::kCount; ++i) l.b[buf][q][PB::k(i)][PB::line(i)] = PB::k(i) < left ? done_b(q, i, fb[q][i]) : -0.f;
    __syncthreads();                                          // (a buffer is written again two steps on, behind the barrier between)
    load(fa, fb, min(s + DEPTH, steps - 1) * STEP);           // (past the end the last again: a branch here would have the compiler wait for all loads)
    ahead(min(s + DEPTH + 1, steps - 1) * STEP);
    const int ks = min(STEP, left);
    // the reads of the next instructions in front of these (left to itself the compiler reads, waits and multiplies in turn)
    struct Operands {
      float a[G], b[NB][G];
    };
    auto read = [&](Operands& o, int g) {
#pragma unroll
      for (int j = 0; j < G; ++j) {
        const int k = (g * G + j) * W::KD + lk;
        o.a[j] = l.a[buf][k][la];
#pragma unroll
        for (int q = 0; q < NB; ++q) o.b[q][j] = l.b[buf][q][k][lb];
      }
    };
    Operands o[2];
    read(o[0], 0);
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
      if (g * G * W::KD >= ks) break;
      if (g + 1 < GROUPS) read(o[(g + 1) & 1], g + 1);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int j = 0; j < G; ++j)
#pragma unroll
        for (int q = 0; q < NB; ++q) acc[q] = W::mul(o[g & 1].a[j], o[g & 1].b[q][j], acc[q]);
      __builtin_amdgcn_sched_barrier(0);
    }
    beside(l.a[buf], ks);
  };
  static_assert(DEPTH == 1 || DEPTH % 2 == 0, "a step's buffer follows from its place in a turn");
  int left = kc;
  for (int s0 = 0; s0 < steps; s0 += DEPTH)
#pragma unroll
    for (int d = 0; d < DEPTH; ++d, left -= STEP) step(s0 + d, left, DEPTH == 1 ? s0 & 1 : d & 1, ra[d], rb[d]);
}
struct F32AsIs {
  __device__ __forceinline__ float operator()(int, float v) const { return v; }
  __device__ __forceinline__ float operator()(int, int, float v) const { return v; }
};

}  // namespace spa
