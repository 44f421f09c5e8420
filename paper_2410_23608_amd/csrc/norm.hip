// The norms in front of and behind a block on packed tokens, with what stands beside them on the way: the gather into packed
// order, and the scatter back onto the residual stream with the residual scale and the token's gate.
//   in front:  a_j = gamma * xh_i + beta, i = gather_idx[j]           xh = (x - mu) r,  r = 1 / sqrt(var + eps)
//   behind:    y_i = res_i + p_i scale * (gamma * zh_j + beta)        (RMS: mu = 0, var = mean x^2),  p = Sigmoid(score)
// and their backward.  With g the gradient of the normed row xh,
//   dx = r (g - mean(g) - xh mean(g xh))                              (RMS: without mean(g))
// All of it is bound by memory: every row is read once and kept in registers (both moments of a row come from there, the
// variance after the mean), G lanes a row, IT chunks of 16 bytes a lane.  Parameter gradients are sums over all rows of
//   A = sum p dy * zh,  B = sum p dy      (in front: da for p dy), from which
//   dgamma = scale * A,  dbeta = scale * B,  dscale = gamma * A + beta * B
// follow; every workgroup adds its rows and writes one partial row, a second launch adds those in a fixed order, all of it in fp32.
// us a launch, TB/s of the bytes it cannot do without (a large copy: 4.6), eight batches in turn so that no rows are left in a
// cache: 134400 bf16 rows of 256, 22 % of them packed, in front 11.0 (2.8) and its backward 33.6 (5.0), behind 34.8 (4.4); 12544 of 768, half
// packed, in front 8.3 (2.3) and 17.0 (3.4), behind 16.6 (2.9) and 11.7 (2.5).
// Small ones are trips to memory: launch, index, rows, and for the backward the fold and the sums' launch of 4 us.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "row_groups.h"
#include "spa_common.h"

namespace spa {

constexpr int kNormThreads = 256;
constexpr int kMaxNormC = 8192;
constexpr int kNormMaxParts = 512;

template <typename T, int G, int IT>
struct NormRow {
  static constexpr int VE = Vec16<T>::kElems, kGroups = kNormThreads / G;
  using Raw = typename Raw16<T>::type;
  static __device__ __forceinline__ void load(const T* row, int gl, int chunks, bool ok, Raw (&r)[IT]) {
#pragma unroll
    for (int it = 0; it < IT; ++it) {
      const int ch = gl + it * G;
      r[it] = {};
      if (ok && ch < chunks) r[it] = *reinterpret_cast<const Raw*>(row + ch * VE);
    }
  }
  static __device__ __forceinline__ void store(T* row, int ch, const float (&f)[VE]) {
    Raw r;
    if constexpr (VE == 8) {
      floatx8 v;
#pragma unroll
      for (int e = 0; e < VE; ++e) v[e] = f[e];
      r = float_to_bf16x8(v);
    } else {
#pragma unroll
      for (int e = 0; e < VE; ++e) r[e] = f[e];
    }
    *reinterpret_cast<Raw*>(row + ch * VE) = r;
  }
};

// K sums over the lanes of a row, in each of them.  A row of the whole workgroup (G = 256): the waves exchange through LDS;
// two sets of slots in turn, so that one barrier a call is enough (a thread comes to write a set again only after the
// barrier of the call between, which every reader of the set has reached).
template <int G, int K>
struct RowSums {
  float* slots;        // [2][K][4]
  int turn = 0;
  __device__ __forceinline__ void operator()(float (&v)[K]) {
    if constexpr (G <= kWave) {
#pragma unroll
      for (int k = 0; k < K; ++k) v[k] = group_sum<G>(v[k]);
    } else {
      float* s = slots + turn * K * 4;
      turn ^= 1;
#pragma unroll
      for (int k = 0; k < K; ++k) {
        v[k] = group_sum<kWave>(v[k]);
        if ((threadIdx.x & 63) == 0) s[k * 4 + (threadIdx.x >> 6)] = v[k];
      }
      __syncthreads();
#pragma unroll
      for (int k = 0; k < K; ++k) v[k] = (s[k * 4] + s[k * 4 + 1]) + (s[k * 4 + 2] + s[k * 4 + 3]);
    }
  }
};

// Moments of a row held in raw chunks; xh = (x - mu) r is left to the caller.
template <typename T, int G, int IT, bool RMS, class Sums>
__device__ __forceinline__ void row_moments(const typename Raw16<T>::type (&raw)[IT], int gl, int chunks, float inv_c, float eps,
                                            Sums& sums, float& mu, float& r) {
  constexpr int VE = Vec16<T>::kElems;
  float v[1] = {0.f};
  mu = 0.f;
  if (!RMS) {
#pragma unroll
    for (int it = 0; it < IT; ++it) {
      float f[VE];
      widen(raw[it], f);
#pragma unroll
      for (int e = 0; e < VE; ++e) v[0] += f[e];
    }
    sums(v);
    mu = v[0] * inv_c;
    v[0] = 0.f;
  }
#pragma unroll
  for (int it = 0; it < IT; ++it) {
    float f[VE];
    widen(raw[it], f);
    float part = 0.f;
#pragma unroll
    for (int e = 0; e < VE; ++e) part = fmaf(f[e] - mu, f[e] - mu, part);
    v[0] += gl + it * G < chunks ? part : 0.f;
  }
  sums(v);
  r = 1.0f / sqrtf(fmaf(v[0], inv_c, eps));
}

// ------------------------------------------------------------------------------- forward
template <typename T>
struct NormFwdArgs {
  const T* rows;                  // in front: x at gather_idx; behind: z, packed
  const int32_t *idx, *total;     // in front: gather_idx or null, total or null; behind: inv_pos or null
  const T *gamma, *beta, *scale, *residual;
  const float* gate;
  float eps;
  long n;                         // in front: M_cap; behind: rows of y
  long cap;                       // packed rows there are
  int C;
  T* out;
  float* stats;                   // [2][cap] or null
};

template <typename T, int G, int IT, int U, bool RMS>
__global__ void __launch_bounds__(kNormThreads) norm_packed_kernel(const NormFwdArgs<T> a) {
  using Row = NormRow<T, G, IT>;
  constexpr int VE = Row::VE, kGroups = Row::kGroups;
  __shared__ float slots[8];
  RowSums<G, 1> sums{slots};
  const int grp = threadIdx.x / G, gl = threadIdx.x % G, chunks = a.C / VE;
  const long M = a.total != nullptr ? min((long)max(*a.total, 0), a.n) : a.n;
  const float inv_c = 1.0f / (float)a.C;
  typename Row::Raw gr[IT], br[IT];
  Row::load(a.gamma, gl, chunks, a.gamma != nullptr, gr);
  Row::load(a.beta, gl, chunks, a.beta != nullptr, br);
  const long step = (long)gridDim.x * kGroups * U;
  for (long base = (long)blockIdx.x * kGroups * U; base < M; base += step) {
    typename Row::Raw xr[U][IT];
    long j[U], i[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      j[u] = base + u * kGroups + grp;
      i[u] = min(j[u], M - 1);
      if (a.idx != nullptr) i[u] = a.idx[i[u]];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) Row::load(a.rows + i[u] * a.C, gl, chunks, j[u] < M, xr[u]);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float mu, r;
      row_moments<T, G, IT, RMS>(xr[u], gl, chunks, inv_c, a.eps, sums, mu, r);
      if (j[u] < M) {
        if (a.stats != nullptr && gl == 0) {
          if (!RMS) a.stats[j[u]] = mu;
          a.stats[a.cap + j[u]] = r;
        }
#pragma unroll
        for (int it = 0; it < IT; ++it) {
          const int ch = gl + it * G;
          float x[VE], g[VE], b[VE];
          widen(xr[u][it], x);
          widen(gr[it], g);
          widen(br[it], b);
#pragma unroll
          for (int e = 0; e < VE; ++e) {
            const float h = (x[e] - mu) * r;
            x[e] = fmaf(h, a.gamma != nullptr ? g[e] : 1.f, b[e]);
          }
          if (ch < chunks) Row::store(a.out + j[u] * a.C, ch, x);
        }
      }
    }
  }
}

// Rows of y in place (y == residual): the others keep what they hold.
template <typename T, int G, int IT, int U, bool RMS>
__global__ void __launch_bounds__(kNormThreads) norm_residual_kernel(const NormFwdArgs<T> a) {
  using Row = NormRow<T, G, IT>;
  constexpr int VE = Row::VE, kGroups = Row::kGroups;
  __shared__ float slots[8];
  RowSums<G, 1> sums{slots};
  const int grp = threadIdx.x / G, gl = threadIdx.x % G, chunks = a.C / VE;
  const float inv_c = 1.0f / (float)a.C;
  const bool in_place = a.residual == a.out;
  typename Row::Raw gr[IT], br[IT], sr[IT];
  Row::load(a.gamma, gl, chunks, a.gamma != nullptr, gr);
  Row::load(a.beta, gl, chunks, a.beta != nullptr, br);
  Row::load(a.scale, gl, chunks, a.scale != nullptr, sr);
  const long step = (long)gridDim.x * kGroups * U;
  for (long base = (long)blockIdx.x * kGroups * U; base < a.n; base += step) {
    typename Row::Raw zr[U][IT], rr[U][IT];
    long i[U], j[U];
    float p[U];
    bool sel[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      i[u] = base + u * kGroups + grp;
      const long ic = min(i[u], a.n - 1);
      j[u] = a.idx != nullptr ? (long)a.idx[ic] : ic;
      p[u] = a.gate != nullptr ? a.gate[ic] : 0.f;
      sel[u] = i[u] < a.n && j[u] >= 0 && j[u] < a.cap;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      Row::load(a.residual + i[u] * a.C, gl, chunks, a.residual != nullptr && i[u] < a.n && (sel[u] || !in_place), rr[u]);
      Row::load(a.rows + j[u] * a.C, gl, chunks, sel[u], zr[u]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float mu, r;
      row_moments<T, G, IT, RMS>(zr[u], gl, chunks, inv_c, a.eps, sums, mu, r);
      if (i[u] < a.n && (sel[u] || !in_place)) {
        if (sel[u] && a.stats != nullptr && gl == 0) {
          if (!RMS) a.stats[j[u]] = mu;
          a.stats[a.cap + j[u]] = r;
        }
        const float w = a.gate != nullptr ? sigmoidf_dev(p[u]) : 1.f;
#pragma unroll
        for (int it = 0; it < IT; ++it) {
          const int ch = gl + it * G;
          if (sel[u]) {
            float z[VE], y[VE], g[VE], b[VE], s[VE];
            widen(zr[u][it], z);
            widen(rr[u][it], y);
            widen(gr[it], g);
            widen(br[it], b);
            widen(sr[it], s);
#pragma unroll
            for (int e = 0; e < VE; ++e) {
              const float v = fmaf((z[e] - mu) * r, a.gamma != nullptr ? g[e] : 1.f, b[e]);
              y[e] = fmaf(w * (a.scale != nullptr ? s[e] : 1.f), v, y[e]);
            }
            if (ch < chunks) Row::store(a.out + i[u] * a.C, ch, y);
          } else if (ch < chunks) {
            *reinterpret_cast<typename Row::Raw*>(a.out + i[u] * a.C + ch * VE) = rr[u][it];
          }
        }
      }
    }
  }
}

// ------------------------------------------------------------------------------- backward
template <typename T>
struct NormBwdArgs {
  const T *rows, *grad;                   // in front: x at token positions, da packed; behind: z packed, dy at token positions
  const int32_t *gather_idx, *inv_pos, *total;
  const T *gamma, *beta, *scale, *residual;
  const float *gate, *stats;
  long n;                                 // token rows
  long cap;                               // packed rows there are
  int C;
  T* out;                                 // in front: dx; behind: dz
  float* d_scores;
  float* partial;                         // [parts][2][C]
};

// The workgroup's sums A and B, held by the groups' lanes, as one partial row.  LDS: a row of C floats a wave, A and B in turn.
template <typename T, int G, int IT>
__device__ __forceinline__ void norm_fold(float (&A)[2][IT][Vec16<T>::kElems], int C, float* partial, float* lds) {
  constexpr int VE = Vec16<T>::kElems, kWaves = kNormThreads / kWave;
  const int gl = threadIdx.x % G, chunks = C / VE, wv = threadIdx.x / kWave;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    float* prow = partial + ((long)blockIdx.x * 2 + k) * C;
    if constexpr (G > kWave) {
#pragma unroll
      for (int it = 0; it < IT; ++it) {
        const int ch = gl + it * G;
        if (ch < chunks) {
#pragma unroll
          for (int e = 0; e < VE; ++e) prow[ch * VE + e] = A[k][it][e];
        }
      }
    } else {
      if (k > 0) __syncthreads();
#pragma unroll
      for (int it = 0; it < IT; ++it) {
        const int ch = gl + it * G;
#pragma unroll
        for (int e = 0; e < VE; ++e) {
          if (G <= 8) A[k][it][e] += dpp_move<0x128>(A[k][it][e]);
          if (G <= 16) A[k][it][e] = add_lane_xor16(A[k][it][e]);
          if (G <= 32) A[k][it][e] = add_lane_xor32(A[k][it][e]);
        }
        if ((threadIdx.x & (kWave - 1)) < G && ch < chunks) {
#pragma unroll
          for (int e = 0; e < VE; e += 4)
            *reinterpret_cast<floatx4*>(&lds[wv * C + ch * VE + e]) = floatx4{A[k][it][e], A[k][it][e + 1], A[k][it][e + 2], A[k][it][e + 3]};
        }
      }
      __syncthreads();
      for (int c = threadIdx.x; c < C; c += kNormThreads) {
        float v = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) v += lds[w * C + c];
        prow[c] = v;
      }
    }
  }
}

template <typename T, int G, int IT, int U, bool RMS>
__global__ void __launch_bounds__(kNormThreads) norm_packed_bwd_kernel(const NormBwdArgs<T> a) {
  using Row = NormRow<T, G, IT>;
  constexpr int VE = Row::VE, kGroups = Row::kGroups;
  extern __shared__ float lds[];
  __shared__ float slots[16];
  RowSums<G, 2> sums{slots};
  const int grp = threadIdx.x / G, gl = threadIdx.x % G, chunks = a.C / VE;
  const long M = a.total != nullptr ? min((long)max(*a.total, 0), a.cap) : a.cap;
  const float inv_c = 1.0f / (float)a.C;
  const bool in_place = a.residual == a.out;
  typename Row::Raw gr[IT];
  Row::load(a.gamma, gl, chunks, a.gamma != nullptr, gr);
  float A[2][IT][VE];
#pragma unroll
  for (int k = 0; k < 2; ++k)
#pragma unroll
    for (int it = 0; it < IT; ++it)
#pragma unroll
      for (int e = 0; e < VE; ++e) A[k][it][e] = 0.f;
  const long step = (long)gridDim.x * kGroups * U;
  int next[U];                                            // the packed rows of the pass to come
  auto ask = [&](long base) {
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (a.inv_pos != nullptr) next[u] = a.inv_pos[min(base + u * kGroups + grp, a.n - 1)];
  };
  ask((long)blockIdx.x * kGroups * U);
  for (long base = (long)blockIdx.x * kGroups * U; base < a.n; base += step) {
    typename Row::Raw xr[U][IT], dr[U][IT], rr[U][IT];
    long i[U], j[U];
    bool sel[U];
    float mu[U], r[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      i[u] = base + u * kGroups + grp;
      j[u] = a.inv_pos != nullptr ? (long)next[u] : min(i[u], a.n - 1);
      sel[u] = i[u] < a.n && j[u] >= 0 && j[u] < M;
    }
    ask(base + step);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      Row::load(a.residual + i[u] * a.C, gl, chunks, a.residual != nullptr && i[u] < a.n && (sel[u] || !in_place), rr[u]);
      Row::load(a.rows + i[u] * a.C, gl, chunks, sel[u], xr[u]);
      Row::load(a.grad + j[u] * a.C, gl, chunks, sel[u], dr[u]);
      mu[u] = !RMS && sel[u] ? a.stats[j[u]] : 0.f;
      r[u] = sel[u] ? a.stats[a.cap + j[u]] : 0.f;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float v[2] = {0.f, 0.f};                            // sums of g and g xh (a row that is not selected: r = 0, da = 0)
#pragma unroll
      for (int it = 0; it < IT; ++it) {
        float x[VE], d[VE], g[VE];
        widen(xr[u][it], x);
        widen(dr[u][it], d);
        widen(gr[it], g);
#pragma unroll
        for (int e = 0; e < VE; ++e) {
          const float xh = (x[e] - mu[u]) * r[u], gg = a.gamma != nullptr ? d[e] * g[e] : d[e];
          v[0] += gg;
          v[1] = fmaf(gg, xh, v[1]);
          A[0][it][e] = fmaf(d[e], xh, A[0][it][e]);
          A[1][it][e] += d[e];
        }
      }
      sums(v);
      const float m1 = RMS ? 0.f : v[0] * inv_c, m2 = v[1] * inv_c;
      if (i[u] < a.n && (sel[u] || !in_place)) {
#pragma unroll
        for (int it = 0; it < IT; ++it) {
          const int ch = gl + it * G;
          float x[VE], d[VE], g[VE], o[VE];
          widen(xr[u][it], x);
          widen(dr[u][it], d);
          widen(gr[it], g);
          widen(rr[u][it], o);
#pragma unroll
          for (int e = 0; e < VE; ++e) {
            const float xh = (x[e] - mu[u]) * r[u], gg = a.gamma != nullptr ? d[e] * g[e] : d[e];
            o[e] = fmaf(r[u], gg - m1 - xh * m2, o[e]);
          }
          if (ch < chunks) {
            if (sel[u]) Row::store(a.out + i[u] * a.C, ch, o);
            else *reinterpret_cast<typename Row::Raw*>(a.out + i[u] * a.C + ch * VE) = rr[u][it];
          }
        }
      }
    }
  }
  norm_fold<T, G, IT>(A, a.C, a.partial, lds);
}

template <typename T, int G, int IT, int U, bool RMS>
__global__ void __launch_bounds__(kNormThreads) norm_residual_bwd_kernel(const NormBwdArgs<T> a) {
  using Row = NormRow<T, G, IT>;
  constexpr int VE = Row::VE, kGroups = Row::kGroups;
  extern __shared__ float lds[];
  __shared__ float slots[24];
  RowSums<G, 3> sums{slots};
  const int grp = threadIdx.x / G, gl = threadIdx.x % G, chunks = a.C / VE;
  const long M = a.total != nullptr ? min((long)max(*a.total, 0), a.cap) : a.cap;
  const float inv_c = 1.0f / (float)a.C;
  // scores of the tokens that were not selected: no gradient (asked for here, written behind the rows: nothing waits in between)
  const bool zeroes = a.d_scores != nullptr && a.inv_pos != nullptr;
  const long token = (long)blockIdx.x * kNormThreads + threadIdx.x;
  const int its = zeroes && token < a.n ? a.inv_pos[token] : 0;
  typename Row::Raw gr[IT], br[IT], sr[IT];
  Row::load(a.gamma, gl, chunks, a.gamma != nullptr, gr);
  Row::load(a.beta, gl, chunks, a.beta != nullptr, br);
  Row::load(a.scale, gl, chunks, a.scale != nullptr, sr);
  float A[2][IT][VE];
#pragma unroll
  for (int k = 0; k < 2; ++k)
#pragma unroll
    for (int it = 0; it < IT; ++it)
#pragma unroll
      for (int e = 0; e < VE; ++e) A[k][it][e] = 0.f;
  const long step = (long)gridDim.x * kGroups * U;
  int next[U];                                            // the tokens of the pass to come
  auto ask = [&](long base) {
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (a.gather_idx != nullptr) next[u] = a.gather_idx[min(base + u * kGroups + grp, a.cap - 1)];      // (does not wait for M)
  };
  ask((long)blockIdx.x * kGroups * U);
  for (long base = (long)blockIdx.x * kGroups * U; base < M; base += step) {
    typename Row::Raw zr[U][IT], dr[U][IT];
    long i[U], j[U];
    bool ok[U];
    float mu[U], r[U], s[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      j[u] = base + u * kGroups + grp;
      ok[u] = j[u] < M;
      j[u] = min(j[u], M - 1);
      i[u] = a.gather_idx != nullptr ? (long)next[u] : j[u];
    }
    ask(base + step);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      Row::load(a.rows + j[u] * a.C, gl, chunks, ok[u], zr[u]);
      Row::load(a.grad + i[u] * a.C, gl, chunks, ok[u], dr[u]);
      mu[u] = !RMS ? a.stats[j[u]] : 0.f;
      r[u] = a.stats[a.cap + j[u]];
      s[u] = a.gate != nullptr && ok[u] ? a.gate[i[u]] : 0.f;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const float p = a.gate != nullptr ? sigmoidf_dev(s[u]) : 1.f;
      float v[3] = {0.f, 0.f, 0.f};                       // of g, g zh and dy scale beta, g = dy scale gamma
#pragma unroll
      for (int it = 0; it < IT; ++it) {
        float z[VE], d[VE], g[VE], b[VE], sc[VE];
        widen(zr[u][it], z);
        widen(dr[u][it], d);
        widen(gr[it], g);
        widen(br[it], b);
        widen(sr[it], sc);
#pragma unroll
        for (int e = 0; e < VE; ++e) {
          const float zh = (z[e] - mu[u]) * r[u];
          const float ds = a.scale != nullptr ? d[e] * sc[e] : d[e], gg = a.gamma != nullptr ? ds * g[e] : ds;
          const float pd = ok[u] ? p * d[e] : 0.f;
          v[0] += gg;
          v[1] = fmaf(gg, zh, v[1]);
          v[2] = fmaf(ds, b[e], v[2]);
          A[0][it][e] = fmaf(pd, zh, A[0][it][e]);
          A[1][it][e] += pd;
        }
      }
      sums(v);
      const float m1 = RMS ? 0.f : v[0] * inv_c, m2 = v[1] * inv_c, pr = p * r[u];
      if (ok[u]) {
        if (a.d_scores != nullptr && gl == 0) a.d_scores[i[u]] = p * (1.f - p) * (v[1] + v[2]);
#pragma unroll
        for (int it = 0; it < IT; ++it) {
          const int ch = gl + it * G;
          float z[VE], d[VE], g[VE], sc[VE], o[VE];
          widen(zr[u][it], z);
          widen(dr[u][it], d);
          widen(gr[it], g);
          widen(sr[it], sc);
#pragma unroll
          for (int e = 0; e < VE; ++e) {
            const float zh = (z[e] - mu[u]) * r[u];
            const float ds = a.scale != nullptr ? d[e] * sc[e] : d[e], gg = a.gamma != nullptr ? ds * g[e] : ds;
            o[e] = pr * (gg - m1 - zh * m2);
          }
          if (ch < chunks) Row::store(a.out + j[u] * a.C, ch, o);
        }
      }
    }
  }
  if (zeroes) {
    int j = its;
    for (long i = token; i < a.n; i += (long)gridDim.x * kNormThreads) {
      if (i != token) j = a.inv_pos[i];
      if (j < 0 || j >= M) a.d_scores[i] = 0.f;
    }
  }
  norm_fold<T, G, IT>(A, a.C, a.partial, lds);
}

// Adds the partial rows in a fixed order: 16 columns a workgroup, SL slices of the rows beside each other, at most 8 rows of both
// sums a thread, whose loads are all in flight at once; the slices of a wave by exchanges, then the waves in order.  Then the
// parameter gradients from the sums A and B.  64 slices, or 16 where these reach all rows.  (16 slices in a loop over the rows,
// 512 rows: 11.2 us.)
template <typename T>
struct NormReduceArgs {
  const float* partial;
  int parts, C;
  const T *gamma, *beta, *scale;
  float *dgamma, *dbeta, *dscale;
};
template <typename T, int SL>
__global__ void __launch_bounds__(16 * SL) norm_reduce_kernel(const NormReduceArgs<T> a) {
  constexpr int kRows = 8, kWaves = SL / 4;
  static_assert(kNormMaxParts <= 64 * kRows, "64 slices reach every row");
  __shared__ float red[2][kWaves][17];
  const int cl = threadIdx.x & 15, sl = threadIdx.x >> 4, c = blockIdx.x * 16 + cl;
  float v[2][kRows];
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    const int r = sl + SL * i;
    const bool in = r < a.parts && c < a.C;
    v[0][i] = in ? a.partial[(long)r * 2 * a.C + c] : 0.f;
    v[1][i] = in ? a.partial[((long)r * 2 + 1) * a.C + c] : 0.f;
  }
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    float t = 0.f;
#pragma unroll
    for (int i = 0; i < kRows; ++i) t += v[k][i];
    t = add_lane_xor32(add_lane_xor16(t));
    if ((threadIdx.x & 63) < 16) red[k][threadIdx.x >> 6][cl] = t;
  }
  __syncthreads();
  if (threadIdx.x >= 16 || c >= a.C) return;
  float A = 0.f, B = 0.f;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    A += red[0][w][cl];
    B += red[1][w][cl];
  }
  const float scale = a.scale != nullptr ? (float)a.scale[c] : 1.f;
  if (a.dgamma != nullptr) a.dgamma[c] = scale * A;
  if (a.dbeta != nullptr) a.dbeta[c] = scale * B;
  if (a.dscale != nullptr)
    a.dscale[c] = fmaf(a.gamma != nullptr ? (float)a.gamma[c] : 1.f, A, a.beta != nullptr ? (float)a.beta[c] * B : 0.f);
}

// ------------------------------------------------------------------------------- host
// The kernel shape of a row length: lanes a row and chunks a lane so that few lanes are without a chunk, up to 4 chunks a
// lane (8 fp32) where the waves of a workgroup share a row.  U rows of a group in flight.  The backward's launch us at 12544 bf16 rows
// of 768, in front: 14.8; with twice the rows in flight 20.3 (fewer waves fit), with eight waves a workgroup 18.4.  Three chunks a
// lane: 64 lanes for up to 192 chunks (forward behind, 100 MB of 1536 bf16 46.7 -> 39.8, backward 46.5 -> 33.0 against four chunks).
template <typename T, class F>
static int norm_shape(const char* fn, int C, F go) {
  const int chunks = C / Vec16<T>::kElems;
#define SPA_SHAPE(G, IT, U) return go(std::integral_constant<int, G>{}, std::integral_constant<int, IT>{}, std::integral_constant<int, U>{})
  if (chunks <= 8) SPA_SHAPE(8, 1, 4);
  if (chunks <= 16) SPA_SHAPE(16, 1, 4);
  if (chunks <= 32) SPA_SHAPE(32, 1, 4);
  if (chunks <= 64) SPA_SHAPE(32, 2, 2);
  if (chunks <= 96) SPA_SHAPE(32, 3, 2);
  if (chunks <= 128) SPA_SHAPE(64, 2, 2);
  if (chunks <= 192) SPA_SHAPE(64, 3, 1);
  if (chunks <= 256) SPA_SHAPE(64, 4, 1);
  if (chunks <= 512) SPA_SHAPE(256, 2, 2);
  if (chunks <= 1024) SPA_SHAPE(256, 4, 1);
  if constexpr (sizeof(T) == 4)
    if (chunks <= 2048) SPA_SHAPE(256, 8, 1);
#undef SPA_SHAPE
  return fail(SPA_ERR_UNSUPPORTED, "%s: C = %d exceeds %d", fn, C, kMaxNormC);
}

static int norm_checks(const char* fn, int kind, int C, int dtype) {
  SPA_REFUSE_IN_GROUP(fn);
  SPA_REQUIRE(kind == SPA_NORM_LAYER || kind == SPA_NORM_RMS, SPA_ERR_INVALID_ARG, "%s: unknown kind of norm %d", fn, kind);
  SPA_REQUIRE(dtype == SPA_F32 || dtype == SPA_BF16, SPA_ERR_UNSUPPORTED, "%s: unknown dtype %d", fn, dtype);
  SPA_REQUIRE(C >= 1, SPA_ERR_INVALID_ARG, "%s: C must be >= 1", fn);
  SPA_REQUIRE(((long)C * elem_size(dtype)) % 16 == 0, SPA_ERR_INVALID_ARG,
              "%s: row length C*elem = %ld bytes is not a multiple of 16", fn, (long)C * elem_size(dtype));
  SPA_REQUIRE(C <= kMaxNormC, SPA_ERR_UNSUPPORTED, "%s: C = %d exceeds %d", fn, C, kMaxNormC);
  return SPA_OK;
}
static bool norm_eps_ok(float eps) { return eps >= 0.f && std::isfinite(eps); }

static unsigned norm_blocks(long rows, int per) { return (unsigned)std::min<long>((rows + per - 1) / per, 4096L); }
// Workgroups of the backward, a partial row each: one for 16 rows, for 4 where a row takes a whole workgroup (us in front | behind, 10 MB
// of packed rows, for 16 and for 4: 2560 bf16 27 | 27 and 22 | 20, 8192 fp32 47 | 48 and 25 | 21).
static int norm_parts(long rows, int C, int dtype) {
  const int each = (long)C * elem_size(dtype) > 256 * 16 ? 4 : 16;
  return (int)std::max<long>(1, std::min<long>((rows + each - 1) / each, kNormMaxParts));
}

template <typename T>
static int launch_norm_fwd(const char* fn, bool behind, int kind, const NormFwdArgs<T>& a, hipStream_t st) {
  return norm_shape<T>(fn, a.C, [&](auto g, auto it, auto u) {
    constexpr int G = decltype(g)::value, IT = decltype(it)::value, U = decltype(u)::value;
    const unsigned blocks = norm_blocks(a.n, kNormThreads / G * U);
#define SPA_NORM(KERNEL, RMS) hipLaunchKernelGGL((KERNEL<T, G, IT, U, RMS>), dim3(blocks), dim3(kNormThreads), 0, st, a)
    if (behind) {
      if (kind == SPA_NORM_RMS) SPA_NORM(norm_residual_kernel, true); else SPA_NORM(norm_residual_kernel, false);
    } else {
      if (kind == SPA_NORM_RMS) SPA_NORM(norm_packed_kernel, true); else SPA_NORM(norm_packed_kernel, false);
    }
#undef SPA_NORM
    return check_launch(fn);
  });
}

template <typename T>
static int launch_norm_bwd(const char* fn, bool behind, int kind, const NormBwdArgs<T>& a, float* dgamma, float* dbeta, float* dscale,
                           hipStream_t st) {
  const int parts = norm_parts(behind ? a.cap : a.n, a.C, sizeof(T) == 4 ? SPA_F32 : SPA_BF16);
  const int rc = norm_shape<T>(fn, a.C, [&](auto g, auto it, auto u) {
    constexpr int G = decltype(g)::value, IT = decltype(it)::value, U = decltype(u)::value;
    const size_t lds = G > kWave ? 0 : (size_t)(kNormThreads / kWave) * a.C * sizeof(float);      // at most 32 KB
#define SPA_NORM(KERNEL, ROWS, RMS) hipLaunchKernelGGL((KERNEL<T, G, IT, ROWS, RMS>), dim3(parts), dim3(kNormThreads), lds, st, a)
    if (behind) {
      // (two rows of three chunks take 273 registers, one wave a SIMD: 62914 rows of 768, half of them packed, 42.3 us, so 32.6)
      constexpr int UB = IT >= 3 ? 1 : U;
      if (kind == SPA_NORM_RMS) SPA_NORM(norm_residual_bwd_kernel, UB, true); else SPA_NORM(norm_residual_bwd_kernel, UB, false);
    } else {
      if (kind == SPA_NORM_RMS) SPA_NORM(norm_packed_bwd_kernel, U, true); else SPA_NORM(norm_packed_bwd_kernel, U, false);
    }
#undef SPA_NORM
    return SPA_OK;
  });
  if (rc != SPA_OK) return rc;
  if (dgamma != nullptr || dbeta != nullptr || dscale != nullptr) {
    const NormReduceArgs<T> r = {a.partial, parts, a.C, a.gamma, a.beta, a.scale, dgamma, dbeta, dscale};
    if (parts <= 128) hipLaunchKernelGGL((norm_reduce_kernel<T, 16>), dim3((a.C + 15) / 16), dim3(256), 0, st, r);
    else hipLaunchKernelGGL((norm_reduce_kernel<T, 64>), dim3((a.C + 15) / 16), dim3(1024), 0, st, r);
  }
  return check_launch(fn);
}

}  // namespace spa

using namespace spa;

extern "C" int spa_norm_packed(const void* x, const int32_t* gather_idx, const int32_t* total, const void* gamma, const void* beta,
                               int kind, float eps, int M_cap, int C, int dtype, void* packed, float* stats, void* stream) {
  const char* fn = "spa_norm_packed";
  SPA_REQUIRE(x && packed, SPA_ERR_INVALID_ARG, "%s: null pointer", fn);
  if (int rc = norm_checks(fn, kind, C, dtype)) return rc;
  SPA_REQUIRE(M_cap >= 1, SPA_ERR_INVALID_ARG, "%s: M_cap must be >= 1", fn);
  SPA_REQUIRE(norm_eps_ok(eps), SPA_ERR_INVALID_ARG, "%s: eps must be finite and >= 0", fn);
  SPA_REQUIRE(aligned16(x) && aligned16(packed) && aligned16(gamma) && aligned16(beta), SPA_ERR_INVALID_ARG,
              "%s: tensors not 16-byte aligned", fn);
#define SPA_ARGS(T)                                                                                                         \
  NormFwdArgs<T> { (const T*)x, gather_idx, total, (const T*)gamma, (const T*)beta, nullptr, nullptr, nullptr, eps, (long)M_cap, \
                   (long)M_cap, C, (T*)packed, stats }
  return dtype == SPA_F32 ? launch_norm_fwd<float>(fn, false, kind, SPA_ARGS(float), as_stream(stream))
                          : launch_norm_fwd<__bf16>(fn, false, kind, SPA_ARGS(__bf16), as_stream(stream));
#undef SPA_ARGS
}

extern "C" int spa_norm_residual_unpack(const void* z, const int32_t* inv_pos, const void* residual, const void* gamma, const void* beta,
                                        const void* scale, const float* gate_scores, int kind, float eps, int M_cap, int64_t rows, int C,
                                        int dtype, void* y, float* stats, void* stream) {
  const char* fn = "spa_norm_residual_unpack";
  SPA_REQUIRE(z && y, SPA_ERR_INVALID_ARG, "%s: null pointer", fn);
  if (int rc = norm_checks(fn, kind, C, dtype)) return rc;
  SPA_REQUIRE(M_cap >= 1 && rows >= 1 && rows < 2147483647L, SPA_ERR_INVALID_ARG, "%s: M_cap and rows must be >= 1 (rows < 2^31)", fn);
  SPA_REQUIRE(norm_eps_ok(eps), SPA_ERR_INVALID_ARG, "%s: eps must be finite and >= 0", fn);
  SPA_REQUIRE(aligned16(z) && aligned16(y) && aligned16(residual) && aligned16(gamma) && aligned16(beta) && aligned16(scale),
              SPA_ERR_INVALID_ARG, "%s: tensors not 16-byte aligned", fn);
#define SPA_ARGS(T)                                                                                                          \
  NormFwdArgs<T> { (const T*)z, inv_pos, nullptr, (const T*)gamma, (const T*)beta, (const T*)scale, (const T*)residual, gate_scores, \
                   eps, (long)rows, (long)M_cap, C, (T*)y, stats }
  return dtype == SPA_F32 ? launch_norm_fwd<float>(fn, true, kind, SPA_ARGS(float), as_stream(stream))
                          : launch_norm_fwd<__bf16>(fn, true, kind, SPA_ARGS(__bf16), as_stream(stream));
#undef SPA_ARGS
}

extern "C" size_t spa_norm_bwd_workspace_bytes(int64_t rows, int C, int dtype) {
  if (rows < 1 || C < 1) return 0;
  return (size_t)norm_parts((long)rows, C, dtype) * 2 * (size_t)C * sizeof(float);
}

extern "C" int spa_norm_packed_bwd(const void* d_packed, const void* x, const int32_t* inv_pos, const int32_t* total, const void* gamma,
                                   int kind, const float* stats, const void* d_residual, int M_cap, int64_t rows, int C, int dtype,
                                   void* dx, float* dgamma, float* dbeta, void* workspace, size_t workspace_bytes, void* stream) {
  const char* fn = "spa_norm_packed_bwd";
  SPA_REQUIRE(d_packed && x && stats && dx, SPA_ERR_INVALID_ARG, "%s: null pointer", fn);
  if (int rc = norm_checks(fn, kind, C, dtype)) return rc;
  SPA_REQUIRE(M_cap >= 1 && rows >= 1 && rows < 2147483647L, SPA_ERR_INVALID_ARG, "%s: M_cap and rows must be >= 1 (rows < 2^31)", fn);
  SPA_REQUIRE(aligned16(d_packed) && aligned16(x) && aligned16(gamma) && aligned16(d_residual) && aligned16(dx), SPA_ERR_INVALID_ARG,
              "%s: tensors not 16-byte aligned", fn);
  const size_t need = spa_norm_bwd_workspace_bytes(rows, C, dtype);
  SPA_REQUIRE(workspace != nullptr && workspace_bytes >= need, SPA_ERR_WORKSPACE, "%s: workspace of %zu bytes needed, %zu given", fn,
              need, workspace_bytes);
#define SPA_ARGS(T)                                                                                                          \
  NormBwdArgs<T> { (const T*)x, (const T*)d_packed, nullptr, inv_pos, total, (const T*)gamma, nullptr, nullptr, (const T*)d_residual, \
                   nullptr, stats, (long)rows, (long)M_cap, C, (T*)dx, nullptr, (float*)workspace }
  return dtype == SPA_F32 ? launch_norm_bwd<float>(fn, false, kind, SPA_ARGS(float), dgamma, dbeta, nullptr, as_stream(stream))
                          : launch_norm_bwd<__bf16>(fn, false, kind, SPA_ARGS(__bf16), dgamma, dbeta, nullptr, as_stream(stream));
#undef SPA_ARGS
}

extern "C" int spa_norm_residual_unpack_bwd(const void* dy, const void* z, const int32_t* gather_idx, const int32_t* inv_pos,
                                            const int32_t* total, const void* gamma, const void* beta, const void* scale,
                                            const float* gate_scores, int kind, const float* stats, int M_cap, int64_t rows, int C,
                                            int dtype, void* dz, float* d_scores, float* dgamma, float* dbeta, float* dscale,
                                            void* workspace, size_t workspace_bytes, void* stream) {
  const char* fn = "spa_norm_residual_unpack_bwd";
  SPA_REQUIRE(dy && z && stats && dz, SPA_ERR_INVALID_ARG, "%s: null pointer", fn);
  if (int rc = norm_checks(fn, kind, C, dtype)) return rc;
  SPA_REQUIRE(M_cap >= 1 && rows >= 1 && rows < 2147483647L, SPA_ERR_INVALID_ARG, "%s: M_cap and rows must be >= 1 (rows < 2^31)", fn);
  SPA_REQUIRE((gather_idx != nullptr) == (inv_pos != nullptr), SPA_ERR_INVALID_ARG,
              "%s: gather_idx and inv_pos are given together or not at all", fn);
  SPA_REQUIRE(inv_pos != nullptr || M_cap <= rows, SPA_ERR_INVALID_ARG, "%s: more packed rows than rows", fn);
  SPA_REQUIRE(d_scores == nullptr || gate_scores != nullptr, SPA_ERR_INVALID_ARG, "%s: d_scores needs gate_scores", fn);
  SPA_REQUIRE(aligned16(dy) && aligned16(z) && aligned16(gamma) && aligned16(beta) && aligned16(scale) && aligned16(dz),
              SPA_ERR_INVALID_ARG, "%s: tensors not 16-byte aligned", fn);
  const size_t need = spa_norm_bwd_workspace_bytes(M_cap, C, dtype);
  SPA_REQUIRE(workspace != nullptr && workspace_bytes >= need, SPA_ERR_WORKSPACE, "%s: workspace of %zu bytes needed, %zu given", fn,
              need, workspace_bytes);
#define SPA_ARGS(T)                                                                                                          \
  NormBwdArgs<T> { (const T*)z, (const T*)dy, gather_idx, inv_pos, total, (const T*)gamma, (const T*)beta, (const T*)scale, nullptr, \
                   gate_scores, stats, (long)rows, (long)M_cap, C, (T*)dz, d_scores, (float*)workspace }
  return dtype == SPA_F32 ? launch_norm_bwd<float>(fn, true, kind, SPA_ARGS(float), dgamma, dbeta, dscale, as_stream(stream))
                          : launch_norm_bwd<__bf16>(fn, true, kind, SPA_ARGS(__bf16), dgamma, dbeta, dscale, as_stream(stream));
#undef SPA_ARGS
}
