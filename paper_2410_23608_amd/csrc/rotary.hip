// Norm of every head of q and k with the rotation by the token's place on its image's map in the same pass, on packed rows.
//   xh = (x - mu) r,  r = 1 / sqrt(var + eps) over the head's elements (RMS: mu = 0, var = mean x^2; none: xh = x)
//   u  = gamma xh + beta,  (y1, y2) = (u1 c - u2 s, u1 s + u2 c) for every pair of elements, c and s of the angle (place on the pair's
// axis) x (the pair's frequency), which a table holds by place and pair: rounded once, from 64 bits, however far the place.
// Backward: du = the pairs of dy turned back,  g = gamma du,  dx = r (g - mean(g) - xh mean(g xh))  (RMS: without mean(g)),
//   dgamma = sum du xh,  dbeta = sum du  over all rows and heads.
// Bound by memory: a head is read once and kept in registers.  LH lanes share a head, a lane has whole pairs of either layout (16 bytes;
// with 32 the backward of video clips took 46.5 us instead of 38); a thread takes up to four heads of a row and looks the row's angles up
// once (two heads: 41).  Launches one by one, half of the tokens live: 64 x 196 tokens of 12 + 12 heads of 64 bf16 10.2 us forward (3.8
// TB/s), 16.4 backward (3.5), 4.5 the sums; 8 clips of 8 x 28 x 28 of 16 + 4 heads 29.6 and 37.7; one image 4.0.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "divisor.h"
#include "row_groups.h"
#include "spa_common.h"

namespace spa {

constexpr int kRotaryThreads = 256, kRotaryHeads = 4, kRotaryMostParts = 512;
constexpr int kMaxRotaryHeads = 256;

// A lane's VE elements of a head: its PAIRS pairs, neighbours (16 bytes) or half a head apart (twice 8 bytes), first ones in front.
template <typename T, int DH, bool HALVES>
struct HeadLanes {
  static constexpr int VE = Vec16<T>::kElems, PAIRS = VE / 2, LH = DH / VE;        // LH: lanes a head
  static_assert(LH == 4 || LH == 8 || LH == 16, "neighbouring lanes");
  using Raw = typename Raw16<T>::type;
  static __device__ __forceinline__ Raw load(const T* head, int c) {
    if constexpr (!HALVES) {
      return *reinterpret_cast<const Raw*>(head + c * VE);
    } else {
      const uintx2 lo = *reinterpret_cast<const uintx2*>(head + c * PAIRS), hi = *reinterpret_cast<const uintx2*>(head + DH / 2 + c * PAIRS);
      return __builtin_bit_cast(Raw, uintx4{lo[0], lo[1], hi[0], hi[1]});
    }
  }
  // place in the head of element e of the lane
  static __device__ __forceinline__ int element(int c, int e) { return !HALVES ? c * VE + e : (e < PAIRS ? 0 : DH / 2 - PAIRS) + c * PAIRS + e; }
  // (the one rounding to the tensors' type)
  static __device__ __forceinline__ void store(T* head, int c, const float (&x)[VE]) {
    Raw r;
    if constexpr (VE == 8) {
      floatx8 v;
#pragma unroll
      for (int e = 0; e < VE; ++e) v[e] = x[e];
      r = float_to_bf16x8(v);
    } else {
#pragma unroll
      for (int e = 0; e < VE; ++e) r[e] = x[e];
    }
    if constexpr (!HALVES) {
      *reinterpret_cast<Raw*>(head + c * VE) = r;
    } else {
      const uintx4 w = __builtin_bit_cast(uintx4, r);
      *reinterpret_cast<uintx2*>(head + c * PAIRS) = uintx2{w[0], w[1]};
      *reinterpret_cast<uintx2*>(head + DH / 2 + c * PAIRS) = uintx2{w[2], w[3]};
    }
  }
  static __device__ __forceinline__ float sum(float v) {
    v += lane_xor<1>(v);
    v += lane_xor<2>(v);
    if (LH > 4) v += dpp_move<0x141>(v);      // a quad holds one value: the half row mirrored, then the row
    if (LH > 8) v += dpp_move<0x140>(v);
    return v;
  }
};

template <typename T>
struct RotarySide {
  const T *x, *d;                // rows of the tensor, and of the gradient of its result
  long xs, ds, os;
  T* out;
  const T *gamma, *beta;
  int heads, slots;              // slots: heads of a row taken beside each other
  unsigned blocks;
  float* partial;                // [blocks][2][DH]
};
template <typename T>
struct RotaryArgs {
  RotarySide<T> side[2];         // q, k
  const int32_t *idx, *total;
  const float* table;            // [places][DH / 2][2] or null
  int pairs_t, pairs_th;         // pairs turned by time, by time or row
  bool even;                     // both are: two pairs a load
  Divisor tokens, plane, width;
  float eps;
  long n;
};

// Cosines and sines of a lane's pairs at the place of a token
template <typename T, int DH, bool HALVES>
struct Turn {
  static constexpr int N = HeadLanes<T, DH, HALVES>::PAIRS, HALF = DH / 2;
  float c[N], s[N];
  // (of plain values: through a lambda's captures the choice is one among addresses, in scratch memory)
  static __device__ __forceinline__ int place(int i, int pairs_t, int pairs_th, int time, int row, int col) {
    return i < pairs_t ? time : i < pairs_th ? row : col;
  }
  __device__ __forceinline__ void look_up(const RotaryArgs<T>& a, int token, int lane) {
    if (a.table == nullptr) {
#pragma unroll
      for (int u = 0; u < N; ++u) c[u] = 1.f, s[u] = 0.f;
      return;
    }
    const uint32_t t = (uint32_t)token & 0x7fffffffu, n = t - quotient(t, a.tokens) * a.tokens.d;
    const uint32_t time = quotient(n, a.plane), at = n - time * a.plane.d, row = quotient(at, a.width), col = at - row * a.width.d;
    if (a.even) {
#pragma unroll
      for (int u = 0; u < N; u += 2) {
        const int i = lane * N + u;
        const floatx4 v = *reinterpret_cast<const floatx4*>(a.table + ((long)place(i, a.pairs_t, a.pairs_th, (int)time, (int)row, (int)col) * HALF + i) * 2);
        c[u] = v[0], s[u] = v[1], c[u + 1] = v[2], s[u + 1] = v[3];
      }
    } else {
#pragma unroll
      for (int u = 0; u < N; ++u) {
        const int i = lane * N + u;
        const floatx2 v = *reinterpret_cast<const floatx2*>(a.table + ((long)place(i, a.pairs_t, a.pairs_th, (int)time, (int)row, (int)col) * HALF + i) * 2);
        c[u] = v[0], s[u] = v[1];
      }
    }
  }
  // SIGN -1: back
  template <int SIGN>
  __device__ __forceinline__ void apply(float (&x)[2 * N]) const {
#pragma unroll
    for (int u = 0; u < N; ++u) {
      float &p = x[HALVES ? u : 2 * u], &q = x[HALVES ? N + u : 2 * u + 1];
      const float sn = SIGN * s[u], y = fmaf(p, c[u], -(q * sn));
      q = fmaf(p, sn, q * c[u]);
      p = y;
    }
  }
};

template <class L, int DH, int KIND>
__device__ __forceinline__ void head_moments(const float (&x)[L::VE], float eps, float& mu, float& r) {
  mu = 0.f;
  r = 1.f;
  if (KIND == SPA_NORM_NONE) return;
  if (KIND == SPA_NORM_LAYER) {
    float v = 0.f;
#pragma unroll
    for (int e = 0; e < L::VE; ++e) v += x[e];
    mu = L::sum(v) * (1.0f / DH);
  }
  float v = 0.f;
#pragma unroll
  for (int e = 0; e < L::VE; ++e) v = fmaf(x[e] - mu, x[e] - mu, v);
  r = 1.0f / sqrtf(fmaf(L::sum(v), 1.0f / DH, eps));
}

// What a thread is: its tensor, the row of its workgroup's, its place among the heads and in a head.
template <typename T, int DH>
struct RotaryPlace {
  int side, group, groups, slot, lane;
  long first, step;              // rows
  __device__ __forceinline__ RotaryPlace(const RotaryArgs<T>& a) {
    constexpr int LH = HeadLanes<T, DH, false>::LH;
    side = blockIdx.x >= a.side[0].blocks;
    const int G = (side ? a.side[1].slots : a.side[0].slots) * LH;
    groups = kRotaryThreads / G;
    group = threadIdx.x / G;
    const int in = threadIdx.x - group * G;
    slot = in / LH;
    lane = in % LH;
    const unsigned b = blockIdx.x - (side ? a.side[0].blocks : 0);
    first = (long)b * groups + group;
    step = (long)(side ? a.side[1].blocks : a.side[0].blocks) * groups;
  }
};

template <typename T, int DH, int KIND, bool HALVES>
__global__ void __launch_bounds__(kRotaryThreads) qk_rotary_kernel(const RotaryArgs<T> a) {
  using L = HeadLanes<T, DH, HALVES>;
  constexpr int VE = L::VE, U = kRotaryHeads;
  const RotaryPlace<T, DH> at(a);
  if (at.group >= at.groups) return;
  const RotarySide<T> side = at.side ? a.side[1] : a.side[0];      // (an index into the arguments would put them into memory)
  typename L::Raw gamma = {}, beta = {};
  if (side.gamma != nullptr) gamma = L::load(side.gamma, at.lane);
  if (side.beta != nullptr) beta = L::load(side.beta, at.lane);
  auto token = [&](long j) { return a.idx != nullptr ? a.idx[min(j, a.n - 1)] : (int)min(j, a.n - 1); };
  int next = token(at.first);
  typename L::Raw raw[U];
  auto load = [&](long j, int h0) {
    const T* row = side.x + j * side.xs;
#pragma unroll
    for (int u = 0; u < U; ++u) raw[u] = L::load(row + min(h0 + u * side.slots, side.heads - 1) * DH, at.lane);
  };
  const long M = a.total != nullptr ? min((long)max(*a.total, 0), a.n) : a.n;
  for (long j = at.first; j < M; j += at.step) {
    load(j, at.slot);                                         // (does not wait for the index)
    Turn<T, DH, HALVES> turn;
    turn.look_up(a, next, at.lane);
    next = token(j + at.step);
    T* out = side.out + j * side.os;
    for (int h0 = at.slot; h0 < side.heads; h0 += U * side.slots) {
      if (h0 != at.slot) load(j, h0);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int h = h0 + u * side.slots;
        if (h >= side.heads) break;
        float x[VE], mu, r;
        widen(raw[u], x);
        head_moments<L, DH, KIND>(x, a.eps, mu, r);
        if (KIND != SPA_NORM_NONE) {
          float g[VE], b[VE];
          widen(gamma, g);
          widen(beta, b);
#pragma unroll
          for (int e = 0; e < VE; ++e) x[e] = fmaf((x[e] - mu) * r, side.gamma != nullptr ? g[e] : 1.f, b[e]);
        }
        turn.template apply<1>(x);
        L::store(out + h * DH, at.lane, x);
      }
    }
  }
}

// Sum over the wave's lanes of the same place in a head, in each of them
template <int LH>
__device__ __forceinline__ float same_place_sum(float v) {
  if (LH <= 4) v += lane_xor<4>(v);
  if (LH <= 8) v += dpp_move<0x128>(v);
  return add_lane_xor32(add_lane_xor16(v));
}

template <typename T, int DH, int KIND, bool HALVES>
__global__ void __launch_bounds__(kRotaryThreads) qk_rotary_bwd_kernel(const RotaryArgs<T> a) {
  using L = HeadLanes<T, DH, HALVES>;
  constexpr int VE = L::VE, U = kRotaryHeads;
  __shared__ float sums[kRotaryThreads / kWave][2][DH];
  const RotaryPlace<T, DH> at(a);
  const RotarySide<T> side = at.side ? a.side[1] : a.side[0];      // (an index into the arguments would put them into memory)
  typename L::Raw gamma = {};
  if (side.gamma != nullptr) gamma = L::load(side.gamma, threadIdx.x % L::LH);
  float A[2][VE];
#pragma unroll
  for (int k = 0; k < 2; ++k)
#pragma unroll
    for (int e = 0; e < VE; ++e) A[k][e] = 0.f;
  if (at.group < at.groups) {
    auto token = [&](long j) { return a.idx != nullptr ? a.idx[min(j, a.n - 1)] : (int)min(j, a.n - 1); };
    int next = token(at.first);
    typename L::Raw xr[U], dr[U];
    auto load = [&](long j, int h0) {
      const T *row = side.x + j * side.xs, *grad = side.d + j * side.ds;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int h = min(h0 + u * side.slots, side.heads - 1) * DH;
        dr[u] = L::load(grad + h, at.lane);
        if (KIND != SPA_NORM_NONE) xr[u] = L::load(row + h, at.lane);
      }
    };
    const long M = a.total != nullptr ? min((long)max(*a.total, 0), a.n) : a.n;
    for (long j = at.first; j < M; j += at.step) {
      load(j, at.slot);                                       // (does not wait for the index)
      Turn<T, DH, HALVES> turn;
      turn.look_up(a, next, at.lane);
      next = token(j + at.step);
      T* out = side.out + j * side.os;
      for (int h0 = at.slot; h0 < side.heads; h0 += U * side.slots) {
        if (h0 != at.slot) load(j, h0);
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int h = h0 + u * side.slots;
          if (h >= side.heads) break;
          float d[VE];
          widen(dr[u], d);
          turn.template apply<-1>(d);
          if (KIND != SPA_NORM_NONE) {
            float x[VE], g[VE], mu, r, v0 = 0.f, v1 = 0.f;
            widen(xr[u], x);
            widen(gamma, g);
            head_moments<L, DH, KIND>(x, a.eps, mu, r);
#pragma unroll
            for (int e = 0; e < VE; ++e) {
              x[e] = (x[e] - mu) * r;
              A[0][e] = fmaf(d[e], x[e], A[0][e]);
              A[1][e] += d[e];
              if (side.gamma != nullptr) d[e] *= g[e];
              v0 += d[e];
              v1 = fmaf(d[e], x[e], v1);
            }
            const float m1 = KIND == SPA_NORM_LAYER ? L::sum(v0) * (1.0f / DH) : 0.f, m2 = L::sum(v1) * (1.0f / DH);
#pragma unroll
            for (int e = 0; e < VE; ++e) d[e] = r * (d[e] - m1 - x[e] * m2);
          }
          L::store(out + h * DH, at.lane, d);
        }
      }
    }
  }
  if (KIND == SPA_NORM_NONE || side.partial == nullptr) return;
  const int lane = threadIdx.x & (kWave - 1), c = lane % L::LH, wv = threadIdx.x / kWave;
#pragma unroll
  for (int k = 0; k < 2; ++k)
#pragma unroll
    for (int e = 0; e < VE; ++e) {
      const float v = same_place_sum<L::LH>(A[k][e]);
      if (lane < L::LH) sums[wv][k][L::element(c, e)] = v;
    }
  __syncthreads();
  const long b = blockIdx.x - (at.side ? a.side[0].blocks : 0);
  for (int i = threadIdx.x; i < 2 * DH; i += kRotaryThreads) {
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < kRotaryThreads / kWave; ++w) v += sums[w][i / DH][i % DH];
    side.partial[b * 2 * DH + i] = v;
  }
}

// Adds a tensor's partial rows in a fixed order: 16 columns a workgroup, 64 slices of the rows beside each other, at most 8 rows a
// thread, whose loads are all in flight at once; the slices of a wave by exchanges, then the waves in order.
struct RotarySums {
  const float* partial[2];
  int parts[2];
  float *dgamma[2], *dbeta[2];
  int dh;
};
__global__ void __launch_bounds__(1024) qk_rotary_sums_kernel(const RotarySums a) {
  constexpr int kRows = kRotaryMostParts / 64;
  __shared__ float red[16][17];
  const int per = 2 * a.dh / 16, k = blockIdx.x / per, c = blockIdx.x % per * 16 + (threadIdx.x & 15), sl = threadIdx.x >> 4;
  const float* partial = k ? a.partial[1] : a.partial[0];
  const int parts = k ? a.parts[1] : a.parts[0];
  float v[kRows], t = 0.f;
#pragma unroll
  for (int i = 0; i < kRows; ++i) v[i] = sl + 64 * i < parts ? partial[(long)(sl + 64 * i) * 2 * a.dh + c] : 0.f;
#pragma unroll
  for (int i = 0; i < kRows; ++i) t += v[i];
  t = add_lane_xor32(add_lane_xor16(t));
  if ((threadIdx.x & 63) < 16) red[threadIdx.x >> 6][threadIdx.x & 15] = t;
  __syncthreads();
  if (threadIdx.x >= 16) return;
  t = 0.f;
#pragma unroll
  for (int w = 0; w < 16; ++w) t += red[w][threadIdx.x];
  float* to = c < a.dh ? (k ? a.dgamma[1] : a.dgamma[0]) : (k ? a.dbeta[1] : a.dbeta[0]);
  if (to != nullptr) to[c < a.dh ? c : c - a.dh] = t;
}

// ------------------------------------------------------------------------------- host
// Heads of a row beside each other so that a thread has at most four, and every group of threads has a row
static int rotary_slots(int heads, int lanes) {
  const int most = kRotaryThreads / lanes;
  return std::max(1, std::min(most, (heads + kRotaryHeads - 1) / kRotaryHeads));
}
static int rotary_lanes(int Dh, int dtype) { return Dh * elem_size(dtype) / 16; }
static int rotary_groups(int heads, int Dh, int dtype) {
  const int lanes = rotary_lanes(Dh, dtype);
  return kRotaryThreads / (rotary_slots(heads, lanes) * lanes);
}
// Workgroups of a tensor: a row a group forward, up to eight a unit (video clips 33.6 us with 8192 workgroups at most, 29.8 with 2048, 30.7
// with 1024); four rows of the backward's, a partial row each
static unsigned rotary_blocks(long rows, int heads, int Dh, int dtype) {
  const int groups = rotary_groups(heads, Dh, dtype);
  return heads == 0 ? 0 : (unsigned)std::min<long>((rows + groups - 1) / groups, 2048L);
}
static unsigned rotary_parts(long rows, int heads, int Dh, int dtype) {
  const int per = 4 * rotary_groups(heads, Dh, dtype);
  return heads == 0 ? 0 : (unsigned)std::min<long>((rows + per - 1) / per, (long)kRotaryMostParts);
}

struct RotaryCall {
  const void *q, *k;
  int64_t q_stride, k_stride;
  const int32_t *idx, *total;
  const void *gamma_q, *beta_q, *gamma_k, *beta_k;
  int kind;
  float eps;
  const float* table;
  int pairs_t, pairs_h, grid_t, grid_h, grid_w, layout, M_cap, H, Hk, Dh, dtype;
  void *q_out, *k_out;
  int64_t qo_stride, ko_stride;
};

static int rotary_rows_ok(const char* fn, const char* name, const void* p, int64_t stride, int heads, int Dh, int dtype) {
  SPA_REQUIRE(p != nullptr, SPA_ERR_INVALID_ARG, "%s: null pointer (%s)", fn, name);
  SPA_REQUIRE(aligned16(p), SPA_ERR_INVALID_ARG, "%s: %s not 16-byte aligned", fn, name);
  SPA_REQUIRE(stride >= (int64_t)heads * Dh && stride < (1LL << 31), SPA_ERR_INVALID_ARG, "%s: row stride %ld of %s out of range", fn, (long)stride, name);
  SPA_REQUIRE(stride * elem_size(dtype) % 16 == 0, SPA_ERR_INVALID_ARG, "%s: row stride of %s is not a multiple of 16 bytes", fn, name);
  return SPA_OK;
}

static int rotary_checks(const char* fn, const RotaryCall& c) {
  SPA_REFUSE_IN_GROUP(fn);
  SPA_REQUIRE(c.dtype == SPA_F32 || c.dtype == SPA_BF16, SPA_ERR_UNSUPPORTED, "%s: unknown dtype %d", fn, c.dtype);
  SPA_REQUIRE(c.Dh == 32 || c.Dh == 64, SPA_ERR_UNSUPPORTED, "%s: head dim %d not supported (32 or 64)", fn, c.Dh);
  SPA_REQUIRE(c.M_cap >= 1, SPA_ERR_INVALID_ARG, "%s: M_cap must be >= 1", fn);
  SPA_REQUIRE(c.H >= 1 && c.Hk >= 0, SPA_ERR_INVALID_ARG, "%s: H must be >= 1 and Hk >= 0", fn);
  SPA_REQUIRE(c.H <= kMaxRotaryHeads && c.Hk <= kMaxRotaryHeads, SPA_ERR_UNSUPPORTED, "%s: more than %d heads", fn, kMaxRotaryHeads);
  SPA_REQUIRE(c.kind == SPA_NORM_LAYER || c.kind == SPA_NORM_RMS || c.kind == SPA_NORM_NONE, SPA_ERR_INVALID_ARG, "%s: unknown kind of norm %d", fn, c.kind);
  SPA_REQUIRE(c.kind != SPA_NORM_NONE || (!c.gamma_q && !c.beta_q && !c.gamma_k && !c.beta_k), SPA_ERR_INVALID_ARG,
              "%s: gamma and beta belong to a norm", fn);
  SPA_REQUIRE(c.eps >= 0.f && std::isfinite(c.eps), SPA_ERR_INVALID_ARG, "%s: eps must be finite and >= 0", fn);
  SPA_REQUIRE(c.layout == SPA_ROTARY_ADJACENT || c.layout == SPA_ROTARY_HALVES, SPA_ERR_INVALID_ARG, "%s: unknown layout of pairs %d", fn, c.layout);
  SPA_REQUIRE(aligned16(c.gamma_q) && aligned16(c.beta_q) && aligned16(c.gamma_k) && aligned16(c.beta_k) && aligned16(c.table),
              SPA_ERR_INVALID_ARG, "%s: gamma / beta / table not 16-byte aligned", fn);
  if (c.table != nullptr) {
    SPA_REQUIRE(c.grid_t >= 1 && c.grid_h >= 1 && c.grid_w >= 1 && (double)c.grid_t * c.grid_h * c.grid_w < 2147483648.0, SPA_ERR_INVALID_ARG,
                "%s: the map's sizes must be >= 1, with fewer than 2^31 tokens", fn);
    SPA_REQUIRE(c.pairs_t >= 0 && c.pairs_h >= 0 && (long)c.pairs_t + c.pairs_h <= c.Dh / 2, SPA_ERR_INVALID_ARG,
                "%s: pairs of the axes must be >= 0 and no more than Dh / 2 together", fn);
  }
  if (int rc = rotary_rows_ok(fn, "q", c.q, c.q_stride, c.H, c.Dh, c.dtype)) return rc;
  if (int rc = rotary_rows_ok(fn, "q's result", c.q_out, c.qo_stride, c.H, c.Dh, c.dtype)) return rc;
  SPA_REQUIRE((c.q != c.q_out || c.q_stride == c.qo_stride) && (c.Hk == 0 || c.k != c.k_out || c.k_stride == c.ko_stride), SPA_ERR_INVALID_ARG,
              "%s: in place the row strides must be the same", fn);
  if (c.Hk > 0) {
    if (int rc = rotary_rows_ok(fn, "k", c.k, c.k_stride, c.Hk, c.Dh, c.dtype)) return rc;
    if (int rc = rotary_rows_ok(fn, "k's result", c.k_out, c.ko_stride, c.Hk, c.Dh, c.dtype)) return rc;
  }
  return SPA_OK;
}

template <typename T>
static RotaryArgs<T> rotary_args(const RotaryCall& c) {
  const int lanes = rotary_lanes(c.Dh, c.dtype);
  const bool map = c.table != nullptr;
  const uint32_t plane = map ? (uint32_t)c.grid_h * c.grid_w : 1;
  RotaryArgs<T> a = {};
  a.side[0] = {(const T*)c.q, nullptr, (long)c.q_stride, 0, (long)c.qo_stride, (T*)c.q_out, (const T*)c.gamma_q, (const T*)c.beta_q, c.H,
               rotary_slots(c.H, lanes), rotary_blocks(c.M_cap, c.H, c.Dh, c.dtype), nullptr};
  a.side[1] = {(const T*)c.k, nullptr, (long)c.k_stride, 0, (long)c.ko_stride, (T*)c.k_out, (const T*)c.gamma_k, (const T*)c.beta_k, c.Hk,
               rotary_slots(c.Hk, lanes), rotary_blocks(c.M_cap, c.Hk, c.Dh, c.dtype), nullptr};
  a.idx = c.idx;
  a.total = c.total;
  a.table = c.table;
  a.pairs_t = c.pairs_t;
  a.pairs_th = c.pairs_t + c.pairs_h;
  a.even = c.pairs_t % 2 == 0 && c.pairs_h % 2 == 0;
  a.plane = divisor(plane);
  a.tokens = divisor(map ? plane * (uint32_t)c.grid_t : 1);
  a.width = divisor(map ? (uint32_t)c.grid_w : 1);
  a.eps = c.eps;
  a.n = c.M_cap;
  return a;
}

template <typename T, int DH, int KIND, bool HALVES>
static void launch_rotary(bool back, const RotaryArgs<T>& a, hipStream_t st) {
  const dim3 grid(a.side[0].blocks + a.side[1].blocks), threads(kRotaryThreads);
  if (back) hipLaunchKernelGGL((qk_rotary_bwd_kernel<T, DH, KIND, HALVES>), grid, threads, 0, st, a);
  else hipLaunchKernelGGL((qk_rotary_kernel<T, DH, KIND, HALVES>), grid, threads, 0, st, a);
}
template <typename T, int DH>
static void launch_rotary_kind(bool back, int kind, bool halves, const RotaryArgs<T>& a, hipStream_t st) {
#define SPA_KIND(K) \
  if (kind == K) return halves ? launch_rotary<T, DH, K, true>(back, a, st) : launch_rotary<T, DH, K, false>(back, a, st)
  SPA_KIND(SPA_NORM_LAYER);
  SPA_KIND(SPA_NORM_RMS);
  SPA_KIND(SPA_NORM_NONE);
#undef SPA_KIND
}

}  // namespace spa

using namespace spa;

extern "C" int spa_qk_norm_rotary(const void* q, const void* k, int64_t q_row_stride, int64_t k_row_stride, const int32_t* gather_idx,
                                  const int32_t* total, const void* gamma_q, const void* beta_q, const void* gamma_k, const void* beta_k,
                                  int kind, float eps, const float* table, int pairs_t, int pairs_h, int grid_t, int grid_h, int grid_w,
                                  int layout, int M_cap, int H, int Hk, int Dh, int dtype, void* q_out, void* k_out,
                                  int64_t q_out_row_stride, int64_t k_out_row_stride, void* stream) {
  const char* fn = "spa_qk_norm_rotary";
  const RotaryCall c = {q, k, q_row_stride, k_row_stride, gather_idx, total, gamma_q, beta_q, gamma_k, beta_k, kind, eps, table, pairs_t, pairs_h,
                        grid_t, grid_h, grid_w, layout, M_cap, H, Hk, Dh, dtype, q_out, k_out, q_out_row_stride, k_out_row_stride};
  if (int rc = rotary_checks(fn, c)) return rc;
  const bool halves = layout == SPA_ROTARY_HALVES;
  hipStream_t st = as_stream(stream);
  if (dtype == SPA_F32) {
    const auto a = rotary_args<float>(c);
    Dh == 32 ? launch_rotary_kind<float, 32>(false, kind, halves, a, st) : launch_rotary_kind<float, 64>(false, kind, halves, a, st);
  } else {
    const auto a = rotary_args<__bf16>(c);
    Dh == 32 ? launch_rotary_kind<__bf16, 32>(false, kind, halves, a, st) : launch_rotary_kind<__bf16, 64>(false, kind, halves, a, st);
  }
  return check_launch(fn);
}

extern "C" size_t spa_qk_norm_rotary_bwd_workspace_bytes(int M_cap, int H, int Hk, int Dh, int dtype) {
  if (M_cap < 1 || H < 1 || Hk < 0 || H > kMaxRotaryHeads || Hk > kMaxRotaryHeads || (Dh != 32 && Dh != 64) ||
      (dtype != SPA_F32 && dtype != SPA_BF16))
    return 0;
  return ((size_t)rotary_parts(M_cap, H, Dh, dtype) + rotary_parts(M_cap, Hk, Dh, dtype)) * 2 * Dh * sizeof(float);
}

template <typename T>
static int rotary_bwd(const char* fn, const RotaryCall& c, const void* dq_out, const void* dk_out, int64_t dqo_stride, int64_t dko_stride,
                      float* dgamma_q, float* dbeta_q, float* dgamma_k, float* dbeta_k, float* ws, hipStream_t st) {
  RotaryArgs<T> a = rotary_args<T>(c);
  const bool sums = c.kind != SPA_NORM_NONE;
  for (int i = 0; i < 2; ++i) {
    RotarySide<T>& s = a.side[i];
    s.d = (const T*)(i ? dk_out : dq_out);
    s.ds = (long)(i ? dko_stride : dqo_stride);
    s.blocks = sums ? rotary_parts(c.M_cap, s.heads, c.Dh, c.dtype) : s.blocks;
    s.partial = !sums ? nullptr : i == 0 ? ws : ws + (size_t)a.side[0].blocks * 2 * c.Dh;
  }
  const bool halves = c.layout == SPA_ROTARY_HALVES;
  if (c.Dh == 32) launch_rotary_kind<T, 32>(true, c.kind, halves, a, st);
  else launch_rotary_kind<T, 64>(true, c.kind, halves, a, st);
  if (sums && (dgamma_q || dbeta_q || dgamma_k || dbeta_k)) {
    const RotarySums r = {{a.side[0].partial, a.side[1].partial}, {(int)a.side[0].blocks, (int)a.side[1].blocks}, {dgamma_q, dgamma_k},
                          {dbeta_q, dbeta_k}, c.Dh};
    hipLaunchKernelGGL(qk_rotary_sums_kernel, dim3((c.Hk > 0 ? 2 : 1) * 2 * c.Dh / 16), dim3(1024), 0, st, r);
  }
  return check_launch(fn);
}

extern "C" int spa_qk_norm_rotary_bwd(const void* dq_out, const void* dk_out, int64_t dq_out_row_stride, int64_t dk_out_row_stride, const void* q,
                                      const void* k, int64_t q_row_stride, int64_t k_row_stride, const int32_t* gather_idx, const int32_t* total,
                                      const void* gamma_q, const void* gamma_k, int kind, float eps, const float* table, int pairs_t,
                                      int pairs_h, int grid_t, int grid_h, int grid_w, int layout, int M_cap, int H, int Hk, int Dh, int dtype,
                                      void* dq, void* dk, int64_t dq_row_stride, int64_t dk_row_stride, float* dgamma_q, float* dbeta_q,
                                      float* dgamma_k, float* dbeta_k, void* workspace, size_t workspace_bytes, void* stream) {
  const char* fn = "spa_qk_norm_rotary_bwd";
  const RotaryCall c = {q, k, q_row_stride, k_row_stride, gather_idx, total, gamma_q, nullptr, gamma_k, nullptr, kind, eps, table, pairs_t, pairs_h,
                        grid_t, grid_h, grid_w, layout, M_cap, H, Hk, Dh, dtype, dq, dk, dq_row_stride, dk_row_stride};
  if (int rc = rotary_checks(fn, c)) return rc;
  if (int rc = rotary_rows_ok(fn, "dq_out", dq_out, dq_out_row_stride, H, Dh, dtype)) return rc;
  if (Hk > 0)
    if (int rc = rotary_rows_ok(fn, "dk_out", dk_out, dk_out_row_stride, Hk, Dh, dtype)) return rc;
  SPA_REQUIRE((dq != dq_out || dq_row_stride == dq_out_row_stride) && (Hk == 0 || dk != dk_out || dk_row_stride == dk_out_row_stride), SPA_ERR_INVALID_ARG,
              "%s: in place the row strides must be the same", fn);
  SPA_REQUIRE(kind != SPA_NORM_NONE || (!dgamma_q && !dbeta_q && !dgamma_k && !dbeta_k), SPA_ERR_INVALID_ARG,
              "%s: gradients of gamma and beta belong to a norm", fn);
  SPA_REQUIRE(Hk > 0 || (!dgamma_k && !dbeta_k), SPA_ERR_INVALID_ARG, "%s: without k there is no gradient of its gamma and beta", fn);
  const size_t need = kind == SPA_NORM_NONE ? 0 : spa_qk_norm_rotary_bwd_workspace_bytes(M_cap, H, Hk, Dh, dtype);
  SPA_REQUIRE(need == 0 || (workspace != nullptr && workspace_bytes >= need), SPA_ERR_WORKSPACE, "%s: workspace of %zu bytes needed, %zu given",
              fn, need, workspace_bytes);
  hipStream_t st = as_stream(stream);
  return dtype == SPA_F32 ? rotary_bwd<float>(fn, c, dq_out, dk_out, dq_out_row_stride, dk_out_row_stride, dgamma_q, dbeta_q, dgamma_k, dbeta_k,
                                              (float*)workspace, st)
                          : rotary_bwd<__bf16>(fn, c, dq_out, dk_out, dq_out_row_stride, dk_out_row_stride, dgamma_q, dbeta_q, dgamma_k,
                                               dbeta_k, (float*)workspace, st);
}
