// Attention of packed rows to the keys of another sequence of another length (an encoder's states, the packed tokens themselves for a few
// queries): O = softmax(scale Q K^T) V, rows of segment b against the keys of segment b, key heads shared by G query heads; segments
// without a key give 0.
//
// A wave owns 32 rows (tokens times heads of a group, cross_attention.h) and computes S^T = K Q^T, so that a lane holds 16 keys of one
// row a 32 x 32 block, and the probabilities (bf16: rounded) are the second product's operand in registers; K and V stream through LDS.
// The maximum and the sum run along, in fp32.  Few rows: the four waves share 32 (or 64) of them, each with its part of every step of keys;
// few units with long keys: the keys are split over workgroups, which leave unnormalised sums, maxima and row sums in fp32 for a
// second launch that joins them in the order of the splits.
// Bound by the vector instructions of the softmax where there is work (of the busy cycles three quarters, the matrix pipe a third): 8 x
// 1568 to 3136 tokens against 410 to 1024 states, 12 and 4 heads of 64, 71 us; by the keys' bytes for few rows (one token of 4 sequences of
// 11200 to 16000 keys, 16 and 4 heads, 14 + 4 us); by chains of trips to memory for short segments (64 x 196 tokens to captions of up to
// 77, 13 us; one image 4.6). fp32: 8 x 1568 to 3136 tokens, 410 to 1024 states, 428 us = 111 of 154 TFLOP/s (backward 1675, 71), to
// captions 41 (132).
#include <algorithm>
#include <cmath>

#include "cross_attention.h"

namespace spa {

template <typename T>
struct CrossFwd {
  const T *q, *k, *v;
  long qs, ks, vs;
  CrossShape s;
  T* out;
  float* lse;
  float* part;                   // [unit][split][row of the unit][DH], then [..][row][2]: maximum and sum; or null
  long part_rows;                // rows of a unit there
  float* part_ms;
};

template <typename T, int DH, int KW>
struct CrossTiles {
  static constexpr int STEP = CrossSteps<KW>::STEP, RS = Ops<T, DH>::RS;
  __attribute__((aligned(16))) T K[2][STEP * RS];
  __attribute__((aligned(16))) T V[2][STEP * RS];
};

// (Maximum and exponentials block by block of 32 keys: two at a time take 147 registers at heads of 64, three waves a SIMD; 64 x 196 tokens
// to captions 14.1 us then, 13.1 so, long keys the same.)
template <typename T, int DH, int KW>
__global__ void __launch_bounds__(kCrossThreads, sizeof(T) == 2 && KW == 1 ? 4 : 1) cross_fwd_kernel(const CrossFwd<T> a) {
  using O = Ops<T, DH>;
  using W = CrossSteps<KW>;
  constexpr int DB = DH / 32, NB = W::TILE / 32;
  extern __shared__ __attribute__((aligned(16))) unsigned char cross_smem[];
  CrossTiles<T, DH, KW>& l = *reinterpret_cast<CrossTiles<T, DH, KW>*>(cross_smem);
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
  const long first = u.k0 + sh.from;
  floatx16 o[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
  float m = -INFINITY, sum = 0.f;
  CrossStage<T, DH, W::STEP, false> st(a.k + first * a.ks + u.hk * DH, a.ks, a.v + first * a.vs + u.hk * DH, a.vs, a.s.G, n - 1);
  if (nt > 0) st.load(0);
  const typename O::Row qf = O::row(a.q + u.q0 * a.qs + (long)u.hk * G * DH + group_row<DH>(a.s.G, rc, a.qs), hh);
  if (nt > 0) st.template store<true>(l.K[0], l.V[0]);
  __syncthreads();
  walk_tiles(nt, [&](int t, auto at) {
    constexpr bool end = decltype(at)::value == kTileLast;
    const int buf = t & 1, left = n - t * W::STEP - part * W::TILE;
    if (!end) st.load(t * W::STEP + W::STEP);
    if (wave_live && (!end || left > 0)) {
      const T *K = &l.K[buf][part * W::TILE * O::RS], *V = &l.V[buf][part * W::TILE * O::RS];
#pragma unroll
      for (int sb = 0; sb < NB; ++sb) {
        if (end && sb * 32 >= left) break;
        floatx16 s;
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = 0.f;
        O::dot(s, O::row(&K[(sb * 32 + l32) * O::RS], hh), qf);
        if (end) {
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (sb * 32 + acc_row(i, hh) >= left) s[i] = -INFINITY;
        }
        float mx = s[0];
#pragma unroll
        for (int i = 0; i < 16; ++i) mx = __builtin_elementwise_maximum(mx, s[i]);
        const float m_new = __builtin_elementwise_maximum(m, max_across_halves(mx));
        // (m, what the exponents are taken from, follows a row's maximum when that is 2^8 past it, or a NaN: of 32 rows one has a new
        // maximum in nearly every block)
        const bool past = !((m_new - m) * a.s.c <= 8.f);
        if (__ballot(past) != 0) {
          const float f = past && m_new != m ? __builtin_amdgcn_exp2f((m - m_new) * a.s.c) : 1.f;
          sum *= f;
#pragma unroll
          for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[d][i] *= f;
          m = past ? m_new : m;
        }
        if (__ballot(fabsf(m) * a.s.scale >= kFarScore) == 0) {
          const float m2 = m * a.s.c;
#pragma unroll
          for (int i = 0; i < 16; ++i) s[i] = __builtin_amdgcn_exp2f(fmaf(s[i], a.s.c, -m2));
        } else {
          const float ref = m == -INFINITY ? 0.f : m;           // (no score yet: weights of 0)
#pragma unroll
          for (int i = 0; i < 16; ++i) s[i] = __builtin_amdgcn_exp2f((s[i] - ref) * a.s.c);
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) sum += s[i];
        O::outer(o, V, sb, s, lane);
      }
    }
    if (!end) st.template store<decltype(at)::value == kTileBeforeLast>(l.K[buf ^ 1], l.V[buf ^ 1]);
    __syncthreads();
  });
  // the waves that share rows: the others hand their sums to the first, which adds them in order
  if constexpr (KW > 1) {
    constexpr int N = DB * 16 + 2;
    static_assert((KW - 1) * W::RW * N * kWave * sizeof(float) <= sizeof(CrossTiles<T, DH, KW>), "the sums of the other waves");
    float* const sums = reinterpret_cast<float*>(cross_smem) + lane;
    if (part > 0) {
      float* mine = sums + ((part - 1) * W::RW + rw) * N * kWave;
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) mine[(d * 16 + i) * kWave] = o[d][i];
      mine[(N - 2) * kWave] = m;
      mine[(N - 1) * kWave] = sum;
    }
    __syncthreads();
    if (part > 0) return;
#pragma unroll
    for (int p = 0; p < KW - 1; ++p) {
      const float* other = sums + (p * W::RW + rw) * N * kWave;
      const float m1 = other[(N - 2) * kWave], both = __builtin_elementwise_maximum(m, m1);
      const float f0 = m == both ? 1.f : __builtin_amdgcn_exp2f((m - both) * a.s.c);
      const float f1 = m1 == both ? 1.f : __builtin_amdgcn_exp2f((m1 - both) * a.s.c);
      m = both;
      sum = sum * f0 + other[(N - 1) * kWave] * f1;
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] = o[d][i] * f0 + other[(d * 16 + i) * kWave] * f1;
    }
  }
  if (!wave_live) return;
  const float total = sum_across_halves(sum);
  if (a.part != nullptr) {
    const long at = (((long)u.b * a.s.Hk + u.hk) * a.s.splits + u.split) * a.part_rows + rc;
    if (!ok) return;
    float* row = a.part + at * DH;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *reinterpret_cast<floatx4*>(row + d * 32 + 8 * g + 4 * hh) = floatx4{o[d][4 * g], o[d][4 * g + 1], o[d][4 * g + 2], o[d][4 * g + 3]};
    if (hh == 0) *reinterpret_cast<floatx2*>(a.part_ms + at * 2) = floatx2{m, total};
    return;
  }
  const float inv = total == 0.f ? 0.f : 1.0f / total;          // (0: no key, all weights 0)
  const long C = (long)a.s.H * DH;
  O::store(o, inv, a.out + u.q0 * C + (long)u.hk * G * DH + group_row<DH>(a.s.G, rc, C), ok, hh);
  if (a.lse != nullptr && ok && hh == 0) {
    const uint32_t i = quotient((uint32_t)rc, a.s.G);
    a.lse[(u.hk * G + (rc - (int)(i * G))) * a.s.stat_stride + u.q0 + i] = total == 0.f ? -INFINITY : m * a.s.scale + logf(total);
  }
}

// Joins the splits of a row: DH / 4 lanes take a row's columns, SL of such groups every SL-th split each, and the first adds the groups'
// sums in their order.  SL 1 for many rows.
template <typename T, int DH, int STEP, int SL>
__global__ void __launch_bounds__(kCrossThreads) cross_join_kernel(const CrossFwd<T> a) {
  constexpr int LANES = DH / 4, ROWS = kCrossThreads / LANES / SL, U = SL > 1 ? 4 : 8;
  __shared__ floatx4 other_o[SL > 1 ? SL - 1 : 1][ROWS][LANES];
  __shared__ floatx2 other_ms[SL > 1 ? SL - 1 : 1][ROWS];
  const int G = (int)a.s.G.d, lane = threadIdx.x % LANES, c = lane * 4, in = threadIdx.x / LANES % ROWS, sl = threadIdx.x / LANES / ROWS;
  const long per = (a.part_rows + ROWS - 1) / ROWS, unit = blockIdx.x / per;
  const int r = (int)(blockIdx.x % per) * ROWS + in, b = (int)(unit / a.s.Hk), hk = (int)(unit % a.s.Hk);
  const int q0 = a.s.cu_q[b];
  int nq, nk, held;
  cross_lengths(a.s, b, q0, a.s.cu_k[b], nq, nk, held);
  const bool ok = r < nq;
  const int live = ok ? share_of<STEP>(nk, a.s.splits, 0).live : 0;
  const long at = unit * a.s.splits * a.part_rows + r;
  float m = -INFINITY, sum = 0.f;
  floatx4 o = {0.f, 0.f, 0.f, 0.f};
  auto add = [&](float m1, float sum1, const floatx4& o1) {
    const float both = __builtin_elementwise_maximum(m, m1);
    const float f0 = m == both ? 1.f : __builtin_amdgcn_exp2f((m - both) * a.s.c);
    const float f1 = m1 == both ? 1.f : __builtin_amdgcn_exp2f((m1 - both) * a.s.c);
    m = both;
    sum = sum * f0 + sum1 * f1;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = o[e] * f0 + o1[e] * f1;
  };
  for (int s0 = sl; s0 < live; s0 += U * SL) {
    floatx2 ms[U];
    floatx4 v[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const long row = at + (long)min(s0 + i * SL, live - 1) * a.part_rows;
      ms[i] = *reinterpret_cast<const floatx2*>(a.part_ms + row * 2);
      v[i] = *reinterpret_cast<const floatx4*>(a.part + row * DH + c);
    }
#pragma unroll
    for (int i = 0; i < U; ++i)
      if (s0 + i * SL < live) add(ms[i][0], ms[i][1], v[i]);
  }
  if constexpr (SL > 1) {
    if (sl > 0) {
      other_o[sl - 1][in][lane] = o;
      if (lane == 0) other_ms[sl - 1][in] = floatx2{m, sum};
    }
    __syncthreads();
    if (sl > 0) return;
    for (int i = 0; i < SL - 1; ++i) add(other_ms[i][in][0], other_ms[i][in][1], other_o[i][in][lane]);
  }
  if (!ok) return;
  const float inv = sum == 0.f ? 0.f : 1.0f / sum;
  const long C = (long)a.s.H * DH;
  const uint32_t i = quotient((uint32_t)r, a.s.G);
  const int h = hk * G + r - (int)(i * G);
  T* to = a.out + ((long)q0 + i) * C + (long)h * DH + c;
  if constexpr (sizeof(T) == 2) *reinterpret_cast<bf16x4*>(to) = __builtin_convertvector(o * inv, bf16x4);
  else *reinterpret_cast<floatx4*>(to) = o * inv;
  if (a.lse != nullptr && c == 0) a.lse[h * a.s.stat_stride + q0 + i] = sum == 0.f ? -INFINITY : m * a.s.scale + logf(sum);
}

// ------------------------------------------------------------------------------- host
size_t cross_up(size_t n) { return (n + 255) & ~(size_t)255; }

bool cross_sizes_ok(int B, int max_q, int max_k, int H, int Hk, int Dh, int dtype) {
  return B >= 1 && B <= 65535 && max_q >= 1 && max_k >= 1 && H >= 1 && H <= 65535 && Hk >= 1 && H % Hk == 0 && (long)B * max_q < 2147483647L &&
         (long)B * max_k < 2147483647L && max_k < 2147483647 - 256 && (long)max_q * (H / Hk) < 2147483647L - 256 && (Dh == 32 || Dh == 64) &&
         (dtype == SPA_F32 || dtype == SPA_BF16);
}

// Few workgroups: the waves of one share its owned rows, two by two or all four, as long as one round of workgroups holds them all.  Fewer
// still and many rows on the other side: these are split, into no less than `least` each, until there are about four workgroups a unit.
CrossPlan cross_plan(long units, long owned, long others, int dtype) {
  CrossPlan p = {1, 1, 1};
  const long least = dtype == SPA_F32 ? 256 : 512;
  auto blocks = [&](int kw) { return (owned + 128 / kw - 1) / (128 / kw); };
  while (p.kw < 4 && (owned <= 64 / p.kw || (dtype == SPA_F32 && units * blocks(2 * p.kw) <= 512))) p.kw *= 2;
  p.blocks = (int)blocks(p.kw);
  const long groups = units * p.blocks;
  if (groups < 512) p.splits = (int)std::max(1L, std::min((1024 + groups - 1) / groups, others / least));
  return p;
}

CrossShape cross_shape(const CrossCall& c, const CrossPlan& p) {
  const float scale = c.softmax_scale > 0.f ? c.softmax_scale : 1.0f / std::sqrt((float)c.Dh);
  return {c.cu_q, c.cu_k, c.key_lens, c.B, c.H, c.Hk, divisor((uint32_t)(c.H / c.Hk)), p.blocks, p.splits, scale, scale * kLog2e,
          (long)c.B * c.max_q, c.max_q, c.max_k};
}

int cross_checks(const char* fn, const CrossCall& c) {
  SPA_REFUSE_IN_GROUP(fn);
  SPA_REQUIRE(c.q && c.k && c.v && c.cu_q && c.cu_k, SPA_ERR_INVALID_ARG, "%s: null pointer", fn);
  SPA_REQUIRE(c.B >= 1 && c.max_q >= 1 && c.max_k >= 1 && c.H >= 1 && c.Hk >= 1, SPA_ERR_INVALID_ARG, "%s: B, max_q, max_k, H, Hk must be >= 1", fn);
  SPA_REQUIRE(c.H % c.Hk == 0, SPA_ERR_INVALID_ARG, "%s: H = %d is not a multiple of Hk = %d", fn, c.H, c.Hk);
  SPA_REQUIRE(c.B <= 65535 && c.H <= 65535, SPA_ERR_INVALID_ARG, "%s: B and H must be <= 65535", fn);
  SPA_REQUIRE((long)c.B * c.max_q < 2147483647L && (long)c.B * c.max_k < 2147483647L, SPA_ERR_INVALID_ARG, "%s: B*max_q and B*max_k must be < 2^31", fn);
  // (a step's places past the last row or key are formed in an int before they are cut)
  SPA_REQUIRE((long)c.max_q * (c.H / c.Hk) < 2147483647L - 256, SPA_ERR_INVALID_ARG, "%s: max_q*H/Hk must be < 2^31 - 257", fn);
  SPA_REQUIRE(c.max_k < 2147483647 - 256, SPA_ERR_INVALID_ARG, "%s: max_k must be < 2^31 - 257", fn);
  SPA_REQUIRE(c.dtype == SPA_F32 || c.dtype == SPA_BF16, SPA_ERR_UNSUPPORTED, "%s: unknown dtype %d", fn, c.dtype);
  SPA_REQUIRE(c.Dh == 32 || c.Dh == 64, SPA_ERR_UNSUPPORTED, "%s: head dim %d not supported (32 or 64)", fn, c.Dh);
  const int64_t strides[3] = {c.qs, c.ks, c.vs};
  for (int i = 0; i < 3; ++i) {
    SPA_REQUIRE(strides[i] >= (int64_t)(i == 0 ? c.H : c.Hk) * c.Dh, SPA_ERR_INVALID_ARG, "%s: row stride %ld < heads * Dh", fn, (long)strides[i]);
    SPA_REQUIRE(strides[i] < (1LL << 31), SPA_ERR_INVALID_ARG, "%s: row stride %ld must be < 2^31 elements", fn, (long)strides[i]);
    SPA_REQUIRE(strides[i] * elem_size(c.dtype) % 16 == 0, SPA_ERR_INVALID_ARG, "%s: row stride is not a multiple of 16 bytes", fn);
  }
  SPA_REQUIRE(aligned16(c.q) && aligned16(c.k) && aligned16(c.v), SPA_ERR_INVALID_ARG, "%s: q/k/v not 16-byte aligned", fn);
  SPA_REQUIRE(c.softmax_scale >= 0.f && std::isfinite(c.softmax_scale), SPA_ERR_INVALID_ARG,
              "%s: softmax_scale must be finite and >= 0 (0 = 1/sqrt(Dh))", fn);
  return SPA_OK;
}

static CrossPlan fwd_plan(int B, int max_q, int max_k, int H, int Hk, int dtype) { return cross_plan((long)B * Hk, (long)max_q * (H / Hk), max_k, dtype); }

template <typename T, int DH, int KW>
static int launch_fwd(const char* fn, const CrossFwd<T>& a, hipStream_t st) {
  constexpr size_t lds = sizeof(CrossTiles<T, DH, KW>);
  const auto kernel = cross_fwd_kernel<T, DH, KW>;
  const hipError_t attr = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
  SPA_REQUIRE(attr == hipSuccess, SPA_ERR_HIP, "%s: cannot reserve %zu bytes of LDS", fn, lds);
  hipLaunchKernelGGL(kernel, dim3((unsigned)cross_grid(a.s)), dim3(kCrossThreads), lds, st, a);
  if (a.part != nullptr) {
    constexpr int many = kCrossThreads / (DH / 4), few = 1;
    const long units = (long)a.s.B * a.s.Hk;
    if (units * a.part_rows <= 4096)
      hipLaunchKernelGGL((cross_join_kernel<T, DH, CrossSteps<KW>::STEP, many>), dim3((unsigned)(units * a.part_rows)), dim3(kCrossThreads), 0, st, a);
    else
      hipLaunchKernelGGL((cross_join_kernel<T, DH, CrossSteps<KW>::STEP, few>), dim3((unsigned)(units * ((a.part_rows + many - 1) / many))),
                         dim3(kCrossThreads), 0, st, a);
  }
  return check_launch(fn);
}

template <typename T>
static int run_fwd(const char* fn, const CrossCall& c, const CrossPlan& p, void* out, float* lse, void* ws, hipStream_t st) {
  CrossFwd<T> a = {(const T*)c.q, (const T*)c.k, (const T*)c.v, (long)c.qs, (long)c.ks, (long)c.vs, cross_shape(c, p), (T*)out, lse, nullptr, 0, nullptr};
  if (p.splits > 1) {
    a.part_rows = (long)c.max_q * (c.H / c.Hk);
    a.part = (float*)ws;
    a.part_ms = (float*)((char*)ws + cross_up((size_t)c.B * c.Hk * p.splits * a.part_rows * c.Dh * sizeof(float)));
  }
#define SPA_KW(D) \
  return p.kw == 1 ? launch_fwd<T, D, 1>(fn, a, st) : p.kw == 2 ? launch_fwd<T, D, 2>(fn, a, st) : launch_fwd<T, D, 4>(fn, a, st)
  if (c.Dh == 32) SPA_KW(32);
  SPA_KW(64);
#undef SPA_KW
}

}  // namespace spa

using namespace spa;

extern "C" size_t spa_cross_attention_workspace_bytes(int B, int max_q, int max_k, int H, int Hk, int Dh, int dtype) {
  if (!cross_sizes_ok(B, max_q, max_k, H, Hk, Dh, dtype)) return 0;
  const CrossPlan p = fwd_plan(B, max_q, max_k, H, Hk, dtype);
  if (p.splits == 1) return 0;
  const size_t rows = (size_t)B * max_q * H * p.splits;
  return cross_up(rows * Dh * sizeof(float)) + cross_up(rows * 2 * sizeof(float));
}

extern "C" int spa_cross_attention(const void* q, const void* k, const void* v, int64_t q_row_stride, int64_t k_row_stride, int64_t v_row_stride,
                                   const int32_t* cu_seqlens_q, const int32_t* cu_seqlens_k, const int32_t* key_lens, int B, int max_q,
                                   int max_k, int H, int Hk, int Dh, int dtype, float softmax_scale, void* out, float* lse, void* workspace,
                                   size_t workspace_bytes, void* stream) {
  const char* fn = "spa_cross_attention";
  const CrossCall c = {q, k, v, q_row_stride, k_row_stride, v_row_stride, cu_seqlens_q, cu_seqlens_k, key_lens, B, max_q, max_k, H, Hk, Dh, dtype,
                       softmax_scale};
  if (int rc = cross_checks(fn, c)) return rc;
  SPA_REQUIRE(out != nullptr, SPA_ERR_INVALID_ARG, "%s: out is null", fn);
  SPA_REQUIRE(aligned16(out), SPA_ERR_INVALID_ARG, "%s: out not 16-byte aligned", fn);
  const CrossPlan p = fwd_plan(B, max_q, max_k, H, Hk, dtype);
  SPA_REQUIRE(((long)Hk * B + 8) * p.blocks * p.splits < 4294967296L / kCrossThreads, SPA_ERR_INVALID_ARG,
              "%s: too many workgroups (B*max_q*H must be < about 2^31)", fn);
  const size_t need = spa_cross_attention_workspace_bytes(B, max_q, max_k, H, Hk, Dh, dtype);
  SPA_REQUIRE(need == 0 || (workspace != nullptr && workspace_bytes >= need), SPA_ERR_WORKSPACE, "%s: workspace of %zu bytes needed, %zu given",
              fn, need, workspace_bytes);
  SPA_REQUIRE(need == 0 || (reinterpret_cast<uintptr_t>(workspace) & 255u) == 0, SPA_ERR_INVALID_ARG, "%s: workspace not 256-byte aligned", fn);
  return dtype == SPA_F32 ? run_fwd<float>(fn, c, p, out, lse, workspace, as_stream(stream))
                          : run_fwd<__bf16>(fn, c, p, out, lse, workspace, as_stream(stream));
}
