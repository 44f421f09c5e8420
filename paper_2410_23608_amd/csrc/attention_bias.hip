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

#include "spa_common.h"

namespace spa {

struct BiasMap {
  const void* table;             // [H, nb]
  const int32_t *buckets, *gather_idx;
  int nb, gw, tokens, offsets, centre;      // tokens = gh gw
};

// Position index of packed row `row`, number j of its segment
__device__ __forceinline__ int bias_position(const BiasMap& m, long row, int j) {
  const unsigned n = m.gather_idx != nullptr ? (unsigned)m.gather_idx[row] % (unsigned)m.tokens : (unsigned)min(j, m.tokens - 1);
  const unsigned r = n / (unsigned)m.gw;
  return (int)(r * (2 * m.gw - 1) + (n - r * m.gw));
}
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
  SPA_REQUIRE(softmax_scale >= 0.f && std::isfinite(softmax_scale), SPA_ERR_INVALID_ARG,
              "%s: softmax_scale must be finite and >= 0 (0 = 1/sqrt(Dh))", fn);
  SPA_REQUIRE(grid_h >= 1 && grid_w >= 1 && (2 * (long)grid_h - 1) * (2 * (long)grid_w - 1) <= (1L << 26), SPA_ERR_INVALID_ARG,
              "%s: grid_h, grid_w must be >= 1, with at most 2^26 offsets", fn);
  const long offsets = (2 * (long)grid_h - 1) * (2 * (long)grid_w - 1);
  SPA_REQUIRE(n_buckets >= 1 && n_buckets <= (1 << 26), SPA_ERR_INVALID_ARG, "%s: n_buckets must lie in 1 .. 2^26", fn);
  SPA_REQUIRE(buckets != nullptr || n_buckets == offsets, SPA_ERR_INVALID_ARG,
              "%s: without a bucket map there is a bucket per offset, %ld of them", fn, offsets);
  SPA_REQUIRE(n_max <= (long)grid_h * grid_w, SPA_ERR_INVALID_ARG, "%s: max_seqlen exceeds the %d x %d map", fn, grid_h, grid_w);
  *m = {table, buckets, gather_idx, n_buckets, grid_w, grid_h * grid_w, (int)offsets, (grid_h - 1) * (2 * grid_w - 1) + grid_w - 1};
  return SPA_OK;
}

// Bits below the bound that a sum of that many values leaves: 62 less those of their number, at most 40.
static int ds_shift(long rows) {
  int bits = 0;
  while ((1L << bits) < rows) ++bits;
  return std::min(40, 62 - bits);
}
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
  const dim3 grid((max_seqlen + kRowThreads - 1) / kRowThreads, H, B);
#define SPA_BIAS(T, D)                                                                                                         \
  hipLaunchKernelGGL((attn_bias_rows_kernel<T, D>), grid, dim3(kRowThreads), 0, st, (const T*)q, (const T*)k, (const T*)v,       \
                     (long)q_row_stride, (long)k_row_stride, (long)v_row_stride, cu_seqlens, m, H, scale, (T*)out, lse, ls)
  if (dtype == SPA_F32) {
    if (Dh == 32) SPA_BIAS(float, 32); else SPA_BIAS(float, 64);
  } else {
    if (Dh == 32) SPA_BIAS(__bf16, 32); else SPA_BIAS(__bf16, 64);
  }
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
