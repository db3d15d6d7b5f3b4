// Attention of many query rows to packed rows that all of them see: cross
// attention (query rows of a sequence against its whole cache) and the decode
// step of a batch that shares a prefix (every sequence's query against the
// prefix's cache and its own).
//
// Both are passes over one form: the query rows of a unit (layer, sequence,
// KV head) against rows [0, len) of one packed cache, the key axis in splits.
// A pass leaves per query row and split (m, l, acc[128]): the maximum of the
// base-2 logits, sum 2^(s - m) and sum 2^(s - m) v in the rotated value
// domain.  Partial states of disjoint row sets merge as
//   m = max m_i,  l = sum l_i 2^(m_i - m),  a = sum a_i 2^(m_i - m),
// so a prefix is one more set of splits.  k_merge joins a row's partials,
// divides by l, rotates back (Pi_V^T) and rounds to the output type.
#include <hip/hip_runtime.h>

#include "kernels.h"
#include "layout.h"

namespace bgtq {
namespace cross_detail {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kNegInf = -__builtin_huge_valf();
constexpr float kRsqrtD = 0.08838834764831845f;  // 1 / sqrt(128)
constexpr int kThreads = 256;
constexpr int kRows = 16;  // query rows of a workgroup

__device__ __forceinline__ float half_bits(uint16_t b) { return static_cast<float>(__builtin_bit_cast(_Float16, b)); }
__device__ __forceinline__ float ld_q(const void* q, size_t i, int dtype) {  // BGTQ_BF16 = 1
  if (dtype == 1) return __uint_as_float(static_cast<uint32_t>(static_cast<const uint16_t*>(q)[i]) << 16);
  return static_cast<const float*>(q)[i];
}

// One-dimensional grid over (layer in call x sequence, KV head, row block,
// split).  fp32 products of a 64-row tile decoded into LDS.
__global__ __launch_bounds__(kThreads) void k_cross(Dims d, const uint8_t* __restrict__ blob, const void* __restrict__ q,
                                                    int n_q, const int32_t* __restrict__ ctx_len, CachePtrs c,
                                                    CrossPass ps) {
  __shared__ float qr[kRows][kHeadDim], s[kRows][kKeyTile];
  __shared__ float kt[kKeyTile][kHeadDim + 1], vt[kKeyTile][kHeadDim];
  __shared__ float mrow[kRows], lrow[kRows], corr[kRows];
  const int tid = threadIdx.x, G = d.group, hq = d.n_kv * G, nr = n_q * G;
  const int n_blocks = (nr + kRows - 1) / kRows;
  long item = blockIdx.x;
  const int split = static_cast<int>(item % ps.n_splits);
  item /= ps.n_splits;
  const int block = static_cast<int>(item % n_blocks);
  item /= n_blocks;
  const int kvh = static_cast<int>(item % d.n_kv), lz = static_cast<int>(item / d.n_kv);
  const int seq = lz % d.batch, layer = d.layer >= 0 ? d.layer : lz / d.batch;
  const int r0 = block * kRows;
  const RowMeta* M = reinterpret_cast<const RowMeta*>(blob + kOffRows) + (layer * d.n_kv + kvh);
  const float* w = reinterpret_cast<const float*>(blob + layout_kdense_offset(d.n_layers * d.n_kv)) +
                   static_cast<size_t>(layer * d.n_kv + kvh) * kMfmaMatFloats;
  const uint16_t* c16 = reinterpret_cast<const uint16_t*>(blob + kOffC16);
  const size_t row = (static_cast<size_t>(layer) * d.batch + seq) * d.n_kv + kvh;
  const uint32_t* kc = c.k_codes + row * d.capacity * d.k_words;
  const uint16_t* kn = c.k_norms + row * kMaxGroups * d.capacity;
  const uint32_t* vc = c.v_codes + row * (d.capacity / kTile) * kHeadDim * d.v_bits;
  const uint16_t* vn = c.v_norms + row * d.capacity;
  const int slots = (M->n_groups + 1) & ~1;
  // q' = W q log2(e) / sqrt(d_g 128)
  for (int i = tid; i < kRows * kHeadDim; i += kThreads) {
    const int r = r0 + i / kHeadDim, p = i % kHeadDim;
    float a = 0.f;
    if (r < nr) {
      const size_t base = ((static_cast<size_t>(lz) * n_q + r / G) * hq + kvh * G + r % G) * kHeadDim;
      for (int k = 0; k < kHeadDim; ++k) a = fmaf(w[mfma_mat_index(p, k)], ld_q(q, base + k, d.in_dtype), a);
    }
    qr[i / kHeadDim][p] = a * kLog2e * rsqrtf(static_cast<float>(M->g_dim[M->grp[p]])) * kRsqrtD;
  }
  if (tid < kRows) {
    mrow[tid] = kNegInf;
    lrow[tid] = 0.f;
  }
  float acc[kRows * kHeadDim / kThreads];  // dim tid % 128 of rows tid / 128 + 2 j
  for (float& a : acc) a = 0.f;
  const int len = ctx_len[seq];
  const bool ok = len >= 0 && len <= ps.max_len;
  const int t0 = split * ps.split_len, t1 = ok ? min(len, t0 + ps.split_len) : t0;
  for (int ta = t0; ta < t1; ta += kKeyTile) {
    __syncthreads();
    for (int i = tid; i < kKeyTile * kHeadDim; i += kThreads) {
      const int tok = i / kHeadDim, p = i % kHeadDim, t = ta + tok;
      const uint32_t* kr = kc + static_cast<size_t>(t) * d.k_words;
      const int off = M->bitoff[p], width = M->width[p];
      uint64_t f = kr[off >> 5];
      if ((off & 31) + width > 32) f |= static_cast<uint64_t>(kr[(off >> 5) + 1]) << 32;
      const uint32_t code = static_cast<uint32_t>(f >> (off & 31)) & ((1u << width) - 1u);
      kt[tok][p] = half_bits(c16[cb_index(width) + code]) * half_bits(kn[static_cast<size_t>(t) * slots + M->grp[p]]);
      const int vo = (t % kTile) * d.v_bits;
      const uint32_t* vr = vc + (static_cast<size_t>(t / kTile) * kHeadDim + p) * d.v_bits;
      f = vr[vo >> 5];
      if ((vo & 31) + d.v_bits > 32) f |= static_cast<uint64_t>(vr[(vo >> 5) + 1]) << 32;
      const uint32_t vcode = static_cast<uint32_t>(f >> (vo & 31)) & ((1u << d.v_bits) - 1u);
      // (rows behind the last one hold whatever was appended there: no product with them)
      vt[tok][p] = t < t1 ? half_bits(c16[cb_index(d.v_bits) + vcode]) * half_bits(vn[t]) : 0.f;
    }
    __syncthreads();
    for (int i = tid; i < kRows * kKeyTile; i += kThreads) {
      const int r = i / kKeyTile, tok = i % kKeyTile;
      float x = 0.f;
      for (int p = 0; p < kHeadDim; ++p) x = fmaf(qr[r][p], kt[tok][p], x);
      s[r][tok] = ta + tok < t1 ? x : kNegInf;
    }
    __syncthreads();
    if (tid < kRows) {
      float m = mrow[tid], l = lrow[tid];
      float mn = m;
      for (int k = 0; k < kKeyTile; ++k) mn = fmaxf(mn, s[tid][k]);
      const float e = m == kNegInf ? 0.f : exp2f(m - mn);
      l *= e;
      const float ref = mn == kNegInf ? 0.f : mn;
      for (int k = 0; k < kKeyTile; ++k) l += s[tid][k] = exp2f(s[tid][k] - ref);
      mrow[tid] = mn;
      lrow[tid] = l;
      corr[tid] = e;
    }
    __syncthreads();
    for (int j = 0; j < kRows * kHeadDim / kThreads; ++j) {
      const int r = tid / kHeadDim + 2 * j;
      float a = acc[j] * corr[r];
      for (int k = 0; k < kKeyTile; ++k) a = fmaf(s[r][k], vt[k][tid % kHeadDim], a);
      acc[j] = a;
    }
  }
  __syncthreads();
  for (int j = 0; j < kRows * kHeadDim / kThreads; ++j) {
    const int rr = tid / kHeadDim + 2 * j, r = r0 + rr;
    if (r >= nr) continue;
    float* o = ps.part + (((static_cast<size_t>(lz) * n_q + r / G) * hq + kvh * G + r % G) * ps.n_slots + ps.slot0 + split) *
                             kPartFloats;
    o[2 + tid % kHeadDim] = acc[j];
    if (tid % kHeadDim == 0) {
      // a length outside [0, max_len] makes the row NaN, and so do logits that
      // are all not a number (fmaxf passes over them: the maximum stays -inf)
      const float l = ok ? lrow[rr] : __builtin_nanf("");
      o[0] = l == 0.f ? kNegInf : (mrow[rr] == kNegInf ? 0.f : mrow[rr]);
      o[1] = l;
    }
  }
}

// One workgroup per query row (128 threads, a dim each).
__global__ __launch_bounds__(kHeadDim) void k_merge(const uint8_t* __restrict__ blob, const float* __restrict__ part,
                                                    int n_slots, void* __restrict__ out, int out_dtype) {
  __shared__ float o[kHeadDim];
  const int dd = threadIdx.x;
  const size_t r = blockIdx.x;
  const float* P = part + r * n_slots * kPartFloats;
  float m = kNegInf;
  for (int i = 0; i < n_slots; ++i) m = fmaxf(m, P[i * kPartFloats]);
  float l = 0.f, a = 0.f;
  if (m != kNegInf) {
    for (int i = 0; i < n_slots; ++i) {
      const float mi = P[i * kPartFloats];
      if (mi == kNegInf) continue;
      const float e = exp2f(mi - m);
      l = fmaf(P[i * kPartFloats + 1], e, l);
      a = fmaf(P[i * kPartFloats + 2 + dd], e, a);
    }
  }
  o[dd] = l == 0.f ? 0.f : a / l * kRsqrtD;
  __syncthreads();
  const float* rv = reinterpret_cast<const float*>(blob + kOffRotV);
  float x = 0.f;
  for (int j = 0; j < kHeadDim; ++j) x = fmaf(rv[j * kHeadDim + dd], o[j], x);
  if (out_dtype == 1) static_cast<__bf16*>(out)[r * kHeadDim + dd] = static_cast<__bf16>(x);
  else static_cast<float*>(out)[r * kHeadDim + dd] = x;
}

}  // namespace cross_detail

long cross_items(const Dims& d, int n_q, int n_splits) {
  const long nr = static_cast<long>(n_q) * d.group;
  return (nr + cross_detail::kRows - 1) / cross_detail::kRows * n_splits * d.n_kv * d.n_lc * d.batch;
}

hipError_t launch_cross_pass(const Dims& d, const void* layout, const void* q, int n_q, const int32_t* ctx_len,
                             const CachePtrs& c, const CrossPass& ps, hipStream_t s) {
  hipLaunchKernelGGL(cross_detail::k_cross, dim3(cross_items(d, n_q, ps.n_splits)), dim3(cross_detail::kThreads), 0, s,
                     d, static_cast<const uint8_t*>(layout), q, n_q, ctx_len, c, ps);
  return hipGetLastError();
}

hipError_t launch_cross_merge(const void* layout, long rows, const float* part, int n_slots, void* out, int out_dtype,
                              hipStream_t s) {
  hipLaunchKernelGGL(cross_detail::k_merge, dim3(rows), dim3(kHeadDim), 0, s, static_cast<const uint8_t*>(layout), part,
                     n_slots, out, out_dtype);
  return hipGetLastError();
}

}  // namespace bgtq
