// Attention of many query rows to packed rows that all of them see: cross
// attention (query rows of a sequence against its whole cache) and the decode
// step of a batch that shares a prefix (every sequence's query against the
// prefix's cache and its own).
//
// Both are passes over one form: the query rows of a unit (layer, sequence,
// KV head) against rows [0, len) of one packed cache, the key axis in splits
// (k_cross, cross_impl.h).  A pass leaves per query row and split (m, l,
// acc[128]): the maximum of the base-2 logits, sum 2^(s - m) and
// sum 2^(s - m) v in the rotated value domain.  Partial states of disjoint row
// sets merge as
//   m = max m_i,  l = sum l_i 2^(m_i - m),  a = sum a_i 2^(m_i - m),
// so a shared prefix is one more set of splits: its pass, whose query rows are
// the batch's, and the sequences' own pass are one launch.  k_cross_merge joins a
// row's partials, divides by l, rotates back (Pi_V^T) and rounds to the output
// type; a row with a single partial is finished by k_cross itself.
#include <hip/hip_runtime.h>

#include "kernels.h"
#include "layout.h"

namespace bgtq {
namespace {

constexpr int kCrossRows = 32;  // query rows of a workgroup
constexpr float kNegInf = -__builtin_huge_valf();
constexpr float kRsqrtD = 0.08838834764831845f;  // 1 / sqrt(128)

// One workgroup per query row (128 threads, a dim each).
__global__ __launch_bounds__(kHeadDim) void k_cross_merge(const uint8_t* __restrict__ blob,
                                                          const float* __restrict__ part, int n_slots,
                                                          void* __restrict__ out, int out_dtype) {
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
      a = fmaf(P[i * kPartFloats + 4 + dd], e, a);
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

}  // namespace

long cross_items(const Dims& d, int n_q, int n_splits) {
  const long nr = static_cast<long>(n_q) * d.group;
  return (nr + kCrossRows - 1) / kCrossRows * n_splits * d.n_kv * d.n_lc * d.batch;
}

hipError_t launch_cross(const Dims& d, const void* layout, const void* q, const CrossCall& call, long rows,
                        hipStream_t s) {
  hipError_t e;
  switch (d.v_bits) {
    case 1: e = launch_cross_bv1(d, layout, q, call, s); break;
    case 2: e = launch_cross_bv2(d, layout, q, call, s); break;
    case 3: e = launch_cross_bv3(d, layout, q, call, s); break;
    case 4: e = launch_cross_bv4(d, layout, q, call, s); break;
    case 5: e = launch_cross_bv5(d, layout, q, call, s); break;
    case 6: e = launch_cross_bv6(d, layout, q, call, s); break;
    case 7: e = launch_cross_bv7(d, layout, q, call, s); break;
    default: e = launch_cross_bv8(d, layout, q, call, s); break;
  }
  if (e != hipSuccess || call.n_slots == 1) return e;
  hipLaunchKernelGGL(k_cross_merge, dim3(rows), dim3(kHeadDim), 0, s, static_cast<const uint8_t*>(layout), call.part,
                     call.n_slots, call.out, call.out_dtype);
  return hipGetLastError();
}

}  // namespace bgtq
