// Attention of a ragged batch's new tokens over pages: the passes of
// paged_pass.h and the join of their splits.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "cross_impl.h"
#include "cross_merge.h"
#include "kernels.h"
#include "paged_pass.h"

namespace bgtq {
namespace {

using namespace cross_detail;

// Partials in the order of the output's rows: those of the pass's sequences.
// (With the whole wave; a lane works out row number lane % 16 of the block.)
struct TokenRows {
  PagedPass pass;
  int hq, group;
  long mine;
  template <int RW>
  __device__ __forceinline__ bool begin(long r0) {
    const int tk = threadIdx.x & 15, t0 = static_cast<int>(r0 / hq), need = static_cast<int>((r0 + RW - 1) / hq) - t0 + 1;
    paged::Seq q = {};
    const int s = paged::seq_of_row(pass.b, t0, tk, need, q), rows = q.n * group;
    const uint64_t live = __builtin_amdgcn_ballot_w64(s >= 0 && rows > pass.lo && rows <= pass.hi);
    const long r = r0 + tk;
    mine = tk < RW && (live >> static_cast<int>(r / hq - t0) & 1) ? r : -1;
    return __builtin_amdgcn_ballot_w64(mine >= 0) != 0;
  }
  __device__ __forceinline__ long out_row(long) const { return mine; }
};
// Partials [sequence][token][head].
struct SeqRows {
  PagedPass pass;
  int hq, group;
  long n_rows;
  long mine;
  template <int RW>
  __device__ __forceinline__ bool begin(long r0) {
    const int tk = threadIdx.x & 15;
    const long r = min(r0 + tk, n_rows - 1);
    const int t = static_cast<int>(r / hq), s = t / pass.most, i = t - s * pass.most;
    const paged::Seq q = paged::seq_of(pass.b, s);
    const int rows = q.n * group;
    const bool live = tk < RW && r0 + tk < n_rows && q.ok && i < q.n && rows > pass.lo && rows <= pass.hi;
    mine = live ? static_cast<long>(q.first + i) * hq + r % hq : -1;
    return __builtin_amdgcn_ballot_w64(live) != 0;
  }
  __device__ __forceinline__ long out_row(long) const { return mine; }
};

hipError_t join(const Dims& d, const void* layout, const CrossCall& call, const PagedPass& pass, hipStream_t s) {
  const int hq = d.n_kv * d.group;
  const long rows = (pass.direct ? static_cast<long>(pass.b.n_seqs) * pass.most : static_cast<long>(pass.b.n_tokens)) * hq;
  const auto go = [&](auto kern, long blocks, auto map) {
    hipLaunchKernelGGL(kern, dim3(blocks), dim3(kThreads), 0, s, static_cast<const uint8_t*>(layout), call.part, call.n_slots,
                       rows, call.out, call.out_dtype, map);
    return hipGetLastError();
  };
  const auto width = [&](auto map) {
    using M = decltype(map);
    if (rows >= 16 * 256) return go(k_cross_merge<16, M>, std::min(kMergeGrid, (rows + 15) / 16), map);
    return go(k_cross_merge<4, M>, (rows + 3) / 4, map);
  };
  return pass.direct ? width(SeqRows{pass, hq, d.group, rows, -1}) : width(TokenRows{pass, hq, d.group, -1});
}

// The query rotation of fp32 rows, as launch_query_rotation's but on the dense
// key rotation over natural dims in operand order: no gather, 16 rows of a wave
// on fp32 MFMAs, their 32 dims of a lane in 16-byte reads.  Bound by those
// products (256 of 32 cycles a wave) and by the staging of the matrix, which
// rows of several heads of the same KV head share.  28768 rows x 8 KV heads:
// 112 us there, 17 here.
constexpr int kRotWaves = 4;
__global__ __launch_bounds__(kRotWaves * 64) void k_paged_rotate(Dims d, const uint8_t* __restrict__ blob,
                                                                 const float* __restrict__ q, int n_tokens, int iters,
                                                                 float* __restrict__ qr) {
  __shared__ float4 wa[kMfmaMatFloats / 4];
  __shared__ float scale[kHeadDim];
  const int tid = threadIdx.x, lane = tid & 63, tk = lane & 15, kk = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int kvh = blockIdx.y, ri = d.layer * d.n_kv + kvh, G = d.group, hq = d.n_kv * G, nr = n_tokens * G;
  const RowMeta* M = reinterpret_cast<const RowMeta*>(blob + kOffRows) + ri;
  {
    const float4* src = reinterpret_cast<const float4*>(blob + layout_kdense_offset(d.n_layers * d.n_kv)) +
                        static_cast<size_t>(ri) * (kMfmaMatFloats / 4);
    constexpr int kPer = kMfmaMatFloats / 4 / (kRotWaves * 64);
    float4 t[kPer];
#pragma unroll
    for (int u = 0; u < kPer; ++u) t[u] = src[tid + u * kRotWaves * 64];
    if (tid < kHeadDim) scale[tid] = kLog2e * rsqrtf(static_cast<float>(M->g_dim[M->grp[tid]]) * kHeadDim);
#pragma unroll
    for (int u = 0; u < kPer; ++u) wa[tid + u * kRotWaves * 64] = t[u];
  }
  __syncthreads();
  for (int it = 0; it < iters; ++it) {
    const int r0 = ((blockIdx.x * iters + it) * kRotWaves + wave) * 16;
    if (r0 >= nr) break;  // wave-uniform
    const int r = r0 + tk, rc = min(r, nr - 1);
    const size_t off = (static_cast<size_t>(rc / G) * hq + kvh * G + rc % G) * kHeadDim;
    float4 x[8];
#pragma unroll
    for (int s4 = 0; s4 < 8; ++s4) x[s4] = *reinterpret_cast<const float4*>(q + off + 32 * kk + 4 * s4);
    float4_t acc[8];
#pragma unroll
    for (int t = 0; t < 8; ++t) acc[t] = float4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s4 = 0; s4 < 8; ++s4)
#pragma unroll
      for (int t = 0; t < 8; ++t) {
        const float4 w = wa[(t * 8 + s4) * 64 + lane];
        acc[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(w.x, x[s4].x, acc[t], 0, 0, 0);
        acc[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(w.y, x[s4].y, acc[t], 0, 0, 0);
        acc[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(w.z, x[s4].z, acc[t], 0, 0, 0);
        acc[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(w.w, x[s4].w, acc[t], 0, 0, 0);
      }
    if (r < nr) {
#pragma unroll
      for (int t = 0; t < 8; ++t)
        *reinterpret_cast<float4_t*>(qr + off + 16 * t + 4 * kk) =
            acc[t] * *reinterpret_cast<const float4_t*>(&scale[16 * t + 4 * kk]);
    }
  }
}

}  // namespace

hipError_t launch_paged_rotation(const Dims& d, const void* layout, const void* q, int n_tokens, float* qr, hipStream_t s) {
  if (d.in_dtype == 1) {
    Dims dq = d;  // (the chunk's tokens are one sequence's query rows)
    dq.batch = 1;
    return launch_query_rotation(dq, layout, q, n_tokens, qr, s);
  }
  const long rows = static_cast<long>(n_tokens) * d.group;
  const int iters = rows * d.n_kv <= 256L * 256 ? 1 : 4, per = kRotWaves * 16 * iters;
  hipLaunchKernelGGL(k_paged_rotate, dim3((rows + per - 1) / per, d.n_kv), dim3(kRotWaves * 64), 0, s, d,
                     static_cast<const uint8_t*>(layout), static_cast<const float*>(q), n_tokens, iters, qr);
  return hipGetLastError();
}

hipError_t launch_paged_pass(const Dims& d, const void* layout, const void* q, const CrossCall& call, const PagedPass& pass,
                             hipStream_t s) {
  hipError_t e;
  if (call.rows0 > 32) {
    e = call.out_dtype == 1 ? launch_paged_tile_bf16(d, layout, call, pass, s) : launch_paged_tile_fp32(d, layout, call, pass, s);
  } else if (call.rows0 == 8) {
    switch (d.v_bits) {
      case 1: e = launch_paged_decode_bv1(d, layout, q, call, pass, s); break;
      case 2: e = launch_paged_decode_bv2(d, layout, q, call, pass, s); break;
      case 3: e = launch_paged_decode_bv3(d, layout, q, call, pass, s); break;
      case 4: e = launch_paged_decode_bv4(d, layout, q, call, pass, s); break;
      case 5: e = launch_paged_decode_bv5(d, layout, q, call, pass, s); break;
      case 6: e = launch_paged_decode_bv6(d, layout, q, call, pass, s); break;
      case 7: e = launch_paged_decode_bv7(d, layout, q, call, pass, s); break;
      default: e = launch_paged_decode_bv8(d, layout, q, call, pass, s); break;
    }
  } else {
    switch (d.v_bits) {
      case 1: e = launch_paged_bv1(d, layout, q, call, pass, s); break;
      case 2: e = launch_paged_bv2(d, layout, q, call, pass, s); break;
      case 3: e = launch_paged_bv3(d, layout, q, call, pass, s); break;
      case 4: e = launch_paged_bv4(d, layout, q, call, pass, s); break;
      case 5: e = launch_paged_bv5(d, layout, q, call, pass, s); break;
      case 6: e = launch_paged_bv6(d, layout, q, call, pass, s); break;
      case 7: e = launch_paged_bv7(d, layout, q, call, pass, s); break;
      default: e = launch_paged_bv8(d, layout, q, call, pass, s); break;
    }
  }
  if (e != hipSuccess || call.n_slots == 1) return e;
  return join(d, layout, call, pass, s);
}

}  // namespace bgtq
