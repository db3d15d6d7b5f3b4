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

// Partials [block][KV head][row of the unit]: those of rows that a sequence has.
template <int R>
struct UnitRows {
  PagedPass pass;
  int n_kv, group;
  paged::Unit u;
  __device__ __forceinline__ bool begin(long r) {
    const int unit = static_cast<int>(r / pass.unit_rows), first = static_cast<int>(r % pass.unit_rows);
    u.kvh = unit % n_kv;
    return paged::find_block<R>(pass, group, unit / n_kv, u) && u.q.ok && u.r0 + first < u.q.n * group;
  }
  __device__ __forceinline__ long out_row(long r) const {
    const int i = u.r0 + static_cast<int>(r % pass.unit_rows);
    return i < u.q.n * group ? (static_cast<long>(u.q.first) + i / group) * n_kv * group + u.kvh * group + i % group : -1;
  }
};

template <int R>
hipError_t join(const Dims& d, const void* layout, const CrossCall& call, const PagedPass& pass, hipStream_t s) {
  const long rows = static_cast<long>(pass.n_blocks) * d.n_kv * pass.unit_rows;
  const UnitRows<R> map{pass, d.n_kv, d.group, {}};
  const auto go = [&](auto kern, long blocks) {
    hipLaunchKernelGGL(kern, dim3(blocks), dim3(kThreads), 0, s, static_cast<const uint8_t*>(layout), call.part, call.n_slots,
                       rows, call.out, call.out_dtype, map);
    return hipGetLastError();
  };
  if (rows >= 16 * 256 && pass.unit_rows % 16 == 0) return go(k_cross_merge<16, UnitRows<R>>, std::min(kMergeGrid, rows / 16));
  return go(k_cross_merge<4, UnitRows<R>>, rows / 4);
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
  if (call.rows0 == 8) return join<8>(d, layout, call, pass, s);
  return call.rows0 == 32 ? join<32>(d, layout, call, pass, s)
                          : call.rows0 == 128 ? join<128>(d, layout, call, pass, s) : join<256>(d, layout, call, pass, s);
}

}  // namespace bgtq
