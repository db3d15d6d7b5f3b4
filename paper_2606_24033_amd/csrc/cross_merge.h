// Join of a query row's partials (m, l, acc[128]) of several splits or passes:
// see cross.hip.
#pragma once
#include <hip/hip_runtime.h>

#include "cross_impl.h"
#include "kernels.h"
#include "layout.h"

namespace bgtq {
namespace cross_detail {

constexpr long kMergeGrid = 512;  // workgroups of a join of many rows: the two of a CU that its registers hold

// RW query rows of a workgroup; a row's partials are shared out to 16 / RW
// groups of 32 threads (4 dims each), four slots at a time.  Bound by reading
// the partials where there are many (32768 rows x 2 slots, 43 MB read and
// written, 18 us: 2.4 TB/s), by its latency (5 us) otherwise.
//
// MAP: where a row's partials belong.  begin<RW>(r), with the whole workgroup: the
// first of the block's rows, false where none is to be joined; out_row(r), in lane
// r % 16 of each quarter of a wave: the row of the output, -1 for none.
template <int RW, class MAP>
__global__ __launch_bounds__(kThreads) void k_cross_merge(const uint8_t* __restrict__ blob, const float* __restrict__ part,
                                                          int n_slots, long n_rows, void* __restrict__ out, int out_dtype, MAP map) {
  constexpr int NG = 16 / RW;
  __shared__ __attribute__((aligned(16))) uint8_t staged2[RW == 16 ? 2 : 1][2 * kHalfPart];
  __shared__ float back2[RW == 16 ? 2 : 1][16];
  __shared__ float gm[16], gl[16];
  __shared__ float4_t ga[16][32];
  const int tid = threadIdx.x, lane = tid & 63, sub = tid >> 5, d4 = tid & 31, rl = sub % RW, grp = sub / RW;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // this wave's 16 output dims of Pi_V^T
  float4_t rot[8];
  half8_t wh[4], wl[4];
  const auto matrix = [&]() {
    const float4_t* src = reinterpret_cast<const float4_t*>(blob + kOffRotVT) +
                          ((16 * wave + (lane & 15)) * kHeadDim + 32 * (lane >> 4)) / 4;
#pragma unroll
    for (int s4 = 0; s4 < 8; ++s4) rot[s4] = src[s4];
  };
  const auto parts = [&]() {
#pragma unroll
    for (int u = 0; u < 4; ++u) matrix_parts(rot, u, wh[u], wl[u]);
  };
  // A workgroup takes every gridDim.x-th block of rows: a wave's part of the
  // matrix is read once.  (Two staging buffers: one barrier a block.)
  int buf = 0;
  bool ready = false;
  for (long block = blockIdx.x; block * RW < n_rows; block += RW == 16 ? static_cast<long>(gridDim.x) : n_rows) {
    if (!map.template begin<RW>(block * RW)) continue;
    if (RW != 16 || !ready) {
      matrix();
      if (RW == 16) parts();  // (else behind the partials' reads)
      ready = true;
    }
    uint8_t* const staged = staged2[buf];
    float* const back = back2[buf];
    const long r = block * RW + rl;
    float m = kNegInf, l = 0.f;
    float4_t a = {0.f, 0.f, 0.f, 0.f};
    if (r < n_rows) {
      const float* P = part + static_cast<size_t>(r) * n_slots * kPartFloats;
      for (int s0 = grp; s0 < n_slots; s0 += 4 * NG) {
        float ms[4], ls[4];
        float4_t as[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const int s = s0 + u * NG;
          const float* p = P + static_cast<size_t>(min(s, n_slots - 1)) * kPartFloats;
          ms[u] = s < n_slots ? p[0] : kNegInf;
          ls[u] = p[1];
          as[u] = *reinterpret_cast<const float4_t*>(p + 4 + 4 * d4);
        }
        const float mn = fmaxf(m, fmaxf(fmaxf(ms[0], ms[1]), fmaxf(ms[2], ms[3])));
        if (mn == kNegInf) continue;
        const float e0 = m == kNegInf ? 0.f : __builtin_amdgcn_exp2f(m - mn);
        l *= e0;
        a *= e0;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          if (ms[u] == kNegInf) continue;
          const float e = __builtin_amdgcn_exp2f(ms[u] - mn);
          l = fmaf(ls[u], e, l);
#pragma unroll
          for (int i = 0; i < 4; ++i) a[i] = fmaf(as[u][i], e, a[i]);
        }
        m = mn;
      }
    }
    if (NG > 1) {
      if (d4 == 0) {
        gm[sub] = m;
        gl[sub] = l;
      }
      ga[sub][d4] = a;
      __syncthreads();
      float mn = kNegInf;
#pragma unroll
      for (int g = 0; g < NG; ++g) mn = fmaxf(mn, gm[rl + g * RW]);
      l = 0.f;
      a = float4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int g = 0; g < NG; ++g) {
        const float mg = gm[rl + g * RW];
        if (mg == kNegInf) continue;
        const float e = __builtin_amdgcn_exp2f(mg - mn);
        l = fmaf(gl[rl + g * RW], e, l);
        const float4_t x = ga[rl + g * RW][d4];
#pragma unroll
        for (int i = 0; i < 4; ++i) a[i] = fmaf(x[i], e, a[i]);
      }
    }
    // (rows past RW of the 16 keep what LDS held: their results are not stored)
    if (grp == 0) {
      a *= l == 0.f ? 0.f : kRsqrtD / l;
      uint32_t mx = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) mx = max(mx, __float_as_uint(a[i]) & 0x7FFFFFFFu);
#pragma unroll
      for (int k = 1; k < 32; k *= 2) mx = max(mx, static_cast<uint32_t>(__shfl_xor(static_cast<int>(mx), k)));
      const int up = up_of(mx);
      a *= two_to(up);
      half4_t hi, lo;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        hi[i] = static_cast<_Float16>(a[i]);
        lo[i] = static_cast<_Float16>(a[i] - static_cast<float>(hi[i]));
      }
      uint8_t* dst = staged + rl * kHalfStride + 8 * d4;
      *reinterpret_cast<half4_t*>(dst) = hi;
      *reinterpret_cast<half4_t*>(dst + kHalfPart) = lo;
      if (d4 == 0) back[rl] = two_to(254 - up) * (1.f / 256.f);
    }
    __syncthreads();
    if (RW != 16) parts();
    float4_t y[1] = {{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int u = 0; u < 4; ++u) staged_step<1>(staged + (lane & 15) * kHalfStride + 64 * (lane >> 4), u, wh[u], wl[u], y);
    const int ro = lane & 15;
    const long rg = block * RW + ro;
    const long to = ro < RW && rg < n_rows ? map.out_row(rg) : -1;
    if (to >= 0)
      store4(out, static_cast<size_t>(to) * kHeadDim + 16 * wave + 4 * (lane >> 4), y[0] * back[ro], out_dtype);
    buf ^= 1;
  }
}

}  // namespace cross_detail
}  // namespace bgtq
