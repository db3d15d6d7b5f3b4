// Root-mean-square norm of every query and key head and the rotation by the
// token's position, in one pass over the rows that a projection wrote:
//   y = x w / sqrt(mean(x^2) + eps)                      (with weights)
//   (y_i, y_{i+64}) rotated by phi_i = pos[axis(i)] theta_i,
// block i = dims (i, i + 64) as in Sec. 2.1.  A token has a position on each
// axis (one for text; time, height and width for pictures and video), and each
// block turns with one of them.
//
// 8 lanes hold a head (lane j: dims 8 j .. + 7 and 64 + 8 j .. + 7, two 16-byte
// reads of bf16), so that a lane has whole blocks and the norm takes three
// exchanges.  A wave takes 8 heads of one token at a time; its lanes work out
// one angle each and hand them round, once for all of the token's heads.  The
// angle is formed and reduced in fp64 turns; only the fraction of a turn is
// rounded to fp32.  Sums, norm and rotation are fp32, rounded once at the store.
//
// What bounds it: reading and writing the rows.  32768 tokens x 40 heads in bf16:
// 126 us, 5.3 TB/s (a copy of 4 GiB reaches 4.8); one token 3.2 us, its latency.
#include <hip/hip_runtime.h>

#include "kernels.h"
#include "layout.h"

namespace bgtq {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kLanes = 8, kHeads = 64 / kLanes;  // lanes of a head, heads of a wave

template <bool BF>
struct Row {  // a lane's 16 values
  uint4 w[BF ? 2 : 4];
};

template <bool BF>
__device__ __forceinline__ void load_row(Row<BF>& r, const void* p, size_t at) {
  if constexpr (BF) {
    const uint16_t* s = static_cast<const uint16_t*>(p) + at;
    r.w[0] = *reinterpret_cast<const uint4*>(s);
    r.w[1] = *reinterpret_cast<const uint4*>(s + 64);
  } else {
    const float* s = static_cast<const float*>(p) + at;
    r.w[0] = *reinterpret_cast<const uint4*>(s);
    r.w[1] = *reinterpret_cast<const uint4*>(s + 4);
    r.w[2] = *reinterpret_cast<const uint4*>(s + 64);
    r.w[3] = *reinterpret_cast<const uint4*>(s + 68);
  }
}

template <bool BF>
__device__ __forceinline__ void values_of(const Row<BF>& r, float (&x)[16]) {
#pragma unroll
  for (int h = 0; h < (BF ? 2 : 4); ++h) {
    const uint32_t w[4] = {r.w[h].x, r.w[h].y, r.w[h].z, r.w[h].w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (BF) {
        x[8 * h + 2 * e] = __uint_as_float(w[e] << 16);
        x[8 * h + 2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u);
      } else {
        x[4 * h + e] = __uint_as_float(w[e]);
      }
    }
  }
}

template <bool BF>
__device__ __forceinline__ void store_row(void* p, size_t at, const float (&x)[16]) {
  if constexpr (BF) {
    typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
    typedef float float8_t __attribute__((ext_vector_type(8)));
    uint16_t* d = static_cast<uint16_t*>(p) + at;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float8_t v;
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = x[8 * h + e];
      *reinterpret_cast<bf16x8_t*>(d + 64 * h) = __builtin_convertvector(v, bf16x8_t);
    }
  } else {
    float* d = static_cast<float*>(p) + at;
#pragma unroll
    for (int h = 0; h < 4; ++h)
      *reinterpret_cast<float4*>(d + 64 * (h >> 1) + 4 * (h & 1)) =
          make_float4(x[4 * h], x[4 * h + 1], x[4 * h + 2], x[4 * h + 3]);
  }
}

// An item = (token, `per` consecutive groups of 8 heads); the query heads'
// groups come first, then the key heads'.  An input may be its own output (no
// __restrict__: a lane reads what it overwrites, before it does).
template <bool IN, bool OUT>
__global__ __launch_bounds__(kThreads) void k_norm_rope(NormRopeArgs a, long items, int n_groups, int per) {
  constexpr int kAhead = IN ? 4 : 2;  // groups whose reads are in flight together
  const int lane = threadIdx.x & 63, j = lane & 7, sub = lane >> 3;
  const long item = static_cast<long>(blockIdx.x) * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (item >= items) return;
  const int chunks = (n_groups + per - 1) / per;
  const long t = item / chunks;
  const int g0 = static_cast<int>(item - t * chunks) * per, g1 = min(g0 + per, n_groups);
  const int q_groups = (a.q.heads + kHeads - 1) / kHeads;

  // this lane's head of group g (the last one again behind the end, not stored)
  const auto head_of = [&](int g, bool& mine) {
    const int n = g < q_groups ? a.q.heads : a.k.heads, h = (g < q_groups ? g : g - q_groups) * kHeads + sub;
    mine = h < n;
    return min(h, n - 1);
  };
  Row<IN> rows[kAhead];
  const auto load_group = [&](int u, int g) {
    bool mine;
    const int h = head_of(g, mine);
    const NormRopeSide& s = g < q_groups ? a.q : a.k;
    load_row<IN>(rows[u], s.in, static_cast<size_t>(t) * s.in_stride + h * kHeadDim + 8 * j);
  };
#pragma unroll
  for (int u = 0; u < kAhead; ++u) load_group(u, min(g0 + u, g1 - 1));

  // the lane's angle (block 8 j + sub), then its 8 blocks' ones
  float cs[8], sn[8];
  {
    const int i = 8 * j + sub;
    const double turns = static_cast<double>(a.pos[t * a.n_axes + a.axis[i]]) * a.turns[i];
    float s1, c1;
    sincospif(static_cast<float>(2.0 * (turns - rint(turns))), &s1, &c1);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      cs[e] = __shfl(c1, 8 * e + j);
      sn[e] = __shfl(s1, 8 * e + j);
    }
  }

  float w[16];
  bool normed = false;
  int side = -1;
  for (int g = g0; g < g1; g += kAhead) {
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      if (g + u >= g1) break;  // wave-uniform
      const bool is_k = g + u >= q_groups;
      const NormRopeSide& s = is_k ? a.k : a.q;
      if (side != static_cast<int>(is_k)) {  // (at most twice)
        side = is_k;
        normed = s.weight != nullptr;
        if (normed) {
#pragma unroll
          for (int h = 0; h < 4; ++h) {
            const float4 v = *reinterpret_cast<const float4*>(s.weight + 64 * (h >> 1) + 8 * j + 4 * (h & 1));
            w[4 * h] = v.x;
            w[4 * h + 1] = v.y;
            w[4 * h + 2] = v.z;
            w[4 * h + 3] = v.w;
          }
        }
      }
      float x[16];
      values_of<IN>(rows[u], x);
      if (g + kAhead + u < g1) load_group(u, g + kAhead + u);
      if (normed) {
        float ss = 0.f;
#pragma unroll
        for (int e = 0; e < 16; ++e) ss = fmaf(x[e], x[e], ss);
#pragma unroll
        for (int o = 1; o < kLanes; o *= 2) ss += __shfl_xor(ss, o);
        const float r = rsqrtf(fmaf(ss, 1.f / kHeadDim, a.eps));
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] = x[e] * r * w[e];
      }
      float y[16];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        y[e] = fmaf(x[e], cs[e], -(x[e + 8] * sn[e]));
        y[e + 8] = fmaf(x[e], sn[e], x[e + 8] * cs[e]);
      }
      bool mine;
      const int h = head_of(g + u, mine);
      if (mine) store_row<OUT>(s.out, static_cast<size_t>(t) * s.out_stride + h * kHeadDim + 8 * j, y);
    }
  }
}

}  // namespace

hipError_t launch_norm_rope(const NormRopeArgs& a, long n_tokens, int in_dtype, int out_dtype, hipStream_t s) {
  const int groups = (a.q.heads + kHeads - 1) / kHeads + (a.k.heads + kHeads - 1) / kHeads;
  // a wave to each group of heads while that leaves CUs idle, else to a token
  const int per = n_tokens * groups <= 256L * 16 ? 1 : groups;
  const long items = n_tokens * ((groups + per - 1) / per);
  const auto go = [&](auto kern) {
    hipLaunchKernelGGL(kern, dim3((items + kWaves - 1) / kWaves), dim3(kThreads), 0, s, a, items, groups, per);
    return hipGetLastError();
  };
  if (in_dtype == 1) return out_dtype == 1 ? go(k_norm_rope<true, true>) : go(k_norm_rope<true, false>);
  return out_dtype == 1 ? go(k_norm_rope<false, true>) : go(k_norm_rope<false, false>);
}

}  // namespace bgtq
