// Append of a ragged batch's bf16 rows to their pages: the TQ-MSE encode of
// quantize.hip, whose two 128 x 128 products per row run on three exact bf16
// products (split.h): the terms are exact, the sums fp32, so codes are as right
// as with fp32 products (a coordinate within their rounding of a threshold may
// fall to either side of it in either).  fp32 inputs and the wider formats,
// whose packing buffers don't fit beside 96 KB of matrix, take quantize.hip's
// kernels; so do sequences of up to 4 rows (k_append_rows).
//
// A wave takes 32 rows at a time, so that each matrix operand read from LDS
// (96 KB per workgroup, split while it is staged) serves two products, and
// finishes the codes of one 16-wide output tile before it starts the next: 16
// accumulator registers, so four waves fit a SIMD.  Codes by counting: up to
// three (width <= 2) or seven (width 3) comparisons against thresholds held per
// position, a branch-free search only for tiles that hold wider codes.  The
// square of a bf16 number is the sum of two: the group radii take two bf16
// products of the rows' squares with the groups' members, exact terms as well.
//
// What bounds it: a wave's chain of reads, products and comparisons, four of
// them to a SIMD (vector instructions 74 %, matrix cores 30 % of the time that a
// CU is busy).  16384 rows x 8 heads of K2V2: 47 us (fp32 products 127; fp32 radii,
// half of the workgroups for each side and a wave's rows read when it needs them
// 61); 65536 rows 178; 4096 rows 21 (32 with all of a workgroup's waves busy
// before the next one starts); up to 1000 rows 16.
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>

#include <algorithm>

#include "kernels.h"
#include "layout.h"
#include "paged.h"
#include "split.h"

namespace bgtq {
namespace {

using namespace split;

constexpr int kSplitKWords = 16, kSplitVBits = 4;
constexpr int kWaves = 16;

struct LdsKeys {
  uint4_t wa[3][kMatOps];                          // W's three parts, A operand order
  uint4_t ma[4 * 64];                              // group membership, A operand order
  float4 ta[kHeadDim], tb[kHeadDim];               // first seven thresholds of each position, NaN past its last
  uint32_t rw[kWaves][kSplitRows * kSplitKWords];  // per wave: packed key rows, k_words apart
  float sc[kWaves][kSplitRows][kMaxGroups];        // per wave: sqrt(d_g) / radius
  uint32_t pm[kHeadDim];                           // bit offset | b << 10 | group << 14
  float thr[kThresholdEntries];
  float gs[kMaxGroups];
  int mw[8];                                       // largest width in each tile of 16 positions
  uint8_t gd[kHeadDim];
};
struct LdsValues {
  uint4_t rb[3][kMatOps];                       // Pi_V's three parts, B operand order
  uint32_t vt[kWaves][kHeadDim * kSplitVBits];  // per wave: words of one value tile
  float nv[kWaves][kSplitRows];
  float thr[kThresholdEntries];
};
static_assert(sizeof(LdsKeys) <= 160 * 1024 && sizeof(LdsValues) <= 160 * 1024, "LDS");

__device__ __forceinline__ void wave_sync() {  // (LDS operations of one wave complete in order)
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// The squares of an operand's 8 numbers, in two parts: what their upper 16 bits
// leave of the product of two 8-bit significands has 8 bits again.
__device__ __forceinline__ void square_parts(const uint4_t& x, uint4_t& hi, uint4_t& lo) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    float a = __uint_as_float(x[j] << 16), b = __uint_as_float(x[j] & 0xFFFF0000u);
    a *= a;
    b *= b;
    const uint32_t ah = __float_as_uint(a) & 0xFFFF0000u, bh = __float_as_uint(b) & 0xFFFF0000u;
    a -= __uint_as_float(ah);
    b -= __uint_as_float(bh);
    hi[j] = bh | ah >> 16;
    lo[j] = __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
  }
}

// Element i of the 32 that four operands hold.
__device__ __forceinline__ float bf16_elem(const uint4_t (&x)[4], int i) {
  const uint32_t w = x[i >> 3][(i & 7) >> 1];
  return __uint_as_float(i & 1 ? w & 0xFFFF0000u : w << 16);
}

// Output tile t of the products of the wave's two sub-tiles, the rows as the
// A operand and the matrix as the B one (split_product: the other way round).
__device__ __forceinline__ void rows_product(const uint4_t (*mat)[kMatOps], int t, int lane, const uint4_t (&x)[2][4],
                                             float4_t (&out)[2]) {
  float4_t hi[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}}, lo[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int o = (t * 4 + q) * 64 + lane;
    const uint4_t w0 = mat[0][o], w1 = mat[1][o], w2 = mat[2][o];
#pragma unroll
    for (int s = 0; s < 2; ++s) lo[s] = mfma_bf16(x[s][q], w2, lo[s]);
#pragma unroll
    for (int s = 0; s < 2; ++s) hi[s] = mfma_bf16(x[s][q], w0, hi[s]);
#pragma unroll
    for (int s = 0; s < 2; ++s) lo[s] = mfma_bf16(x[s][q], w1, lo[s]);
  }
#pragma unroll
  for (int s = 0; s < 2; ++s) out[s] = hi[s] + lo[s];
}

// ---------------------------------------------------------------- keys
__device__ __forceinline__ void quant_keys(LdsKeys& S, int bx, int n_wg, const Dims& d,
                                           const uint8_t* __restrict__ blob, const void* __restrict__ kin,
                                           const PagedRows& rows, const CachePtrs& c) {
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int head = blockIdx.y;
  const int cap = d.capacity, n = rows.b.n_tokens;
  constexpr int kThreads = kWaves * 64;
  const int n_rows_blob = d.n_layers * d.n_kv, ri = d.layer * d.n_kv + head;
  const RowMeta* M = reinterpret_cast<const RowMeta*>(blob + kOffRows) + ri;
  const float* gthr = reinterpret_cast<const float*>(blob + kOffThr);
  const int ng = M->n_groups, kw = d.k_words;

  for (int i = tid; i < kWaves * kSplitRows * kSplitKWords; i += kThreads) (&S.rw[0][0])[i] = 0u;
  for (int i = tid; i < kThresholdEntries; i += kThreads) S.thr[i] = gthr[i];
  if (tid < kHeadDim) {
    const int g = M->grp[tid], b = M->width[tid], nt = (1 << b) - 1;
    S.gd[M->dim[tid]] = static_cast<uint8_t>(g);
    S.pm[tid] = static_cast<uint32_t>(M->bitoff[tid]) | (static_cast<uint32_t>(b) << 10) | (static_cast<uint32_t>(g) << 14);
    float th[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) th[j] = j < nt ? gthr[thr_index(b) + j] : __builtin_nanf("");
    S.ta[tid] = make_float4(th[0], th[1], th[2], th[3]);
    S.tb[tid] = make_float4(th[4], th[5], th[6], th[7]);
  }
  if (tid < kMaxGroups) {
    S.gs[tid] = tid < ng ? sqrtf(static_cast<float>(M->g_dim[tid])) : 0.f;
    int w = 0;
    for (int j = 0; j < 16; ++j) w = max(w, static_cast<int>(M->width[16 * tid + j]));
    S.mw[tid] = w;
  }
  // A wave's next rows: read before the staging ends, and before the last
  // rows' codes are written.
  const int tk = lane & 15, kk = lane >> 4;
  uint4_t x[2][4];
  int2 at = make_int2(-1, 0);  // page and place of row lane % 32
  const auto load_rows = [&](int r0) {
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const int r = r0 + kSub * s + tk;
      load_operands(kin, min(r, n - 1) * rows.k_stride + head * kHeadDim + 32 * kk, r < n, x[s]);
    }
    at = paged::page_of_row<kSplitRows>(rows.b, d.batch, cap, r0, lane & 31);
    if (r0 + (lane & 31) >= n) at.x = -1;
  };
  // (the last waves of all workgroups are those that have a block less)
  int r0 = (wave * n_wg + bx) * kSplitRows;
  if (r0 < n) load_rows(r0);
  stage_split<kWaves>(
      S.wa, reinterpret_cast<const float4*>(blob + layout_kdense_offset(n_rows_blob)) + static_cast<size_t>(ri) * kMatF4, tid);
  __syncthreads();
  for (int i = tid; i < 4 * 64; i += kThreads) {
    // row 4 m + e of the product is group 2 m + e (e < 2): two groups to each
    // quarter of the wave instead of four to two of them
    const int l = i & 63, d0 = 32 * (l >> 4) + 8 * (i >> 6);
    const int g = (l & 3) < 2 ? 2 * ((l >> 2) & 3) + (l & 3) : -1;
    uint4_t m;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      m[j] = (S.gd[d0 + 2 * j] == g ? 0x3F80u : 0u) | (S.gd[d0 + 2 * j + 1] == g ? 0x3F800000u : 0u);
    S.ma[i] = m;
  }
  __syncthreads();

  const float gs[2] = {S.gs[2 * kk], S.gs[2 * kk + 1]};
  const int nslot = (ng + 1) & ~1;
  const auto cache_row = [&](int page) { return (static_cast<size_t>(d.layer) * d.batch + page) * d.n_kv + head; };
  while (r0 < n) {  // (wave-uniform)
    // group radii: R2[g][row] = sum_d [group(d) = g] x[row][d]^2
    float4_t n2[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const uint4_t m = S.ma[q * 64 + lane];
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        uint4_t hi, lo;
        square_parts(x[s][q], hi, lo);
        n2[s] = mfma_bf16(m, lo, n2[s]);
        n2[s] = mfma_bf16(m, hi, n2[s]);
      }
    }
    // this lane holds R2 of rows tk, 16 + tk for groups 2 kk, 2 kk + 1 (zero
    // past the last group)
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      float nrm[2];
      uint16_t h[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        nrm[i] = sqrtf(n2[s][i]);
        S.sc[wave][kSub * s + tk][2 * kk + i] = nrm[i] > 0.f ? gs[i] / nrm[i] : 0.f;
        h[i] = __half_as_ushort(__float2half_rn(nrm[i]));
      }
      const int page = __shfl(at.x, kSub * s + tk), place = __shfl(at.y, kSub * s + tk);
      if (page >= 0 && 2 * kk < ng) {
        uint16_t* dst = c.k_norms + cache_row(page) * kMaxGroups * cap + static_cast<size_t>(place) * nslot + 2 * kk;
        if (2 * kk + 1 < ng) *reinterpret_cast<uint32_t*>(dst) = h[0] | static_cast<uint32_t>(h[1]) << 16;
        else *dst = h[0];
      }
    }
    wave_sync();
    // Z[p][row] = sum_d W[p][d] x[row][d]; codes of stream positions
    // 16 t + 4 kk + i of a row: one bit field
#pragma unroll 1
    for (int t = 0; t < 8; ++t) {
      const int p0 = 16 * t + 4 * kk;
      float4_t z[2];
      split_product(S.wa, t, lane, x, z);
      uint32_t pm[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) pm[i] = S.pm[p0 + i];
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int i = 0; i < 4; ++i) z[s][i] *= S.sc[wave][kSub * s + tk][(pm[i] >> 14) & 7];
      const int mw = __builtin_amdgcn_readfirstlane(S.mw[t]);
      uint32_t code[2][4];
      if (mw <= 3) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float4 th = S.ta[p0 + i];
#pragma unroll
          for (int s = 0; s < 2; ++s)
            code[s][i] = (th.x <= z[s][i] ? 1u : 0u) + (th.y <= z[s][i] ? 1u : 0u) + (th.z <= z[s][i] ? 1u : 0u);
        }
        if (mw == 3) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float t3 = S.ta[p0 + i].w;
            const float4 th = S.tb[p0 + i];
#pragma unroll
            for (int s = 0; s < 2; ++s)
              code[s][i] += (t3 <= z[s][i] ? 1u : 0u) + (th.x <= z[s][i] ? 1u : 0u) + (th.y <= z[s][i] ? 1u : 0u) +
                            (th.z <= z[s][i] ? 1u : 0u);
          }
        }
      } else {
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int i = 0; i < 4; ++i) code[s][i] = 0u;
        // all lanes read on every step (a narrow position's index stays inside
        // the table: thr_index(7) + 127 at most) and the eight reads of a step
        // are in flight together
#pragma unroll 1
        for (uint32_t step = 1u << (mw - 1); step > 0; step >>= 1) {
          float tv[2][4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int first = thr_index((pm[i] >> 10) & 15) + static_cast<int>(step) - 1;
#pragma unroll
            for (int s = 0; s < 2; ++s) tv[s][i] = S.thr[min(first + static_cast<int>(code[s][i]), kThresholdEntries - 1)];
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t add = (step >> ((pm[i] >> 10) & 15)) == 0 ? step : 0u;
#pragma unroll
            for (int s = 0; s < 2; ++s) code[s][i] += tv[s][i] <= z[s][i] ? add : 0u;
          }
        }
      }
      const int b0 = (pm[0] >> 10) & 15, b1 = b0 + ((pm[1] >> 10) & 15), b2 = b1 + ((pm[2] >> 10) & 15);
      const int nb = b2 + ((pm[3] >> 10) & 15), bo = pm[0] & 1023, w = bo >> 5, sh = bo & 31;
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const uint32_t field = code[s][0] | code[s][1] << b0 | code[s][2] << b1 | code[s][3] << b2;
        uint32_t* dst = &S.rw[wave][(kSub * s + tk) * kw + w];
        atomicOr(dst, field << sh);
        if (sh + nb > 32) atomicOr(dst + 1, field >> (32 - sh));
      }
    }
    wave_sync();
    const int2 was = at;
    r0 += n_wg * kWaves * kSplitRows;
    if (r0 < n) load_rows(r0);
    for (int idx = lane; idx < kSplitRows * kw; idx += 64) {
      const int t2 = idx / kw, w = idx - t2 * kw;
      // (lanes 0 .. 31 take part in every round)
      const int2 a = make_int2(__shfl(was.x, t2), __shfl(was.y, t2));
      if (a.x >= 0) c.k_codes[(cache_row(a.x) * cap + a.y) * kw + w] = S.rw[wave][idx];
      S.rw[wave][idx] = 0u;
    }
    wave_sync();
  }
}

// ---------------------------------------------------------------- values
// The BV-bit codes of one value tile, ORed into its words.
template <int BV>
__device__ __forceinline__ void tile_codes(LdsValues& S, int wave, int lane, const uint4_t (&x)[2][4], int s_lo, int s_hi) {
  constexpr int kThr = (1 << BV) - 1;
  const int tk = lane & 15, kk = lane >> 4;
  const float sq = sqrtf(static_cast<float>(kHeadDim));
  float scl[2][4], thr[kThr];
  uint32_t keep[2] = {0u, 0u};
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int s = kSub * h + 4 * kk + i;
      const float n = S.nv[wave][s];
      scl[h][i] = n > 0.f ? sq / n : 0.f;
      keep[h] |= (s >= s_lo && s < s_hi ? ((1u << BV) - 1u) : 0u) << (i * BV);
    }
#pragma unroll
  for (int j = 0; j < kThr; ++j)
    thr[j] = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(S.thr[thr_index(BV) + j])));
#pragma unroll 1
  for (int t = 0; t < 8; ++t) {
    // Z[row][j] = sum_d x[row][d] Pi_V[j][d]; this lane: coordinate j of
    // rows 16 h + 4 kk + i
    float4_t z[2];
    rows_product(S.rb, t, lane, x, z);
    const int j = 16 * t + tk;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int bit = (kSub * h + 4 * kk) * BV, w = bit >> 5, sh = bit & 31;
      uint32_t field = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float v = z[h][i] * scl[h][i];
        uint32_t code = 0;
#pragma unroll
        for (int e = 0; e < kThr; ++e) code += thr[e] <= v ? 1u : 0u;
        field |= code << (i * BV);
      }
      field &= keep[h];
      atomicOr(&S.vt[wave][j * BV + w], field << sh);
      if (sh + 4 * BV > 32) atomicOr(&S.vt[wave][j * BV + w + 1], field >> (32 - sh));
    }
  }
}

template <int BV>
__device__ __forceinline__ void quant_values(LdsValues& S, int bx, int n_wg, long n_tiles, const Dims& d,
                                             const uint8_t* __restrict__ blob, const void* __restrict__ vin,
                                             const PagedRows& rows, const CachePtrs& c) {
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int head = blockIdx.y, cap = d.capacity;
  const float* gthr = reinterpret_cast<const float*>(blob + kOffThr);
  for (int i = tid; i < kThresholdEntries; i += kWaves * 64) S.thr[i] = gthr[i];
  // as in quant_keys: a wave's next tile is read early
  const int tk = lane & 15, kk = lane >> 4;
  uint4_t x[2][4];
  paged::Tile next = {};
  bool there = false;
  const auto load_tile = [&](int i) {
    there = paged::tile_of(rows.b, d.batch, cap, i, next);  // wave-uniform
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int slot = kSub * h + tk;
      load_operands(vin, (next.in0 + next.P0 + slot) * rows.v_stride + head * kHeadDim + 32 * kk,
                    there && slot >= next.lo && slot < next.hi, x[h]);
    }
  };
  int i = wave * n_wg + bx;
  if (i < n_tiles) load_tile(i);
  stage_split<kWaves>(S.rb, reinterpret_cast<const float4*>(blob + layout_rotv_mfma_offset(d.n_layers * d.n_kv)), tid);
  __syncthreads();

  while (i < n_tiles) {
    const paged::Tile t = next;
    i += n_wg * kWaves;
    if (!there) {
      if (i < n_tiles) load_tile(i);
      continue;
    }
    const size_t row = (static_cast<size_t>(d.layer) * d.batch + t.page) * d.n_kv + head;
    const int P0 = t.P0 % cap;
    uint32_t* gv = c.v_codes + (row * (cap / kTile) + P0 / kTile) * kHeadDim * static_cast<size_t>(BV);
    // tile words: zero, or the old words with the new rows' bits cleared
    if (t.lo == 0 && t.hi == kTile) {
      for (int idx = lane; idx < kHeadDim * BV; idx += 64) S.vt[wave][idx] = 0u;
    } else {
      for (int idx = lane; idx < kHeadDim * BV; idx += 64) {
        const int w = idx % BV;
        const int lo_b = max(t.lo * BV - 32 * w, 0), hi_b = min(t.hi * BV - 32 * w, 32);
        const uint32_t mask = hi_b <= lo_b ? 0u : (hi_b - lo_b == 32 ? ~0u : ((1u << (hi_b - lo_b)) - 1u) << lo_b);
        S.vt[wave][idx] = gv[idx] & ~mask;
      }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int slot = kSub * h + tk;
      float ss = 0.f;
#pragma unroll
      for (int i = 0; i < 32; ++i) ss = fmaf(bf16_elem(x[h], i), bf16_elem(x[h], i), ss);
      ss += __shfl_xor(ss, 16, 64);
      ss += __shfl_xor(ss, 32, 64);
      const float nrm = sqrtf(ss);
      if (kk == 0) {
        S.nv[wave][slot] = nrm;
        if (slot >= t.lo && slot < t.hi) c.v_norms[row * cap + P0 + slot] = __half_as_ushort(__float2half_rn(nrm));
      }
    }
    wave_sync();
    tile_codes<BV>(S, wave, lane, x, t.lo, t.hi);
    wave_sync();
    there = false;
    if (i < n_tiles) load_tile(i);
    for (int idx = lane; idx < kHeadDim * BV; idx += 64) gv[idx] = S.vt[wave][idx];
    wave_sync();
  }
}

// The key workgroups (the longer ones) come first.
template <int BV>
__global__ __launch_bounds__(kWaves * 64) void k_paged_quantize(Dims d, const uint8_t* __restrict__ blob,
                                                           const void* __restrict__ kin, const void* __restrict__ vin,
                                                           PagedRows rows, CachePtrs c, int n_kwg, int n_vwg, int n_tiles) {
  constexpr size_t kBytes = sizeof(LdsKeys) > sizeof(LdsValues) ? sizeof(LdsKeys) : sizeof(LdsValues);
  __shared__ __attribute__((aligned(16))) uint8_t smem[kBytes];
  const int bx = static_cast<int>(blockIdx.x);
  if (bx < n_kwg) quant_keys(*reinterpret_cast<LdsKeys*>(smem), bx, n_kwg, d, blob, kin, rows, c);
  else quant_values<BV>(*reinterpret_cast<LdsValues*>(smem), bx - n_kwg, n_vwg, n_tiles, d, blob, vin, rows, c);
}

}  // namespace

bool paged_quantize_fits(const Dims& d) { return d.in_dtype == 1 && d.k_words <= kSplitKWords && d.v_bits <= kSplitVBits; }

// One workgroup runs per CU: 256 of them, or fewer for few rows, share the rows
// of all heads, so that each stages its matrix once.  160 are for keys, whose
// blocks of 32 rows take about 1.6 times as long as the values' (65536 rows x 8
// heads: 205 us with 128, 178 with 160, 193 with 176).
hipError_t launch_paged_quantize_bf16(const Dims& d, const void* layout, const void* k, const void* v, const PagedRows& rows,
                                      const CachePtrs& c, hipStream_t s) {
  constexpr long kKeyShare = 160;
  const long n = rows.b.n_tokens, tiles = std::min(n, (n + 62L * rows.b.n_seqs) / kTile);
  const auto go = [&](auto kern) {
    const int n_kwg = static_cast<int>(std::min(std::max(1l, kKeyShare / d.n_kv), (n + kSplitRows - 1) / kSplitRows));
    const int n_vwg = static_cast<int>(std::min(std::max(1l, (256 - kKeyShare) / d.n_kv), tiles));
    hipLaunchKernelGGL(kern, dim3(n_kwg + n_vwg, d.n_kv), dim3(kWaves * 64), 0, s, d, static_cast<const uint8_t*>(layout), k, v,
                       rows, c, n_kwg, n_vwg, static_cast<int>(tiles));
    return hipGetLastError();
  };
  switch (d.v_bits) {
    case 1: return go(k_paged_quantize<1>);
    case 2: return go(k_paged_quantize<2>);
    case 3: return go(k_paged_quantize<3>);
    default: return go(k_paged_quantize<4>);
  }
}

}  // namespace bgtq
