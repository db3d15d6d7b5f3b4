// Attention of one generated token a sequence to the rows that its pages hold:
// the pass of a batch's single tokens (paged_pass.h), up to 8 query rows (one
// token's heads of one KV head).
//
// The products are the packed decode's (decode_impl.h): a wave takes 64-row
// tiles, lane = token, whose codes become the operands of 4x4x4 f16 MFMAs with
// the query heads broadcast; 4 or 8 columns instead of the 32 of cross_impl.h,
// whose scaling and softmax of columns that one token does not have cost more
// instructions than the decode of the tile.  What differs from the packed decode:
//  * the rows' pages: a wave reads the page number of a tile one tile ahead of
//    the loads that need it;
//  * query rows and value radii are scaled by powers of two (mix.h), every query
//    product has its lo part and fp32 outputs (EX) have their weights in two fp16
//    parts, so that both output types have the precision of cross_impl.h;
//  * numbers that are not finite are kept (these files are compiled without the
//    packed decode's no-NaN flags);
//  * splits leave partials for a join instead of counting one another.
//
// What bounds it: vector instructions, some 560 a 64-row tile with 16 waves, and the
// set-up (10 us: the sequence's numbers, then its first page, then rows; rotation
// and tables meanwhile).  32 sequences of 500 to 8200 K2V2 rows x 8 KV heads x 4:
// 47 us, decided by the longest (107 in 32-row workgroups, 55 with a set-up that
// waits for each read in turn); one sequence of 500 rows 14.
#pragma once
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>
#include <utility>

#include "cross_impl.h"
#include "decode_impl.h"
#include "kernels.h"
#include "layout.h"
#include "mix.h"
#include "paged_pass.h"

namespace bgtq {
namespace paged_decode_detail {

using namespace split_detail;

template <int NSET, int KWB>
constexpr int waves_of() { return NSET == 1 && KWB <= 16 ? 16 : 12; }

using cross_detail::half8_t;
using cross_detail::matrix_parts;
using cross_detail::split8;
using cross_detail::staged_product;
using cross_detail::top16;
using cross_detail::two_to;
using cross_detail::up_of;

// ---- LDS: the packed decode's tables and query image, then per query row its
// largest rotated magnitude, as bits, and what its staged copy is multiplied with
constexpr int kTop = split_detail::kLdsBytes;
constexpr int kBack = kTop + 16 * 4;
constexpr int kLds = kBack + 16 * 4;
static_assert(kLds <= 160 * 1024, "LDS of one workgroup");
// rows staged as fp16 hi and lo parts (cross_impl.h), in the image's place
// before the rotation, behind the joined states at the end
static_assert(cross_detail::kHalfPart + 16 * cross_detail::kHalfStride <= kQimgBytes, "staged queries in the image's place");

// Tables of the widths in `used` (bit b - 1): see decode_impl.h.  A thread works
// out all its entries of a table before it writes one (the codebooks that it
// reads and the tables lie in the same LDS: the compiler would wait for each).
template <int THREADS, int N, class T, class F>
__device__ __forceinline__ void fill_table(uint8_t* dst, int tid, const F& entry) {
  constexpr int kPer = (N + THREADS - 1) / THREADS;
  T v[kPer];
#pragma unroll
  for (int k = 0; k < kPer; ++k) v[k] = entry(min(tid + k * THREADS, N - 1));
#pragma unroll
  for (int k = 0; k < kPer; ++k)
    if (N % THREADS == 0 || tid + k * THREADS < N) reinterpret_cast<T*>(dst)[tid + k * THREADS] = v[k];
}
template <int THREADS, bool T12>
__device__ __forceinline__ void build_tables(uint8_t* smem, const uint16_t* cbs, uint32_t used, int tid) {
  const auto pair = [](const uint16_t* cb, int i, int b) {
    const int m = (1 << b) - 1;
    return cb[i & m] | static_cast<uint32_t>(cb[(i >> b) & m]) << 16;
  };
  // two codes of 1 or 2 bits: bytes of the codebook's words
  const uint32_t c1 = *reinterpret_cast<const uint32_t*>(cbs + cb_index(1));
  const uint32_t c2a = *reinterpret_cast<const uint32_t*>(cbs + cb_index(2)), c2b = *reinterpret_cast<const uint32_t*>(cbs + cb_index(2) + 2);
  const auto pair1 = [&](int i) {
    return __builtin_amdgcn_perm(0u, c1, 0x01000100u + 0x0202u * (i & 1) + 0x02020000u * ((i >> 1) & 1));
  };
  const auto pair2 = [&](int i) {
    return __builtin_amdgcn_perm(c2b, c2a, 0x01000100u + 0x0202u * (i & 3) + 0x02020000u * ((i >> 2) & 3));
  };
  if (used & 2u)  // 16 lanes write an entry's 32 replicas
    fill_table<THREADS, 256 * 16, uint4>(smem + kLut2, tid, [&](int i) {
      const uint32_t lo = pair2(i >> 4), hi = pair2(i >> 8);
      return make_uint4(lo, hi, lo, hi);
    });
  if (used & 1u) {
    fill_table<THREADS, 16 * 16, uint2>(smem + kLut1, tid, [&](int i) { return make_uint2(pair1(i >> 4), pair1(i >> 6)); });
    if constexpr (!T12)
      fill_table<THREADS, 256 * 8, uint4>(smem + kLut1B, tid, [&](int i) {
        const int e = i >> 3;
        return make_uint4(pair1(e), pair1(e >> 2), pair1(e >> 4), pair1(e >> 6));
      });
  }
  if (used & 4u) {
    const uint16_t* cb = cbs + cb_index(3);
    if constexpr (T12)
      fill_table<THREADS, 4096, uint2>(smem + kLut1B, tid, [&](int i) { return make_uint2(pair(cb, i, 3), pair(cb, i >> 6, 3)); });
    else
      fill_table<THREADS, 64 * 32, uint32_t>(smem + kLut3, tid, [&](int i) { return pair(cb, i >> 5, 3); });
  }
  if (used & 8u)
    fill_table<THREADS, 256 * 8, uint32_t>(smem + kLut4, tid, [&](int i) { return pair(cbs + cb_index(4), i >> 3, 4); });
  if (used & 16u)
    fill_table<THREADS, 32 * 32, uint32_t>(smem + kLut5, tid, [&](int i) { return static_cast<uint32_t>(cbs[cb_index(5) + (i >> 5)]); });
  if (used & 0xE0u)
    fill_table<THREADS, 256 + 128 + 64, uint16_t>(smem + kLutF, tid, [&](int i) {
      const int b = i < 256 ? 8 : (i < 384 ? 7 : 6), k = i < 256 ? i : (i < 384 ? i - 256 : i - 384);
      return cbs[cb_index(b) + k];
    });
}

// PV with weights in two parts, each decoded operand used for both.
template <int BV, int NSET, bool T12, int ST>
__device__ __forceinline__ void pv_step_both(const uint8_t* smem, const uint32_t (&vw)[4][pv_words<BV>()], const LaneRep& rep,
                                             const half4_t (&hi)[NSET], const half4_t (&lo)[NSET], float4_t (&O)[NSET][2]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const half4_t vv = decode4<BV, 4 * BV * (ST & 7), T12>(smem, vw[(ST >> 3) * 2 + h], rep);
#pragma unroll
    for (int s = 0; s < NSET; ++s) {
      O[s][h] = __builtin_amdgcn_mfma_f32_4x4x4f16(hi[s], vv, O[s][h], 4, ST, 0);
      O[s][h] = __builtin_amdgcn_mfma_f32_4x4x4f16(lo[s], vv, O[s][h], 4, ST, 0);
    }
  }
}
template <int BV, int NSET, bool T12, int... ST>
__device__ __forceinline__ void pv_both(std::integer_sequence<int, ST...>, const uint8_t* smem,
                                        const uint32_t (&vw)[4][pv_words<BV>()], const LaneRep& rep,
                                        const half4_t (&hi)[NSET], const half4_t (&lo)[NSET], float4_t (&O)[NSET][2]) {
  (pv_step_both<BV, NSET, T12, ST>(smem, vw, rep, hi, lo, O), ...);
}

template <int NSET, int KWB, int BV, bool EX, bool MODS>
__global__ __launch_bounds__((waves_of<NSET, KWB>() * 64))
__attribute__((amdgpu_waves_per_eu((waves_of<NSET, KWB>() / 4)))) void k_paged_decode(
    Dims d, const uint8_t* __restrict__ blob, const void* __restrict__ q, CrossCall call, paged::Mode<MODS> mode) {
  constexpr int kWaves = waves_of<NSET, KWB>(), kThreads = kWaves * 64;
  constexpr bool T12 = BV == 3;
  __shared__ __attribute__((aligned(16))) uint8_t smem[kLds];
  const CrossSide& S = call.side[0];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int bq = lane >> 2, jq = lane & 3;
  const int G = d.group, hq = d.n_kv * G, kw = d.k_words;
  paged::Unit U;
  const int block = paged::unit_at(mode, d, call.n_slots, static_cast<int>(blockIdx.x), U);
  const RowMeta* M = reinterpret_cast<const RowMeta*>(blob + kOffRows) + (d.layer * d.n_kv + U.kvh);
  // the reads that need no sequence, before its numbers are there
  const uint16_t cv = reinterpret_cast<const uint16_t*>(blob + kOffC16)[min(tid, kCodebookEntries - 1)];
  float4_t rk[8];
  if (wave < 8) {
    const float4_t* w = reinterpret_cast<const float4_t*>(blob + layout_kdense_offset(d.n_layers * d.n_kv)) +
                        static_cast<size_t>(d.layer * d.n_kv + U.kvh) * (kMfmaMatFloats / 4) + wave * 8 * 64 + lane;
#pragma unroll
    for (int s4 = 0; s4 < 8; ++s4) rk[s4] = w[s4 * 64];
  }
  const int ng = M->n_groups;
  int gdim[kMaxGroups], gpos[kMaxGroups];
  uint32_t used = 1u << (BV - 1);
#pragma unroll
  for (int g = 0; g < kMaxGroups; ++g) {
    const int a = M->g_dim[g], b = M->g_pos[g];
    gdim[g] = g < ng ? a : 0;
    gpos[g] = g < ng ? b : kHeadDim;
    used |= (M->gm[g] >> 31) << g;
  }
  if (!paged::find_unit<8>(mode, d, call, block, U, kThreads)) return;
  const int kvh = U.kvh, split = U.split;
  const size_t out_row = static_cast<size_t>(U.q.first) * hq + kvh * G;  // head 0's row of q and out
  const int t_begin = split * S.split_len, t_end = min(U.q.len, t_begin + S.split_len), pos = U.q.len - 1;
  float* const part = call.part + (paged::part_row(mode, U, hq, 0, kvh * G) * call.n_slots + split) * kPartFloats;
  const size_t part_step = static_cast<size_t>(call.n_slots) * kPartFloats;  // from a head's partial to the next one's
  if (t_begin >= t_end) {  // (more than one split: a sequence has a row at least)
    if (tid < G) {
      part[tid * part_step] = kNegInf;
      part[tid * part_step + 1] = 0.f;
    }
    return;
  }

  // ---- set-up, in few rounds of global reads, those of the first tile among
  // them: the query heads staged as cross_impl.h does and rotated by three fp16
  // products (8 of the waves, 16 positions each), written into the image as hi
  // and lo parts scaled by a power of two; the lookup tables meanwhile.
  const int stride = kWaves * 64;
  int t0 = t_begin + wave * 64;
  int page_next = 0;
  bool lost = false;  // a page outside the pool: the rows that attend it are not numbers
  const auto read_page = [&](int t) {
    page_next = paged::page_ahead(mode.b, U.seq, t, S.capacity);
  };
  const auto after = [&](int t) { return t + stride < t_end ? t + stride : t; };
  if (t0 < t_end) read_page(t0);
  const int nslot = (ng + 1) & ~1;
  uint16_t* const cbs = reinterpret_cast<uint16_t*>(smem + kCbStage);
  uint32_t* const top = reinterpret_cast<uint32_t*>(smem + kTop);
  float* const fix = reinterpret_cast<float*>(smem + kBack);
  uint4 x0 = make_uint4(0, 0, 0, 0), x1 = x0;
  const bool bf = d.in_dtype == 1;
  if (tid < G * 16) {  // thread = row tid / 16, dims 8 (tid % 16) .. + 7
    const size_t at = (out_row + (tid >> 4)) * kHeadDim + 8 * (tid & 15);
    const uint4* qp = reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(q) + at * (bf ? 2 : 4));
    x0 = qp[0];
    if (!bf) x1 = qp[1];
  }
  const size_t cap = S.capacity;
  const auto turn_to = [&](RowPtrs& R) {  // the page whose number was read
    const int page = __builtin_amdgcn_readfirstlane(page_next);
    lost |= static_cast<uint32_t>(page) >= static_cast<uint32_t>(S.batch);
    const size_t row = (static_cast<size_t>(d.layer) * S.batch + (lost ? 0 : page)) * d.n_kv + kvh;
    R = {S.c.k_codes + row * cap * kw, S.c.k_norms + row * kMaxGroups * cap, S.c.v_codes + row * (cap / kTile) * kHeadDim * BV,
         S.c.v_norms + row * cap};
  };
  RowPtrs R, R2;
  constexpr bool kValuesAhead = NSET == 1 && KWB <= 8 && BV <= 2 && !EX;
  uint32_t rw[KWB + kRowPad], knp[4], rw2[KWB], knp2[4], vw[4][pv_words<BV>()];
  uint32_t vw2[kValuesAhead ? 4 : 1][kValuesAhead ? pv_words<BV>() : 1];
  uint2 vn, vn2;
#pragma unroll
  for (int i = KWB; i < KWB + kRowPad; ++i) rw[i] = 0u;
  if (t0 < t_end) {
    turn_to(R2);
    load_keys<KWB>(rw2, knp2, nslot, R2, kw, t0 % S.capacity, lane);
    if constexpr (kValuesAhead) load_values<BV>(vn2, vw2, R2, t0 % S.capacity, lane);
    read_page(after(t0));
  }
  if (tid < kCodebookEntries) cbs[tid] = cv;
  if (tid < 16) top[tid] = 0;
  if (tid < G * 16) {
    const uint32_t y0[4] = {x0.x, x0.y, x0.z, x0.w}, y1[4] = {x1.x, x1.y, x1.z, x1.w};
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t half = e & 1 ? y0[e >> 1] & 0xFFFF0000u : y0[e >> 1] << 16;
      x[e] = __uint_as_float(bf ? half : (e < 4 ? y0[e & 3] : y1[e & 3]));
    }
    const int up = up_of(top16(x));
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] *= two_to(up);
    half8_t hi, lo;
    split8(x, hi, lo);
    uint8_t* dst = smem + kQimg + (tid >> 4) * cross_detail::kHalfStride + 16 * (tid & 15);
    *reinterpret_cast<half8_t*>(dst) = hi;
    *reinterpret_cast<half8_t*>(dst + cross_detail::kHalfPart) = lo;
    if ((tid & 15) == 0) fix[tid >> 4] = two_to(254 - up) * (1.f / 256.f);
  }
  __syncthreads();
  const int hr = lane & 15, p0 = 16 * (wave & 7) + 4 * (lane >> 4);  // the lane's row and 4 positions
  float4_t rq[1];
  uint32_t img_at[2];
  if (wave < 8) {
    // (rows from G on are what LDS held: their products are not used)
    staged_product<1>(smem + kQimg, rk, lane, rq);
    // place of the lane's position pairs in the image (group sizes are even)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      int sl = 0, at = 0, dg = 2, base = 0;
#pragma unroll
      for (int g = 0; g < kMaxGroups; ++g) {
        if (p0 + 2 * h >= gpos[g]) {
          at = p0 + 2 * h - gpos[g];
          dg = gdim[g];
          sl = base;
        }
        base += ((gdim[g] + 3) / 4 + 15) / 16;
      }
      const int step = at >> 2;
      img_at[h] = kQimg + ((((sl + (step >> 4)) * 2 + (hr >> 2)) * 2) * 64 + 4 * (step & 15) + (hr & 3)) * 8 + (at & 3) * 2;
      const float scale = kLog2e * cross_detail::kRsqrtD * rsqrtf(static_cast<float>(dg));
      rq[0][2 * h] *= scale;
      rq[0][2 * h + 1] *= scale;
    }
    uint32_t mx = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) mx = max(mx, __float_as_uint(rq[0][i]) & 0x7FFFFFFFu);
    mx = max(mx, static_cast<uint32_t>(__shfl_xor(static_cast<int>(mx), 16)));
    mx = max(mx, static_cast<uint32_t>(__shfl_xor(static_cast<int>(mx), 32)));
    if (lane < 16) atomicMax(top + lane, mx);
  }
  build_tables<kThreads, T12>(smem, cbs, used, tid);
  __syncthreads();
  // (the image takes the staged queries' place)
  if (wave < 8 && hr < 4 * NSET) {
    const float to = two_to(up_of(top[hr]));
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      _Float16 hi[2], lo[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const float x = hr < G ? rq[0][2 * h + j] * to : 0.f;
        hi[j] = static_cast<_Float16>(x);
        lo[j] = static_cast<_Float16>(x - static_cast<float>(hi[j]));
      }
      typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
      *reinterpret_cast<half2_t*>(smem + img_at[h]) = half2_t{hi[0], hi[1]};
      *reinterpret_cast<half2_t*>(smem + img_at[h] + 64 * 8) = half2_t{lo[0], lo[1]};
    }
  } else if (wave == 8 && lane < 8 * kMaxGroups) {
    // zeros behind a group's end: lane = (group, row)
    int base = 0, gd = 0, sl = 0;
#pragma unroll
    for (int g = 0; g < kMaxGroups; ++g) {
      if (lane >> 3 == g) {
        gd = gdim[g];
        sl = base;
      }
      base += ((gdim[g] + 3) / 4 + 15) / 16;
    }
    if (gd & 2) {
      const int step = gd >> 2, r = lane & 7;
      uint8_t* dst = smem + kQimg + ((((sl + (step >> 4)) * 2 + (r >> 2)) * 2) * 64 + 4 * (step & 15) + (r & 3)) * 8 + 4;
      *reinterpret_cast<uint32_t*>(dst) = 0;
      *reinterpret_cast<uint32_t*>(dst + 64 * 8) = 0;
    }
  }
  __syncthreads();

  LaneRep rep{static_cast<uint32_t>(kLut1 + (lane & 15) * 8), static_cast<uint32_t>(kLut3 + (lane & 31) * 4),
              static_cast<uint32_t>(kLut4 + (lane & 7) * 4),   static_cast<uint32_t>(kLut5 + (lane & 31) * 4),
              static_cast<uint32_t>(kLut2 + (lane & 31) * 8),  static_cast<uint32_t>(kLut1B + (T12 ? 0 : (lane & 7) * 16)),
              static_cast<uint32_t>(kQimg + lane * 8)};
  asm volatile("" : "+v"(rep.r1), "+v"(rep.r3), "+v"(rep.r4), "+v"(rep.r5), "+v"(rep.r2), "+v"(rep.r1b));

  // what undoes the scales: head r of each set while lane = token (registers are
  // heads), uniform; the slopes likewise
  float back[NSET][4], slope[MODS ? NSET : 1][4];
#pragma unroll
  for (int s = 0; s < NSET; ++s)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      back[s][r] = two_to(254 - up_of(__builtin_amdgcn_readfirstlane(top[4 * s + r]))) *
                   (4 * s + r < G ? __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(fix[4 * s + r]))) : 0.f);
      if constexpr (MODS) slope[s][r] = mode.m.slopes && 4 * s + r < G ? kLog2e * mode.m.slopes[kvh * G + 4 * s + r] : 0.f;
    }

  float m_run[NSET], l_run[NSET];
  float4_t O[NSET][2];
#pragma unroll
  for (int s = 0; s < NSET; ++s) {
    m_run[s] = kNegInf;
    l_run[s] = 0.f;
    O[s][0] = float4_t{0.f, 0.f, 0.f, 0.f};
    O[s][1] = float4_t{0.f, 0.f, 0.f, 0.f};
  }
  int v_top = 0;  // (see radius_top)

  uint32_t gmb[8];
  for (; t0 < t_end; t0 += stride) {
#pragma unroll
    for (int i = 0; i < KWB; ++i) rw[i] = rw2[i];
    // (an infinite key radius becomes not a number: see cross_impl.h)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
      const half2_t r = __builtin_bit_cast(half2_t, knp2[g]);
      knp[g] = __builtin_bit_cast(uint32_t, r + (r - r));
    }
    R = R2;
    if constexpr (kValuesAhead) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int w = 0; w < pv_words<BV>(); ++w) vw[i][w] = vw2[i][w];
      vn = vn2;
    } else {
      load_values<BV>(vn, vw, R, t0 % S.capacity, lane);
    }
    if (t0 + stride < t_end) {
      const int tn = t0 + stride;
      __builtin_amdgcn_s_setprio(3);
      turn_to(R2);
      load_keys<KWB>(rw2, knp2, nslot, R2, kw, tn % S.capacity, lane);
      if constexpr (kValuesAhead) load_values<BV>(vn2, vw2, R2, tn % S.capacity, lane);
      read_page(after(tn));
      __builtin_amdgcn_s_setprio(0);
    }
    const int tk = t0 + lane;
    {
      uint32_t goff = 0;
      asm volatile("" : "+s"(goff));
      const uint32_t* gmt = reinterpret_cast<const uint32_t*>(reinterpret_cast<const uint8_t*>(M->gm) + goff);
#pragma unroll
      for (int b = 0; b < 8; ++b) {
        gmb[b] = gmt[b] & ~(1u << 23);  // every product's lo part
      }
    }
    float4_t L[NSET];
#pragma unroll
    for (int s = 0; s < NSET; ++s) L[s] = float4_t{0.f, 0.f, 0.f, 0.f};
    __builtin_amdgcn_s_setprio(2);
    qk_all<NSET, T12, KWB>(std::make_integer_sequence<int, 8>{}, smem, rw, knp, gmb, rep, lane, L);
    __builtin_amdgcn_s_setprio(0);

    const bool full = t0 + 64 <= t_end;
    uint2 vr = vn;
    if (!full) vr = paged::seen(vr, t_end - (t0 + 4 * bq));
    // radii to the running power of two (the tile's largest: any lane has four)
    {
      const auto field = [](uint32_t r) {
        const int a = static_cast<int>(r >> 10 & 31u), b = static_cast<int>(r >> 26 & 31u);
        return max(a == 31 ? 0 : a, b == 31 ? 0 : b);
      };
      const int was = v_top;
      v_top = raise_top(was, max(field(vr.x), field(vr.y)));
      if (v_top != was && was > 0) {
        const float down = two_to(127 + was - v_top);
#pragma unroll
        for (int s = 0; s < NSET; ++s) {
          O[s][0] *= down;
          O[s][1] *= down;
        }
      }
      const int up = radius_up(v_top);
      vr.x = radius_times(vr.x & 0xFFFFu, up) | radius_times(vr.x >> 16, up) << 16;
      vr.y = radius_times(vr.y & 0xFFFFu, up) | radius_times(vr.y >> 16, up) << 16;
    }
    half4_t pp[NSET], pl[EX ? NSET : 1];
#pragma unroll
    for (int s = 0; s < NSET; ++s) {
      float4_t x = L[s];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        x[r] *= back[s][r];
        if constexpr (MODS) x[r] = paged::changed(mode.m.cap, slope[s][r], x[r], static_cast<float>(pos - tk));
      }
      if (!full) {
        if (tk >= t_end) x = float4_t{kNegInf, kNegInf, kNegInf, kNegInf};
        asm volatile("" : "+v"(x));
      }
      quad_transpose(x, lane);
      const float mx = fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]));
      float mn = m_run[s], corr = 1.f;
      const bool raise = __builtin_amdgcn_ballot_w64(mx > mn) != 0;
      if (raise) {
        mn = fmaxf(mn, xmax16(mx));
        corr = m_run[s] == kNegInf ? 0.f : exp2_hw(m_run[s] - mn);
      }
      const float mref = mn == kNegInf ? 0.f : mn;  // (logits that are all not a number)
      float e[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) e[r] = exp2_hw(x[r] - mref);
      const float ps = ((e[0] + e[1]) + e[2]) + e[3];
      const uint32_t w0 = mix_pair(e[0], e[1], vr.x), w1 = mix_pair(e[2], e[3], vr.y);
      pp[s] = as_half4(w0, w1);
      if constexpr (EX) {
        typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const half2_t r = __builtin_bit_cast(half2_t, k ? vr.y : vr.x);
#pragma unroll
          for (int j = 0; j < 2; ++j)
            pl[s][2 * k + j] =
                static_cast<_Float16>(fmaf(e[2 * k + j], static_cast<float>(r[j]), -static_cast<float>(pp[s][2 * k + j])));
        }
      }
      l_run[s] = fmaf(l_run[s], corr, ps);
      if (raise) {
        const float c0 = qperm<0x00>(corr), c1 = qperm<0x55>(corr), c2 = qperm<0xAA>(corr), c3 = qperm<0xFF>(corr);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          O[s][h][0] *= c0;
          O[s][h][1] *= c1;
          O[s][h][2] *= c2;
          O[s][h][3] *= c3;
        }
        m_run[s] = mn;
      }
    }
    __builtin_amdgcn_s_setprio(1);
    if constexpr (EX) pv_both<BV, NSET, T12>(std::make_integer_sequence<int, 16>{}, smem, vw, rep, pp, pl, O);
    else pv_steps<BV, NSET, T12>(std::make_integer_sequence<int, 16>{}, smem, vw, rep, pp, O);
    __builtin_amdgcn_s_setprio(0);
  }

  // ---- the waves' states joined in LDS (over the tables), then a partial or
  // the output
#pragma unroll
  for (int s = 0; s < NSET; ++s) {
    l_run[s] = xsum16(l_run[s]);
    if (lost) l_run[s] = __builtin_nanf("");
  }
  __syncthreads();
  float* const fm = reinterpret_cast<float*>(smem);  // [wave][8] maxima
  float* const fl = fm + kWaves * 8;                 // [wave][8] sums
  float* const fo = fl + kWaves * 8;                 // [wave][8][128] accumulators
  constexpr int kEnd = (16 * 8 * 2 + 16 * 8 * kHeadDim) * 4;  // result rows in fp32, then staged
  float* const os = reinterpret_cast<float*>(smem + kEnd);
  constexpr int kStaged = kEnd + 8 * kHeadDim * 4;
  static_assert(kStaged + cross_detail::kHalfPart + 16 * cross_detail::kHalfStride <= kTop, "join area");
  float4_t rot[8];  // this wave's 16 output dims of Pi_V^T
  if (call.n_slots == 1 && wave < 8) {
    const float4_t* src = reinterpret_cast<const float4_t*>(blob + kOffRotVT) +
                          ((16 * wave + (lane & 15)) * kHeadDim + 32 * (lane >> 4)) / 4;
#pragma unroll
    for (int s4 = 0; s4 < 8; ++s4) rot[s4] = src[s4];
  }
  const float v_back = two_to(127 - radius_up(v_top));
#pragma unroll
  for (int s = 0; s < NSET; ++s) {
    if (bq == 0) {
      fm[wave * 8 + s * 4 + jq] = m_run[s];
      fl[wave * 8 + s * 4 + jq] = l_run[s];
    }
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int r = 0; r < 4; ++r) fo[(wave * 8 + s * 4 + r) * kHeadDim + 64 * h + lane] = O[s][h][r] * v_back;
  }
  __syncthreads();
  const int n_act = min(kWaves, (t_end - t_begin + 63) / 64);  // waves that had a tile
  for (int i = tid; i < G * kHeadDim; i += kThreads) {
    const int h = i >> 7, dd = i & 127;
    float mx = kNegInf;
    for (int w = 0; w < n_act; ++w) mx = fmaxf(mx, fm[w * 8 + h]);
    const float mref = mx == kNegInf ? 0.f : mx;
    float l = 0.f, a = 0.f;
    for (int w = 0; w < n_act; ++w) {
      const float e = exp2_hw(fm[w * 8 + h] - mref);
      l = fmaf(fl[w * 8 + h], e, l);
      a = fmaf(fo[(w * 8 + h) * kHeadDim + dd], e, a);
    }
    if (call.n_slots > 1) {
      float* P = part + h * part_step;
      if (dd == 0) {
        P[0] = l == 0.f ? kNegInf : mref;
        P[1] = l;
      }
      P[4 + dd] = a;
    } else {
      os[i] = l == 0.f ? 0.f : a * (0.08838834764831845f / l);
    }
  }
  if (call.n_slots > 1) return;
  __syncthreads();
  // out = Pi_V^T (a / l), in three fp16 products of the rows scaled as the queries were
  if (tid < G * 16) {
    const float* o = os + (tid >> 4) * kHeadDim + 8 * (tid & 15);
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = o[e];
    const int up = up_of(top16(x));
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] *= two_to(up);
    half8_t hi, lo;
    split8(x, hi, lo);
    uint8_t* dst = smem + kStaged + (tid >> 4) * cross_detail::kHalfStride + 16 * (tid & 15);
    *reinterpret_cast<half8_t*>(dst) = hi;
    *reinterpret_cast<half8_t*>(dst + cross_detail::kHalfPart) = lo;
    if ((tid & 15) == 0) fix[tid >> 4] = two_to(254 - up) * (1.f / 256.f);
  }
  __syncthreads();
  if (wave < 8) {
    float4_t y[1];
    staged_product<1>(smem + kStaged, rot, lane, y);
    if (hr < G)
      cross_detail::store4(call.out, (out_row + hr) * kHeadDim + 16 * wave + 4 * (lane >> 4), y[0] * fix[hr], call.out_dtype);
  }
}

template <int BV>
hipError_t launch_bv(const Dims& d, const void* layout, const void* q, const CrossCall& call, const PagedPass& pass,
                     hipStream_t s) {
  const auto go = [&](auto kern, int threads, auto mode) {
    hipLaunchKernelGGL(kern, dim3(call.side[0].items), dim3(threads), 0, s, d, static_cast<const uint8_t*>(layout), q, call, mode);
    return hipGetLastError();
  };
  const auto width = [&](auto set, auto ex, auto mode) {
    constexpr int N = decltype(set)::value;
    constexpr bool E = decltype(ex)::value, M = decltype(mode)::kMods;
    if (d.k_words <= 8) return go(k_paged_decode<N, 8, BV, E, M>, 64 * waves_of<N, 8>(), mode);
    if (d.k_words <= 12) return go(k_paged_decode<N, 12, BV, E, M>, 64 * waves_of<N, 12>(), mode);
    if (d.k_words <= 16) return go(k_paged_decode<N, 16, BV, E, M>, 64 * waves_of<N, 16>(), mode);
    return go(k_paged_decode<N, 32, BV, E, M>, 64 * waves_of<N, 32>(), mode);
  };
  const auto mods = [&](auto set, auto ex) {
    return pass.m.cap > 0.f || pass.m.slopes ? width(set, ex, paged::Mode<true>{pass}) : width(set, ex, paged::Mode<false>{pass});
  };
  const auto type = [&](auto set) { return call.out_dtype == 0 ? mods(set, std::true_type{}) : mods(set, std::false_type{}); };
  return d.group <= 4 ? type(std::integral_constant<int, 1>{}) : type(std::integral_constant<int, 2>{});
}

}  // namespace paged_decode_detail
}  // namespace bgtq
