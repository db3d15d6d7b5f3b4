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
//  * query rows and value radii are scaled by powers of two (mix.h), and fp32
//    outputs (EX) have their weights in two fp16 parts and every query product's
//    lo part, so that both output types have the precision of cross_impl.h;
//  * numbers that are not finite are kept (these files are compiled without the
//    packed decode's no-NaN flags);
//  * splits leave partials for a join instead of counting one another.
#pragma once
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>
#include <utility>

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

// ---- LDS: the packed decode's tables and query image; before them, while the
// tables are not yet built, what the query rotation needs
constexpr int kIn = 0;                                 // [8][128] query rows in stream order
constexpr int kSum = kIn + 8 * kHeadDim * 4;           // [4][8][128] quarter sums
constexpr int kRot = kSum + 4 * 8 * kHeadDim * 4;      // [8][128] rotated rows
static_assert(kRot + 8 * kHeadDim * 4 <= kQimg, "set-up below the query image");
constexpr int kTop = split_detail::kLdsBytes;          // [8] largest magnitudes, as bits
constexpr int kLds = kTop + 8 * 4;
static_assert(kLds <= 160 * 1024, "LDS of one workgroup");

__device__ __forceinline__ int up_of(uint32_t bits) {  // biased exponent of the power that brings it to [2^13, 2^14)
  const int e = static_cast<int>(bits >> 23);
  return e == 0 || e == 255 ? 127 : max(1, min(253, 127 + 13 + 127 - e));
}
__device__ __forceinline__ float two_to(int biased) { return __uint_as_float(static_cast<uint32_t>(biased) << 23); }

// Tables of the widths in `used` (bit b - 1): see decode_impl.h.
template <int THREADS, bool T12>
__device__ __forceinline__ void build_tables(uint8_t* smem, const uint16_t* cbs, uint32_t used, int tid) {
  const auto pair = [](const uint16_t* cb, int i, int b) {
    const int m = (1 << b) - 1;
    return cb[i & m] | static_cast<uint32_t>(cb[(i >> b) & m]) << 16;
  };
  if (used & 1u) {
    for (int i = tid; i < 16 * 16; i += THREADS)
      *reinterpret_cast<uint2*>(smem + kLut1 + i * 8) =
          make_uint2(pair(cbs + cb_index(1), i >> 4, 1), pair(cbs + cb_index(1), i >> 6, 1));
    if constexpr (!T12)
      for (int i = tid; i < 256 * 8; i += THREADS) {
        const int e = i >> 3;
        const uint16_t* cb = cbs + cb_index(1);
        *reinterpret_cast<uint4*>(smem + kLut1B + i * 16) =
            make_uint4(pair(cb, e, 1), pair(cb, e >> 2, 1), pair(cb, e >> 4, 1), pair(cb, e >> 6, 1));
      }
  }
  if (used & 2u)  // 16 lanes write an entry's 32 replicas
    for (int i = tid; i < 256 * 16; i += THREADS) {
      const uint32_t lo = pair(cbs + cb_index(2), i >> 4, 2), hi = pair(cbs + cb_index(2), i >> 8, 2);
      *reinterpret_cast<uint4*>(smem + kLut2 + i * 16) = make_uint4(lo, hi, lo, hi);
    }
  if (used & 4u) {
    if constexpr (T12)
      for (int i = tid; i < 4096; i += THREADS)
        *reinterpret_cast<uint2*>(smem + kLut1B + i * 8) =
            make_uint2(pair(cbs + cb_index(3), i, 3), pair(cbs + cb_index(3), i >> 6, 3));
    else
      for (int i = tid; i < 64 * 32; i += THREADS)
        *reinterpret_cast<uint32_t*>(smem + kLut3 + i * 4) = pair(cbs + cb_index(3), i >> 5, 3);
  }
  if (used & 8u)
    for (int i = tid; i < 256 * 8; i += THREADS)
      *reinterpret_cast<uint32_t*>(smem + kLut4 + i * 4) = pair(cbs + cb_index(4), i >> 3, 4);
  if (used & 16u)
    for (int i = tid; i < 32 * 32; i += THREADS)
      *reinterpret_cast<uint32_t*>(smem + kLut5 + i * 4) = cbs[cb_index(5) + (i >> 5)];
  if (used & 0xE0u)
    for (int i = tid; i < 256 + 128 + 64; i += THREADS) {
      const int b = i < 256 ? 8 : (i < 384 ? 7 : 6), k = i < 256 ? i : (i < 384 ? i - 256 : i - 384);
      *reinterpret_cast<uint16_t*>(smem + kLutF + i * 2) = cbs[cb_index(b) + k];
    }
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
  if (!paged::unit_of<8>(mode, d, static_cast<int>(blockIdx.x), U)) return;
  if (!U.q.ok) {
    if (U.split == 0) paged::refuse(U, d, U.kvh, call.out, call.out_dtype, tid, kThreads);
    return;
  }
  const int kvh = U.kvh, split = U.split, ri = d.layer * d.n_kv + kvh;
  const size_t out_row = static_cast<size_t>(U.q.first) * hq + kvh * G;  // head 0's row of q and out
  const RowMeta* M = reinterpret_cast<const RowMeta*>(blob + kOffRows) + ri;
  const int t_begin = split * S.split_len, t_end = min(U.q.len, t_begin + S.split_len), pos = U.q.len - 1;
  float* const part = call.part + ((static_cast<size_t>(U.block) * d.n_kv + kvh) * mode.unit_rows * call.n_slots + split) * kPartFloats;
  const size_t part_step = static_cast<size_t>(call.n_slots) * kPartFloats;  // from a head's partial to the next one's
  if (t_begin >= t_end) {  // (more than one split: a sequence has a row at least)
    if (tid < G) {
      part[tid * part_step] = kNegInf;
      part[tid * part_step + 1] = 0.f;
    }
    return;
  }

  // ---- set-up: the query heads in stream order, rotated as k_append_rows
  // rotates key rows (each of 512 threads a position and a quarter of the
  // products, its coefficients in flight together), scaled by a power of two
  // and split into fp16 hi and lo parts; then the lookup tables.
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
  uint16_t* const cbs = reinterpret_cast<uint16_t*>(smem + kCbStage);
  float* const xin = reinterpret_cast<float*>(smem + kIn);
  float* const sum = reinterpret_cast<float*>(smem + kSum);
  float* const rotd = reinterpret_cast<float*>(smem + kRot);
  uint32_t* const top = reinterpret_cast<uint32_t*>(smem + kTop);
  const int p = tid & 127, qq = (tid >> 7) & 3;
  int dg = gdim[0], p0 = 0;
#pragma unroll
  for (int h = 1; h < kMaxGroups; ++h)
    if (p >= gpos[h]) {
      dg = gdim[h];
      p0 = gpos[h];
    }
  float rc[32];
  {
    const float* rsrc = reinterpret_cast<const float*>(blob + kOffRotKT) + rotk_index(dg) + (p - p0);
#pragma unroll
    for (int u = 0; u < 32; ++u) rc[u] = rsrc[min(32 * qq + u, dg - 1) * dg];
  }
  {
    const uint16_t cv = reinterpret_cast<const uint16_t*>(blob + kOffC16)[min(tid, kCodebookEntries - 1)];
    const int src = M->dim[p];
    for (int i = tid; i < G * kHeadDim; i += kThreads)  // (kThreads is a multiple of 128: i % 128 = p)
      xin[i] = ld_q(q, (out_row + (i >> 7)) * kHeadDim + src, d.in_dtype);
    if (tid < kCodebookEntries) cbs[tid] = cv;
    if (tid < 8) top[tid] = 0;
  }
  __syncthreads();
  if (tid < 512) {
#pragma unroll
    for (int h = 0; h < 4 * NSET; ++h) {
      if (h >= G) break;
      float a = 0.f;
#pragma unroll
      for (int u = 0; u < 32; ++u)
        a = 32 * qq + u < dg ? fmaf(rc[u], xin[h * kHeadDim + p0 + 32 * qq + u], a) : a;
      sum[(qq * 8 + h) * kHeadDim + p] = a;
    }
  }
  __syncthreads();
  for (int i = tid; i < G * kHeadDim; i += kThreads) {
    const float* s = sum + i;
    const float v = ((s[0] + s[8 * kHeadDim]) + (s[16 * kHeadDim] + s[24 * kHeadDim])) *
                    (kLog2e * rsqrtf(static_cast<float>(dg) * kHeadDim));
    rotd[i] = v;
    atomicMax(top + (i >> 7), __float_as_uint(v) & 0x7FFFFFFFu);
  }
  __syncthreads();
  {
    int sl0[kMaxGroups], nslots = 0;
#pragma unroll
    for (int g = 0; g < kMaxGroups; ++g) {
      sl0[g] = nslots;
      nslots += ((gdim[g] + 3) / 4 + 15) / 16;
    }
    for (int i = tid; i < nslots * NSET * 64; i += kThreads) {
      const int l = i & 63, set = (i >> 6) % NSET, slot = (i >> 6) / NSET;
      int gd = gdim[0], gp = 0, s0 = 0;
#pragma unroll
      for (int g = 1; g < kMaxGroups; ++g)
        if (g < ng && slot >= sl0[g]) {
          gd = gdim[g];
          gp = gpos[g];
          s0 = sl0[g];
        }
      const int coord = 4 * (16 * (slot - s0) + (l >> 2)), h = 4 * set + (l & 3);
      const float to = two_to(up_of(top[min(h, 7)]));
      half4_t hi, lo;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float v = coord + k < gd && h < G ? rotd[h * kHeadDim + gp + coord + k] * to : 0.f;
        hi[k] = static_cast<_Float16>(v);
        lo[k] = static_cast<_Float16>(v - static_cast<float>(hi[k]));
      }
      uint8_t* dst = smem + kQimg + (((slot * 2 + set) * 2) * 64 + l) * 8;
      *reinterpret_cast<half4_t*>(dst) = hi;
      *reinterpret_cast<half4_t*>(dst + 64 * 8) = lo;
    }
  }
  __syncthreads();
  build_tables<kThreads, T12>(smem, cbs, used, tid);
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
      back[s][r] = two_to(254 - up_of(__builtin_amdgcn_readfirstlane(top[4 * s + r])));
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

  const int stride = kWaves * 64, nslot = (ng + 1) & ~1;
  int t0 = t_begin + wave * 64;
  int page_next = 0;
  bool lost = false;  // a page outside the pool: the rows that attend it are not numbers
  const auto read_page = [&](int t) {
    page_next = mode.b.pages[static_cast<size_t>(U.seq) * mode.b.max_pages + t / S.capacity];
  };
  const auto after = [&](int t) { return t + stride < t_end ? t + stride : t; };
  const size_t cap = S.capacity;
  const auto turn_to = [&](RowPtrs& R) {  // the page whose number was read
    lost |= static_cast<uint32_t>(page_next) >= static_cast<uint32_t>(S.batch);
    const size_t row = (static_cast<size_t>(d.layer) * S.batch + (lost ? 0 : page_next)) * d.n_kv + kvh;
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
    read_page(t0);
    turn_to(R2);
    load_keys<KWB>(rw2, knp2, nslot, R2, kw, t0 % S.capacity, lane);
    if constexpr (kValuesAhead) load_values<BV>(vn2, vw2, R2, t0 % S.capacity, lane);
    read_page(after(t0));
  }
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
        gmb[b] = gmt[b];
        if constexpr (EX) gmb[b] &= ~(1u << 23);  // every product's lo part
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
        if constexpr (MODS) x[r] = paged::changed<EX>(mode.m.cap, slope[s][r], x[r], static_cast<float>(pos - tk));
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
  float* const os = fo + kWaves * 8 * kHeadDim;      // [8][128] the result in the rotated domain
  static_assert((16 * 8 * 2 + 17 * 8 * kHeadDim) * 4 <= kLds, "join area");
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
  const float* rotv = reinterpret_cast<const float*>(blob + kOffRotV);
  for (int i = tid; i < G * kHeadDim; i += kThreads) {
    const int dd = i & 127;
    const float* o = os + (i & ~127);
    float r[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int j = 0; j < kHeadDim; j += 4)
#pragma unroll
      for (int u = 0; u < 4; ++u) r[u] = fmaf(rotv[(j + u) * kHeadDim + dd], o[j + u], r[u]);
    const float y = (r[0] + r[1]) + (r[2] + r[3]);
    const size_t at = out_row * kHeadDim + i;
    if (call.out_dtype == 1) {
      const __bf16 b = static_cast<__bf16>(y);
      static_cast<uint16_t*>(call.out)[at] = __builtin_bit_cast(uint16_t, b);
    } else {
      static_cast<float*>(call.out)[at] = y;
    }
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
