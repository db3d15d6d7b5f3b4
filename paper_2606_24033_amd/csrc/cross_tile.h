// Attention of many query rows of one (layer, sequence, KV head) to a range of
// packed rows that all of them see: the wide form of cross_impl.h, for units of
// some hundred query rows and more.
//
// As in the causal prefill attention (attn_tile.h has the shared parts), a
// workgroup's 8 waves decode each 64-row tile once into LDS, double-buffered,
// for 256 query rows (128 with two waves to 32 rows, KS = 2), so that a row
// pays 1/256 of the decode.  Here there is no causal mask, the key axis can be
// in splits, query rows and the radii of keys and values are scaled by powers of
// two (their fp16 lo parts stay above the subnormals), and the results are
// partials or, with one split, outputs.
//
// What bounds it: the matrix cores (53 % busy) and the decode beside them; QK takes
// three fp16 products and PV one (two for fp32 outputs) where fp16 attention
// takes two in all.  A 64-row tile takes 2.75 us for 256 query rows with few CUs
// busy, 3.65 with all.  2 x 8 heads x 2048 query positions on 16385 K3V3 rows: 521 us
// a call, 527 TFLOP/s.  An 8192-token prompt over pages, 8 KV heads x 4 query heads,
// causal: 1092 us, matrix cores and vector instructions 51 % busy each.  256 or 128
// rows: the former pay less decode, the latter give twice the workgroups (32768
// rows, 8 KV heads, in us for 128 / 256: 128 query rows a head 71 / 86, 512 171 /
// 155, 2048 614 / 497).
#pragma once
#include <hip/hip_runtime.h>

#include "attn_tile.h"
#include "kernels.h"
#include "layout.h"
#include "mix.h"
#include "paged_pass.h"

namespace bgtq {
namespace cross_tile_detail {

using namespace prefill_detail;
constexpr float kRsqrtD = 0.08838834764831845f;  // 1 / sqrt(128)
// the epilogue's Pi_V^T in fp16 hi and lo parts, operand [part][dim block][step][lane] x 16 B
constexpr int kRotPart = 4 * 8 * 1024;
static_assert(2 * kRotPart <= kLdsBytes, "Pi_V in LDS");

__device__ __forceinline__ void store4(void* out, size_t i, const float4_t& y, int dtype) {  // BGTQ_BF16 = 1
  if (dtype == 1) {
    typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
    *reinterpret_cast<bf16x4_t*>(static_cast<uint16_t*>(out) + i) = __builtin_convertvector(y, bf16x4_t);
  } else {
    *reinterpret_cast<float4_t*>(static_cast<float*>(out) + i) = y;
  }
}

// The power of two 2^up that brings a magnitude to [2^13, 2^14), as a float,
// and 2^-up; 1 for zeros and what is not finite.
__device__ __forceinline__ void scale_of(float mx, float& to, float& back) {
  const int e = static_cast<int>(__float_as_uint(mx) >> 23);
  const int up = e == 0 || e == 255 ? 127 : max(1, min(253, 127 + 13 + 127 - e));
  to = __uint_as_float(static_cast<uint32_t>(up) << 23);
  back = __uint_as_float(static_cast<uint32_t>(254 - up) << 23);
}

// EX: the softmax weights in two fp16 parts, for fp32 outputs (see cross_impl.h).
// MODE: WholeCache, or the new rows of a ragged batch over pages (paged_pass.h).
template <int BV, int KS, bool EX, class MODE>
__global__ __launch_bounds__(kAttnThreads) __attribute__((amdgpu_waves_per_eu(2, 2))) void k_cross_tile(
    Dims d, const uint8_t* __restrict__ blob, const float* __restrict__ qr, CrossCall call, MODE mode) {
  constexpr bool kPaged = MODE::kPaged, kMods = MODE::kMods;
  constexpr int kWgRows = kAttnWaves / KS * kWaveRows, NB = 2 / KS;  // query rows; token blocks of a wave
  __shared__ __attribute__((aligned(16))) uint8_t smem[kLdsBytes];
  const CrossSide& S = call.side[0];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, hf = lane >> 5;
  const int G = d.group, hq = d.n_kv * G, kw = d.k_words;
  int item = blockIdx.x;  // (row blocks fastest, splits slowest: see k_cross)
  int nr, first, kvh, lz = 0, split, seq, layer;  // query rows of the unit, the workgroup's first one
  paged::Unit U = {};
  if constexpr (kPaged) {
    if (!paged::find_unit<kWgRows>(mode, d, call, paged::unit_at(mode, d, call.n_slots, item, U), U, kAttnThreads)) return;
    nr = U.q.n * G;
    first = U.r0;
    kvh = U.kvh;
    split = U.split;
    seq = U.seq;
    layer = d.layer;
  } else {
    nr = S.n_q * G;
    const int n_blocks = (nr + kWgRows - 1) / kWgRows;
    first = item % n_blocks * kWgRows;
    item /= n_blocks;
    kvh = item % d.n_kv;
    item /= d.n_kv;
    const int n_lz = d.n_lc * S.batch;
    lz = item % n_lz;
    split = item / n_lz;
    seq = lz % S.batch;
    layer = d.layer >= 0 ? d.layer : lz / S.batch;
  }
  const RowMeta* M = reinterpret_cast<const RowMeta*>(blob + kOffRows) + (layer * d.n_kv + kvh);
  const int nslot = (M->n_groups + 1) & ~1;
  const int rw = KS == 1 ? wave : wave & 3;   // the wave's row block
  const int blk0 = KS == 1 ? 0 : wave >> 2;   // its first token block of a tile
  const int r = first + rw * kWaveRows + l32;  // this lane's query row of the unit
  const int rc = min(r, nr - 1);
  const size_t row_at = ((kPaged ? static_cast<size_t>(U.q.first) : static_cast<size_t>(lz) * S.n_q) + rc / G) * hq + kvh * G + rc % G;
  const auto part_of = [&]() {
    if constexpr (kPaged)
      return call.part + (paged::part_row(mode, U, hq, rc / G, kvh * G + rc % G) * call.n_slots + split) * kPartFloats;
    else return call.part + (row_at * call.n_slots + S.slot0 + split) * kPartFloats;
  };

  // a length outside [0, max_len] (the host's bound) makes the rows NaN
  const int len = kPaged ? U.q.len : S.len[seq];
  const bool ok = kPaged || (len >= 0 && len <= S.max_len);
  const int t_begin = split * S.split_len;
  // the rows that the last query row sees; each row's own end, and the wave's
  // first row's (paged)
  paged::Sight sight = {};
  int t_end, lim = 0, lim0 = 0;
  float slope = 0.f;
  if constexpr (kPaged) {
    sight = paged::sight_of(mode, U, seq);
    t_end = min(sight.end((min(first + kWgRows, nr) - 1) / G), t_begin + S.split_len);
    lim = min(sight.end(rc / G), t_end);
    lim0 = min(sight.end(min(first + rw * kWaveRows, nr - 1) / G), t_end);
    if (kMods && mode.m.slopes) slope = kLog2e * mode.m.slopes[kvh * G + rc % G];
  } else {
    t_end = ok ? min(len, t_begin + S.split_len) : t_begin;
  }
  const int n_kt = (max(t_end - t_begin, 0) + kKeyTile - 1) / kKeyTile;

  if (t_begin >= t_end && call.n_slots > 1) {  // no row of the sequence in this split: an empty partial
    if (r < nr && hf == 0 && (KS == 1 || wave < 4)) {
      float* P = part_of();
      P[0] = ok ? kNegInf : 0.f;
      P[1] = ok ? 0.f : __builtin_nanf("");
    }
    return;
  }

  // query operands (B of S^T = K Q^T): dims 16 ks + 8 hf .. +7 of the row,
  // scaled, in fp16 hi and lo parts.
  half8_t qh[8], ql[8];
  float sc;
  {
    const float4_t* src = reinterpret_cast<const float4_t*>(qr + row_at * kHeadDim + 8 * hf);
    float4_t v[16];
    float mx = 0.f;
    bool bad = false;
#pragma unroll
    for (int ks = 0; ks < 16; ++ks) {
      v[ks] = src[4 * (ks >> 1) + (ks & 1)];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        mx = fmaxf(mx, fabsf(v[ks][e]));
        bad = bad || v[ks][e] != v[ks][e];
      }
    }
    mx = max2g(bad ? __builtin_huge_valf() : mx);
    float to;
    scale_of(mx, to, sc);
#pragma unroll
    for (int ks = 0; ks < 8; ++ks)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float x = v[2 * ks + (e >> 2)][e & 3] * to;
        const _Float16 h = static_cast<_Float16>(x);
        qh[ks][e] = h;
        ql[ks][e] = static_cast<_Float16>(x - static_cast<float>(h));
      }
  }
  const KeyItems items = key_items(M, wave, kw);
  {
    const uint16_t* c16 = reinterpret_cast<const uint16_t*>(blob + kOffC16);
    uint16_t* cbs = reinterpret_cast<uint16_t*>(smem + kOffCb);
    for (int i = tid; i < kCodebookEntries; i += kAttnThreads) cbs[i] = c16[i];
    __syncthreads();
#pragma unroll
    for (int b = 1; b <= kMaxPair; ++b)
      for (int i = tid; i < (1 << (2 * b)); i += kAttnThreads)
        *reinterpret_cast<uint32_t*>(smem + kOffPair + pair_offset(b) + 4 * i) =
            cbs[cb_index(b) + (i & ((1 << b) - 1))] | (static_cast<uint32_t>(cbs[cb_index(b) + (i >> b)]) << 16);
  }

  const size_t cap = S.capacity;
  const uint8_t *kc, *kn, *vc;
  const uint16_t* vnp;
  const auto rows_of = [&](size_t row) {  // (layer, sequence or page, head)
    kc = reinterpret_cast<const uint8_t*>(S.c.k_codes + row * cap * kw);
    kn = reinterpret_cast<const uint8_t*>(S.c.k_norms + row * kMaxGroups * cap);
    vc = reinterpret_cast<const uint8_t*>(S.c.v_codes + row * (cap / kTile) * kHeadDim * BV);
    vnp = S.c.v_norms + row * cap;
  };
  const uint64_t row0 = static_cast<uint64_t>(layer) * S.batch * d.n_kv + kvh;  // the layer's first page
  int page_next = 0;  // page number of the next tile to load, read a tile ahead of it
  bool lost = false;  // a page outside the pool: the rows that attend it are not numbers
  const auto read_page = [&](int t) {
    if constexpr (kPaged) page_next = paged::page_ahead(mode.b, seq, t, S.capacity);
  };
  if constexpr (!kPaged) rows_of((static_cast<size_t>(layer) * S.batch + seq) * d.n_kv + kvh);

  float m_run = kNegInf, l_run = 0.f;
  int v_top = 0, v_acc = 0;  // see radius_top: of the tiles decoded so far, and of those in o
  float16_t o[4];
#pragma unroll
  for (int cc = 0; cc < 4; ++cc)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[cc][i] = 0.f;

  // Raw words of one tile: straight from memory to the registers of the lane
  // that decodes them (see k_prefill_attn).
  const int quarter = wave >> 1;
  const auto opaque_tid = [&]() {
    int t = tid;
    asm volatile("" : "+v"(t));
    return t;
  };
  Raw<BV> raw;
  const auto load_raw = [&](int t) {
    const int tt = opaque_tid();
    const uint8_t *ks, *ns, *vs;
    const uint16_t* rs;
    if constexpr (kPaged) {
      const int page = __builtin_amdgcn_readfirstlane(page_next);
      lost |= static_cast<uint32_t>(page) >= static_cast<uint32_t>(S.batch);
      const int ta = t % S.capacity;  // the tile's place in its page
      // (all rows of a cache numbered in turn: few multiplications)
      const uint64_t x = (row0 + static_cast<uint64_t>(lost ? 0u : static_cast<uint32_t>(page)) * static_cast<uint32_t>(d.n_kv)) *
                             static_cast<uint32_t>(S.capacity) + static_cast<uint32_t>(ta);
      ks = reinterpret_cast<const uint8_t*>(S.c.k_codes) + x * static_cast<uint32_t>(kw) * 4;
      ns = reinterpret_cast<const uint8_t*>(S.c.k_norms) + x * (kMaxGroups * 2) -
           static_cast<uint64_t>(static_cast<uint32_t>(ta)) * static_cast<uint32_t>((kMaxGroups - nslot) * 2);
      vs = reinterpret_cast<const uint8_t*>(S.c.v_codes) + x * (kHeadDim / kTile * BV * 4);
      rs = S.c.v_norms + x;
    } else {
      ks = kc + static_cast<size_t>(t) * kw * 4;
      ns = kn + static_cast<size_t>(t) * nslot * 2;
      vs = vc + static_cast<size_t>(t / kTile) * kHeadDim * BV * 4;
      rs = vnp + t;
    }
    uint32_t k_at = static_cast<uint32_t>((tt & 63) * kw * 4), n_at = static_cast<uint32_t>((tt & 63) * nslot * 2);
    uint32_t v_lane = static_cast<uint32_t>((tt & 127) * BV * 4), vn_lane = static_cast<uint32_t>((tt & 63) * 2);
#pragma unroll
    for (int j = 0; j < kItemsPer; ++j) {
      raw.k[j].x = ld_at<uint32_t>(ks + items.word[j], k_at);
      raw.k[j].y = ld_at<uint32_t>(ks + items.word[j] + 4, k_at);
    }
    raw.kn.x = ld_at<uint32_t>(ns, n_at);
    raw.kn.y = ld_at<uint32_t>(ns + 4, n_at);
    raw.kn.z = ld_at<uint32_t>(ns + 8, n_at);
    raw.kn.w = ld_at<uint32_t>(ns + 12, n_at);
    constexpr int NW = Raw<BV>::kVW;
    vs += (quarter >> 1) * kHeadDim * BV * 4 + 4 * (BV * (quarter & 1) / 2);
#pragma unroll
    for (int i = 0; i < NW; ++i) raw.v[i] = ld_at<uint32_t>(vs + 4 * i, v_lane);
    raw.vn = ld_at<uint16_t>(rs, vn_lane);
    // what lies behind the last row may be large, infinite or not a number: no radii
    if (t + kKeyTile > t_end) {
      const uint32_t in = t + (tt & 63) < t_end ? ~0u : 0u;
      raw.vn &= in;
      raw.kn = make_uint4(raw.kn.x & in, raw.kn.y & in, raw.kn.z & in, raw.kn.w & in);
    }
  };
  // Key radii come in times a power of two that brings the largest one so far to
  // [2^12, 2^13): their products with centroids (below 5) stay in fp16's range,
  // and the lo parts of those hold 2^-37 of the largest product, whatever the
  // size of the keys.  k_top: the running maximum of the radii's exponent fields,
  // plus one.  A tile's logits are multiplied back by its own power.
  int k_top = 2;
  const auto key_up = [](int top) { return max(-3, min(26, 28 - top)); };
  const auto scaled_keys = [&]() {
    // (a token's 16 bytes reach into the next ones' where the row has fewer than 8 slots)
    typedef uint16_t ushort2_t __attribute__((ext_vector_type(2)));
    const auto fields = [](uint32_t x) {  // exponent fields plus one, 0 for what is not finite
      return __builtin_bit_cast(ushort2_t, ((x & 0x7C007C00u) + 0x04000400u) & 0x7C007C00u);
    };
    const ushort2_t f = __builtin_elementwise_max(
        __builtin_elementwise_max(fields(raw.kn.x), fields(nslot > 2 ? raw.kn.y : 0u)),
        __builtin_elementwise_max(fields(nslot > 4 ? raw.kn.z : 0u), fields(nslot > 6 ? raw.kn.w : 0u)));
    k_top = raise_top(k_top, max(f[0] >> 10, f[1] >> 10));
    const int up = key_up(k_top);
    const auto times = [&](const uint4& x, int n) {
      const _Float16 p = __builtin_bit_cast(_Float16, static_cast<uint16_t>((n + 15) << 10));
      const half2_t pp = {p, p};
      const auto one = [&](uint32_t r) { return __builtin_bit_cast(uint32_t, __builtin_bit_cast(half2_t, r) * pp); };
      return make_uint4(one(x.x), one(x.y), one(x.z), one(x.w));
    };
    uint4 r = times(raw.kn, min(up, 15));
    if (up > 15) r = times(r, up - 15);
    return r;
  };
  const auto decode = [&](uint8_t* dec) {
    const int tt = opaque_tid();
    uint4 va, vb;
    uint2 code[kItemsPer];
    if (items.wide) key_lookups<true>(smem, items, raw.k, code);
    else key_lookups<false>(smem, items, raw.k, code);
    value_lookups<BV>(smem, raw, quarter, va, vb);
    uint8_t* dst = dec + (tt & 63) * (2 * kKStride) + 8 * wave;
    const uint4 radii = scaled_keys();
#pragma unroll
    for (int j = 0; j < kItemsPer; ++j) key_store(dst + 8 * kAttnWaves * j, items, j, radii, code[j]);
    v_top = radius_top(v_top, raw.vn);  // (the same in every wave: each has the tile's 64 radii)
    raw.vn = radius_times(raw.vn, radius_up(v_top));
    store_values<BV>(dec, raw, tt, quarter, va, vb);
  };

  float16_t s[NB];
  const auto products_qk = [&](const uint8_t* dcur) {
    const int tt = opaque_tid();
    const uint8_t* kb = dcur + (32 * blk0 + (tt & 31)) * (2 * kKStride) + ((tt & 32) >> 1);
    half8_t ka[3][2];
    const auto read_keys = [&](int u) {
      const uint8_t* at = kb + u % NB * 32 * 2 * kKStride + 32 * (u / NB);
      ka[u % 3][0] = *reinterpret_cast<const half8_t*>(at + kDecKH);
      ka[u % 3][1] = *reinterpret_cast<const half8_t*>(at + kDecKL);
    };
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[n][i] = 0.f;
    read_keys(0);
    read_keys(1);
#pragma unroll
    for (int u = 0; u < 8 * NB; ++u) {
      if (u + 2 < 8 * NB) read_keys(u + 2);
      __builtin_amdgcn_sched_barrier(0);
      const int n = u % NB, ks = u / NB;
      s[n] = __builtin_amdgcn_mfma_f32_32x32x16_f16(ka[u % 3][0], qh[ks], s[n], 0, 0, 0);
      s[n] = __builtin_amdgcn_mfma_f32_32x32x16_f16(ka[u % 3][1], qh[ks], s[n], 0, 0, 0);
      s[n] = __builtin_amdgcn_mfma_f32_32x32x16_f16(ka[u % 3][0], ql[ks], s[n], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
  };

  // Online softmax (base 2), then O^T += V^T P^T; only a tile that reaches past
  // the end masks anything.
  const auto softmax_pv = [&](const uint8_t* dcur, int t0, int k_cur, int v_cur) {
    const int tt = opaque_tid(), hf4 = (tt & 32) >> 3;  // 4 hf
    if (v_cur != v_acc) {
      if (v_acc > 0) {
        const float down = __uint_as_float(static_cast<uint32_t>(127 + v_acc - v_cur) << 23);
#pragma unroll
        for (int cc = 0; cc < 4; ++cc) o[cc] *= down;
      }
      v_acc = v_cur;
    }
    float st = sc * __uint_as_float(static_cast<uint32_t>(127 - key_up(k_cur)) << 23);
    if constexpr (kMods) {
      const float at = static_cast<float>(sight.pos(rc / G) - t0 - hf4);
#pragma unroll
      for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          s[n][i] = paged::changed(mode.m.cap, slope, s[n][i] * st,
                                       at - static_cast<float>(32 * (blk0 + n) + 8 * (i >> 2) + (i & 3)));
      st = 1.f;
    }
    const bool cut = t0 + 32 * (blk0 + NB) > (kPaged ? lim0 : t_end);  // wave-uniform
    if (cut) {
#pragma unroll
      for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int tok = t0 + 32 * (blk0 + n) + 8 * (i >> 2) + hf4 + (i & 3);
          s[n][i] = tok >= (kPaged ? lim : t_end) ? kNegInf : s[n][i];
        }
    }
    uint2 vr[4];
    const auto read_radii = [&](int n) {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        vr[q] = *reinterpret_cast<const uint2*>(dcur + kDecVN + 2 * (32 * (blk0 + n) + 8 * q + hf4));
        // (a radius that the row does not see may be infinite or not a number)
        if (kPaged && cut) vr[q] = paged::seen(vr[q], lim - (t0 + 32 * (blk0 + n) + 8 * q + hf4));
      }
    };
    float mp[4];
#pragma unroll
    for (int c4 = 0; c4 < 4; ++c4) {
      mp[c4] = fmaxf(s[0][4 * c4], s[0][4 * c4 + 1]);
      mp[c4] = fmaxf(fmaxf(mp[c4], s[0][4 * c4 + 2]), s[0][4 * c4 + 3]);
      if constexpr (NB == 2) {
        mp[c4] = fmaxf(fmaxf(mp[c4], s[1][4 * c4]), s[1][4 * c4 + 1]);
        mp[c4] = fmaxf(fmaxf(mp[c4], s[1][4 * c4 + 2]), s[1][4 * c4 + 3]);
      }
    }
    const float mx = fmaxf(fmaxf(mp[0], mp[1]), fmaxf(mp[2], mp[3])) * st;
    if (__builtin_amdgcn_ballot_w64(mx > m_run) != 0) {
      const float mn = fmaxf(m_run, max2g(mx));
      const float corr = m_run == kNegInf ? 0.f : __builtin_amdgcn_exp2f(m_run - mn);
      m_run = mn;
      l_run *= corr;
#pragma unroll
      for (int cc = 0; cc < 4; ++cc) o[cc] *= corr;
    }
    const float mref = m_run == kNegInf ? 0.f : m_run;
    float ps = 0.f;
    half8_t pb[NB][2], pe[EX ? NB : 1][2];
    const auto weights = [&](int n) {
      uint32_t pw[8], pl[8];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        float p[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) p[i] = __builtin_amdgcn_exp2f(fmaf(s[n][4 * q + i], st, -mref));
        ps += (p[0] + p[1]) + (p[2] + p[3]);
        pw[2 * q] = mix_pair(p[0], p[1], vr[q].x);
        pw[2 * q + 1] = mix_pair(p[2], p[3], vr[q].y);
        if constexpr (EX) {
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const half2_t h = __builtin_bit_cast(half2_t, pw[2 * q + k]);
            const half2_t w = __builtin_bit_cast(half2_t, k ? vr[q].y : vr[q].x);
            const half2_t x = {
                static_cast<_Float16>(fmaf(p[2 * k], static_cast<float>(w[0]), -static_cast<float>(h[0]))),
                static_cast<_Float16>(fmaf(p[2 * k + 1], static_cast<float>(w[1]), -static_cast<float>(h[1])))};
            pl[2 * q + k] = __builtin_bit_cast(uint32_t, x);
          }
        }
      }
      pb[n][0] = __builtin_bit_cast(half8_t, make_uint4(pw[0], pw[1], pw[2], pw[3]));
      pb[n][1] = __builtin_bit_cast(half8_t, make_uint4(pw[4], pw[5], pw[6], pw[7]));
      if constexpr (EX) {
        pe[n][0] = __builtin_bit_cast(half8_t, make_uint4(pl[0], pl[1], pl[2], pl[3]));
        pe[n][1] = __builtin_bit_cast(half8_t, make_uint4(pl[4], pl[5], pl[6], pl[7]));
      }
    };
    const uint8_t* vb = dcur + kDecV + (tt & 31) * (2 * kVStride) + 64 * blk0 + 4 * hf4;
    half8_t va[2][4];
    const auto read_values = [&](int st16) {
#pragma unroll
      for (int cc = 0; cc < 4; ++cc)
        va[st16 & 1][cc] = *reinterpret_cast<const half8_t*>(vb + 32 * cc * (2 * kVStride) + 32 * st16);
    };
    read_radii(0);
    read_values(0);
    __builtin_amdgcn_sched_barrier(0);
    weights(0);
#pragma unroll
    for (int st16 = 0; st16 < 2 * NB; ++st16) {
      if (NB == 2 && st16 == 0) read_radii(1);
      if (st16 + 1 < 2 * NB) read_values(st16 + 1);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int cc = 0; cc < 4; ++cc)
        o[cc] = __builtin_amdgcn_mfma_f32_32x32x16_f16(va[st16 & 1][cc], pb[st16 >> 1][st16 & 1], o[cc], 0, 0, 0);
      if constexpr (EX) {
#pragma unroll
        for (int cc = 0; cc < 4; ++cc)
          o[cc] = __builtin_amdgcn_mfma_f32_32x32x16_f16(va[st16 & 1][cc], pe[st16 >> 1][st16 & 1], o[cc], 0, 0, 0);
      }
      if (NB == 2 && st16 == 0) weights(1);
      __builtin_amdgcn_sched_barrier(0);
    }
    l_run += ps;
  };

  // Pipeline as in k_prefill_attn: tile kt's products beside the decode of tile
  // kt + 1, waves 0-3 decoding before and waves 4-7 after them, one barrier a
  // tile.  (A split without a tile loads and decodes its first one for nobody.)
  const auto tile_start = [&](int kt) { return t_begin + min(kt, max(n_kt - 1, 0)) * kKeyTile; };
  read_page(t_begin);
  load_raw(t_begin);
  read_page(tile_start(1));
  __syncthreads();
  decode(smem + kOffDec);
  load_raw(tile_start(1));
  read_page(tile_start(2));
  __syncthreads();
  if (wave >= 4) __builtin_amdgcn_s_setprio(2);
  for (int kt = 0; kt < n_kt; ++kt) {
    const uint8_t* const dcur = smem + kOffDec + (kt & 1) * kDecBytes;
    uint8_t* const dnxt = smem + kOffDec + (~kt & 1) * kDecBytes;
    const int k_cur = k_top, v_cur = v_top;
    if (wave < 4) {
      decode(dnxt);
      load_raw(tile_start(kt + 2));
      read_page(tile_start(kt + 3));
    }
    products_qk(dcur);
    softmax_pv(dcur, t_begin + kt * kKeyTile, k_cur, v_cur);
    if (wave >= 4) {
      decode(dnxt);
      load_raw(tile_start(kt + 2));
      read_page(tile_start(kt + 3));
    }
    __syncthreads();
  }

  // ---- KS = 2: waves 4-7 hand their states over to waves 0-3
  l_run = sum2g(l_run);
  if constexpr (KS == 2) {
    float* mg = reinterpret_cast<float*>(smem) + (wave & 3) * 66 * 64 + lane;
    if (wave >= 4) {
      mg[0] = m_run;
      mg[64] = l_run;
#pragma unroll
      for (int cc = 0; cc < 4; ++cc)
#pragma unroll
        for (int i = 0; i < 16; ++i) mg[64 * (2 + 16 * cc + i)] = o[cc][i];
    }
    __syncthreads();
    if (wave < 4) {
      const float m2 = mg[0], l2 = mg[64], mn = fmaxf(m_run, m2);
      const float e1 = m_run == kNegInf ? 0.f : __builtin_amdgcn_exp2f(m_run - mn);
      const float e2 = m2 == kNegInf ? 0.f : __builtin_amdgcn_exp2f(m2 - mn);
      m_run = mn;
      l_run = l_run * e1 + l2 * e2;
#pragma unroll
      for (int cc = 0; cc < 4; ++cc)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[cc][i] = o[cc][i] * e1 + mg[64 * (2 + 16 * cc + i)] * e2;
    }
    __syncthreads();
  }
  if (!ok || (kPaged && lost)) l_run = __builtin_nanf("");
  const bool mine = r < nr && (KS == 1 || wave < 4);
  const float v_back = __uint_as_float(static_cast<uint32_t>(127 - radius_up(v_acc)) << 23);

  if (call.n_slots > 1) {
    if (!mine) return;
    float* P = part_of();
    if (hf == 0) {
      // (no row seen, or logits that are all not a number: see k_cross)
      P[0] = l_run == 0.f ? kNegInf : m_run == kNegInf ? 0.f : m_run;
      P[1] = l_run;
    }
#pragma unroll
    for (int cc = 0; cc < 4; ++cc)
#pragma unroll
      for (int u = 0; u < 4; ++u)
        *reinterpret_cast<float4_t*>(P + 4 + 32 * cc + 8 * u + 4 * hf) =
            float4_t{o[cc][4 * u], o[cc][4 * u + 1], o[cc][4 * u + 2], o[cc][4 * u + 3]} * v_back;
    return;
  }

  // ---- the only partial: out = Pi_V^T (o / l).  A row's o / l, scaled as the
  // query rows were, is the B operand of three fp16 products as it lies in the
  // accumulators (k runs over dims 16 st + {4 hf + i, 8 + 4 hf + i} of block
  // cc); A = Pi_V^T in that order, hi and lo parts.
  {
    const float* rot = reinterpret_cast<const float*>(blob + kOffRotVT);
    for (int it = tid; it < 4 * 8 * 64; it += kAttnThreads) {
      const int l = it & 63, st = (it >> 6) & 7, c2 = it >> 9;
      const float* src = rot + (32 * c2 + (l & 31)) * kHeadDim + 16 * st + 4 * (l >> 5);
      const float4_t a = *reinterpret_cast<const float4_t*>(src) * 256.f, b = *reinterpret_cast<const float4_t*>(src + 8) * 256.f;
      half8_t hi, lo;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float x = e < 4 ? a[e & 3] : b[e & 3];
        hi[e] = static_cast<_Float16>(x);
        lo[e] = static_cast<_Float16>(x - static_cast<float>(hi[e]));
      }
      *reinterpret_cast<half8_t*>(smem + it * 16) = hi;
      *reinterpret_cast<half8_t*>(smem + kRotPart + it * 16) = lo;
    }
  }
  __syncthreads();
  if (KS == 2 && wave >= 4) return;
  float mx = 0.f;
#pragma unroll
  for (int cc = 0; cc < 4; ++cc)
#pragma unroll
    for (int i = 0; i < 16; ++i) mx = fmaxf(mx, fabsf(o[cc][i]));
  float to, back;
  scale_of(max2g(mx), to, back);
  // (not a number in l: every output is)
  const float scale = l_run == 0.f ? 0.f : back * (v_back * (kRsqrtD / 256.f)) / l_run;
  half8_t oh[8], ol[8];
#pragma unroll
  for (int st = 0; st < 8; ++st)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float x = o[st >> 1][8 * (st & 1) + e] * to;
      const _Float16 h = static_cast<_Float16>(x);
      oh[st][e] = h;
      ol[st][e] = static_cast<_Float16>(x - static_cast<float>(h));
    }
#pragma unroll 1
  for (int c2 = 0; c2 < 4; ++c2) {
    float16_t y;
#pragma unroll
    for (int i = 0; i < 16; ++i) y[i] = 0.f;
#pragma unroll
    for (int st = 0; st < 8; ++st) {
      const half8_t ah = *reinterpret_cast<const half8_t*>(smem + ((c2 * 8 + st) * 64 + lane) * 16);
      const half8_t al = *reinterpret_cast<const half8_t*>(smem + kRotPart + ((c2 * 8 + st) * 64 + lane) * 16);
      y = __builtin_amdgcn_mfma_f32_32x32x16_f16(ah, oh[st], y, 0, 0, 0);
      y = __builtin_amdgcn_mfma_f32_32x32x16_f16(al, oh[st], y, 0, 0, 0);
      y = __builtin_amdgcn_mfma_f32_32x32x16_f16(ah, ol[st], y, 0, 0, 0);
    }
    if (mine) {
#pragma unroll
      for (int u = 0; u < 4; ++u)
        store4(call.out, row_at * kHeadDim + 32 * c2 + 8 * u + 4 * hf,
               float4_t{y[4 * u], y[4 * u + 1], y[4 * u + 2], y[4 * u + 3]} * scale, call.out_dtype);
    }
  }
}

template <int BV, bool EX, class MODE>
hipError_t launch_tile_bv(const Dims& d, const uint8_t* blob, const float* qr, const CrossCall& call, bool half,
                          const MODE& mode, hipStream_t s) {
  const auto go = [&](auto kern) {
    hipLaunchKernelGGL(kern, dim3(call.side[0].items), dim3(kAttnThreads), 0, s, d, blob, qr, call, mode);
    return hipGetLastError();
  };
  return half ? go(k_cross_tile<BV, 2, EX, MODE>) : go(k_cross_tile<BV, 1, EX, MODE>);
}
template <bool EX, class MODE>
hipError_t launch_tile(const Dims& d, const void* layout, const float* qr, const CrossCall& call, bool half,
                       const MODE& mode, hipStream_t s) {
  const uint8_t* blob = static_cast<const uint8_t*>(layout);
  switch (d.v_bits) {
    case 1: return launch_tile_bv<1, EX>(d, blob, qr, call, half, mode, s);
    case 2: return launch_tile_bv<2, EX>(d, blob, qr, call, half, mode, s);
    case 3: return launch_tile_bv<3, EX>(d, blob, qr, call, half, mode, s);
    case 4: return launch_tile_bv<4, EX>(d, blob, qr, call, half, mode, s);
    case 5: return launch_tile_bv<5, EX>(d, blob, qr, call, half, mode, s);
    case 6: return launch_tile_bv<6, EX>(d, blob, qr, call, half, mode, s);
    case 7: return launch_tile_bv<7, EX>(d, blob, qr, call, half, mode, s);
    default: return launch_tile_bv<8, EX>(d, blob, qr, call, half, mode, s);
  }
}

}  // namespace cross_tile_detail
}  // namespace bgtq
