// Packed K/V tiles decoded into LDS for many query rows: what the causal
// prefill attention (prefill.hip) and the wide attention passes
// (cross_tile.h) share.
#pragma once
#include <hip/hip_runtime.h>

#include "kernels.h"
#include "layout.h"
#include "mix.h"

namespace bgtq {
namespace prefill_detail {

typedef _Float16 half8_t __attribute__((ext_vector_type(8)));
typedef float float4_t __attribute__((ext_vector_type(4)));

typedef float float16_t __attribute__((ext_vector_type(16)));
typedef _Float16 half2_t __attribute__((ext_vector_type(2)));

constexpr int kAttnWaves = 8;      // attention kernel: 8 waves (2 per SIMD)
constexpr int kAttnThreads = kAttnWaves * 64;
constexpr int kWaveRows = 32;      // query rows (position x head) of a wave: one 32x32 column block
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kNegInf = -__builtin_huge_valf();
// ---- LDS map of the attention kernel (bytes)
constexpr int kKStride = 136;  // halves per decoded key row (128 + 8 pad)
constexpr int kVStride = 72;   // halves per decoded value row (64 + 8 pad: 16-byte aligned, conflict-free reads)
// decoded tile (two buffers): keys hi, lo [64 tokens][kKStride] fp16, values
// [128 dims][kVStride] fp16, value radii [64] fp16
constexpr int kDecKH = 0;
constexpr int kDecKL = kDecKH + 64 * kKStride * 2;
constexpr int kDecV = kDecKL + 64 * kKStride * 2;
constexpr int kDecVN = kDecV + 128 * kVStride * 2;
constexpr int kDecBytes = kDecVN + 64 * 2;
constexpr int kOffCb = 0;                        // fp16 codebooks
constexpr int kOffPair = kOffCb + 1024;          // pair tables of the widths 1 .. kMaxPair
constexpr int kMaxPair = 6;
// byte offset of the pair table of width b: 4^b entries of two fp16 centroids
__host__ __device__ constexpr int pair_offset(int b) { return 4 * (((1 << (2 * b)) - 4) / 3); }
// (the tables lie below 64 KB: their offsets fit the immediate of an LDS read)
constexpr int kOffDec = (kOffPair + pair_offset(kMaxPair + 1) + 15) / 16 * 16;
constexpr int kTileLds = kOffDec + 2 * kDecBytes;
constexpr int kRotVLds = kHeadDim * kHeadDim * 4;  // Pi_V staged for the epilogue
constexpr int kMergeLds = (kAttnWaves / 2) * 64 * 66 * 4;  // states of the waves that hand theirs over (KS = 2)
constexpr int kLdsBytes = kTileLds > kRotVLds ? (kTileLds > kMergeLds ? kTileLds : kMergeLds)
                                              : (kRotVLds > kMergeLds ? kRotVLds : kMergeLds);
static_assert(kLdsBytes <= 160 * 1024, "LDS of one workgroup");
static_assert(kDecBytes % 16 == 0 && kDecV % 16 == 0 && kOffDec % 16 == 0, "aligned buffers");
static_assert(2 * kCodebookEntries <= 1024, "codebook staging");

// Load of a T at a 32-bit byte offset from a wave-uniform base (the global
// load form with a scalar base and a 32-bit vector offset).
template <class T>
__device__ __forceinline__ T ld_at(const void* base, uint32_t byte_off) {
  return *reinterpret_cast<const T*>(static_cast<const char*>(base) + byte_off);
}

// r0, r1 = the values of lanes l % 32 and l % 32 + 32 (the two lanes that hold
// the same query row of an accumulator); gfx950 lane swap
__device__ __forceinline__ void swap32(float v, float& r0, float& r1) {
  unsigned x = __builtin_bit_cast(unsigned, v), y = x;
  asm volatile("s_nop 1\n\tv_permlane32_swap_b32 %0, %1\n\ts_nop 1" : "+v"(x), "+v"(y));
  r0 = __builtin_bit_cast(float, x);
  r1 = __builtin_bit_cast(float, y);
}
__device__ __forceinline__ float max2g(float v) {
  float a, b;
  swap32(v, a, b);
  return fmaxf(a, b);
}
__device__ __forceinline__ float sum2g(float v) {
  float a, b;
  swap32(v, a, b);
  return a + b;
}


// Lane roles in the products (32x32x16 f16 MFMAs; l32 = lane % 32, hf =
// lane / 32): the A operand comes from the decoded tile (token or dim l32 of
// a 32-block, 8 consecutive k from 8 hf), the B operand is the wave's 32 query
// rows (row l32, the same k), and an accumulator's register r holds token
// (S^T) or dim (O^T) 8 (r / 4) + 4 hf + r % 4 of its 32-block for row l32.
// The softmax weights of a lane are therefore, 8 registers at a time, a B
// operand of O^T = V^T P^T whose k runs over tokens {4 hf + i, 8 + 4 hf + i}
// of a 16-token step; the value tile stores the tokens of a step in that
// order (0-3, 8-11, 4-7, 12-15), so that its operand is one 16-byte read.

// Bits [POS, POS + LEN) of the little-endian word array w, placed at bit SH.
template <int POS, int LEN, int SH, int N>
__device__ __forceinline__ uint32_t field_at(const uint32_t (&w)[N]) {
  constexpr int wi = POS / 32, sh = POS % 32;
  static_assert(wi < N && SH + LEN <= 32, "field");
  uint32_t v;
  if constexpr (sh + LEN > 32) {
    static_assert(wi + 1 < N && sh >= SH, "field word");
    v = __builtin_amdgcn_alignbit(w[wi + 1], w[wi], sh - SH);
  } else if constexpr (sh >= SH) {
    v = w[wi] >> (sh - SH);
  } else {
    v = w[wi] << (SH - sh);
  }
  return v & (((1u << LEN) - 1u) << SH);
}

// Two consecutive BV-bit codes at bit POS of w -> two fp16 centroids.
template <int BV, int POS, int N>
__device__ __forceinline__ uint32_t value_pair(const uint8_t* smem, const uint32_t (&w)[N]) {
  if constexpr (BV <= kMaxPair) {
    return *reinterpret_cast<const uint32_t*>(smem + kOffPair + pair_offset(BV) + field_at<POS, 2 * BV, 2>(w));
  } else {
    const uint32_t c0 = *reinterpret_cast<const uint16_t*>(smem + kOffCb + 2 * cb_index(BV) + field_at<POS, BV, 1>(w));
    const uint32_t c1 =
        *reinterpret_cast<const uint16_t*>(smem + kOffCb + 2 * cb_index(BV) + field_at<POS + BV, BV, 1>(w));
    return c0 | (c1 << 16);
  }
}

// Key decode.  A key row is 32 items of 4 consecutive stream positions: two
// pairs, each inside one group (groups have even sizes), whose codes are one
// dense field of 2 bA + 2 bB <= 32 bits.  Lane = token; a wave decodes the
// items wave + 8 j, so that everything that describes an item is
// wave-uniform, and stores 8 bytes per item and token.
constexpr int kItemsPer = kHeadDim / 4 / kAttnWaves;
struct KeyItems {
  uint32_t word[kItemsPer];                     // byte offset of the first of the two words that are loaded
  uint32_t sh[kItemsPer];                       // first bit of the field in them
  uint32_t wa[kItemsPer], wb[kItemsPer];        // 2 bA, 2 bB
  uint32_t ta[kItemsPer], tb[kItemsPer];        // offsets of the widths' pair tables
  uint32_t sel_lo[kItemsPer], sel_hi[kItemsPer];  // byte selectors that pick (rA, rB) from the token's 8 radii:
                                                // groups 0-3 and 4-7, a radius in the other half selects zero
  bool wide;                                    // some width is above kMaxPair: codes looked up one by one
};
// Raw words of a thread's share of one tile.
template <int BV>
struct Raw {
  static constexpr int kVW = (BV + 1) / 2;  // words of 16 value codes
  uint2 k[kItemsPer];
  uint4 kn;
  uint32_t v[kVW];
  uint32_t vn;
};
__device__ __forceinline__ KeyItems key_items(const RowMeta* M, int wave, int kw) {
  KeyItems k;
  k.wide = false;
#pragma unroll
  for (int j = 0; j < kItemsPer; ++j) {
    const int p = 4 * (wave + kAttnWaves * j);
    const auto uni = [](uint32_t v) { return static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(v))); };
    const uint32_t off = uni(M->bitoff[p]), ba = uni(M->width[p]), bb = uni(M->width[p + 2]), ga = uni(M->grp[p]),
                   gb = uni(M->grp[p + 2]);
    const uint32_t w0 = min(off >> 5, static_cast<uint32_t>(kw - 2));  // (a row has at least 4 words)
    const auto tab = [](uint32_t b) { return static_cast<uint32_t>(kOffPair) + 4 * (((1u << (2 * b)) - 4u) / 3u); };
    const auto sel = [](uint32_t g) { return 2 * (g & 3u) | (2 * (g & 3u) + 1) << 8; };
    k.word[j] = 4 * w0;
    k.sh[j] = off - 32 * w0;
    k.wa[j] = 2 * ba;
    k.wb[j] = 2 * bb;
    k.ta[j] = tab(ba);
    k.tb[j] = tab(bb);
    k.sel_lo[j] = (ga < 4 ? sel(ga) : 0x0C0Cu) | (gb < 4 ? sel(gb) : 0x0C0Cu) << 16;
    k.sel_hi[j] = (ga < 4 ? 0x0C0Cu : sel(ga)) | (gb < 4 ? 0x0C0Cu : sel(gb)) << 16;
    k.wide = k.wide || ba > kMaxPair || bb > kMaxPair;
  }
  return k;
}
// The centroids of the wave's items (c.x: pair A, c.y: pair B).
template <bool WIDE>
__device__ __forceinline__ void key_lookups(const uint8_t* smem, const KeyItems& it, const uint2 (&w)[kItemsPer],
                                            uint2 (&c)[kItemsPer]) {
#pragma unroll
  for (int j = 0; j < kItemsPer; ++j) {
    const uint32_t f = static_cast<uint32_t>((static_cast<uint64_t>(w[j].y) << 32 | w[j].x) >> it.sh[j]);
    if constexpr (!WIDE) {
      c[j].x = *reinterpret_cast<const uint32_t*>(smem + it.ta[j] + 4 * __builtin_amdgcn_ubfe(f, 0, it.wa[j]));
      c[j].y = *reinterpret_cast<const uint32_t*>(smem + it.tb[j] + 4 * __builtin_amdgcn_ubfe(f, it.wa[j], it.wb[j]));
    } else {
      const uint32_t ba = it.wa[j] >> 1, bb = it.wb[j] >> 1;
      const auto one = [&](uint32_t at, uint32_t b) {
        return static_cast<uint32_t>(*reinterpret_cast<const uint16_t*>(
            smem + kOffCb + 2 * ((1u << b) - 2u + __builtin_amdgcn_ubfe(f, at, b))));
      };
      c[j].x = one(0, ba) | one(ba, ba) << 16;
      c[j].y = one(2 * ba, bb) | one(2 * ba + bb, bb) << 16;
    }
  }
}
// Item j: centroids times the groups' radii, as fp16 hi and lo parts.  The
// product of two fp16 numbers has at most 22 significant bits: hi =
// fp16(r c) and the fused residual lo = fp16(r c - hi) carry all of them above
// fp16's subnormal step.  dst: the item's place in the token's decoded row.
__device__ __forceinline__ void key_store(uint8_t* dst, const KeyItems& it, int j, const uint4& radii, const uint2& c) {
  const uint32_t r =
      __builtin_amdgcn_perm(radii.y, radii.x, it.sel_lo[j]) | __builtin_amdgcn_perm(radii.w, radii.z, it.sel_hi[j]);
  const half2_t rr = __builtin_bit_cast(half2_t, r);
  const half2_t ra = {rr[0], rr[0]}, rb = {rr[1], rr[1]};
  const half2_t ca = __builtin_bit_cast(half2_t, c.x), cb = __builtin_bit_cast(half2_t, c.y);
  const half2_t ha = ra * ca, hb = rb * cb;
  const half2_t la = __builtin_elementwise_fma(ra, ca, -ha), lb = __builtin_elementwise_fma(rb, cb, -hb);
  *reinterpret_cast<uint2*>(dst + kDecKH) =
      make_uint2(__builtin_bit_cast(uint32_t, ha), __builtin_bit_cast(uint32_t, hb));
  *reinterpret_cast<uint2*>(dst + kDecKL) =
      make_uint2(__builtin_bit_cast(uint32_t, la), __builtin_bit_cast(uint32_t, lb));
}

// Value decode: thread = (dim tid % 128, 16-token step tid / 128); a holds
// tokens 0-3 and 8-11 of the step, b tokens 4-7 and 12-15.
template <int BV>
__device__ __forceinline__ void value_lookups(const uint8_t* smem, const Raw<BV>& raw, int quarter, uint4& a, uint4& b) {
  constexpr int NW = Raw<BV>::kVW;
  uint32_t w[NW];
  if constexpr (BV % 2 == 0) {
#pragma unroll
    for (int i = 0; i < NW; ++i) w[i] = raw.v[i];
  } else {
    const int sh = 16 * (quarter & 1);  // uniform
#pragma unroll
    for (int i = 0; i < NW; ++i) w[i] = __builtin_amdgcn_alignbit(i + 1 < NW ? raw.v[i + 1] : 0u, raw.v[i], sh);
  }
  a.x = value_pair<BV, 0 * BV>(smem, w);
  a.y = value_pair<BV, 2 * BV>(smem, w);
  b.x = value_pair<BV, 4 * BV>(smem, w);
  b.y = value_pair<BV, 6 * BV>(smem, w);
  a.z = value_pair<BV, 8 * BV>(smem, w);
  a.w = value_pair<BV, 10 * BV>(smem, w);
  b.z = value_pair<BV, 12 * BV>(smem, w);
  b.w = value_pair<BV, 14 * BV>(smem, w);
}
template <int BV>
__device__ __forceinline__ void store_values(uint8_t* dec, const Raw<BV>& raw, int tid, int quarter, const uint4& a,
                                             const uint4& b) {
  uint4* dst = reinterpret_cast<uint4*>(dec + kDecV + (tid & 127) * (2 * kVStride) + 32 * quarter);
  dst[0] = a;
  dst[1] = b;
  // every wave stores the 64 value radii it loaded (the same ones; no branch)
  reinterpret_cast<uint16_t*>(dec + kDecVN)[tid & 63] = static_cast<uint16_t>(raw.vn);
}

}  // namespace prefill_detail
}  // namespace bgtq
