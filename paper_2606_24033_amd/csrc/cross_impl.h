// Attention of up to 32 query rows of one (layer, sequence, KV head) to a range
// of packed rows that all of them see (cross.hip has the passes it serves).
//
// Work mapping.  A workgroup of 8 waves (two per SIMD; its lookup tables fill
// the LDS) = one (unit, block of 32 query rows, split of the key axis).  A wave
// owns 64-row tiles and decodes their codes straight into the operands of
// 32x32x16 f16 MFMAs: the decode of a tile costs a wave the same whether 4 or
// 32 query rows use it, nothing decoded passes through LDS and the waves meet
// only at the end.
//  * QK, S^T = K Q^T: lane = token decodes 16 coordinates of one group (a code
//    width is uniform in the wave); v_permlane32_swap exchanges the halves, so
//    that the registers of all 64 tokens become the A operands of two 32-token
//    blocks.  B = the query rows from an image in LDS (fp16 hi and lo parts,
//    groups padded to 16 coordinates with zeros).  The operands are the bare
//    centroids (exact in fp16); a group's products are scaled by its radii as
//    they are added to S, in fp32.
//  * The accumulator's layout (lane = query row, registers = tokens 8 (i / 4) +
//    4 hf + i % 4, hf = lane / 32) makes the softmax weights the B operand of
//    O^T = V^T P^T as they are.  Its k runs over the tokens {4 hf + i, 8 + 4 hf
//    + i} of a 16-token step, and a lane (dim, hf) decodes just those from the
//    value tile, where the codes of a dim lie one after the other.
//
// What bounds it.  A small call is one chain of latencies, 16 us (38K cycles)
// for a workgroup with a tile per wave: 15K of set-up (arguments, tables, the
// query rotation), 9K the tile (5.3K QK, 0.8K the maximum, 1.9K PV: lookups that
// wait on LDS with two waves a SIMD), 8K for joining the waves, the output
// rotation and the store.  A long pass takes 5.4 to 6.2 us for every tile of
// each wave, 13 where key rows have more than 16 words (they and some 60 other
// registers lie in scratch memory).  32 query rows are one column block of the product; a second
// block's accumulators and operands do not fit the 256 registers of two waves
// a SIMD, and one wave a SIMD waits on each lookup.  Measured in a call: 8
// sequences x 8 KV heads x 4 query rows on 150 to 1500 rows 21 us; 64 query rows
// of 32 layers x 8 heads on 4001 rows and 4 each on 20 to 300 rows 189 us, 743
// GB/s and 185 TFLOP/s of what the definition asks for.
#pragma once
#include <hip/hip_runtime.h>

#include "decode_impl.h"
#include "kernels.h"
#include "layout.h"
#include "mix.h"
#include "paged_pass.h"

namespace bgtq {
namespace cross_detail {

using split_detail::decode4;
using split_detail::half4_t;
using split_detail::LaneRep;
using split_detail::ld_at;
using split_detail::swap32;
typedef _Float16 half8_t __attribute__((ext_vector_type(8)));
typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
typedef float float4_t __attribute__((ext_vector_type(4)));
typedef float float16_t __attribute__((ext_vector_type(16)));

constexpr int kWaves = 8, kThreads = kWaves * 64;
constexpr int kRows = 32;      // query rows of a workgroup
constexpr int kMaxSteps = 15;  // 16-coordinate steps of a key row: at most (128 + 8 * 14) / 16
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kNegInf = -__builtin_huge_valf();
constexpr float kRsqrtD = 0.08838834764831845f;  // 1 / sqrt(128)

// ---- LDS map (bytes).  The lookup tables keep the decode kernel's places
// (split_detail::kLut*), then
constexpr int kImg = split_detail::kQimg;                // query image [step][hi, lo][lane] x 16 B
constexpr int kRad = kImg + kMaxSteps * 2048;            // per wave: radii [8 groups, values][64 tokens] fp16
constexpr int kRadBytes = 9 * 64 * 2;
constexpr int kBooks = kRad + kWaves * kRadBytes;        // fp16 codebooks
constexpr int kTop = kBooks + 1024;                      // per query row: largest rotated magnitude, as bits,
constexpr int kBack = kTop + kRows * 4;                  // and what its staged copy is to be multiplied with
constexpr int kLds = kBack + kRows * 4;
// rows staged as fp16 hi and lo parts, [part][row][128 + 8 pad]: the query rows
// in the image's place before the rotation, the result rows at 0 after the loop
constexpr int kHalfStride = (kHeadDim + 8) * 2;
constexpr int kHalfPart = kRows * kHalfStride;
static_assert(2 * kHalfPart <= kMaxSteps * 2048, "staged queries in the image's place");
static_assert(kLds <= 160 * 1024, "LDS of one workgroup");
// at the end: [wave][row] accumulators, then maxima and sums
constexpr int kAccStride = kHeadDim + 4;
constexpr int kEndM = kWaves * kRows * kAccStride * 4;
constexpr int kEndTiles = kEndM + 2 * kWaves * kRows * 4;  // per wave: tiles of its sequence, -1 for a refused length
constexpr int kEndBack = kEndTiles + kWaves * 4;           // per wave: what undoes the scale of its value radii
static_assert(kEndBack + kWaves * 4 <= kLds, "merge area");

__device__ __forceinline__ void store4(void* out, size_t i, const float4_t& y, int dtype) {  // BGTQ_BF16 = 1
  if (dtype == 1) {
    typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
    *reinterpret_cast<bf16x4_t*>(static_cast<uint16_t*>(out) + i) = __builtin_convertvector(y, bf16x4_t);
  } else {
    *reinterpret_cast<float4_t*>(static_cast<float*>(out) + i) = y;
  }
}

// x, y = 4 registers each: exchanges the upper half-wave of x with the lower
// one of y (s_nop: the wait states around a lane swap and before an MFMA).
__device__ __forceinline__ void swap_halves(uint2& x0, uint2& x1, uint2& y0, uint2& y1) {
  asm("s_nop 1\n\t"
      "v_permlane32_swap_b32 %0, %4\n\t"
      "v_permlane32_swap_b32 %1, %5\n\t"
      "v_permlane32_swap_b32 %2, %6\n\t"
      "v_permlane32_swap_b32 %3, %7\n\t"
      "s_nop 1"
      : "+v"(x0.x), "+v"(x0.y), "+v"(x1.x), "+v"(x1.y), "+v"(y0.x), "+v"(y0.y), "+v"(y1.x), "+v"(y1.y));
}

// x = the lower half-wave's value, y = the upper one's, in both.
__device__ __forceinline__ void spread_halves(uint32_t (&x)[4], uint32_t (&y)[4]) {
  asm("v_mov_b32 %4, %0\n\tv_mov_b32 %5, %1\n\tv_mov_b32 %6, %2\n\tv_mov_b32 %7, %3\n\t"
      "s_nop 1\n\t"
      "v_permlane32_swap_b32 %0, %4\n\t"
      "v_permlane32_swap_b32 %1, %5\n\t"
      "v_permlane32_swap_b32 %2, %6\n\t"
      "v_permlane32_swap_b32 %3, %7\n\t"
      "s_nop 1"
      : "+v"(x[0]), "+v"(x[1]), "+v"(x[2]), "+v"(x[3]), "=&v"(y[0]), "=&v"(y[1]), "=&v"(y[2]), "=&v"(y[3]));
}

// The power of two 2^up that brings a magnitude (as bits, sign cleared) to
// [2^13, 2^14), and its inverse; 1 for zeros and what is not finite.
__device__ __forceinline__ int up_of(uint32_t bits) {  // biased
  const int e = static_cast<int>(bits >> 23);
  return e == 0 || e == 255 ? 127 : max(1, min(253, 127 + 13 + 127 - e));
}
__device__ __forceinline__ float two_to(int biased) { return __uint_as_float(static_cast<uint32_t>(biased) << 23); }

// fp16 parts of 8 floats
__device__ __forceinline__ void split8(const float (&x)[8], half8_t& hi, half8_t& lo) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    hi[j] = static_cast<_Float16>(x[j]);
    lo[j] = static_cast<_Float16>(x[j] - static_cast<float>(hi[j]));
  }
}

// largest magnitude (as bits: infinities and not-a-numbers rank above every
// number) over the 16 lanes of a row of threads
__device__ __forceinline__ uint32_t top16(const float (&x)[8]) {
  uint32_t mx = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) mx = max(mx, __float_as_uint(x[j]) & 0x7FFFFFFFu);
#pragma unroll
  for (int k = 1; k < 16; k *= 2) mx = max(mx, static_cast<uint32_t>(__shfl_xor(static_cast<int>(mx), k)));
  return mx;
}

// A 16 x 128 block of a matrix (the lane's operands: row lane % 16, columns 32
// (lane / 16) .. + 31 in m, times 2^8) times 16 NC staged rows, three fp16
// products: acc[c] = rows 16 c + lane % 16 of the 16 results 4 (lane / 16) ..
// Its 32 columns in four steps of 8 a lane: step u's operand parts, and products.
__device__ __forceinline__ void matrix_parts(const float4_t (&m)[8], int u, half8_t& hi, half8_t& lo) {
  float x[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) x[j] = m[2 * u + (j >> 2)][j & 3] * 256.f;
  split8(x, hi, lo);
}
template <int NC>
__device__ __forceinline__ void staged_step(const uint8_t* src, int u, const half8_t& wh, const half8_t& wl,
                                            float4_t (&acc)[NC]) {
  half8_t bh[NC], bl[NC];
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    bh[c] = *reinterpret_cast<const half8_t*>(src + 16 * c * kHalfStride + 16 * u);
    bl[c] = *reinterpret_cast<const half8_t*>(src + kHalfPart + 16 * c * kHalfStride + 16 * u);
  }
#pragma unroll
  for (int c = 0; c < NC; ++c) acc[c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(wh, bh[c], acc[c], 0, 0, 0);
#pragma unroll
  for (int c = 0; c < NC; ++c) acc[c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(wl, bh[c], acc[c], 0, 0, 0);
#pragma unroll
  for (int c = 0; c < NC; ++c) acc[c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(wh, bl[c], acc[c], 0, 0, 0);
}
template <int NC>
__device__ __forceinline__ void staged_product(const uint8_t* staged, const float4_t (&m)[8], int lane, float4_t (&acc)[NC]) {
  const uint8_t* src = staged + (lane & 15) * kHalfStride + 64 * (lane >> 4);
#pragma unroll
  for (int c = 0; c < NC; ++c) acc[c] = float4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    half8_t wh, wl;
    matrix_parts(m, u, wh, wl);
    staged_step<NC>(src, u, wh, wl, acc);
  }
}

// N consecutive words (4-byte aligned) in as few loads as they take.
template <int N>
__device__ __forceinline__ void load_words(const uint32_t* base, uint32_t byte_off, uint32_t (&w)[N]) {
  typedef uint32_t u3_t __attribute__((ext_vector_type(3), aligned(4)));
  constexpr int F = N / 4 * 4;
#pragma unroll
  for (int i = 0; i < F; i += 4) {
    const uint4 v = ld_at<uint4>(base, byte_off + 4 * i);
    w[i] = v.x;
    w[i + 1] = v.y;
    w[i + 2] = v.z;
    w[i + 3] = v.w;
  }
  if constexpr (N % 4 == 3) {
    const u3_t v = ld_at<u3_t>(base, byte_off + 4 * F);
    w[F] = v[0];
    w[F + 1] = v[1];
    w[F + 2] = v[2];
  } else if constexpr (N % 4 == 2) {
    const uint2 v = ld_at<uint2>(base, byte_off + 4 * F);
    w[F] = v.x;
    w[F + 1] = v.y;
  } else if constexpr (N % 4 == 1) {
    w[F] = ld_at<uint32_t>(base, byte_off + 4 * F);
  }
}

__device__ __forceinline__ half8_t as_half8(const uint2& a, const uint2& b) {
  return __builtin_bit_cast(half8_t, make_uint4(a.x, a.y, b.x, b.y));
}

// ---------------------------------------------------------------- QK
// 16 coordinates of all 64 tokens: four lookups of four codes (bits POS .. of
// aw), or the operands of both token blocks once the half-waves have changed.
struct Step {
  uint2 a0, a1, b0, b1;
};
template <int B, int POS, int N>
__device__ __forceinline__ Step step_lookups(const uint8_t* smem, const uint32_t (&aw)[N], const LaneRep& rep) {
  return {__builtin_bit_cast(uint2, decode4<B, POS, true>(smem, aw, rep)),
          __builtin_bit_cast(uint2, decode4<B, POS + 4 * B, true>(smem, aw, rep)),
          __builtin_bit_cast(uint2, decode4<B, POS + 8 * B, true>(smem, aw, rep)),
          __builtin_bit_cast(uint2, decode4<B, POS + 12 * B, true>(smem, aw, rep))};
}
// The step's products: hi and lo query parts into the accumulators of the two
// token blocks.
template <bool Z>
__device__ __forceinline__ void step_products(const Step& k, const half8_t& qh, const half8_t& ql, float16_t (&part)[2]) {
  const half8_t k0 = as_half8(k.a0, k.a1), k1 = as_half8(k.b0, k.b1);
  if constexpr (Z) {  // the group's first product starts its accumulators
    const float16_t zero = {};
    part[0] = __builtin_amdgcn_mfma_f32_32x32x16_f16(k0, qh, zero, 0, 0, 0);
    part[1] = __builtin_amdgcn_mfma_f32_32x32x16_f16(k1, qh, zero, 0, 0, 0);
  } else {
    part[0] = __builtin_amdgcn_mfma_f32_32x32x16_f16(k0, qh, part[0], 0, 0, 0);
    part[1] = __builtin_amdgcn_mfma_f32_32x32x16_f16(k1, qh, part[1], 0, 0, 0);
  }
  part[0] = __builtin_amdgcn_mfma_f32_32x32x16_f16(k0, ql, part[0], 0, 0, 0);
  part[1] = __builtin_amdgcn_mfma_f32_32x32x16_f16(k1, ql, part[1], 0, 0, 0);
}

// S += radius * (the products of a group)
__device__ __forceinline__ void add_scaled(const half4_t (&r)[2][4], const float16_t (&part)[2], float16_t (&s)[2]) {
#pragma unroll
  for (int n = 0; n < 2; ++n)
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        s[n][4 * q + i] = fmaf(static_cast<float>(r[n][q][i]), part[n][4 * q + i], s[n][4 * q + i]);
}

// The group of width B (metadata gm): part = codes x query rows.  Its bits are
// realigned to bit 0 of a small word array, 32 coordinates at a time (16 for
// the wide codes); the lookups of both steps are in flight before the first
// product (a step past the group's end decodes other bits of the row for
// nobody), and the last group's products are added to S behind this one's first
// lookups.
template <int B, int KWB>
__device__ __forceinline__ void qk_group(const uint8_t* smem, const uint32_t (&rw)[KWB + split_detail::kRowPad],
                                         uint32_t gm, int step0, const uint8_t* radii, const LaneRep& rep, int lane,
                                         half4_t (&r)[2][4], float16_t (&part)[2], float16_t (&s)[2]) {
  constexpr int CH = B <= 4 ? 2 : 1;             // steps per chunk
  constexpr int NW = (CH * 16 * B + 31) / 32;    // its words
  const int o = split_detail::gm_off(gm), n16 = (split_detail::gm_steps(gm) + 3) >> 2;
  const auto chunk = [&](auto first, int c) __attribute__((always_inline)) {
    const int at = o + c * 16 * B, w0 = at >> 5, sh = at & 31;
    uint32_t aw[NW + 1];
#pragma unroll
    for (int i = 0; i < NW; ++i) aw[i] = __builtin_amdgcn_alignbit(rw[w0 + i + 1], rw[w0 + i], sh);
    aw[NW] = 0;
    const uint32_t img = kImg + (step0 + c) * 2048 + lane * 16;
    Step k0 = step_lookups<B, 0>(smem, aw, rep), k1;
    const half8_t qh = *reinterpret_cast<const half8_t*>(smem + img);
    const half8_t ql = *reinterpret_cast<const half8_t*>(smem + img + 1024);
    if constexpr (CH == 2) k1 = step_lookups<B, 16 * B>(smem, aw, rep);
    __builtin_amdgcn_sched_barrier(0);  // (every read of the chunk is issued before the first wait)
    if constexpr (decltype(first)::value) {
      if (step0 > 0) add_scaled(r, part, s);
      // radii of the lane's tokens: 8 q + 4 hf .. + 3 of each block
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int q = 0; q < 4; ++q) r[n][q] = *reinterpret_cast<const half4_t*>(radii + 2 * (32 * n + 8 * q));
    }
    swap_halves(k0.a0, k0.a1, k0.b0, k0.b1);
    if constexpr (CH == 2) swap_halves(k1.a0, k1.a1, k1.b0, k1.b1);
    step_products<decltype(first)::value>(k0, qh, ql, part);
    if constexpr (CH == 2) {
      if (c + 1 < n16) {
        const half8_t qh1 = *reinterpret_cast<const half8_t*>(smem + img + 2048);
        const half8_t ql1 = *reinterpret_cast<const half8_t*>(smem + img + 3072);
        step_products<false>(k1, qh1, ql1, part);
      }
    }
  };
  chunk(std::true_type{}, 0);
  for (int c = CH; c < n16; c += CH) chunk(std::false_type{}, c);
}

template <int KWB, int... BM1>
__device__ __forceinline__ void qk_all(std::integer_sequence<int, BM1...>, const uint8_t* smem,
                                       const uint32_t (&rw)[KWB + split_detail::kRowPad], const uint32_t (&gm)[8],
                                       const uint8_t* radii, const LaneRep& rep, int lane, float16_t (&s)[2]) {
  int step0 = 0;
  half4_t r[2][4];
  float16_t part[2];
  const auto one = [&](auto bm1) __attribute__((always_inline)) {
    constexpr int b = decltype(bm1)::value;
    if (gm[b] >> 31) {
      qk_group<b + 1, KWB>(smem, rw, gm[b], step0, radii + split_detail::gm_plane(gm[b]) * 128, rep, lane, r, part, s);
      step0 += (split_detail::gm_steps(gm[b]) + 3) >> 2;
    }
  };
  (one(std::integral_constant<int, BM1>{}), ...);
  add_scaled(r, part, s);
}

// ---------------------------------------------------------------- lookup tables
// Entries of the widths in `used` (bit b - 1), in the decode kernel's layout:
// four codes an entry for 1, 2 and 3 bits, two for 4, one above.
__device__ __forceinline__ void build_tables(uint8_t* smem, const uint16_t* cbs, uint32_t used, int tid) {
  using namespace split_detail;
  const auto pair = [](const uint16_t* cb, int i, int b) {
    const int m = (1 << b) - 1;
    return cb[i & m] | static_cast<uint32_t>(cb[(i >> b) & m]) << 16;
  };
  if (used & 2u) {
    // 16 lanes write an entry's 32 replicas; a thread keeps its low code pair
    const int e0 = tid >> 4;
    const uint32_t lo = pair(cbs + cb_index(2), e0, 2);
    uint32_t hi[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) hi[k] = pair(cbs + cb_index(2), (e0 + 32 * k) >> 4, 2);
#pragma unroll
    for (int k = 0; k < 8; ++k)
      *reinterpret_cast<uint4*>(smem + kLut2 + (e0 + 32 * k) * 256 + (tid & 15) * 16) = make_uint4(lo, hi[k], lo, hi[k]);
  }
  if (used & 4u) {
    const uint32_t lo = pair(cbs + cb_index(3), tid & 63, 3);
    uint32_t hi[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) hi[k] = pair(cbs + cb_index(3), (tid >> 6) + 8 * k, 3);
#pragma unroll
    for (int k = 0; k < 8; ++k) *reinterpret_cast<uint2*>(smem + kLut1B + (tid + 512 * k) * 8) = make_uint2(lo, hi[k]);
  }
  if (used & 1u)
    if (tid < 256)  // 16 entries x 16 replicas
      *reinterpret_cast<uint2*>(smem + kLut1 + tid * 8) =
          make_uint2(pair(cbs + cb_index(1), tid >> 4, 1), pair(cbs + cb_index(1), tid >> 6, 1));
  if (used & 8u)
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int i = tid + 512 * k;
      *reinterpret_cast<uint32_t*>(smem + kLut4 + i * 4) = pair(cbs + cb_index(4), i >> 3, 4);
    }
  if (used & 16u)
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int i = tid + 512 * k;
      *reinterpret_cast<uint32_t*>(smem + kLut5 + i * 4) = cbs[cb_index(5) + (i >> 5)];
    }
  if (used & 0xE0u) {
    const int i = tid;
    if (i < 256 + 128 + 64) {
      const int b = i < 256 ? 8 : (i < 384 ? 7 : 6), k = i < 256 ? i : (i < 384 ? i - 256 : i - 384);
      *reinterpret_cast<uint16_t*>(smem + kLutF + i * 2) = cbs[cb_index(b) + k];
    }
  }
}

// ---------------------------------------------------------------- kernel
// EX: the softmax weights times their radii in two fp16 parts (22 bits) for fp32
// outputs; one part is off by 2^-11 of a weight at most, an eighth of the
// output's own rounding to bf16.
// PACK: a side may have several sequences in a workgroup (what it takes to find
// a row's sequence is 0.5 us of a call of 16 without it).
// MODE: WholeCache, or the new rows of a ragged batch over pages (paged_pass.h).
template <int KWB, int BV, bool EX, bool PACK, class MODE>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2, 2))) void k_cross(
    Dims d, const uint8_t* __restrict__ blob, const void* __restrict__ q, CrossCall call, MODE mode) {
  constexpr bool kPaged = MODE::kPaged, kMods = MODE::kMods;
  __shared__ __attribute__((aligned(16))) uint8_t smem[kLds];
  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, hf = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int G = d.group, hq = d.n_kv * G, kw = d.k_words;
  const bool second = static_cast<int>(blockIdx.x) >= call.side[0].items;
  CrossSide S;  // (of both sides' arguments, read at once: no address waits for the choice)
  {
    const CrossSide &a = call.side[0], &b = call.side[1];
    S.c = {second ? b.c.k_codes : a.c.k_codes, second ? b.c.k_norms : a.c.k_norms, second ? b.c.v_codes : a.c.v_codes,
           second ? b.c.v_norms : a.c.v_norms};
    S.len = second ? b.len : a.len;
    S.batch = second ? b.batch : a.batch;
    S.capacity = second ? b.capacity : a.capacity;
    S.n_q = second ? b.n_q : a.n_q;
    S.split_len = second ? b.split_len : a.split_len;
    S.max_len = second ? b.max_len : a.max_len;
    S.slot0 = second ? b.slot0 : a.slot0;
    S.pack = !PACK ? 0 : second ? b.pack : a.pack;
  }
  // Row blocks vary fastest and splits slowest: workgroups go to the 8 XCDs in
  // turn, and a ragged batch's late splits, often empty, would leave some XCDs
  // without work if the split chose the XCD.
  int item = static_cast<int>(blockIdx.x) - (second ? call.side[0].items : 0);
  // 2^pack sequences of few query rows to a workgroup: their query rows lie one
  // after the other in the 32, a wave walks the tiles of one of them, and the
  // other sequences' columns of its products are not used.
  const int per = 1 << S.pack, wps = kWaves >> S.pack;  // sequences; waves to a sequence
  int r0, kvh, split, seq0 = 0, lz = 0, layer, sub = 0, seq, nr;  // nr: query rows
  paged::Unit U = {};
  if constexpr (kPaged) {
    if (!paged::find_unit<kRows>(mode, d, call, paged::unit_at(mode, d, call.n_slots, item, U), U, kThreads)) return;
    r0 = U.r0;
    kvh = U.kvh;
    split = U.split;
    layer = d.layer;
    seq = U.seq;
    nr = U.q.n * G;
  } else {
    const int n_blocks = (S.n_q * G + kRows - 1) / kRows, n_seq = (S.batch + per - 1) >> S.pack;
    r0 = item % n_blocks * kRows;
    item /= n_blocks;
    kvh = item % d.n_kv;
    item /= d.n_kv;
    const int n_lz = d.n_lc * n_seq, z = item % n_lz;
    split = item / n_lz;
    seq0 = z % n_seq << S.pack;
    lz = z / n_seq * S.batch + seq0;
    layer = d.layer >= 0 ? d.layer : z / n_seq;
    sub = wave >> (3 - S.pack);
    seq = min(seq0 + sub, S.batch - 1);  // the wave's sequence
    nr = S.n_q * G * min(per, S.batch - seq0);
  }
  const int ri = layer * d.n_kv + kvh;
  const RowMeta* M = reinterpret_cast<const RowMeta*>(blob + kOffRows) + ri;
  const auto row_at = [&](int r) {  // query row r of the unit (or its sequences), in q, out and the partials
    if constexpr (kPaged) return (static_cast<size_t>(U.q.first) + r / G) * hq + kvh * G + r % G;
    else return (static_cast<size_t>(lz) * S.n_q + r / G) * hq + kvh * G + r % G;
  };
  const auto part_of = [&](int r) {  // its partial
    if constexpr (kPaged)
      return call.part + (paged::part_row(mode, U, hq, r / G, kvh * G + r % G) * call.n_slots + split) * kPartFloats;
    else return call.part + (row_at(r) * call.n_slots + S.slot0 + split) * kPartFloats;
  };

  // The reads of the set-up that need no length, before the length is there (a
  // read that misses every cache takes about 1 us): fp16 codebooks, the wave's
  // 16 positions of the rotation, the query rows (thread = row tid / 16, dims 8
  // (tid % 16) .. + 7).
  const bool bf = d.in_dtype == 1;
  const uint16_t cv = reinterpret_cast<const uint16_t*>(blob + kOffC16)[min(tid, kCodebookEntries - 1)];
  float4_t rk[8];
  uint4 x0, x1;
  {
    const float4_t* w = reinterpret_cast<const float4_t*>(blob + layout_kdense_offset(d.n_layers * d.n_kv)) +
                        static_cast<size_t>(ri) * (kMfmaMatFloats / 4) + wave * 8 * 64 + lane;
    const size_t at = row_at(min(r0 + (tid >> 4), nr - 1)) * kHeadDim + 8 * (tid & 15);
    const uint4* qp = reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(q) + at * (bf ? 2 : 4));
    x0 = qp[0];
    x1 = bf ? make_uint4(0, 0, 0, 0) : qp[1];
#pragma unroll
    for (int s4 = 0; s4 < 8; ++s4) rk[s4] = w[s4 * 64];
  }

  // The length and the row's groups, read together (the asm keeps the compiler
  // from reading each group where it is used, one wait after the other).
  int len = kPaged ? U.q.len : S.len[seq], ng = M->n_groups;
  uint32_t gm[8], used = 1u << (BV - 1);
  int gd[8], gp[8];
#pragma unroll
  for (int b = 0; b < 8; ++b) {
    gm[b] = M->gm[b];
    gd[b] = M->g_dim[b];
    gp[b] = M->g_pos[b];
  }
  asm volatile("" : "+s"(len), "+s"(ng), "+s"(gm[0]), "+s"(gm[1]), "+s"(gm[2]), "+s"(gm[3]), "+s"(gm[4]), "+s"(gm[5]),
               "+s"(gm[6]), "+s"(gm[7]));
  asm volatile("" : "+s"(gd[0]), "+s"(gd[1]), "+s"(gd[2]), "+s"(gd[3]), "+s"(gd[4]), "+s"(gd[5]), "+s"(gd[6]), "+s"(gd[7]),
               "+s"(gp[0]), "+s"(gp[1]), "+s"(gp[2]), "+s"(gp[3]), "+s"(gp[4]), "+s"(gp[5]), "+s"(gp[6]), "+s"(gp[7]));
#pragma unroll
  for (int b = 0; b < 8; ++b) {
    used |= (gm[b] >> 31) << b;
    gd[b] = b < ng ? gd[b] : 0;
  }
  const int nslot = (ng + 1) & ~1;
  // a length outside [0, max_len] (the host's bound) makes the rows NaN
  const bool ok = kPaged || (len >= 0 && len <= S.max_len);
  const int t_begin = split * S.split_len;
  // the rows that the last query row sees; each row's own end (paged)
  paged::Sight sight = {};
  int t_end, lim = 0, lim0 = 0;
  float slope = 0.f;
  if constexpr (kPaged) {
    sight = paged::sight_of(mode, U, seq);
    t_end = min(sight.end((min(r0 + kRows, nr) - 1) / G), t_begin + S.split_len);
    const int rl = min(r0 + l32, nr - 1);
    lim = min(sight.end(rl / G), t_end);
    lim0 = min(sight.end(r0 / G), t_end);
    if (kMods && mode.m.slopes) slope = kLog2e * mode.m.slopes[kvh * G + rl % G];
  } else {
    t_end = ok && seq0 + sub < S.batch ? min(len, t_begin + S.split_len) : t_begin;
  }

  if (t_begin >= t_end && call.n_slots > 1 && S.pack == 0) {  // no row of the sequence in this split: an empty partial
    if (tid < kRows && r0 + tid < nr) {
      float* P = part_of(r0 + tid);
      P[0] = ok ? kNegInf : 0.f;
      P[1] = ok ? 0.f : __builtin_nanf("");
    }
    return;
  }
  const size_t cap = S.capacity;
  const uint32_t *kc, *vc;
  const uint16_t *kn, *vn;
  const auto rows_of = [&](size_t row) {  // (layer, sequence or page, head)
    kc = S.c.k_codes + row * cap * kw;
    kn = S.c.k_norms + row * kMaxGroups * cap;
    vc = S.c.v_codes + row * (cap / kTile) * kHeadDim * BV;
    vn = S.c.v_norms + row * cap;
  };
  // The wave's page numbers are read a tile ahead of the rows that need them.
  int page_next = 0;
  bool lost = false;  // a page outside the pool: the rows that attend it are not numbers
  const auto turn_to = [&](int t) {  // rows [t, t + 64) of the sequence: the page whose number was read, and t there
    const int number = __builtin_amdgcn_readfirstlane(page_next);
    lost |= static_cast<uint32_t>(number) >= static_cast<uint32_t>(S.batch);
    const int page = lost ? 0 : number;
    rows_of((static_cast<size_t>(layer) * S.batch + page) * d.n_kv + kvh);
    return t % S.capacity;
  };
  if constexpr (!kPaged) rows_of((static_cast<size_t>(layer) * S.batch + seq) * d.n_kv + kvh);
  uint32_t nw[KWB], knp[4], vnw, vw[4][BV];  // (a half-wave loads the values of its own 32-row tile)
  const auto load_keys = [&](int t0) {
    const uint32_t* src = kc + static_cast<size_t>(t0) * kw;
    const uint32_t at = static_cast<uint32_t>(lane * kw * 4);
    if ((kw & 3) == 0) {
#pragma unroll
      for (int i = 0; i < KWB; i += 4) {
        const uint4 v = i < kw ? ld_at<uint4>(src, at + 4 * i) : make_uint4(0, 0, 0, 0);
        nw[i] = v.x;
        nw[i + 1] = v.y;
        nw[i + 2] = v.z;
        nw[i + 3] = v.w;
      }
    } else {
#pragma unroll
      for (int i = 0; i < KWB; ++i) nw[i] = i < kw ? ld_at<uint32_t>(src, at + 4 * i) : 0u;
    }
    // (a token's 16 bytes of radii stay inside the row's 8 slots per token)
    const uint4 r = ld_at<uint4>(kn + static_cast<size_t>(t0) * nslot, static_cast<uint32_t>(lane * nslot * 2));
    knp[0] = r.x;
    knp[1] = r.y;
    knp[2] = r.z;
    knp[3] = r.w;
    vnw = ld_at<uint16_t>(vn + t0, static_cast<uint32_t>(lane * 2));
  };
  const auto load_values = [&](int t0) {
    const uint32_t* src = vc + static_cast<size_t>(t0 / kTile) * kHeadDim * BV;
#pragma unroll
    for (int cc = 0; cc < 4; ++cc)
      load_words(src + 32 * cc * BV, static_cast<uint32_t>((hf * kHeadDim + l32) * BV * 4), vw[cc]);
  };
  int t0 = t_begin + (wave & (wps - 1)) * kKeyTile;
  const int stride = wps * kKeyTile;
  const auto read_page = [&](int t) {
    if constexpr (kPaged) page_next = paged::page_ahead(mode.b, seq, t, S.capacity);
  };
  // (without a next tile this one again: the loads in flight stay countable)
  const auto after = [&](int t) { return t + stride < t_end ? t + stride : t; };

  // ---- set-up: the query rows rotated into stream order,
  //   q'[p] = log2 e / sqrt(d_g d_h) sum_d W[p][d] q[d],
  // in three fp16 products (wave = 16 positions), and written into the image,
  // before and after scaled by the power of two that brings the row's largest
  // coordinate to [2^13, 2^14): the lo parts stay above fp16's subnormals.
  // Every global read of the set-up and the first tile's are issued at once
  // (few and wide ones: the 8 waves' loads pass one by one).
  const int p0 = 16 * wave + 4 * (lane >> 4);  // the lane's 4 positions of the rotation
  float4_t rq[2];                              // rows 16 c + lane % 16
  {
    // (the lane's 128 bytes of Pi_V^T for the end, brought near)
    float near = 0.f;
    if (call.n_slots == 1)
      near = reinterpret_cast<const float*>(blob + kOffRotVT)[(16 * wave + (lane & 15)) * kHeadDim + 32 * (lane >> 4)];
    if (t0 < t_end) {
      read_page(t0);
      const int at = kPaged ? turn_to(t0) : t0;
      load_keys(at);
      load_values(at);
      read_page(after(t0));
    }
    uint16_t* cbs = reinterpret_cast<uint16_t*>(smem + kBooks);
    if (tid < kCodebookEntries) cbs[tid] = cv;
    if (tid < kRows) reinterpret_cast<uint32_t*>(smem + kTop)[tid] = 0;
    {
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
      uint8_t* dst = smem + kImg + (tid >> 4) * kHalfStride + 16 * (tid & 15);
      *reinterpret_cast<half8_t*>(dst) = hi;
      *reinterpret_cast<half8_t*>(dst + kHalfPart) = lo;
      if ((tid & 15) == 0) reinterpret_cast<float*>(smem + kBack)[tid >> 4] = two_to(254 - up) * (1.f / 256.f);
    }
    __syncthreads();
    build_tables(smem, cbs, used, tid);
    staged_product<2>(smem + kImg, rk, lane, rq);
    asm volatile("" ::"v"(near));
  }
  // place of the lane's position pairs in the image (group sizes are even)
  uint32_t img_at[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    int st = 0, at = 0, dg = 2, base = 0;
#pragma unroll
    for (int g = 0; g < 8; ++g) {
      if (g < ng && p0 + 2 * h >= gp[g]) {
        at = p0 + 2 * h - gp[g];
        dg = gd[g];
        st = base;
      }
      base += (gd[g] + 15) >> 4;
    }
    img_at[h] = kImg + (st + (at >> 4)) * 2048 + ((at >> 3) & 1) * 512 + (at & 7) * 2;
    const float scale = kLog2e * kRsqrtD * rsqrtf(static_cast<float>(dg));
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      rq[c][2 * h] *= scale;
      rq[c][2 * h + 1] *= scale;
    }
  }
  uint32_t* const top = reinterpret_cast<uint32_t*>(smem + kTop);
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    uint32_t mx = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) mx = max(mx, __float_as_uint(rq[c][i]) & 0x7FFFFFFFu);
    mx = max(mx, static_cast<uint32_t>(__shfl_xor(static_cast<int>(mx), 16)));
    mx = max(mx, static_cast<uint32_t>(__shfl_xor(static_cast<int>(mx), 32)));
    if (lane < 16) atomicMax(top + 16 * c + lane, mx);
  }
  __syncthreads();
  // (the image takes the staged queries' place)
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    const int r = 16 * c + (lane & 15);
    const float to = two_to(up_of(top[r]));
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      half2_t hi, lo;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const float x = rq[c][2 * h + j] * to;
        hi[j] = static_cast<_Float16>(x);
        lo[j] = static_cast<_Float16>(x - static_cast<float>(hi[j]));
      }
      *reinterpret_cast<half2_t*>(smem + img_at[h] + r * 16) = hi;
      *reinterpret_cast<half2_t*>(smem + img_at[h] + r * 16 + 1024) = lo;
    }
  }
  // zeros behind the groups' ends: thread = (position pair tid / 32 from the end, row)
  if (tid < 7 * 32) {
    int base = 0;
#pragma unroll
    for (int g = 0; g < 8; ++g) {
      const int at = gd[g] + 2 * (tid >> 5), n16 = (gd[g] + 15) >> 4;
      if (at < 16 * n16) {
        uint8_t* dst = smem + kImg + (base + (at >> 4)) * 2048 + ((at >> 3) & 1) * 512 + (at & 7) * 2 + (tid & 31) * 16;
        *reinterpret_cast<uint32_t*>(dst) = 0;
        *reinterpret_cast<uint32_t*>(dst + 1024) = 0;
      }
      base += n16;
    }
  }
  __syncthreads();

  LaneRep rep{static_cast<uint32_t>(split_detail::kLut1 + (lane & 15) * 8),
              static_cast<uint32_t>(split_detail::kLut3 + (lane & 31) * 4),
              static_cast<uint32_t>(split_detail::kLut4 + (lane & 7) * 4),
              static_cast<uint32_t>(split_detail::kLut5 + (lane & 31) * 4),
              static_cast<uint32_t>(split_detail::kLut2 + (lane & 31) * 8),
              static_cast<uint32_t>(split_detail::kLut1B), 0u};
  asm volatile("" : "+v"(rep.r1), "+v"(rep.r3), "+v"(rep.r4), "+v"(rep.r5), "+v"(rep.r2), "+v"(rep.r1b));
  // the row's scales, undone on its logits
  const float sc = two_to(254 - up_of(top[l32])) * reinterpret_cast<const float*>(smem + kBack)[l32];
  uint8_t* const rad = smem + kRad + wave * kRadBytes;
  const uint8_t* const rad_l = rad + 8 * hf;  // the lane's tokens start at 4 hf

  float m_run = kNegInf, l_run = 0.f;
  int v_top = 0;  // (see radius_top)
  float16_t o[4];
#pragma unroll
  for (int cc = 0; cc < 4; ++cc)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[cc][i] = 0.f;

  for (; t0 < t_end; t0 += stride) {
    const bool full = t0 + kKeyTile <= (kPaged ? lim0 : t_end);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // the last tile's reads of the radii come first
    // this tile's radii, token-minor, for the wave's own reads (LDS operations
    // of a wave complete in order); a token past the end has value radius 0:
    // what lies there may be infinite or not a number
    // (an infinite key radius becomes not a number: the coordinates that it
    // scales have both signs, so the row's logits are not numbers, where the sum
    // of a group's products, scaled afterwards, would be infinite)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const half2_t r = __builtin_bit_cast(half2_t, knp[g]);
      knp[g] = __builtin_bit_cast(uint32_t, r + (r - r));
    }
#pragma unroll
    for (int g = 0; g < 8; ++g)
      if (g < ng) *reinterpret_cast<uint16_t*>(rad + 128 * g + 2 * lane) = static_cast<uint16_t>(knp[g >> 1] >> (16 * (g & 1)));
    const uint32_t vr_now = t0 + lane < t_end ? vnw : 0u;
    if (const int was = v_top; (v_top = radius_top(was, vr_now)) != was && was > 0) {
      const float down = two_to(127 + was - v_top);
#pragma unroll
      for (int cc = 0; cc < 4; ++cc) o[cc] *= down;
    }
    *reinterpret_cast<uint16_t*>(rad + 128 * 8 + 2 * lane) = static_cast<uint16_t>(radius_times(vr_now, radius_up(v_top)));
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    {
      // the row's width table re-read every tile (scalar loads through an
      // opaque offset): hoisted, its derived scalars exhaust the SGPRs
      uint32_t goff = 0;
      asm volatile("" : "+s"(goff));
      const uint32_t* gmt = reinterpret_cast<const uint32_t*>(reinterpret_cast<const uint8_t*>(M->gm) + goff);
#pragma unroll
      for (int b = 0; b < 8; ++b) gm[b] = gmt[b];
    }
    uint32_t rw[KWB + split_detail::kRowPad];
#pragma unroll
    for (int i = 0; i < KWB; ++i) rw[i] = nw[i];
#pragma unroll
    for (int i = KWB; i < KWB + split_detail::kRowPad; ++i) rw[i] = 0u;
    float16_t s[2];
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[n][i] = 0.f;
    qk_all<KWB>(std::make_integer_sequence<int, 8>{}, smem, rw, gm, rad_l, rep, lane, s);
    int t_next = after(t0);
    if constexpr (kPaged) {
      const int t = t_next;
      t_next = turn_to(t);
      read_page(after(t));
    }
    load_keys(t_next);

    const float sx = kMods ? 1.f : sc;  // what is left to multiply the logits with
    if constexpr (kMods) {
      const float at = static_cast<float>(sight.pos(min(r0 + l32, nr - 1) / G) - t0 - 4 * hf);
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          s[n][i] = paged::changed(mode.m.cap, slope, s[n][i] * sc, at - static_cast<float>(32 * n + 8 * (i >> 2) + (i & 3)));
    }

    // ---- online softmax, base 2
    if (!full) {
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int tok = t0 + 32 * n + 8 * (i >> 2) + 4 * hf + (i & 3);
          s[n][i] = tok >= (kPaged ? lim : t_end) ? kNegInf : s[n][i];
        }
    }
    float mp[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      mp[c] = fmaxf(s[0][4 * c], s[0][4 * c + 1]);
      mp[c] = fmaxf(fmaxf(mp[c], s[0][4 * c + 2]), s[0][4 * c + 3]);
      mp[c] = fmaxf(fmaxf(mp[c], s[1][4 * c]), s[1][4 * c + 1]);
      mp[c] = fmaxf(fmaxf(mp[c], s[1][4 * c + 2]), s[1][4 * c + 3]);
    }
    const float mx = fmaxf(fmaxf(mp[0], mp[1]), fmaxf(mp[2], mp[3])) * sx;
    // a tile that raises no running maximum of the wave skips the rescale
    if (__builtin_amdgcn_ballot_w64(mx > m_run) != 0) {
      float x, y;
      swap32(mx, x, y);
      const float mn = fmaxf(m_run, fmaxf(x, y));
      const float corr = m_run == kNegInf ? 0.f : __builtin_amdgcn_exp2f(m_run - mn);
      m_run = mn;
      l_run *= corr;
#pragma unroll
      for (int cc = 0; cc < 4; ++cc) o[cc] *= corr;
    }
    const float mref = m_run == kNegInf ? 0.f : m_run;
    // the values of both 32-row tiles into both half-waves
    uint32_t v1[4 * BV];
#pragma unroll
    for (int i = 0; i < BV; ++i) {
      uint32_t x[4] = {vw[0][i], vw[1][i], vw[2][i], vw[3][i]}, y[4];
      spread_halves(x, y);
#pragma unroll
      for (int cc = 0; cc < 4; ++cc) {
        vw[cc][i] = x[cc];
        v1[cc * BV + i] = y[cc];
      }
    }
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      uint32_t pw[8], pl[EX ? 8 : 1];
      float ps = 0.f;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        uint2 vr = *reinterpret_cast<const uint2*>(rad_l + 128 * 8 + 2 * (32 * n + 8 * u));
        // (a radius that the row does not see may be infinite or not a number)
        if (kPaged && !full) vr = paged::seen(vr, lim - (t0 + 32 * n + 8 * u + 4 * hf));
        float p[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) p[i] = __builtin_amdgcn_exp2f(fmaf(s[n][4 * u + i], sx, -mref));
        ps += (p[0] + p[1]) + (p[2] + p[3]);
        pw[2 * u] = mix_pair(p[0], p[1], vr.x);
        pw[2 * u + 1] = mix_pair(p[2], p[3], vr.y);
        if constexpr (EX) {
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const half2_t h = __builtin_bit_cast(half2_t, pw[2 * u + k]), r = __builtin_bit_cast(half2_t, k ? vr.y : vr.x);
            const half2_t x = {
                static_cast<_Float16>(fmaf(p[2 * k], static_cast<float>(r[0]), -static_cast<float>(h[0]))),
                static_cast<_Float16>(fmaf(p[2 * k + 1], static_cast<float>(r[1]), -static_cast<float>(h[1])))};
            pl[2 * u + k] = __builtin_bit_cast(uint32_t, x);
          }
        }
      }
      l_run += ps;
#pragma unroll
      for (int cc = 0; cc < 4; ++cc) {
        // the codes of tokens 8 k + 4 hf .. + 3 to bit 8 k BV
        uint32_t w[BV + 1];
#pragma unroll
        for (int i = 0; i < BV; ++i) {
          const uint32_t up = i + 1 < BV ? (n ? v1[cc * BV + i + 1] : vw[cc][i + 1]) : 0u;
          if constexpr (BV == 8) w[i] = hf ? up : (n ? v1[cc * BV + i] : vw[cc][i]);
          else w[i] = __builtin_amdgcn_alignbit(up, (n ? v1[cc * BV + i] : vw[cc][i]), 4 * BV * hf);
        }
        w[BV] = 0;
        const half4_t v0 = decode4<BV, 0, true>(smem, w, rep), v1 = decode4<BV, 8 * BV, true>(smem, w, rep);
        const half4_t v2 = decode4<BV, 16 * BV, true>(smem, w, rep), v3 = decode4<BV, 24 * BV, true>(smem, w, rep);
        const half8_t a0 = {v0[0], v0[1], v0[2], v0[3], v1[0], v1[1], v1[2], v1[3]};
        const half8_t a1 = {v2[0], v2[1], v2[2], v2[3], v3[0], v3[1], v3[2], v3[3]};
        const half8_t b0 = __builtin_bit_cast(half8_t, make_uint4(pw[0], pw[1], pw[2], pw[3]));
        const half8_t b1 = __builtin_bit_cast(half8_t, make_uint4(pw[4], pw[5], pw[6], pw[7]));
        o[cc] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a0, b0, o[cc], 0, 0, 0);
        o[cc] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a1, b1, o[cc], 0, 0, 0);
        if constexpr (EX) {
          const half8_t c0 = __builtin_bit_cast(half8_t, make_uint4(pl[0], pl[1], pl[2], pl[3]));
          const half8_t c1 = __builtin_bit_cast(half8_t, make_uint4(pl[4], pl[5], pl[6], pl[7]));
          o[cc] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a0, c0, o[cc], 0, 0, 0);
          o[cc] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a1, c1, o[cc], 0, 0, 0);
        }
      }
    }
    load_values(t_next);
  }
  {
    float x, y;
    swap32(l_run, x, y);
    l_run = x + y;
  }
  if (kPaged && lost) l_run = __builtin_nanf("");

  // ---- the waves' states joined in LDS (over the tables)
  float4_t rot[8];  // this wave's 16 output dims of Pi_V^T, for the output rotation
  if (call.n_slots == 1) {
    const float4_t* src = reinterpret_cast<const float4_t*>(blob + kOffRotVT) +
                          ((16 * wave + (lane & 15)) * kHeadDim + 32 * (lane >> 4)) / 4;
#pragma unroll
    for (int s4 = 0; s4 < 8; ++s4) rot[s4] = src[s4];
  }
  __syncthreads();
  float* const acc = reinterpret_cast<float*>(smem);
  float* const ms = reinterpret_cast<float*>(smem + kEndM);
  float* const ls = ms + kWaves * kRows;
  int* const tiles = reinterpret_cast<int*>(smem + kEndTiles);
  float* const vback = reinterpret_cast<float*>(smem + kEndBack);
  const int n_tiles = max(t_end - t_begin + kKeyTile - 1, 0) / kKeyTile;
  if (S.pack && lane == 0) tiles[wave] = ok ? n_tiles : -1;
  if (lane == 0) vback[wave] = two_to(127 - radius_up(v_top));
  if ((wave & (wps - 1)) < n_tiles) {
#pragma unroll
    for (int cc = 0; cc < 4; ++cc)
#pragma unroll
      for (int u = 0; u < 4; ++u)
        *reinterpret_cast<float4_t*>(acc + (wave * kRows + l32) * kAccStride + 32 * cc + 8 * u + 4 * hf) =
            float4_t{o[cc][4 * u], o[cc][4 * u + 1], o[cc][4 * u + 2], o[cc][4 * u + 3]};
  }
  if (hf == 0) {
    ms[wave * kRows + l32] = m_run;
    ls[wave * kRows + l32] = l_run;
  }
  __syncthreads();
  const int r = tid >> 4, d0 = (tid & 15) * 8;  // dims d0 .. + 7 of row r
  float m = kNegInf, l = 0.f;
  float4_t a[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
  // the waves of the row's sequence that had a tile
  const int w0 = S.pack == 0 ? 0 : min(r / (S.n_q * G), per - 1) * wps;
  const int n_row = S.pack == 0 ? (ok ? n_tiles : -1) : tiles[w0], n_act = min(wps, n_row);
#pragma unroll
  for (int w = 0; w < kWaves; ++w)
    if (w < n_act) m = fmaxf(m, ms[(w0 + w) * kRows + r]);
  const float mref = m == kNegInf ? 0.f : m;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    if (w >= n_act) break;
    const float e = __builtin_amdgcn_exp2f(ms[(w0 + w) * kRows + r] - mref);
    l = fmaf(ls[(w0 + w) * kRows + r], e, l);
    const float ea = e * vback[w0 + w];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const float4_t x = *reinterpret_cast<const float4_t*>(acc + ((w0 + w) * kRows + r) * kAccStride + 4 * h + d0);
#pragma unroll
      for (int i = 0; i < 4; ++i) a[h][i] = fmaf(x[i], ea, a[h][i]);
    }
  }
  if (n_row < 0) l = __builtin_nanf("");
  if (call.n_slots > 1) {
    if (r0 + r < nr) {
      float* P = part_of(r0 + r);
      if (d0 == 0) {
        // no row seen: -inf; logits that are all not a number leave the
        // maximum at -inf (fmaxf passes over them) but not the sum at 0
        P[0] = l == 0.f ? kNegInf : mref;
        P[1] = l;
      }
      *reinterpret_cast<float4_t*>(P + 4 + d0) = a[0];
      *reinterpret_cast<float4_t*>(P + 8 + d0) = a[1];
    }
    return;
  }
  // ---- the only partial: out = Pi_V^T (a / l), in three fp16 products of the
  // rows scaled as the queries were
  __syncthreads();
  {
    const float inv = l == 0.f ? 0.f : kRsqrtD / l;
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = a[e >> 2][e & 3] * inv;
    const int up = up_of(top16(x));
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] *= two_to(up);
    half8_t hi, lo;
    split8(x, hi, lo);
    uint8_t* dst = smem + r * kHalfStride + 16 * (tid & 15);
    *reinterpret_cast<half8_t*>(dst) = hi;
    *reinterpret_cast<half8_t*>(dst + kHalfPart) = lo;
    if ((tid & 15) == 0) reinterpret_cast<float*>(smem + 2 * kHalfPart)[r] = two_to(254 - up) * (1.f / 256.f);
  }
  __syncthreads();
  float4_t y[2];
  staged_product<2>(smem, rot, lane, y);
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    const int rl = 16 * c + (lane & 15);
    if (r0 + rl < nr)
      store4(call.out, row_at(r0 + rl) * kHeadDim + 16 * wave + 4 * (lane >> 4),
             y[c] * reinterpret_cast<const float*>(smem + 2 * kHalfPart)[rl], call.out_dtype);
  }
}

template <int BV>
hipError_t launch_bv(const Dims& d, const void* layout, const void* q, const CrossCall& call, hipStream_t s) {
  const int items = call.side[0].items + call.side[1].items;
  const auto go = [&](auto kern) {
    hipLaunchKernelGGL(kern, dim3(items), dim3(kThreads), 0, s, d, static_cast<const uint8_t*>(layout), q, call, paged::WholeCache{});
    return hipGetLastError();
  };
  const auto width = [&](auto ex, auto pack) {
    constexpr bool E = decltype(ex)::value, P = decltype(pack)::value;
    using W = paged::WholeCache;
    if (d.k_words <= 8) return go(k_cross<8, BV, E, P, W>);
    if (d.k_words <= 12) return go(k_cross<12, BV, E, P, W>);
    if (d.k_words <= 16) return go(k_cross<16, BV, E, P, W>);
    return go(k_cross<32, BV, E, P, W>);
  };
  const bool pack = call.side[0].pack || call.side[1].pack;
  if (call.out_dtype == 0)  // BGTQ_FP32
    return pack ? width(std::true_type{}, std::true_type{}) : width(std::true_type{}, std::false_type{});
  return pack ? width(std::false_type{}, std::true_type{}) : width(std::false_type{}, std::false_type{});
}

template <int BV>
hipError_t launch_paged_bv(const Dims& d, const void* layout, const void* q, const CrossCall& call, const PagedPass& pass,
                           hipStream_t s) {
  const auto go = [&](auto kern, auto mode) {
    hipLaunchKernelGGL(kern, dim3(call.side[0].items), dim3(kThreads), 0, s, d, static_cast<const uint8_t*>(layout), q, call,
                       mode);
    return hipGetLastError();
  };
  const auto width = [&](auto ex, auto mode) {
    constexpr bool E = decltype(ex)::value;
    using M = decltype(mode);
    if (d.k_words <= 8) return go(k_cross<8, BV, E, false, M>, mode);
    if (d.k_words <= 12) return go(k_cross<12, BV, E, false, M>, mode);
    if (d.k_words <= 16) return go(k_cross<16, BV, E, false, M>, mode);
    return go(k_cross<32, BV, E, false, M>, mode);
  };
  const auto mods = [&](auto ex) {
    return pass.m.cap > 0.f || pass.m.slopes ? width(ex, paged::Mode<true>{pass}) : width(ex, paged::Mode<false>{pass});
  };
  return call.out_dtype == 0 ? mods(std::true_type{}) : mods(std::false_type{});  // BGTQ_FP32
}

}  // namespace cross_detail
}  // namespace bgtq
