// Cache rows read back as plain keys and values: the inverse of
// blockgtq_quantize_append.
//
//   k_hat[d] = sum_p W[p][d] y[p],   y[p] = r_g C_b(code_p) / sqrt(d_g)
//   v_hat[d] = sum_j Pi_V[j][d] y[j], y[j] = n_V C_bV(code_j) / sqrt(128)
//
// with W the row's key rotation on the natural dims (zero outside position
// p's group g, so its transpose is its inverse).
//
// Both are products with a 128 x 128 matrix on 32x32x16 f16 MFMAs,
// D[dim][token] = A[dim][p] B[p][token], the matrix in fp16 in LDS (scaled by
// 2^8 and 1 / sqrt(d_g)), built once per workgroup, which then walks many
// tiles.  A workgroup does keys or values.
//  * Keys: lane = token decodes 16 positions of one group, two codes a lookup,
//    and v_permlane32_swap turns the 64 tokens' registers into B operands of
//    two 32-token blocks.  A dim's row of the matrix is zero outside its own
//    group, so the group's radius scales the result, dim by dim, in fp32: a
//    group's dims are as exact as its own radius whatever the others are, and a
//    radius that is not finite stays in its group's dims.
//  * Values: codes lie dim after dim, so a 32-token tile is decoded lane = dim
//    into LDS and read back lane = token.  The bare centroids are the operand;
//    the radius scales the result.
// Centroids are fp16 numbers, exact as operands; the matrix is in hi and lo
// parts (22 bits, two products).  bf16 outputs are the fp32 result rounded: with
// the hi part alone, 2^-11 of each term, 12 % of them would be another bf16 number
// and elements whose terms cancel off by many of their own steps.
//
// What bounds it: writing the rows, and the decode and products that wait while a
// wave stores.  65536 rows x 8 heads of K2V2 to bf16: 112 us for 308 MB, 2.7 TB/s.  A
// few rows: the keys' matrix, more than half of the 20 us of 16 rows of 32 layers x
// 8 heads, whose 512 workgroups take two rounds of the CUs.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "decode_impl.h"
#include "kernels.h"
#include "layout.h"

namespace bgtq {
namespace {

using split_detail::field_at;
typedef _Float16 half8_t __attribute__((ext_vector_type(8)));
typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
typedef float float4_t __attribute__((ext_vector_type(4)));
typedef float float2_t __attribute__((ext_vector_type(2)));
typedef float float16_t __attribute__((ext_vector_type(16)));

constexpr int kWaves = 8, kThreads = kWaves * 64;
constexpr int kMaxSteps = 15;       // 16-position steps of a key row, groups padded: at most (128 + 8 * 14) / 16
constexpr float kMatScale = 256.f;  // keeps the matrix's lo parts above fp16's subnormals
// ---- LDS map (bytes): codebooks, pair tables of the widths 1 .. 6 (entry i
// of width b: the centroids of codes i % 2^b and i / 2^b), then the matrix
// [part][step][dim block][lane] x 16 B, and behind it the values' tiles
constexpr int kBooks = 0;
constexpr int kPair = 1024;
constexpr int kMaxPair = 6;
__host__ __device__ constexpr int pair_offset(int b) { return kPair + 4 * (((1 << (2 * b)) - 4) / 3); }
constexpr int kDims = pair_offset(kMaxPair + 1);  // a key row's stream position -> dim
// by 4 dims, 16 bytes: byte selectors that pick the dims' radii (2 bytes each)
// from the token's 8: among groups 0-3, then 4-7 (the other half's select zero)
constexpr int kSel = (kDims + kHeadDim + 15) / 16 * 16;
constexpr int kMat = kSel + kHeadDim / 4 * 16;
constexpr int kVSteps = kHeadDim / 16;
constexpr int kTileStride = (kHeadDim + 8) * 2;  // bytes of a decoded token
constexpr int kTileBytes = kTile * kTileStride;
constexpr int kKeyBytes = 2 * kMaxSteps * 4096, kValueBytes = 2 * kVSteps * 4096 + kWaves * kTileBytes;
constexpr int kLds = kMat + (kKeyBytes > kValueBytes ? kKeyBytes : kValueBytes);
static_assert(kLds <= 160 * 1024, "LDS of one workgroup");

struct RowsCall {
  CachePtrs c;
  const int32_t* read_pos;
  const int32_t* ctx_len;  // or null
  void* out[2];            // keys, values; a null one has no workgroups
  int n_rows;
  int chunks[2], tiles[2];  // workgroups per unit and tiles (64 keys, 32 values) per workgroup
  int key_items;            // workgroups of the keys
};

// Two consecutive B-bit codes at bit POS of w -> two fp16 centroids.
template <int B, int POS, int N>
__device__ __forceinline__ half2_t pair_at(const uint8_t* smem, const uint32_t (&w)[N]) {
  if constexpr (B <= kMaxPair) {
    return *reinterpret_cast<const half2_t*>(smem + pair_offset(B) + field_at<POS, 2 * B, 2>(w));
  } else {
    const half2_t r = {*reinterpret_cast<const _Float16*>(smem + kBooks + 2 * cb_index(B) + field_at<POS, B, 1>(w)),
                       *reinterpret_cast<const _Float16*>(smem + kBooks + 2 * cb_index(B) + field_at<POS + B, B, 1>(w))};
    return r;
  }
}

__device__ __forceinline__ void swap4(uint32_t (&x)[4], uint32_t (&y)[4]) {
  asm("s_nop 1\n\t"
      "v_permlane32_swap_b32 %0, %4\n\t"
      "v_permlane32_swap_b32 %1, %5\n\t"
      "v_permlane32_swap_b32 %2, %6\n\t"
      "v_permlane32_swap_b32 %3, %7\n\t"
      "s_nop 1"
      : "+v"(x[0]), "+v"(x[1]), "+v"(x[2]), "+v"(x[3]), "+v"(y[0]), "+v"(y[1]), "+v"(y[2]), "+v"(y[3]));
}
// x = the lower half-wave's value, y = the upper one's, in both.
__device__ __forceinline__ void spread4(uint32_t (&x)[4], uint32_t (&y)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) y[i] = x[i];
  swap4(x, y);
}
__device__ __forceinline__ half8_t as_half8(const uint32_t (&x)[4]) {
  return __builtin_bit_cast(half8_t, make_uint4(x[0], x[1], x[2], x[3]));
}

// Pair tables of the widths in `used` (bit b - 1).
__device__ __forceinline__ void build_pairs(uint8_t* smem, uint32_t used, int tid) {
  const uint16_t* cbs = reinterpret_cast<const uint16_t*>(smem + kBooks);
#pragma unroll
  for (int b = 1; b <= kMaxPair; ++b)
    if ((used >> (b - 1)) & 1u)
#pragma unroll
      for (int i0 = 0; i0 < (1 << (2 * b)); i0 += kThreads) {
        const int i = i0 + tid;
        if ((1 << (2 * b)) >= kThreads || i < (1 << (2 * b)))
          *reinterpret_cast<uint32_t*>(smem + pair_offset(b) + 4 * i) =
              cbs[cb_index(b) + (i & ((1 << b) - 1))] | (static_cast<uint32_t>(cbs[cb_index(b) + (i >> b)]) << 16);
      }
}

// One operand of the matrix: 8 numbers, rounded, and their residuals.
__device__ __forceinline__ void store_operand(uint8_t* dst, int part_bytes, float (&x)[8]) {
  half8_t hi, lo;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    // (x as fp32, opaque: a product rounded to fp16 at once in one place and by
    // way of fp32 in the other gives two different hi parts next to a tie)
    asm volatile("" : "+v"(x[j]));
    hi[j] = static_cast<_Float16>(x[j]);
    lo[j] = static_cast<_Float16>(x[j] - static_cast<float>(hi[j]));
  }
  *reinterpret_cast<half8_t*>(dst) = hi;
  *reinterpret_cast<half8_t*>(dst + part_bytes) = lo;
}

// Rows of 16 lanes: the odd ones of x change places with the even ones of y.
__device__ __forceinline__ void swap_rows4(uint32_t (&x)[4], uint32_t (&y)[4]) {
  asm("s_nop 1\n\t"
      "v_permlane16_swap_b32 %0, %4\n\t"
      "v_permlane16_swap_b32 %1, %5\n\t"
      "v_permlane16_swap_b32 %2, %6\n\t"
      "v_permlane16_swap_b32 %3, %7\n\t"
      "s_nop 1"
      : "+v"(x[0]), "+v"(x[1]), "+v"(x[2]), "+v"(x[3]), "+v"(y[0]), "+v"(y[1]), "+v"(y[2]), "+v"(y[3]));
}

// acc (lane = token l32, registers = dims 32 cc + 8 (i / 4) + 4 hf + i % 4)
// times scale, to the output rows of the valid tokens (bit j: token j, at
// element at0 + j stride).  A store as the registers lie has 16 bytes of a row
// from each half-wave; lanes change places until it has 64 contiguous ones of
// 16 rows (the memory takes 32-byte pieces at half the rate).
template <bool F32>
__device__ __forceinline__ void store_rows(const float16_t (&acc)[4], float scale, void* out, long at0, long stride,
                                           uint32_t valid, int lane) {
  const int l16 = lane & 15, r1 = (lane >> 4) & 1, hf = lane >> 5;
  const bool ok[2] = {((valid >> l16) & 1u) != 0, ((valid >> (16 + l16)) & 1u) != 0};
#pragma unroll
  for (int cc = 0; cc < 4; ++cc) {
    float16_t y = acc[cc];
    y *= scale;
    if constexpr (F32) {
#pragma unroll
      for (int v = 0; v < 2; ++v) {  // dims 16 v .. + 15 of the block
        uint32_t a[4], b[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          a[i] = __float_as_uint(y[8 * v + i]);
          b[i] = __float_as_uint(y[8 * v + 4 + i]);
        }
        swap_rows4(a, b);
        const long at = at0 + 32 * cc + 16 * v + 8 * r1 + 4 * hf;
        if (ok[0])
          *reinterpret_cast<uint4*>(static_cast<float*>(out) + at + l16 * stride) = make_uint4(a[0], a[1], a[2], a[3]);
        if (ok[1])
          *reinterpret_cast<uint4*>(static_cast<float*>(out) + at + (16 + l16) * stride) = make_uint4(b[0], b[1], b[2], b[3]);
      }
    } else {
      typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
      uint32_t a[4], b[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const float4_t f = {y[4 * u], y[4 * u + 1], y[4 * u + 2], y[4 * u + 3]};
        const uint2 p = __builtin_bit_cast(uint2, __builtin_convertvector(f, bf16x4_t));
        (u & 1 ? b : a)[u & ~1] = p.x;
        (u & 1 ? b : a)[u | 1] = p.y;
      }
      swap4(a, b);  // a lane has dims 8 hf .. + 7 of the block's first and second 16
      uint32_t x[4] = {a[0], a[1], b[0], b[1]}, z[4] = {a[2], a[3], b[2], b[3]};
      swap_rows4(x, z);
      const long at = at0 + 32 * cc + 16 * r1 + 8 * hf;
      if (ok[0])
        *reinterpret_cast<uint4*>(static_cast<uint16_t*>(out) + at + l16 * stride) = make_uint4(x[0], x[1], x[2], x[3]);
      if (ok[1])
        *reinterpret_cast<uint4*>(static_cast<uint16_t*>(out) + at + (16 + l16) * stride) = make_uint4(z[0], z[1], z[2], z[3]);
    }
  }
}

// ---------------------------------------------------------------- keys
// Group of width B: its positions of the 64 tokens into the accumulators.
template <int B, int KWB>
__device__ __forceinline__ void key_group(const uint8_t* smem, const uint32_t (&rw)[KWB + split_detail::kRowPad],
                                          uint32_t gm, int step0, int lane, float16_t (&acc)[2][4]) {
  constexpr int NW = (16 * B + 31) / 32;
  const int o = split_detail::gm_off(gm), n16 = (split_detail::gm_steps(gm) + 3) >> 2;
  for (int c = 0; c < n16; ++c) {
    const int at = o + c * 16 * B, w0 = at >> 5, sh = at & 31;
    uint32_t aw[NW + 1];
#pragma unroll
    for (int i = 0; i < NW; ++i) aw[i] = __builtin_amdgcn_alignbit(rw[w0 + i + 1], rw[w0 + i], sh);
    aw[NW] = 0;
    const half2_t y[8] = {pair_at<B, 0>(smem, aw),      pair_at<B, 2 * B>(smem, aw),  pair_at<B, 4 * B>(smem, aw),
                          pair_at<B, 6 * B>(smem, aw),  pair_at<B, 8 * B>(smem, aw),  pair_at<B, 10 * B>(smem, aw),
                          pair_at<B, 12 * B>(smem, aw), pair_at<B, 14 * B>(smem, aw)};
    // the step's matrix operands, in flight with the lookups
    const uint8_t* mat = smem + kMat + (step0 + c) * 4096 + lane * 16;
    half8_t ops[4], lows[4];
#pragma unroll
    for (int cc = 0; cc < 4; ++cc) {
      ops[cc] = *reinterpret_cast<const half8_t*>(mat + cc * 1024);
      lows[cc] = *reinterpret_cast<const half8_t*>(mat + kMaxSteps * 4096 + cc * 1024);
    }
    __builtin_amdgcn_sched_barrier(0);
    uint32_t code[2][4];
#pragma unroll
    for (int u = 0; u < 8; ++u) code[u >> 2][u & 3] = __builtin_bit_cast(uint32_t, y[u]);
    swap4(code[0], code[1]);
#pragma unroll
    for (int cc = 0; cc < 4; ++cc) {
#pragma unroll
      for (int n = 0; n < 2; ++n)
        acc[n][cc] = __builtin_amdgcn_mfma_f32_32x32x16_f16(ops[cc], as_half8(code[n]), acc[n][cc], 0, 0, 0);
#pragma unroll
      for (int n = 0; n < 2; ++n)
        acc[n][cc] = __builtin_amdgcn_mfma_f32_32x32x16_f16(lows[cc], as_half8(code[n]), acc[n][cc], 0, 0, 0);
    }
  }
}

template <int KWB, int... BM1>
__device__ __forceinline__ void key_groups(std::integer_sequence<int, BM1...>, const uint8_t* smem,
                                           const uint32_t (&rw)[KWB + split_detail::kRowPad], const uint32_t (&gm)[8],
                                           int lane, float16_t (&acc)[2][4]) {
  int step0 = 0;
  const auto one = [&](auto bm1) __attribute__((always_inline)) {
    constexpr int b = decltype(bm1)::value;
    if (gm[b] >> 31) {
      key_group<b + 1, KWB>(smem, rw, gm[b], step0, lane, acc);
      step0 += (split_detail::gm_steps(gm[b]) + 3) >> 2;
    }
  };
  (one(std::integral_constant<int, BM1>{}), ...);
}

// Each dim times its group's radius: r[n] = the 8 radii of token l32 of block n.
__device__ __forceinline__ void scale_keys(const uint8_t* smem, const uint32_t (&r)[2][4], int lane, float16_t (&acc)[2][4]) {
#pragma unroll
  for (int cc = 0; cc < 4; ++cc)
#pragma unroll
    for (int u = 0; u < 4; ++u) {  // dims 32 cc + 8 u + 4 hf .. + 3
      const uint4 sel = *reinterpret_cast<const uint4*>(smem + kSel + (8 * cc + 2 * u + (lane >> 5)) * 16);
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        const half2_t x = __builtin_bit_cast(half2_t, __builtin_amdgcn_perm(r[n][1], r[n][0], sel.x) |
                                                          __builtin_amdgcn_perm(r[n][3], r[n][2], sel.z));
        const half2_t y = __builtin_bit_cast(half2_t, __builtin_amdgcn_perm(r[n][1], r[n][0], sel.y) |
                                                          __builtin_amdgcn_perm(r[n][3], r[n][2], sel.w));
        acc[n][cc][4 * u] *= static_cast<float>(x[0]);
        acc[n][cc][4 * u + 1] *= static_cast<float>(x[1]);
        acc[n][cc][4 * u + 2] *= static_cast<float>(y[0]);
        acc[n][cc][4 * u + 3] *= static_cast<float>(y[1]);
      }
    }
}

template <int KWB, bool F32>
__device__ __forceinline__ void read_keys(uint8_t* smem, const Dims& d, const uint8_t* __restrict__ blob,
                                          const RowsCall& call, int lz, int kvh, int chunk, long pos, int end) {
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int layer = d.layer >= 0 ? d.layer : lz / d.batch, seq = lz % d.batch, ri = layer * d.n_kv + kvh;
  const RowMeta* M = reinterpret_cast<const RowMeta*>(blob + kOffRows) + ri;
  const int ng = M->n_groups, nslot = (ng + 1) & ~1, kw = d.k_words;
  uint32_t gm[8], used = 0;
  int gd[8], gp[8];
#pragma unroll
  for (int b = 0; b < 8; ++b) {
    gm[b] = M->gm[b];
    used |= (gm[b] >> 31) << b;
    gd[b] = b < ng ? M->g_dim[b] : 0;
    gp[b] = M->g_pos[b];
  }
  const size_t row = (static_cast<size_t>(layer) * d.batch + seq) * d.n_kv + kvh;
  const size_t cap = d.capacity;
  const uint32_t* kc = call.c.k_codes + row * cap * kw;
  const uint16_t* kn = call.c.k_norms + row * kMaxGroups * cap;
  const int n_tiles = (call.n_rows + 63) / 64, first = chunk * call.tiles[0];
  const int last = min(n_tiles, first + call.tiles[0]);
  uint32_t nw[KWB], next_radii[4];
  bool next_valid;
  // a tile's words, a tile ahead (past the last one, row 0 again: in bounds, for nobody)
  const auto load = [&](int tile) {
    const int i = tile * 64 + lane;
    const long t = pos + i;
    next_valid = tile < last && i < call.n_rows && t >= 0 && t < end;
    const size_t tr = next_valid ? static_cast<size_t>(t) : 0;  // (any row of the cache: its result is not stored)
    const uint32_t* src = kc + tr * kw;
    if ((kw & 3) == 0) {
#pragma unroll
      for (int k = 0; k < KWB; k += 4) {
        const uint4 v = k < kw ? *reinterpret_cast<const uint4*>(src + k) : make_uint4(0, 0, 0, 0);
        nw[k] = v.x;
        nw[k + 1] = v.y;
        nw[k + 2] = v.z;
        nw[k + 3] = v.w;
      }
    } else {
#pragma unroll
      for (int k = 0; k < KWB; ++k) nw[k] = k < kw ? src[k] : 0u;
    }
    // (a token's 16 bytes of radii stay inside the row's 8 slots per token)
    const uint32_t* r = reinterpret_cast<const uint32_t*>(kn + tr * nslot);
#pragma unroll
    for (int k = 0; k < 4; ++k) next_radii[k] = r[k];
  };
  load(first + wave);

  // ---- the matrix A[dim][p] = 2^8 / sqrt(d_g) Pi_g[p - p_g][index of dim in
  // g], zero for dims of other groups and past a group's end; operand (step,
  // dim block cc, lane) = dim 32 cc + lane % 32, positions 8 (lane / 32) .. + 7
  // of the step.  The row's slot of the layout holds each Pi_g transposed.
  // Item = 8 numbers of one Pi_g, in memory order (dim after dim, contiguous
  // reads); the rest of the matrix is cleared.
  {
    const float* rot = reinterpret_cast<const float*>(blob + layout_rowrot_offset(d.n_layers * d.n_kv)) +
                       static_cast<size_t>(ri) * kRowRotFloats;
    const uint16_t* c16 = reinterpret_cast<const uint16_t*>(blob + kOffC16);
    const uint16_t cv = c16[min(tid, kCodebookEntries - 1)];
    const uint8_t dv = M->dim[tid & 127], gv = M->grp[tid & 127];
    int n_steps = 0, n_items = 0;
#pragma unroll
    for (int g = 0; g < 8; ++g) {
      n_steps += (gd[g] + 15) >> 4;
      n_items += gd[g] * 2 * ((gd[g] + 15) >> 4);
    }
    if (tid < kCodebookEntries) reinterpret_cast<uint16_t*>(smem + kBooks)[tid] = cv;
    for (int i = tid; i < n_steps * 256; i += kThreads) {
      *reinterpret_cast<uint4*>(smem + kMat + i * 16) = make_uint4(0, 0, 0, 0);
      *reinterpret_cast<uint4*>(smem + kMat + kMaxSteps * 4096 + i * 16) = make_uint4(0, 0, 0, 0);
    }
    if (tid < kHeadDim) {
      smem[kDims + tid] = dv;
      const uint16_t sel = static_cast<uint16_t>(2 * (gv & 3) | (2 * (gv & 3) + 1) << 8);
      uint8_t* at = smem + kSel + (dv >> 2) * 16 + (dv & 3) * 2;
      *reinterpret_cast<uint16_t*>(at) = gv < 4 ? sel : 0x0C0C;
      *reinterpret_cast<uint16_t*>(at + 8) = gv < 4 ? 0x0C0C : sel;
    }
    __syncthreads();
    build_pairs(smem, used, tid);
    for (int i0 = tid; i0 < n_items; i0 += kThreads) {
      int left = i0, dg = 2, p0 = 0, at = 0, st = 0, off = 0, base = 0;
      bool found = false;
#pragma unroll
      for (int g = 0; g < 8; ++g) {
        const int n16 = (gd[g] + 15) >> 4, n = gd[g] * 2 * n16;
        if (!found && left < n) {
          found = true;
          dg = gd[g];
          p0 = gp[g];
          at = off;
          st = base;
        }
        if (!found) left -= n;
        off += gd[g] * gd[g];
        base += n16;
      }
      const int per = 2 * ((dg + 15) >> 4), k = left / per, j0 = 8 * (left - k * per), dim = smem[kDims + p0 + k];
      const float* src = rot + at + k * dg + j0;
      const float scale = kMatScale * rsqrtf(static_cast<float>(dg));
      float x[8];
#pragma unroll
      for (int j = 0; j < 8; j += 2) {  // (group sizes are even, and so are the blocks' offsets)
        const float2_t v = j0 + j < dg ? *reinterpret_cast<const float2_t*>(src + j) : float2_t{0.f, 0.f};
        x[j] = v[0] * scale;
        x[j + 1] = v[1] * scale;
      }
      store_operand(smem + kMat + (st + (j0 >> 4)) * 4096 + (dim >> 5) * 1024 + (((j0 >> 3) & 1) * 32 + (dim & 31)) * 16,
                        kMaxSteps * 4096, x);
    }
  }
  __syncthreads();

  for (int tile = first + wave; tile < last; tile += kWaves) {
    uint32_t rw[KWB + split_detail::kRowPad], radii[4];
#pragma unroll
    for (int k = 0; k < KWB; ++k) rw[k] = nw[k];
#pragma unroll
    for (int k = KWB; k < KWB + split_detail::kRowPad; ++k) rw[k] = 0u;
#pragma unroll
    for (int k = 0; k < 4; ++k) radii[k] = next_radii[k];
    const bool valid = next_valid;
    load(tile + kWaves);
    float16_t acc[2][4];
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int cc = 0; cc < 4; ++cc)
#pragma unroll
        for (int k = 0; k < 16; ++k) acc[n][cc][k] = 0.f;
    key_groups<KWB>(std::make_integer_sequence<int, 8>{}, smem, rw, gm, lane, acc);
    uint32_t r[2][4];
#pragma unroll
    for (int k = 0; k < 4; ++k) r[0][k] = radii[k];
    spread4(r[0], r[1]);
    scale_keys(smem, r, lane, acc);
    const unsigned long long ok = __builtin_amdgcn_ballot_w64(valid);
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      // lane = token 32 n + l32 of the tile
      const long at = ((static_cast<long>(lz) * call.n_rows + tile * 64 + 32 * n) * d.n_kv + kvh) * kHeadDim;
      store_rows<F32>(acc[n], 1.f / kMatScale, call.out[0], at, static_cast<long>(d.n_kv) * kHeadDim,
                     static_cast<uint32_t>(ok >> (32 * n)), lane);
    }
  }
}

// ---------------------------------------------------------------- values
// A tile's codes (words of dims lane and 64 + lane) as fp16 centroids in LDS,
// token after token.
template <int BV>
__device__ __forceinline__ void decode_values(const uint8_t* smem, uint8_t* tile, const uint32_t (&words)[2][BV], int lane) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int dim = 64 * h + lane;
    uint32_t w[BV + 1];
#pragma unroll
    for (int i = 0; i < BV; ++i) w[i] = words[h][i];
    w[BV] = 0;
    const half2_t y[16] = {pair_at<BV, 0>(smem, w),       pair_at<BV, 2 * BV>(smem, w),  pair_at<BV, 4 * BV>(smem, w),
                           pair_at<BV, 6 * BV>(smem, w),  pair_at<BV, 8 * BV>(smem, w),  pair_at<BV, 10 * BV>(smem, w),
                           pair_at<BV, 12 * BV>(smem, w), pair_at<BV, 14 * BV>(smem, w), pair_at<BV, 16 * BV>(smem, w),
                           pair_at<BV, 18 * BV>(smem, w), pair_at<BV, 20 * BV>(smem, w), pair_at<BV, 22 * BV>(smem, w),
                           pair_at<BV, 24 * BV>(smem, w), pair_at<BV, 26 * BV>(smem, w), pair_at<BV, 28 * BV>(smem, w),
                           pair_at<BV, 30 * BV>(smem, w)};
#pragma unroll
    for (int u = 0; u < 16; ++u) {
      *reinterpret_cast<_Float16*>(tile + (2 * u) * kTileStride + 2 * dim) = y[u][0];
      *reinterpret_cast<_Float16*>(tile + (2 * u + 1) * kTileStride + 2 * dim) = y[u][1];
    }
  }
}

// The wave's tiles first, first + 8, .. below last, of cache tiles that hold a
// row below end; the next one's words are in flight.
template <bool F32, int BV>
__device__ __forceinline__ void value_tiles(const uint8_t* smem, uint8_t* mine, const Dims& d, const RowsCall& call,
                                            const uint32_t* __restrict__ vc, const uint16_t* __restrict__ vn, long first,
                                            long last, long pos, int end, int lz, int kvh, int lane) {
  const int l32 = lane & 31, hf = lane >> 5;
  uint32_t w[2][BV];
  uint16_t radius;
  const auto load = [&](long tile) {
    const size_t t = static_cast<size_t>(tile < last && tile >= 0 && tile * kTile < end ? tile : 0);  // (else for nobody)
    const uint32_t* src = vc + t * kHeadDim * BV;
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < BV; ++i) w[h][i] = src[(64 * h + lane) * BV + i];
    radius = vn[t * kTile + l32];
  };
  load(first);
  for (long tile = first; tile < last; tile += kWaves) {
    if (tile < 0 || tile * kTile >= end) {  // uniform
      load(tile + kWaves);
      continue;
    }
    const long t = tile * kTile + l32;
    const float scale = static_cast<float>(__builtin_bit_cast(_Float16, radius)) / kMatScale;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // the last tile's reads come before this one's writes
    decode_values<BV>(smem, mine, w, lane);
    load(tile + kWaves);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // a wave's LDS operations complete in order
    __builtin_amdgcn_wave_barrier();
    float16_t acc[4];
#pragma unroll
    for (int cc = 0; cc < 4; ++cc)
#pragma unroll
      for (int k = 0; k < 16; ++k) acc[cc][k] = 0.f;
#pragma unroll
    for (int st = 0; st < kVSteps; ++st) {
      const half8_t y = *reinterpret_cast<const half8_t*>(mine + l32 * kTileStride + 32 * st + 16 * hf);
      const uint8_t* mat = smem + kMat + st * 4096 + lane * 16;
#pragma unroll
      for (int cc = 0; cc < 4; ++cc)
        acc[cc] = __builtin_amdgcn_mfma_f32_32x32x16_f16(*reinterpret_cast<const half8_t*>(mat + cc * 1024), y, acc[cc], 0, 0, 0);
#pragma unroll
      for (int cc = 0; cc < 4; ++cc)
        acc[cc] = __builtin_amdgcn_mfma_f32_32x32x16_f16(
            *reinterpret_cast<const half8_t*>(mat + kVSteps * 4096 + cc * 1024), y, acc[cc], 0, 0, 0);
    }
    const long i = t - pos;
    const unsigned long long ok = __builtin_amdgcn_ballot_w64(i >= 0 && i < call.n_rows && t < end);
    const long at = ((static_cast<long>(lz) * call.n_rows + tile * kTile - pos) * d.n_kv + kvh) * kHeadDim;
    store_rows<F32>(acc, scale, call.out[1], at, static_cast<long>(d.n_kv) * kHeadDim, static_cast<uint32_t>(ok), lane);
  }
}

template <bool F32>
__device__ __forceinline__ void read_values(uint8_t* smem, const Dims& d, const uint8_t* __restrict__ blob,
                                            const RowsCall& call, int lz, int kvh, int chunk, long pos, int end) {
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int layer = d.layer >= 0 ? d.layer : lz / d.batch, seq = lz % d.batch;
  // A[dim][j] = 2^8 / sqrt(128) Pi_V[j][dim], read from the transposed Pi_V
  {
    const uint16_t* c16 = reinterpret_cast<const uint16_t*>(blob + kOffC16);
    const uint16_t cv = c16[min(tid, kCodebookEntries - 1)];
    const float* rot = reinterpret_cast<const float*>(blob + kOffRotVT);
    constexpr int kPer = kVSteps * 4 * 64 / kThreads;
    float4_t v[kPer][2];
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
      const int it = tid + u * kThreads, l = it & 63, cc = (it >> 6) & 3, st = it >> 8;
      const float4_t* src = reinterpret_cast<const float4_t*>(rot + (32 * cc + (l & 31)) * kHeadDim + 16 * st + 8 * (l >> 5));
      v[u][0] = src[0];
      v[u][1] = src[1];
    }
    if (tid < kCodebookEntries) reinterpret_cast<uint16_t*>(smem + kBooks)[tid] = cv;
    __syncthreads();
    build_pairs(smem, 1u << (d.v_bits - 1), tid);
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
      float x[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = v[u][j >> 2][j & 3] * (kMatScale * 0.08838834764831845f);
      store_operand(smem + kMat + (tid + u * kThreads) * 16, kVSteps * 4096, x);
    }
  }
  __syncthreads();
  const size_t row = (static_cast<size_t>(layer) * d.batch + seq) * d.n_kv + kvh;
  const size_t cap = d.capacity;
  const int bv = d.v_bits;
  const uint32_t* vc = call.c.v_codes + row * (cap / kTile) * kHeadDim * bv;
  const uint16_t* vn = call.c.v_norms + row * cap;
  uint8_t* const mine = smem + kMat + 2 * kVSteps * 4096 + wave * kTileBytes;
  // cache tiles from the one that holds the first row
  const long tile0 = pos >> 5, tile_end = (pos + call.n_rows + kTile - 1) >> 5;
  const long at = tile0 + chunk * static_cast<long>(call.tiles[1]), last = min(tile_end, at + call.tiles[1]);
  const auto go = [&](auto b) __attribute__((always_inline)) {
    value_tiles<F32, decltype(b)::value>(smem, mine, d, call, vc, vn, at + wave, last, pos, end, lz, kvh, lane);
  };
  switch (bv) {
    case 1: go(std::integral_constant<int, 1>{}); break;
    case 2: go(std::integral_constant<int, 2>{}); break;
    case 3: go(std::integral_constant<int, 3>{}); break;
    case 4: go(std::integral_constant<int, 4>{}); break;
    case 5: go(std::integral_constant<int, 5>{}); break;
    case 6: go(std::integral_constant<int, 6>{}); break;
    case 7: go(std::integral_constant<int, 7>{}); break;
    default: go(std::integral_constant<int, 8>{}); break;
  }
}

// One-dimensional grid: the keys' (unit, chunk) items, then the values'.
template <int KWB, bool F32>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2, 2))) void k_read_rows(
    Dims d, const uint8_t* __restrict__ blob, RowsCall call) {
  __shared__ __attribute__((aligned(16))) uint8_t smem[kLds];
  const bool keys = static_cast<int>(blockIdx.x) < call.key_items;
  int item = static_cast<int>(blockIdx.x) - (keys ? 0 : call.key_items);
  const int chunks = keys ? call.chunks[0] : call.chunks[1];
  const int chunk = item % chunks;
  item /= chunks;
  const int kvh = item % d.n_kv, lz = item / d.n_kv, seq = lz % d.batch;
  const long pos = call.read_pos[seq];
  const int end = min(d.capacity, call.ctx_len ? call.ctx_len[seq] : d.capacity);
  if (keys) read_keys<KWB, F32>(smem, d, blob, call, lz, kvh, chunk, pos, end);
  else read_values<F32>(smem, d, blob, call, lz, kvh, chunk, pos, end);
}

}  // namespace

hipError_t launch_dequantize_rows(const Dims& d, const void* layout, const CachePtrs& c, int n_rows,
                                  const int32_t* read_pos, const int32_t* ctx_len, void* k_out, void* v_out,
                                  int out_dtype, hipStream_t s) {
  RowsCall call = {};
  call.c = c;
  call.read_pos = read_pos;
  call.ctx_len = ctx_len;
  call.out[0] = k_out;
  call.out[1] = v_out;
  call.n_rows = n_rows;
  // One workgroup per CU: 256 of them share the units' tiles, a multiple of 8
  // (a tile per wave) each; of both sides' the keys get 9 / 16 (65536 random K2V2
  // rows x 8 heads to bf16, one side alone on all CUs: keys 64 us, values 49).  In
  // fp32 (83 and 97) 120 : 136 instead takes 175 us for 188 at 8 heads, but 55 for
  // 42 at 2, where it rounds to one tile more a wave: the same share for both.
  const long units = static_cast<long>(d.n_kv) * d.n_lc * d.batch;
  const bool both = k_out && v_out;
  long items = 0;
  for (int k = 0; k < 2; ++k) {
    const long n = k == 0 ? (n_rows + 63l) / 64 : (n_rows + 2l * kTile - 2) / kTile;  // (unaligned rows reach one tile more)
    const long want = std::max(1l, (both ? (k == 0 ? 144 : 112) : 256) / std::max(1l, units));
    call.tiles[k] = static_cast<int>(((n + want - 1) / want + kWaves - 1) / kWaves * kWaves);
    call.chunks[k] = static_cast<int>((n + call.tiles[k] - 1) / call.tiles[k]);
    if (call.out[k]) items += units * call.chunks[k];
    if (k == 0) call.key_items = static_cast<int>(items);
  }
  const auto go = [&](auto kern) {
    hipLaunchKernelGGL(kern, dim3(items), dim3(kThreads), 0, s, d, static_cast<const uint8_t*>(layout), call);
    return hipGetLastError();
  };
  const bool f32 = out_dtype == 0;  // BGTQ_FP32
  if (d.k_words <= 8) return f32 ? go(k_read_rows<8, true>) : go(k_read_rows<8, false>);
  if (d.k_words <= 12) return f32 ? go(k_read_rows<12, true>) : go(k_read_rows<12, false>);
  if (d.k_words <= 16) return f32 ? go(k_read_rows<16, true>) : go(k_read_rows<16, false>);
  return f32 ? go(k_read_rows<32, true>) : go(k_read_rows<32, false>);
}

}  // namespace bgtq
