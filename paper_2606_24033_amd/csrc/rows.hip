// Cache rows read back as plain keys and values: the inverse of
// blockgtq_quantize_append.
//
//   k_hat[d] = sum_p W[p][d] y[p],   y[p] = r_g C_b(code_p) / sqrt(d_g)
//   v_hat[d] = sum_j Pi_V[j][d] y[j], y[j] = n_V C_bV(code_j) / sqrt(128)
//
// with W the row's key rotation on the natural dims (zero outside position
// p's group g, so its transpose is its inverse).
#include <hip/hip_runtime.h>

#include "kernels.h"
#include "layout.h"

namespace bgtq {
namespace {

constexpr int kThreads = 128;  // one output dim per thread
constexpr int kRowsPerWg = 16;

__device__ __forceinline__ float half_bits(uint16_t b) { return static_cast<float>(__builtin_bit_cast(_Float16, b)); }

__device__ __forceinline__ void store_out(void* out, size_t i, float v, int dtype) {  // BGTQ_BF16 = 1
  if (dtype == 1) static_cast<__bf16*>(out)[i] = static_cast<__bf16>(v);
  else static_cast<float*>(out)[i] = v;
}

// grid (ceil(n_rows / kRowsPerWg), n_kv, n_lc * batch): fp32 sums, one row at a time.
__global__ __launch_bounds__(kThreads) void k_dequant_rows(Dims d, const uint8_t* __restrict__ blob, CachePtrs c,
                                                           int n_rows, const int32_t* __restrict__ read_pos,
                                                           const int32_t* __restrict__ ctx_len, void* __restrict__ k_out,
                                                           void* __restrict__ v_out, int out_dtype) {
  __shared__ float y[2][kHeadDim];
  const int p = threadIdx.x, kvh = blockIdx.y, lz = blockIdx.z;
  const int seq = lz % d.batch, layer = d.layer >= 0 ? d.layer : lz / d.batch;
  const RowMeta* M = reinterpret_cast<const RowMeta*>(blob + kOffRows) + (layer * d.n_kv + kvh);
  const int n_meta = d.n_layers * d.n_kv;
  const float* w = reinterpret_cast<const float*>(blob + layout_kdense_offset(n_meta)) +
                   static_cast<size_t>(layer * d.n_kv + kvh) * kMfmaMatFloats;
  const float* rv = reinterpret_cast<const float*>(blob + kOffRotV);
  const uint16_t* c16 = reinterpret_cast<const uint16_t*>(blob + kOffC16);
  const size_t row = (static_cast<size_t>(layer) * d.batch + seq) * d.n_kv + kvh;
  const uint32_t* kc = c.k_codes + row * d.capacity * d.k_words;
  const uint16_t* kn = c.k_norms + row * kMaxGroups * d.capacity;
  const uint32_t* vc = c.v_codes + row * (d.capacity / kTile) * kHeadDim * d.v_bits;
  const uint16_t* vn = c.v_norms + row * d.capacity;
  const int slots = (M->n_groups + 1) & ~1, width = M->width[p], off = M->bitoff[p], g = M->grp[p];
  const float kscale = rsqrtf(static_cast<float>(M->g_dim[g]));
  const int end = min(d.capacity, ctx_len ? ctx_len[seq] : d.capacity);
  for (int i = blockIdx.x * kRowsPerWg; i < min(n_rows, (static_cast<int>(blockIdx.x) + 1) * kRowsPerWg); ++i) {
    const long t = static_cast<long>(read_pos[seq]) + i;
    if (t < 0 || t >= end) continue;  // uniform
    const uint32_t* kr = kc + static_cast<size_t>(t) * d.k_words;
    const int k0 = off >> 5;
    uint64_t f = kr[k0];
    if ((off & 31) + width > 32) f |= static_cast<uint64_t>(kr[k0 + 1]) << 32;
    const uint32_t code = static_cast<uint32_t>(f >> (off & 31)) & ((1u << width) - 1u);
    y[0][p] = half_bits(c16[cb_index(width) + code]) * (half_bits(kn[static_cast<size_t>(t) * slots + g]) * kscale);
    const int vo = static_cast<int>(t % kTile) * d.v_bits, v0 = vo >> 5;
    const uint32_t* vr = vc + (static_cast<size_t>(t / kTile) * kHeadDim + p) * d.v_bits;
    f = vr[v0];
    if ((vo & 31) + d.v_bits > 32) f |= static_cast<uint64_t>(vr[v0 + 1]) << 32;
    const uint32_t vcode = static_cast<uint32_t>(f >> (vo & 31)) & ((1u << d.v_bits) - 1u);
    y[1][p] = half_bits(c16[cb_index(d.v_bits) + vcode]) * (half_bits(vn[t]) * 0.08838834764831845f);
    __syncthreads();
    float k = 0.f, v = 0.f;
    for (int j = 0; j < kHeadDim; ++j) {
      k = fmaf(w[mfma_mat_index(j, p)], y[0][j], k);
      v = fmaf(rv[j * kHeadDim + p], y[1][j], v);
    }
    const size_t o = ((static_cast<size_t>(lz) * n_rows + i) * d.n_kv + kvh) * kHeadDim + p;
    if (k_out) store_out(k_out, o, k, out_dtype);
    if (v_out) store_out(v_out, o, v, out_dtype);
    __syncthreads();
  }
}

}  // namespace

hipError_t launch_dequantize_rows(const Dims& d, const void* layout, const CachePtrs& c, int n_rows,
                                  const int32_t* read_pos, const int32_t* ctx_len, void* k_out, void* v_out,
                                  int out_dtype, hipStream_t s) {
  hipLaunchKernelGGL(k_dequant_rows, dim3((n_rows + kRowsPerWg - 1) / kRowsPerWg, d.n_kv, d.n_lc * d.batch),
                     dim3(kThreads), 0, s, d, static_cast<const uint8_t*>(layout), c, n_rows, read_pos, ctx_len, k_out,
                     v_out, out_dtype);
  return hipGetLastError();
}

}  // namespace bgtq
