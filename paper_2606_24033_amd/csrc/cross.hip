// Attention of many query rows to packed rows that all of them see: cross
// attention (query rows of a sequence against its whole cache) and the decode
// step of a batch that shares a prefix (every sequence's query against the
// prefix's cache and its own).
//
// Both are passes over one form: the query rows of a unit (layer, sequence,
// KV head) against rows [0, len) of one packed cache, the key axis in splits
// (k_cross, cross_impl.h).  A pass leaves per query row and split (m, l,
// acc[128]): the maximum of the base-2 logits, sum 2^(s - m) and
// sum 2^(s - m) v in the rotated value domain.  Partial states of disjoint row
// sets merge as
//   m = max m_i,  l = sum l_i 2^(m_i - m),  a = sum a_i 2^(m_i - m),
// so a shared prefix is one more set of splits: its pass, whose query rows are
// the batch's, and the sequences' own pass are one launch.  k_cross_merge joins a
// row's partials, divides by l, rotates back (Pi_V^T) and rounds to the output
// type; a row with a single partial is finished by k_cross itself.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "cross_impl.h"
#include "cross_merge.h"
#include "kernels.h"
#include "layout.h"

namespace bgtq {
namespace {

using namespace cross_detail;

struct RowsInOrder {  // partials of the output's rows, one after the other
  template <int RW>
  __device__ __forceinline__ bool begin(long) { return true; }
  __device__ __forceinline__ long out_row(long r) const { return r; }
};

}  // namespace

hipError_t launch_cross(const Dims& d, const void* layout, const void* q, const CrossCall& call, long rows,
                        hipStream_t s) {
  hipError_t e = hipSuccess;
  CrossCall rest = call;
  if (call.rows0 > 32) {
    Dims d0 = d;
    d0.batch = call.side[0].batch;
    e = launch_query_rotation(d0, layout, q, call.side[0].n_q, call.qr, s);
    if (e != hipSuccess) return e;
    e = call.out_dtype == 1 ? launch_cross_tile_bf16(d, layout, call.qr, call, call.rows0 == 128, s)
                            : launch_cross_tile_fp32(d, layout, call.qr, call, call.rows0 == 128, s);
    rest.side[0].items = 0;
  }
  if (e == hipSuccess && rest.side[0].items + rest.side[1].items > 0) {
    switch (d.v_bits) {
      case 1: e = launch_cross_bv1(d, layout, q, rest, s); break;
      case 2: e = launch_cross_bv2(d, layout, q, rest, s); break;
      case 3: e = launch_cross_bv3(d, layout, q, rest, s); break;
      case 4: e = launch_cross_bv4(d, layout, q, rest, s); break;
      case 5: e = launch_cross_bv5(d, layout, q, rest, s); break;
      case 6: e = launch_cross_bv6(d, layout, q, rest, s); break;
      case 7: e = launch_cross_bv7(d, layout, q, rest, s); break;
      default: e = launch_cross_bv8(d, layout, q, rest, s); break;
    }
  }
  if (e != hipSuccess || call.n_slots == 1) return e;
  // 16 rows to a workgroup where that fills the CUs; below, 4 rows, whose
  // partials four groups of threads read at once
  const auto merge = [&](auto kern, long blocks) {
    hipLaunchKernelGGL(kern, dim3(blocks), dim3(kThreads), 0, s, static_cast<const uint8_t*>(layout),
                       call.part, call.n_slots, rows, call.out, call.out_dtype, RowsInOrder{});
  };
  if (rows >= 16 * 256) merge(k_cross_merge<16, RowsInOrder>, std::min(kMergeGrid, (rows + 15) / 16));
  else merge(k_cross_merge<4, RowsInOrder>, (rows + 3) / 4);
  return hipGetLastError();
}

}  // namespace bgtq
