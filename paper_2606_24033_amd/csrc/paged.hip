// Attention of a ragged batch's new tokens over pages: the passes of
// paged_pass.h and the join of their splits.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "cross_impl.h"
#include "cross_merge.h"
#include "kernels.h"
#include "paged_pass.h"

namespace bgtq {
namespace {

using namespace cross_detail;

// Partials [block][KV head][row of the unit]: those of rows that a sequence has.
template <int R>
struct UnitRows {
  PagedPass pass;
  int n_kv, group;
  paged::Unit u;
  __device__ __forceinline__ bool begin(long r) {
    const int unit = static_cast<int>(r / pass.unit_rows), first = static_cast<int>(r % pass.unit_rows);
    u.kvh = unit % n_kv;
    return paged::find_block<R>(pass, group, unit / n_kv, u) && u.q.ok && u.r0 + first < u.q.n * group;
  }
  __device__ __forceinline__ long out_row(long r) const {
    const int i = u.r0 + static_cast<int>(r % pass.unit_rows);
    return i < u.q.n * group ? (static_cast<long>(u.q.first) + i / group) * n_kv * group + u.kvh * group + i % group : -1;
  }
};

template <int R>
hipError_t join(const Dims& d, const void* layout, const CrossCall& call, const PagedPass& pass, hipStream_t s) {
  const long rows = static_cast<long>(pass.n_blocks) * d.n_kv * pass.unit_rows;
  const UnitRows<R> map{pass, d.n_kv, d.group, {}};
  const auto go = [&](auto kern, long blocks) {
    hipLaunchKernelGGL(kern, dim3(blocks), dim3(kThreads), 0, s, static_cast<const uint8_t*>(layout), call.part, call.n_slots,
                       rows, call.out, call.out_dtype, map);
    return hipGetLastError();
  };
  if (rows >= 16 * 256 && pass.unit_rows % 16 == 0) return go(k_cross_merge<16, UnitRows<R>>, std::min(kMergeGrid, rows / 16));
  return go(k_cross_merge<4, UnitRows<R>>, rows / 4);
}

}  // namespace

hipError_t launch_paged_pass(const Dims& d, const void* layout, const void* q, const CrossCall& call, const PagedPass& pass,
                             hipStream_t s) {
  hipError_t e;
  if (call.rows0 > 32) {
    e = call.out_dtype == 1 ? launch_paged_tile_bf16(d, layout, call, pass, s) : launch_paged_tile_fp32(d, layout, call, pass, s);
  } else if (call.rows0 == 8) {
    switch (d.v_bits) {
      case 1: e = launch_paged_decode_bv1(d, layout, q, call, pass, s); break;
      case 2: e = launch_paged_decode_bv2(d, layout, q, call, pass, s); break;
      case 3: e = launch_paged_decode_bv3(d, layout, q, call, pass, s); break;
      case 4: e = launch_paged_decode_bv4(d, layout, q, call, pass, s); break;
      case 5: e = launch_paged_decode_bv5(d, layout, q, call, pass, s); break;
      case 6: e = launch_paged_decode_bv6(d, layout, q, call, pass, s); break;
      case 7: e = launch_paged_decode_bv7(d, layout, q, call, pass, s); break;
      default: e = launch_paged_decode_bv8(d, layout, q, call, pass, s); break;
    }
  } else {
    switch (d.v_bits) {
      case 1: e = launch_paged_bv1(d, layout, q, call, pass, s); break;
      case 2: e = launch_paged_bv2(d, layout, q, call, pass, s); break;
      case 3: e = launch_paged_bv3(d, layout, q, call, pass, s); break;
      case 4: e = launch_paged_bv4(d, layout, q, call, pass, s); break;
      case 5: e = launch_paged_bv5(d, layout, q, call, pass, s); break;
      case 6: e = launch_paged_bv6(d, layout, q, call, pass, s); break;
      case 7: e = launch_paged_bv7(d, layout, q, call, pass, s); break;
      default: e = launch_paged_bv8(d, layout, q, call, pass, s); break;
    }
  }
  if (e != hipSuccess || call.n_slots == 1) return e;
  if (call.rows0 == 8) return join<8>(d, layout, call, pass, s);
  return call.rows0 == 32 ? join<32>(d, layout, call, pass, s)
                          : call.rows0 == 128 ? join<128>(d, layout, call, pass, s) : join<256>(d, layout, call, pass, s);
}

}  // namespace bgtq
