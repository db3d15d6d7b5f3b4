// Wide attention passes over pages (cross_tile.h) for bf16 outputs.
#include "cross_tile.h"

namespace bgtq {
hipError_t launch_paged_tile_bf16(const Dims& d, const void* layout, const CrossCall& call, const PagedPass& pass,
                                hipStream_t s) {
  const bool half = call.rows0 == 128;
  if (pass.m.cap > 0.f || pass.m.slopes)
    return cross_tile_detail::launch_tile<false>(d, layout, call.qr, call, half, paged::Mode<true>{pass}, s);
  return cross_tile_detail::launch_tile<false>(d, layout, call.qr, call, half, paged::Mode<false>{pass}, s);
}
}  // namespace bgtq
