// Wide attention passes (cross_tile.h) for bf16 outputs.
#include "cross_tile.h"

namespace bgtq {
hipError_t launch_cross_tile_bf16(const Dims& d, const void* layout, const float* qr, const CrossCall& call, bool half,
                                hipStream_t s) {
  return cross_tile_detail::launch_tile<false>(d, layout, qr, call, half, paged::WholeCache{}, s);
}
}  // namespace bgtq
