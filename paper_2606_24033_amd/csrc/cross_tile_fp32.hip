// Wide attention passes (cross_tile.h) for fp32 outputs.
#include "cross_tile.h"

namespace bgtq {
hipError_t launch_cross_tile_fp32(const Dims& d, const void* layout, const float* qr, const CrossCall& call, bool half,
                                hipStream_t s) {
  return cross_tile_detail::launch_tile<true>(d, layout, qr, call, half, s);
}
}  // namespace bgtq
