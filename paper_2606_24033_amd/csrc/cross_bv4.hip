// Packed-row attention instantiation for value code width 4 (see cross_impl.h).
#include "cross_impl.h"

namespace bgtq {
hipError_t launch_cross_bv4(const Dims& d, const void* layout, const void* q, const CrossCall& call, hipStream_t s) {
  return cross_detail::launch_bv<4>(d, layout, q, call, s);
}
}  // namespace bgtq
