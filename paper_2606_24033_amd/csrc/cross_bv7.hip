// Packed-row attention instantiation for value code width 7 (see cross_impl.h).
#include "cross_impl.h"

namespace bgtq {
hipError_t launch_cross_bv7(const Dims& d, const void* layout, const void* q, const CrossCall& call, hipStream_t s) {
  return cross_detail::launch_bv<7>(d, layout, q, call, s);
}
}  // namespace bgtq
