// Attention over pages, instantiation for value code width 3 (see cross_impl.h).
#include "cross_impl.h"

namespace bgtq {
hipError_t launch_paged_bv3(const Dims& d, const void* layout, const void* q, const CrossCall& call, const PagedPass& pass,
                            hipStream_t s) {
  return cross_detail::launch_paged_bv<3>(d, layout, q, call, pass, s);
}
}  // namespace bgtq
