// Attention over pages, instantiation for value code width 1 (see cross_impl.h).
#include "cross_impl.h"

namespace bgtq {
hipError_t launch_paged_bv1(const Dims& d, const void* layout, const void* q, const CrossCall& call, const PagedPass& pass,
                            hipStream_t s) {
  return cross_detail::launch_paged_bv<1>(d, layout, q, call, pass, s);
}
}  // namespace bgtq
