// Single tokens over pages, instantiation for value code width 1 (see paged_decode.h).
#include "paged_decode.h"

namespace bgtq {
hipError_t launch_paged_decode_bv1(const Dims& d, const void* layout, const void* q, const CrossCall& call,
                                   const PagedPass& pass, hipStream_t s) {
  return paged_decode_detail::launch_bv<1>(d, layout, q, call, pass, s);
}
}  // namespace bgtq
