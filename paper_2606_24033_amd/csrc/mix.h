// Softmax weights times value radii, packed as fp16 operands (prefill.hip,
// decode_impl.h).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace bgtq {

// fp16(p0 lo(w)) | fp16(p1 hi(w)) << 16, w = two fp16: one mixed-precision
// product into each half (v_fma_mixlo_f16, v_fma_mixhi_f16).  In C++ and not in
// inline asm: p0 and p1 come straight from v_exp_f32, and gfx950 wants a wait
// state between a transcendental instruction and a plain VALU one that reads
// its result.  The compiler keeps it only for instructions that it knows; with
// asm here every prefill attention kernel had a product right behind its
// exponential.
__device__ __forceinline__ uint32_t mix_pair(float p0, float p1, uint32_t w) {
  typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
  const half2_t h = __builtin_bit_cast(half2_t, w);
  const half2_t r = {static_cast<_Float16>(__builtin_fmaf(p0, static_cast<float>(h[0]), 0.f)),
                     static_cast<_Float16>(__builtin_fmaf(p1, static_cast<float>(h[1]), 0.f))};
  return __builtin_bit_cast(uint32_t, r);
}

// Value radii enter a pass's products times a power of two that brings the
// largest one so far to [2^14, 2^15): weight times radius then keeps fp16's full
// precision for weights down to 2^-28 of the largest, whatever size the values
// have.  `top` is the running maximum of the radii's exponent fields (0: none
// yet); when it rises the accumulators are rescaled, as for a running maximum of
// the logits.
__device__ __forceinline__ int raise_top(int top, int e) {  // the largest of top and the lanes' e (0 .. 31)
  for (uint64_t more; (more = __builtin_amdgcn_ballot_w64(e > top)) != 0;)  // (each turn raises top)
    top = __builtin_amdgcn_readlane(e, __builtin_ctzll(more));
  return top;
}
__device__ __forceinline__ int radius_top(int top, uint32_t bits) {  // bits: a lane's radius, fp16
  const int f = static_cast<int>(bits >> 10 & 31u);
  return raise_top(top, f == 31 ? 0 : f);  // (not finite: no size)
}
__device__ __forceinline__ int radius_up(int top) { return 29 - max(top, 1); }
__device__ __forceinline__ uint32_t radius_times(uint32_t bits, int up) {  // 2^up times an fp16 number, as fp16
  const float r = static_cast<float>(__builtin_bit_cast(_Float16, static_cast<uint16_t>(bits)));
  return __builtin_bit_cast(uint16_t, static_cast<_Float16>(__builtin_amdgcn_ldexpf(r, up)));
}

}  // namespace bgtq
