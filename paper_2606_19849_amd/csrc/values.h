// Pairs of bf16 values, looked at for those that are not finite (gfx950).
#pragma once

#include <stdint.h>

namespace vico {

// The largest exponent fields of the pairs seen so far, and the pair with zeros in the place of what is not finite.
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ void largest_exponents(u16x2& most, uint32_t x) {
  most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, x & 0x7F807F80u));
}
__device__ __forceinline__ bool not_finite(u16x2 most) { return (most[0] == 0x7F80) | (most[1] == 0x7F80); }
__device__ __forceinline__ uint32_t finite_or_zero(uint32_t x) {
  return x & ((x & 0x7F80u) == 0x7F80u ? 0xFFFF0000u : ~0u) & ((x & 0x7F800000u) == 0x7F800000u ? 0xFFFFu : ~0u);
}

}  // namespace vico
