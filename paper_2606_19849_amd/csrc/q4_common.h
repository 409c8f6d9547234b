// The 4-bit store of keys and values (gfx950), and what its kernels share.
//
// A token's row of one head is D/2 bytes of codes and D/32 scale bytes:
// element 2i in the low four bits of byte i, element 2i+1 in the high four; a
// code is a sign and one of 0, .5, 1, 1.5, 2, 3, 4, 6 (e2m1); every 32
// elements share a power of two 2^(byte - 127), byte 255 makes them all NaN.
// The matrix cores' own conversion (v_cvt_scalef32_pk_bf16_fp4) turns two
// codes and their scale into two bf16 values, exactly: a value has two
// significant bits.
#pragma once

#include "attn_common.h"

namespace vico {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int kQ4Group = 32;             // elements that share a scale
constexpr uint32_t kQ4MinScale = 4;      // 2^-123: no value of the store, and none rounded to it, is subnormal in bf16
constexpr uint32_t kQ4MaxScale = 252;    // 2^125: 6 * 2^125 is the store's largest value
constexpr uint32_t kQ4Nan = 255;

// Codes 2*sel and 2*sel + 1 of w, times `scale` (a power of two), as two bf16 values.
template <int SEL>
__device__ __forceinline__ uint32_t q4_pair(uint32_t w, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, SEL));
}

// The eight codes of w as bf16 values, in order.
__device__ __forceinline__ u32x4 q4_eight(uint32_t w, float scale) {
  return u32x4{q4_pair<0>(w, scale), q4_pair<1>(w, scale), q4_pair<2>(w, scale), q4_pair<3>(w, scale)};
}

__device__ __forceinline__ float q4_scale(uint32_t byte) { return __uint_as_float(byte << 23); }

}  // namespace vico
