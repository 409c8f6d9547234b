// The 4-bit store of keys and values (gfx950), and what its kernels share.
//
// A token's row of one head is D/2 bytes of codes and D/32 scale bytes:
// element 2i in the low four bits of byte i, element 2i+1 in the high four; a
// code is a sign and one of 0, .5, 1, 1.5, 2, 3, 4, 6 (e2m1); every 32
// elements share a power of two 2^(byte - 127), byte 255 makes them all NaN.
// The matrix cores' own conversion (v_cvt_scalef32_pk_bf16_fp4) turns two
// codes and their scale into two bf16 values, exactly: a value has two
// significant bits.  The append writes bytes 4 .. 252 and 255; of the others, 0
// to 3 make exact subnormals, 253 and 254 infinities of values from 2^128 on.
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

// The kernel's arguments, read again from memory where they are used: what only the start, the end or the bf16
// blocks need takes no scalar registers (and, spilled, no vector ones) in the store's loop.
typedef const __attribute__((address_space(4))) RowsQ4Args* late_args;
__device__ __forceinline__ late_args late() {
  late_args p = (late_args)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  return p;
}

// Pairs of bf16 values that are not finite: the largest exponent fields of the pairs seen so far, and the pair with
// zeros in their place.
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ void largest_exponents(u16x2& most, uint32_t x) {
  most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, x & 0x7F807F80u));
}
__device__ __forceinline__ bool not_finite(u16x2 most) { return (most[0] == 0x7F80) | (most[1] == 0x7F80); }
__device__ __forceinline__ uint32_t finite_or_zero(uint32_t x) {
  return x & ((x & 0x7F80u) == 0x7F80u ? 0xFFFF0000u : ~0u) & ((x & 0x7F800000u) == 0x7F800000u ? 0xFFFFu : ~0u);
}

// The segment table of a work-group of NT threads.  The lanes of every wave
// hold a window of 64 segments: `incl`, keys up to a segment's end, and
// `shift`, from gathered key to slot.  Up to 64 segments that is all, and no
// LDS or barrier stands between the table and the first key load; more are
// scanned by the work-group into LDS, and a wave moves its window as it goes:
// keys are asked for in rising order.  Segments are clipped to the store.
template <int NT>
struct Segments {
  static constexpr int PER = kMaxSegments / NT;
  static_assert(PER * NT == kMaxSegments, "segments of a thread");
  struct Lds {
    int incl[kMaxSegments], shift[kMaxSegments], wave[NT / 64];
  };
  static __device__ __forceinline__ int clipped(const int64_t* start, const int32_t* length, int s, int cap, int& slot) {
    const int64_t st = start[s], en = st + (int64_t)length[s];
    const int64_t lo = st > 0 ? st : 0, hi = en < (int64_t)cap ? en : (int64_t)cap;
    slot = hi > lo ? (int)lo : 0;
    return hi > lo ? (int)(hi - lo) : 0;
  }
  // inclusive sum over the lanes up to this one: inside the rows of 16, then across them
  static __device__ __forceinline__ int scan(int x) {
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, true);       // row_shr 1, 2, 4, 8: 0 from outside of the row
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xA, 0xF, false);      // lane 15 of a row to the next one: rows 1, 3
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xC, 0xF, false);      // lane 31 to rows 2, 3
    return x;
  }
  // The state is the kernel's locals, the table in LDS, the lanes' window of it and the window's first segment:
  Lds& l;
  int &incl, &shift, &win;

  // every thread of the work-group calls this; returns the keys of all segments
  __device__ __forceinline__ int build(const int64_t* start, const int32_t* length, int n, int cap) const {
    const int tid = threadIdx.x, lane = tid & 63;
    win = 0;
    int slot = 0;
    if (n <= 64) {
      const int len = lane < n ? clipped(start, length, lane, cap, slot) : 0;
      incl = scan(len);
      shift = slot - (incl - len);
      return __builtin_amdgcn_readlane(incl, 63);
    }
    int len[PER], run = 0;
#pragma unroll
    for (int e = 0; e < PER; ++e) {
      const int s = tid * PER + e;
      len[e] = s < n ? clipped(start, length, s, cap, slot) : 0;
      l.shift[s] = slot;
      run += len[e];
    }
    const int upto = scan(run);
    if (lane == 63) l.wave[tid >> 6] = upto;
    __syncthreads();
    int base = upto - run;
    for (int w = 0; w < (tid >> 6); ++w) base += l.wave[w];
#pragma unroll
    for (int e = 0; e < PER; ++e) {
      const int s = tid * PER + e;
      l.shift[s] -= base;
      base += len[e];
      l.incl[s] = base;
    }
    __syncthreads();
    incl = l.incl[lane];
    shift = l.shift[lane];
    return __builtin_amdgcn_readfirstlane(l.incl[kMaxSegments - 1]);
  }
  // segment of gathered key i (0 <= i < the total) inside the window, which moves there
  __device__ __forceinline__ int find(int i) const {
    while (__builtin_amdgcn_readlane(incl, 63) <= i) {      // entries past the last segment hold the total
      win += 64;
      incl = l.incl[win + (threadIdx.x & 63)];
      shift = l.shift[win + (threadIdx.x & 63)];
    }
    return __builtin_popcountll(__builtin_amdgcn_ballot_w64(incl <= i));
  }
  // how many keys from i on lie in consecutive slots, from slot0
  __device__ __forceinline__ int straight(int i, int& slot0) const {
    const int s = find(i);
    slot0 = i + __builtin_amdgcn_readlane(shift, s);
    return __builtin_amdgcn_readlane(incl, s) - i;
  }
  // slot of key i0 + lane % n (n: a power of two); a key past the last, `total` - 1, has its slot and real = false
  __device__ __forceinline__ int slot_of_lane(int i0, int n, int total, bool& real) const {
    const int i = i0 + (int)(threadIdx.x & (n - 1)), end = min(i0 + n, total);
    int s = find(i0), slot = 0, last = 0, begin = i0;
    while (begin < end) {
      const int e = __builtin_amdgcn_readlane(incl, s), d = __builtin_amdgcn_readlane(shift, s);
      slot = ((i >= begin) & (i < e)) ? i + d : slot;
      last = e > begin ? min(e, end) - 1 + d : last;
      begin = max(begin, e);
      if (++s == 64 && begin < end) s = find(begin);
    }
    real = i < end;
    return real ? slot : last;
  }
};

}  // namespace vico
