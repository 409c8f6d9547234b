// The 4-bit store of keys and values: writing a chunk, reading segments back
// (gfx950).  The paper keeps every past chunk's visual K/V for query-time
// retrieval (ViCoStream Sec. 3); held in 4 bits that store takes 34 bytes for
// 64 values instead of 128.
//
// Append: ring slot (hist_len + j) mod R <- chunk token j, for K and V.  A
// group of 32 elements has amax = max |x|; its scale is the smallest power of
// two s with amax <= 7 s, so that the largest element, which may round down to
// 6 s, is no further off than half the last step (4 s to 6 s).  On bf16 bits
// that is one addition: (bits(amax) + 0x1F) >> 7 raises the exponent where the
// fraction is above 1.75.  The codes are x / s to the nearest, ties to the
// even code, by v_cvt_scalef32_pk_fp4_bf16.
//
// Both kernels move bytes: 2.5 bytes of work per value of which 2 are bf16.  A
// thread takes 8 elements: 16 bytes on the bf16 side, 4 of codes; four lanes
// share a group (amax and the scale byte by two DPP steps).

#include "q4_common.h"

namespace vico {
namespace {

constexpr int kQ4Threads = 256;

// max over the four lanes of a quad
__device__ __forceinline__ uint32_t quad_max(uint32_t x) {
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0xB1, 0xF, 0xF, false));   // lanes 1 0 3 2
  return max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x4E, 0xF, 0xF, false)); // lanes 2 3 0 1
}

__device__ __forceinline__ uint32_t abs_max(u32x4 x) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) m = max(m, max((x[i] << 16) & 0x7FFF0000u, x[i] & 0x7FFF0000u));
  return m >> 16;
}

// The scale byte of a group with largest magnitude `amax` (bf16 bits without the sign).
__device__ __forceinline__ uint32_t q4_scale_byte(uint32_t amax) {
  const int b = (int)((amax + 0x1F) >> 7) - 2;
  return amax >= 0x7F80 ? kQ4Nan : (uint32_t)min(max(b, (int)kQ4MinScale), (int)kQ4MaxScale);
}

__device__ __forceinline__ uint32_t q4_encode(u32x4 x, uint32_t byte) {
  if (byte == kQ4Nan) return 0;
  const float s = q4_scale(byte);
  // by value: a bit cast of a vector's element would take the vector's first one
  auto two = [&](uint32_t p) __attribute__((always_inline)) { return __builtin_bit_cast(bf16x2, p); };
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, two(x[0]), s, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, two(x[1]), s, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, two(x[2]), s, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, two(x[3]), s, 3);
  return w;
}

// blockIdx.y picks K (0) or V (1).  A thread's unit is 8 elements; the four
// lanes of a group are always in range together (32 divides the row).
__global__ __launch_bounds__(kQ4Threads) void kv_append_q4_kernel(AppendQ4Args a) {
  const int upt = a.row_elems >> 3;
  const int64_t total = (int64_t)a.C * upt;
  const uint16_t* src = blockIdx.y ? a.vc : a.kc;
  uint8_t* dst = blockIdx.y ? a.v4 : a.k4;
  uint8_t* dsc = blockIdx.y ? a.vs : a.ks;
  const int64_t step = (int64_t)gridDim.x * blockDim.x;
  for (int64_t u = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; u < total; u += step) {
    const int j = (int)(u / upt);
    const int c = (int)(u - (int64_t)j * upt);
    int64_t slot = (int64_t)a.p0 + j;
    if (slot >= a.R) slot -= a.R;
    const u32x4 x = *(const u32x4*)(src + u * 8);
    const uint32_t byte = q4_scale_byte(quad_max(abs_max(x)));
    const int64_t at = slot * upt + c;
    *(uint32_t*)(dst + at * 4) = q4_encode(x, byte);
    if ((c & 3) == 0) dsc[at >> 2] = (uint8_t)byte;
  }
}

// Rows of the concatenated segments, as bf16.  Every work-group builds the
// prefix sums of the clipped segment lengths in LDS; a row's segment is found
// by bisection.
__global__ __launch_bounds__(kQ4Threads) void kv_load_q4_kernel(LoadQ4Args a) {
  constexpr int PER = kMaxSegments / kQ4Threads;
  __shared__ int incl_s[kMaxSegments], shift_s[kMaxSegments];
  __shared__ int wave_s[kQ4Threads / 64];
  const int tid = threadIdx.x, lane = tid & 63;
  int len[PER], run = 0;
#pragma unroll
  for (int e = 0; e < PER; ++e) {
    const int i = tid * PER + e;
    len[e] = 0;
    int slot = 0;
    if (i < a.n_segs) {
      const int64_t st = a.seg_start[i], en = st + a.seg_len[i];
      const int64_t lo = st > 0 ? st : 0, hi = en < a.cap ? en : a.cap;
      if (hi > lo) { len[e] = (int)(hi - lo); slot = (int)lo; }
    }
    shift_s[i] = slot;
    run += len[e];
  }
  int incl = run;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(incl, o, 64);
    if (lane >= o) incl += y;
  }
  if (lane == 63) wave_s[tid >> 6] = incl;
  __syncthreads();
  int base = incl - run;
  for (int w = 0; w < (tid >> 6); ++w) base += wave_s[w];
#pragma unroll
  for (int e = 0; e < PER; ++e) {
    const int i = tid * PER + e;
    shift_s[i] -= base;
    base += len[e];
    incl_s[i] = base;
  }
  __syncthreads();
  const int G = incl_s[kMaxSegments - 1], rows = min(G, a.out_rows);
  if (a.out_count && blockIdx.x == 0 && blockIdx.y == 0 && tid == 0) *a.out_count = G;

  const int upt = a.row_elems >> 3;
  const uint8_t* src = blockIdx.y ? a.v4 : a.k4;
  const uint8_t* ssc = blockIdx.y ? a.vs : a.ks;
  uint16_t* dst = blockIdx.y ? a.v : a.k;
  const int64_t total = (int64_t)rows * upt, step = (int64_t)gridDim.x * blockDim.x;
  for (int64_t u = (int64_t)blockIdx.x * blockDim.x + tid; u < total; u += step) {
    const int i = (int)(u / upt);
    const int c = (int)(u - (int64_t)i * upt);
    int s = 0;                           // the first segment whose end is past i
#pragma unroll
    for (int h = kMaxSegments / 2; h > 0; h >>= 1)
      if (incl_s[s + h - 1] <= i) s += h;
    const int64_t at = (int64_t)(i + shift_s[s]) * upt + c;
    *(u32x4*)(dst + u * 8) = q4_eight(*(const uint32_t*)(src + at * 4), q4_scale(ssc[at >> 2]));
  }
}

unsigned blocks_for(int64_t units) {
  const int64_t b = (units + kQ4Threads - 1) / kQ4Threads;
  return (unsigned)(b > 4096 ? 4096 : b < 1 ? 1 : b);
}

}  // namespace

hipError_t launch_append_q4(const AppendQ4Args& a, hipStream_t stream) {
  hipLaunchKernelGGL(kv_append_q4_kernel, dim3(blocks_for((int64_t)a.C * (a.row_elems >> 3)), 2), dim3(kQ4Threads), 0,
                     stream, a);
  return hipGetLastError();
}

hipError_t launch_load_q4(const LoadQ4Args& a, hipStream_t stream) {
  hipLaunchKernelGGL(kv_load_q4_kernel, dim3(blocks_for((int64_t)a.out_rows * (a.row_elems >> 3)), 2),
                     dim3(kQ4Threads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace vico
