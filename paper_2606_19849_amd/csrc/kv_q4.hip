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
// Both kernels move bytes, 2.53 a value, and are bound by memory or, for one
// chunk, by the launch.  A thread takes units of 8 elements: 16 bytes on the bf16
// side, 4 of codes; four lanes share a group (amax and the scale byte by two DPP
// steps).  7B heads, medians of a trace: append of 2048 tokens (5.3 MB) 3.5 us, of 77
// tokens (3B heads) 2.6; load of 32 chunks, 17.6k rows (45.5 MB), 8.4 to 9.4 us by the
// box, 4.9 to 5.4 TB/s.

#include <algorithm>

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

// Rows of the concatenated segments, as bf16; blockIdx.y picks K or V.  A wave
// takes `per_wave` rows: lane l finds the slot of row l, then the wave walks the
// rows' 8-element units, 64 at a time, kLoadAhead of them on the way.
constexpr int kLoadRows = 16, kLoadAhead = 4;      // most rows of a wave
constexpr int kLoadWaves = 4096;                   // 16 a CU: as many as hide the loads' latency

__global__ __launch_bounds__(kQ4Threads) void kv_load_q4_kernel(LoadQ4Args a) {
  __shared__ Segments<kQ4Threads>::Lds seg_s;
  const int tid = threadIdx.x, lane = tid & 63;
  int incl, shift, win;
  const Segments<kQ4Threads> seg{seg_s, incl, shift, win};
  const int G = seg.build(a.seg_start, a.seg_len, a.n_segs, a.cap), rows = min(G, a.out_rows);
  if (a.out_count && blockIdx.x == 0 && blockIdx.y == 0 && tid == 0) *a.out_count = G;

  const int upt = a.row_elems >> 3;
  const uint8_t* src = blockIdx.y ? a.v4 : a.k4;
  const uint8_t* ssc = blockIdx.y ? a.vs : a.ks;
  uint16_t* dst = blockIdx.y ? a.v : a.k;
  const int wave = __builtin_amdgcn_readfirstlane(blockIdx.x * (kQ4Threads / 64) + (tid >> 6));
  const int64_t first = (int64_t)wave * a.per_wave;
  if (first >= rows) return;
  const int r0 = (int)first;
  bool real;
  const int slot = seg.slot_of_lane(r0, a.per_wave, G, real);
  const int units = min(a.per_wave, rows - r0) * upt;
  uint16_t* const out = dst + (int64_t)r0 * a.row_elems;
  for (int u0 = lane; u0 - lane < units; u0 += 64 * kLoadAhead) {
    uint32_t w[kLoadAhead], b[kLoadAhead];
#pragma unroll
    for (int k = 0; k < kLoadAhead; ++k) {
      const int u = min(u0 + 64 * k, units - 1), r = a.by_units(u);     // past the end: the last unit, not stored
      const int64_t at = (int64_t)__shfl(slot, r, 64) * upt + (u - r * upt);
      w[k] = *(const uint32_t*)(src + at * 4);
      b[k] = ssc[at >> 2];
    }
#pragma unroll
    for (int k = 0; k < kLoadAhead; ++k)
      if (u0 + 64 * k < units) *(u32x4*)(out + (int64_t)(u0 + 64 * k) * 8) = q4_eight(w[k], q4_scale(b[k]));
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

hipError_t launch_load_q4(const LoadQ4Args& args, hipStream_t stream) {
  LoadQ4Args a = args;
  a.by_units = FastDiv::by(a.row_elems >> 3);
  // Rows of a wave: enough for a load of 64 units, and more (a power of two) where that leaves kLoadWaves waves.
  // 2048 rows of 64 units 6.0 us with 16 rows a wave, 2.9 with 1; 17.8k rows 8.6 / 8.6.
  a.per_wave = 1;
  while (a.per_wave < kLoadRows && (a.per_wave * (a.row_elems >> 3) < 64 || int64_t(a.out_rows) >= int64_t(a.per_wave) * kLoadWaves))
    a.per_wave *= 2;
  const int64_t per_block = (int64_t)a.per_wave * (kQ4Threads / 64);
  const unsigned blocks = (unsigned)std::max<int64_t>((a.out_rows + per_block - 1) / per_block, 1);
  hipLaunchKernelGGL(kv_load_q4_kernel, dim3(blocks, 2), dim3(kQ4Threads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace vico
