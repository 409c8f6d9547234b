// Norms of queries and keys for each head with the position rotation, from
// the packed projection to the dense q, k, v of the attention calls (gfx950).
//
// For a token and a head, in fp32, rounded to bf16 once at the end:
//     x' = x * w / sqrt(mean(x^2) + eps)                  (x' = x without w)
//     y0 = x0' cos a - x1' sin a,  y1 = x1' cos a + x0' sin a
// for every pair (x0, x1) of the first `rot` elements: elements i and i + rot/2,
// or 2i and 2i + 1; a = position(t, axis of i) * inv_freq[i].  A streaming
// video's positions grow without bound, and an fp32 product of a position of
// 10^6 is off by up to 0.03 rad: the angle is an fp64 product (31 + 24 bits),
// reduced to half turns there, and only the remainder is an fp32 number.
//
// A byte of work per byte moved, so it is bound by memory and, for one token,
// by the launch.  A lane holds 8 pairs (two 16-byte units), D/16 lanes a head;
// the heads of all tokens, q, k and v alike, are one list.

#include "attn_common.h"

namespace vico {
namespace {

constexpr int kRopeThreads = 256;

__device__ __forceinline__ void unpack(u32x4 x, float (&f)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = __uint_as_float(x[i] << 16);
    f[2 * i + 1] = __uint_as_float(x[i] & 0xFFFF0000u);
  }
}

__device__ __forceinline__ u32x4 pack(const float (&f)[8]) {
  bf16x8 b;
#pragma unroll
  for (int i = 0; i < 8; ++i) b[i] = (__bf16)f[i];
  return __builtin_bit_cast(u32x4, b);
}

__device__ __forceinline__ void weights(const void* w, int f32, int at, float (&f)[8]) {
  if (f32) {
    const f32x4 a = *(const f32x4*)((const float*)w + at), b = *(const f32x4*)((const float*)w + at + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) { f[i] = a[i]; f[4 + i] = b[i]; }
  } else {
    unpack(*(const u32x4*)((const uint16_t*)w + at), f);
  }
}

template <int D>
__global__ __launch_bounds__(kRopeThreads) void qk_norm_rope_kernel(RopeArgs a) {
  constexpr int LPH = D / 16;            // lanes of a head
  const int HT = a.Hq + a.Hkv + (a.v ? a.Hkv : 0);
  const int64_t total = (int64_t)a.T * HT;
  const int64_t item = ((int64_t)blockIdx.x * kRopeThreads + threadIdx.x) / LPH;
  if (item >= total) return;             // whole heads: the lanes of a head stay together
  const int u = threadIdx.x % LPH;
  const int t = (int)(item / HT), ht = (int)(item - (int64_t)t * HT);
  const int kind = ht < a.Hq ? 0 : ht < a.Hq + a.Hkv ? 1 : 2;
  const int h = ht - (kind == 0 ? 0 : kind == 1 ? a.Hq : a.Hq + a.Hkv);
  const uint16_t* src = (kind == 0 ? a.q + (int64_t)t * a.q_stride : kind == 1 ? a.k + (int64_t)t * a.k_stride
                                   : a.v + (int64_t)t * a.v_stride) + h * D;
  uint16_t* dst = (kind == 0 ? a.q_out + (int64_t)t * a.Hq * D : (kind == 1 ? a.k_out : a.v_out) + (int64_t)t * a.Hkv * D) + h * D;

  // this lane's two units of 8 elements
  const bool turned = kind < 2 && 16 * u < a.rot;
  const bool halves = turned && !a.adjacent;
  const int ea = halves ? 8 * u : 16 * u, eb = halves ? a.rot / 2 + 8 * u : 16 * u + 8;
  const u32x4 xa = *(const u32x4*)(src + ea), xb = *(const u32x4*)(src + eb);
  if (kind == 2) {
    *(u32x4*)(dst + ea) = xa;
    *(u32x4*)(dst + eb) = xb;
    return;
  }
  float fa[8], fb[8];
  unpack(xa, fa);
  unpack(xb, fb);
  const void* w = kind == 0 ? a.q_weight : a.k_weight;
  if (w) {
    float ss = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) ss = __builtin_fmaf(fa[i], fa[i], __builtin_fmaf(fb[i], fb[i], ss));
#pragma unroll
    for (int o = 1; o < LPH; o <<= 1) ss += __shfl_xor(ss, o, 64);
    const float r = 1.f / sqrtf(ss * (1.f / D) + a.eps);
    float wa[8], wb[8];
    weights(w, a.weight_f32, ea, wa);
    weights(w, a.weight_f32, eb, wb);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      fa[i] = fa[i] * r * wa[i];
      fb[i] = fb[i] * r * wb[i];
    }
  }
  if (turned) {
    float c[8], s[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int p = 8 * u + i;
      const int axis = a.axes == 1 ? 0 : a.strided ? (p % 3 == 1 && p < 3 * a.s1 ? 1 : p % 3 == 2 && p < 3 * a.s2 ? 2 : 0)
                                                   : (p >= a.s0) + (p >= a.s0 + a.s1);
      const double turns = (double)a.positions[(int64_t)axis * a.T + t] * (double)a.inv_freq[p] * 0.31830988618379067154;
      sincospif((float)(turns - 2.0 * rint(turns * 0.5)), &s[i], &c[i]);
    }
    if (a.adjacent) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float a0 = fa[2 * i], a1 = fa[2 * i + 1], b0 = fb[2 * i], b1 = fb[2 * i + 1];
        fa[2 * i] = a0 * c[i] - a1 * s[i];
        fa[2 * i + 1] = a1 * c[i] + a0 * s[i];
        fb[2 * i] = b0 * c[4 + i] - b1 * s[4 + i];
        fb[2 * i + 1] = b1 * c[4 + i] + b0 * s[4 + i];
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float x0 = fa[i], x1 = fb[i];
        fa[i] = x0 * c[i] - x1 * s[i];
        fb[i] = x1 * c[i] + x0 * s[i];
      }
    }
  }
  *(u32x4*)(dst + ea) = pack(fa);
  *(u32x4*)(dst + eb) = pack(fb);
}

}  // namespace

hipError_t launch_qk_norm_rope(const RopeArgs& a, hipStream_t stream) {
  const int64_t threads = (int64_t)a.T * (a.Hq + a.Hkv + (a.v ? a.Hkv : 0)) * (a.D / 16);
  const dim3 grid((unsigned)((threads + kRopeThreads - 1) / kRopeThreads));
  if (a.D == 128) hipLaunchKernelGGL(qk_norm_rope_kernel<128>, grid, dim3(kRopeThreads), 0, stream, a);
  else hipLaunchKernelGGL(qk_norm_rope_kernel<64>, grid, dim3(kRopeThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace vico
