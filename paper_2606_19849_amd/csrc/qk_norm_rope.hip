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
// The operator moves four bytes for every element and computes little, so it
// is bound by memory and, for few tokens, by the launch -- as long as a
// token's angles are not computed for each of its heads: fp64 products, sines
// and cosines of 64 pairs for 32 heads each took 16.4 us a call for a 2048-token
// chunk (7B heads, 38 MB), computed once 10.7 (traced kernel: median 11.1 to 11.4,
// least 10.0).  A work-group takes one token, computes its sines and cosines once, one
// pair a thread, into LDS, and its heads, q, k and v alike, D/16 lanes a head; a
// lane holds 8 pairs (two 16-byte units), loaded before the angles are ready.
// The next head is loaded after this one's stores: loaded before its arithmetic it
// costs registers, and waves (0.2 us more).  That chunk again and again in a
// graph, the same inputs / eight in turn: 9.8 / 12.9 us; two tokens a work-group,
// as a variant of this kernel, 9.1 / 12.2, four 10.2 / 13.8.

#include "attn_common.h"

namespace vico {
namespace {

constexpr int kRopeThreads = 512;     // most threads of a work-group

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

// The norm of a head whose squares leave fp32 (a mean below 2^-100 has lost some of them, an infinite one all): x and
// the squares scaled by powers of two.  Returns the factor that is still to be applied.
template <int LPH>
__device__ __forceinline__ float scaled_norm(float (&fa)[8], float (&fb)[8], float mean, float eps) {
  const bool tiny = mean < 1.f;
  const float up = tiny ? 0x1p100f : 1.f, down = tiny ? 1.f : 0x1p-70f, sc = up * down;
  float ss = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    fa[i] *= up;                         // exact: at most 2^-46 before
    fb[i] *= up;
    const float u = fa[i] * down, v = fb[i] * down;
    ss = __builtin_fmaf(u, u, __builtin_fmaf(v, v, ss));
  }
#pragma unroll
  for (int o = 1; o < LPH; o <<= 1) ss += __shfl_xor(ss, o, 64);
  const float r = 1.f / sqrtf(ss * (1.f / (16 * LPH)) + eps * sc * sc);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    fa[i] *= r;
    fb[i] *= r;
  }
  return down;
}

template <int D>
__global__ __launch_bounds__(kRopeThreads) void qk_norm_rope_kernel(RopeArgs a) {
  constexpr int LPH = D / 16;            // lanes of a head
  __shared__ __attribute__((aligned(16))) float cos_s[D / 2], sin_s[D / 2];
  const int tid = threadIdx.x, u = tid % LPH, step = (int)blockDim.x / LPH;
  const int heads = a.Hq + a.Hkv + (a.v ? a.Hkv : 0);
  const int64_t t = blockIdx.x;

  // a head: its place, and this lane's two units of 8 elements
  struct Head {
    u32x4 xa, xb;
    uint16_t* dst;
    int kind, ea, eb;                    // kind: q, k, v
  };
  auto load = [&](int i, Head& x) __attribute__((always_inline)) {
    x.kind = i < a.Hq ? 0 : i < a.Hq + a.Hkv ? 1 : 2;
    const int h = i - (x.kind == 0 ? 0 : x.kind == 1 ? a.Hq : a.Hq + a.Hkv);
    const uint16_t* src = (x.kind == 0 ? a.q + t * a.q_stride : x.kind == 1 ? a.k + t * a.k_stride : a.v + t * a.v_stride) + h * D;
    x.dst = (x.kind == 0 ? a.q_out + t * a.Hq * D : (x.kind == 1 ? a.k_out : a.v_out) + t * a.Hkv * D) + h * D;
    const bool halves = x.kind < 2 && 16 * u < a.rot && !a.adjacent;
    x.ea = halves ? 8 * u : 16 * u;
    x.eb = halves ? a.rot / 2 + 8 * u : 16 * u + 8;
    x.xa = *(const u32x4*)(src + x.ea);
    x.xb = *(const u32x4*)(src + x.eb);
  };
  Head x;
  int head = tid / LPH;
  if (head < heads) load(head, x);

  // ---- sines and cosines of the token's angles
  for (int p = tid; p < a.rot / 2; p += (int)blockDim.x) {
    const int axis = a.axes == 1 ? 0 : a.strided ? (p % 3 == 1 && p < 3 * a.s1 ? 1 : p % 3 == 2 && p < 3 * a.s2 ? 2 : 0)
                                                 : (p >= a.s0) + (p >= a.s0 + a.s1);
    const double turns = (double)a.positions[(int64_t)axis * a.T + t] * (double)a.inv_freq[p] * 0.31830988618379067154;
    sincospif((float)(turns - 2.0 * rint(turns * 0.5)), &sin_s[p], &cos_s[p]);
  }
  __syncthreads();

  while (head < heads) {                 // whole heads: the lanes of a head stay together
    if (x.kind == 2) {
      *(u32x4*)(x.dst + x.ea) = x.xa;
      *(u32x4*)(x.dst + x.eb) = x.xb;
      if ((head += step) < heads) load(head, x);
      continue;
    }
    float fa[8], fb[8];
    unpack(x.xa, fa);
    unpack(x.xb, fb);
    const void* w = x.kind == 0 ? a.q_weight : a.k_weight;
    if (w) {
      float wa[8], wb[8];
      weights(w, a.weight_f32, x.ea, wa);
      weights(w, a.weight_f32, x.eb, wb);
      float ss = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) ss = __builtin_fmaf(fa[i], fa[i], __builtin_fmaf(fb[i], fb[i], ss));
#pragma unroll
      for (int o = 1; o < LPH; o <<= 1) ss += __shfl_xor(ss, o, 64);
      const float mean = ss * (1.f / D) + a.eps;
      float r = 1.f / sqrtf(mean);
      // (alike in all lanes of a head)
      if (__builtin_expect(!(mean >= 0x1p-100f && mean < INFINITY), 0)) r = scaled_norm<LPH>(fa, fb, mean, a.eps);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        fa[i] = fa[i] * r * wa[i];
        fb[i] = fb[i] * r * wb[i];
      }
    }
    if (16 * u < a.rot) {
      float c[8], s[8];
#pragma unroll
      for (int k = 0; k < 8; k += 4) {
        const f32x4 cv = *(const f32x4*)&cos_s[8 * u + k], sv = *(const f32x4*)&sin_s[8 * u + k];
#pragma unroll
        for (int e = 0; e < 4; ++e) { c[k + e] = cv[e]; s[k + e] = sv[e]; }
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
    *(u32x4*)(x.dst + x.ea) = pack(fa);
    *(u32x4*)(x.dst + x.eb) = pack(fb);
    if ((head += step) < heads) load(head, x);
  }
}

}  // namespace

hipError_t launch_qk_norm_rope(const RopeArgs& a, hipStream_t stream) {
  // equal rounds of heads, as few as kRopeThreads allow
  const int lanes = (a.Hq + a.Hkv + (a.v ? a.Hkv : 0)) * (a.D / 16), rounds = (lanes + kRopeThreads - 1) / kRopeThreads;
  const dim3 grid(a.T), block(((lanes + rounds - 1) / rounds + 63) / 64 * 64);
  if (a.D == 128) hipLaunchKernelGGL(qk_norm_rope_kernel<128>, grid, block, 0, stream, a);
  else hipLaunchKernelGGL(qk_norm_rope_kernel<64>, grid, block, 0, stream, a);
  return hipGetLastError();
}

}  // namespace vico
