// Attention over a 4-bit store: query rows against [sink | store segments |
// tail, causal], the store's keys and values in 4 bits (q4_common.h), sink and
// tail in bf16 (ViCoStream Sec. 3, query-time decoding; query rows of Eq. (4)).
//
//   O = softmax(scale Q K^T) V,  K, V of a store row = code * 2^(scale byte - 127)
//
// Every wave takes 32-key blocks of its work-group's key range in turn, loads
// them into registers, turns the codes into bf16 there (exactly) and keeps a
// running softmax of its own; the waves' states are merged through LDS at the
// end.  A block lies in one region, so the three regions' last blocks may be
// part-filled.
//   * S^T = K Q^T with v_mfma_f32_16x16x32_bf16.  Lane (n, j), n = lane % 16,
//     j = lane / 16, holds D/4 consecutive dims of one key: one load of its
//     codes, and one scale for all of them.  The order of the dims inside the
//     k-steps differs from memory's for that; Q is loaded in the same order.
//     Key rows are ordered so that lane group j ends with the logits of keys
//     8j .. 8j+7, and P^T is the second product's B operand as it stands.
//   * O^T = V^T P^T: the lane holds D/16 dims of its 8 keys, converted two dims
//     at a time and transposed with one v_perm_b32 per two values.  The scale
//     bytes of a quad's 4 lanes cover the quad's 8 keys; a DPP step broadcasts
//     each.
// Probabilities are rounded to bf16 for the second product, as in the bf16
// kernels: its operands are 16-bit, and a second term for the rest would double
// it.  Each is off by 2^-8 of itself at most, a result by 2^-8 of the weighted mean
// of |v|: over the norm 2.1e-3 to 2.3e-3 from 64 bits, with the bf16 output's own
// 1.7e-3, for 1.7e-3 with fp32 ones.  Logits, softmax state and sums are fp32.
//
// What bounds it (the kernel alone, medians of a trace).  A decode step streams the store: 16 waves a CU, one 16-row
// block each, have 16 blocks on the way, and 7B heads over 256 chunks (262k keys,
// 143 MB) take 35.4 us, loads alone 34.4 (4.6 TB/s between the first load and the
// last).  8 waves with the next block loaded ahead took 39; with the heads of a
// key range on different XCDs 48: a token's codes are 64 bytes a head, and two
// heads share a cache line.  Over 32 chunks the launch, the table, a memory latency
// and the waves' merge are most of its 7.9 us.  Above 16 rows, two row
// blocks a wave use each converted block twice, at 8 waves' registers: 224 rows
// over 17.8k keys (a 32-token query, 7B heads) 21.1 us, against 30.4 with one row
// block; what bounds those is issue, of conversion and softmax between the matrix
// products (the matrix cores are busy for 18 % of the cycles), and the start.
//
// A masked key's probability is 0, but 0 times a NaN or an infinity is not: in
// a block that the causal mask cuts, such values of V are zeros and are added at
// the end for the rows that see them (whatever its weight, such a value is the
// row's result).

#include "q4_common.h"

namespace vico {
namespace {

template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_mov_dpp((int)x, CTRL, 0xF, 0xF, true);
}

// A row tile's state and block bodies; D dims a head, NRB blocks of 16 rows.
template <int D, int NRB, int NW>
__global__ __launch_bounds__(NW * 64, 1) void attn_rows_q4_kernel(RowsQ4Args a) {
  constexpr int NKS = D / 32;              // k-steps of Q K^T
  constexpr int DPL = D / 4;               // dims of a key per lane
  constexpr int VE = D / 16;               // dims per lane of a V row
  constexpr int RT = 16 * NRB;             // rows of the work-group
  constexpr int BK = kRowsBlock;           // keys per block
  constexpr int OS = D + 8;                // row stride of the merge buffer (floats)
  static_assert(BK == 32, "two 16-key products per block");
  typedef uint32_t krow_t __attribute__((ext_vector_type(DPL / 8)));
  typedef uint32_t vrow_t __attribute__((ext_vector_type(VE / 2)));
  typedef const __attribute__((address_space(1))) char* gptr;

  __shared__ __attribute__((aligned(16))) float o_s[NW][RT][OS];
  __shared__ float m_s[NW][RT], l_s[NW][RT];
  __shared__ typename Segments<NW * 64>::Lds seg_s;
  __shared__ int odd_s;

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 15, j = lane >> 4;
  const int g = a.Hq / a.Hkv;
  const int NR = g * a.Lq;

  // ---- work item: the row tiles of one key range side by side, then its KV heads: they share its codes, and the
  // heads the cache lines (a head's codes of a token are 64 or 32 bytes), in an XCD's L2
  const int L = xcd_remap(blockIdx.x, gridDim.x);
  const int group = a.by_rt(L), rt = L - group * a.n_rt, part = a.by_kv(group);
  const int kv = group - part * a.Hkv;

  if (tid == 0) odd_s = 0;
  int incl, shift, win;
  const Segments<NW * 64> seg{seg_s, incl, shift, win};
  const int G = seg.build(a.seg_start, a.seg_len, a.n_segs, a.cap);

  // ---- Q rows as B fragments; rows past the end repeat the last one and are never stored
  bf16x8 qf[NRB][NKS];
  int tok[NRB];
#pragma unroll
  for (int rb = 0; rb < NRB; ++rb) {
    const int r = min(rt * RT + rb * 16 + n, NR - 1);
    tok[rb] = a.by_g(r);
    const uint16_t* qp = a.q + ((int64_t)tok[rb] * a.Hq + kv * g + r - tok[rb] * g) * D + j * DPL;
#pragma unroll
    for (int ks = 0; ks < NKS; ++ks) qf[rb][ks] = __builtin_bit_cast(bf16x8, *(const u32x4*)(qp + ks * 8));
  }

  // ---- blocks: sink, store, tail
  const int tail0 = a.T - a.Lq;                                // tail key `tail0 + t` is row t's last
  const int tail_first = tail0 + a.by_g(min(rt * RT, NR - 1)), tail_last = tail0 + a.by_g(min((rt + 1) * RT, NR) - 1);
  const int nb_s = (a.S + BK - 1) / BK, nb_g = (G + BK - 1) / BK, nb_t = tail_last / BK + 1;
  const int n_blocks = nb_s + nb_g + nb_t;
  const int per_part = a.by_parts(n_blocks + a.parts - 1);
  const int b_lo = min(per_part * part, n_blocks), b_hi = min(b_lo + per_part, n_blocks);

  const int rbytes = a.Hkv * D * 2, cbytes = a.Hkv * (D / 2), sbytes = a.Hkv * (D / kQ4Group);
  const int ka = 8 * (n >> 2) + (n & 3);                       // this lane's key of the first product; second: + 4
  const int kg = j * DPL / kQ4Group, vg = n * VE / kQ4Group;   // scale groups of this lane's dims

  // ---- running state: row n of each 16-row block, shared by the lanes n, n+16, n+32, n+48
  f32x4 o[NRB][VE];
  float m_run[NRB], l_run[NRB], neg_m[NRB];        // neg_m: -m_run, +inf while there is no max
#pragma unroll
  for (int rb = 0; rb < NRB; ++rb) {
#pragma unroll
    for (int e = 0; e < VE; ++e) o[rb][e] = f32x4{0.f, 0.f, 0.f, 0.f};
    m_run[rb] = -INFINITY;
    neg_m[rb] = INFINITY;
    l_run[rb] = 0.f;
  }
  const float c = a.scale_log2;

  // Softmax of the block's logits (key 8j + v in s[v / 4][v % 4]); key index past lim[rb] is masked.
  auto softmax = [&](f32x4 (&s)[2], int rb, int lim, bool masked) __attribute__((always_inline)) {
    if (__builtin_expect(masked, 0)) {
#pragma unroll
      for (int v = 0; v < 8; ++v) s[v / 4][v % 4] = 8 * j + v > lim ? -INFINITY : s[v / 4][v % 4];
    }
    float e[8], sum;
    auto expo = [&](float nm) __attribute__((always_inline)) {
#pragma unroll
      for (int v = 0; v < 8; ++v) e[v] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[v / 4][v % 4], c, nm));
      sum = ((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7]));
    };
    expo(neg_m[rb]);
    // the max is raised when a lane's sum of 8 (which bounds each) passes kLaneSumLimit, or there is none yet
    if (__builtin_amdgcn_ballot_w64(!(sum <= kLaneSumLimit))) {
      float mx = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])),
                       fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
      mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
      mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
      const float m_new = fmaxf(m_run[rb], mx * c);
      const float alpha = (m_new == m_run[rb]) ? 1.f : __builtin_amdgcn_exp2f(m_run[rb] - m_new);
      l_run[rb] *= alpha;
#pragma unroll
      for (int d = 0; d < VE; ++d) o[rb][d] *= alpha;
      m_run[rb] = m_new;
      neg_m[rb] = -m_new;
      expo(m_new == -INFINITY ? 0.f : -m_new);
    }
    l_run[rb] += sum;
    bf16x8 p;
#pragma unroll
    for (int v = 0; v < 8; ++v) p[v] = (__bf16)e[v];
    return p;
  };

  // ---- a block of keys as bf16: K fragments of keys ka, ka + 4, V rows of keys 8j .. 8j + 7
  auto probabilities = [&](const u32x4 (&kr)[2][NKS], bf16x8 (&pf)[NRB], const int (&lim)[NRB], bool masked)
      __attribute__((always_inline)) {
    f32x4 s[NRB][2];
#pragma unroll
    for (int rb = 0; rb < NRB; ++rb)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        s[rb][h] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ks = 0; ks < NKS; ++ks)
          s[rb][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kr[h][ks]), qf[rb][ks], s[rb][h], 0, 0, 0);
      }
#pragma unroll
    for (int rb = 0; rb < NRB; ++rb) pf[rb] = softmax(s[rb], rb, lim[rb], masked);
  };
  auto values = [&](const vrow_t (&vr)[8], const bf16x8 (&pf)[NRB]) __attribute__((always_inline)) {
#pragma unroll
    for (int e = 0; e < VE; ++e) {
      u32x4 w;           // value e of this lane's 8 keys
#pragma unroll
      for (int p = 0; p < 4; ++p)
        w[p] = __builtin_amdgcn_perm(vr[2 * p + 1][e / 2], vr[2 * p][e / 2], (e & 1) ? 0x07060302u : 0x05040100u);
      const bf16x8 vf = __builtin_bit_cast(bf16x8, w);
#pragma unroll
      for (int rb = 0; rb < NRB; ++rb) o[rb][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[rb], o[rb][e], 0, 0, 0);
    }
  };

  // ---- rows row0 .. row0 + 31 of a bf16 tensor with `rows` (rows past it read as zero); lim counts from row0
  bool odd = false;                                // a value of the tail that is not finite
  auto bf16_block = [&](const uint16_t* bk, const uint16_t* bv, int rows, int row0, const int (&lim)[NRB],
                        bool masked, bool tail) __attribute__((always_inline)) {
    const int left = min(rows - row0, BK) * rbytes;
    const rsrc_t rk = make_rsrc((const char*)bk + (int64_t)row0 * rbytes, left);
    const rsrc_t rv = make_rsrc((const char*)bv + (int64_t)row0 * rbytes, left);
    const uint32_t k_off = (uint32_t)(ka * rbytes + kv * D * 2 + j * DPL * 2);
    const uint32_t v_off = (uint32_t)(8 * j * rbytes + kv * D * 2 + n * VE * 2);
    bf16x8 pf[NRB];
    {
      u32x4 kr[2][NKS];
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int ks = 0; ks < NKS; ++ks)
          kr[h][ks] = __builtin_amdgcn_raw_buffer_load_b128(rk, k_off + h * 4 * rbytes + ks * 16, 0, 0);
      probabilities(kr, pf, lim, masked);
    }
    vrow_t vr[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if constexpr (VE == 8) vr[i] = __builtin_amdgcn_raw_buffer_load_b128(rv, v_off + i * rbytes, 0, 0);
      else vr[i] = __builtin_amdgcn_raw_buffer_load_b64(rv, v_off + i * rbytes, 0, 0);
    }
    if (masked && tail) {
      u16x2 most{0, 0};
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int d = 0; d < VE / 2; ++d) largest_exponents(most, vr[i][d]);
      if (__builtin_expect(__builtin_amdgcn_ballot_w64(not_finite(most)) != 0, 0)) {
        odd = true;
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
          for (int d = 0; d < VE / 2; ++d) vr[i][d] = finite_or_zero(vr[i][d]);
      }
    }
    values(vr, pf);
  };

  // ---- a block of the store: what its loads bring
  struct Codes {
    krow_t k[2];                  // this lane's dims of keys ka, ka + 4
    uint32_t v[8];                // its dims of keys 8j .. 8j + 7
    uint32_t ks[2], vs[2];        // scale bytes: K of the two keys; V of keys 8j + n%4, 8j + 4 + n%4
  };
  const uint32_t kc = (uint32_t)(kv * (D / 2) + j * (DPL / 2)), vc = (uint32_t)(kv * (D / 2) + n * (VE / 2));
  const uint32_t ksc = (uint32_t)(kv * (D / kQ4Group) + kg), vsc = (uint32_t)(kv * (D / kQ4Group) + vg);
  const uint32_t k_at = (uint32_t)(ka * cbytes) + kc, v_at = (uint32_t)(8 * j * cbytes) + vc;
  const uint32_t ks_at = (uint32_t)(ka * sbytes) + ksc, vs_at = (uint32_t)((8 * j + (n & 3)) * sbytes) + vsc;
  auto load_codes = [&](int i0, Codes& x) __attribute__((always_inline)) {      // gathered keys i0 .. i0 + 31, i0 < G
    int slot0;
    if (seg.straight(i0, slot0) >= BK) {
      // consecutive slots: base + fixed per-lane offsets
      const int64_t slot = slot0;
      const rsrc_t rk = make_rsrc(a.k4 + slot * cbytes, BK * cbytes), rv = make_rsrc(a.v4 + slot * cbytes, BK * cbytes);
      const rsrc_t rks = make_rsrc(a.ks + slot * sbytes, BK * sbytes), rvs = make_rsrc(a.vs + slot * sbytes, BK * sbytes);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if constexpr (D == 128) x.k[h] = __builtin_amdgcn_raw_buffer_load_b128(rk, k_at, h * 4 * cbytes, 0);
        else x.k[h] = __builtin_amdgcn_raw_buffer_load_b64(rk, k_at, h * 4 * cbytes, 0);
        x.ks[h] = __builtin_amdgcn_raw_buffer_load_b8(rks, ks_at, h * 4 * sbytes, 0);
        x.vs[h] = __builtin_amdgcn_raw_buffer_load_b8(rvs, vs_at, h * 4 * sbytes, 0);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if constexpr (D == 128) x.v[i] = __builtin_amdgcn_raw_buffer_load_b32(rv, v_at, i * cbytes, 0);
        else x.v[i] = __builtin_amdgcn_raw_buffer_load_b16(rv, v_at, i * cbytes, 0);
      }
      return;
    }
    // several segments, or the last ones: keys past the last read its slot and count as zero
    bool real;
    const int slot = seg.slot_of_lane(i0, BK, G, real);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int64_t r = __shfl(slot, ka + 4 * h, 64);
      x.k[h] = *(const __attribute__((address_space(1))) krow_t*)((gptr)a.k4 + r * cbytes + kc);
      x.ks[h] = *(const __attribute__((address_space(1))) uint8_t*)((gptr)a.ks + r * sbytes + ksc);
      const int64_t rv = __shfl(slot, 8 * j + 4 * h + (n & 3), 64);
      const bool ok = __shfl((int)real, 8 * j + 4 * h + (n & 3), 64);
      const uint32_t b = *(const __attribute__((address_space(1))) uint8_t*)((gptr)a.vs + rv * sbytes + vsc);
      x.vs[h] = ok ? b : 127;
    }
#pragma unroll
    for (int i8 = 0; i8 < 8; ++i8) {
      const int64_t r = __shfl(slot, 8 * j + i8, 64);
      const bool ok = __shfl((int)real, 8 * j + i8, 64);
      uint32_t w;
      if constexpr (D == 128) w = *(const __attribute__((address_space(1))) uint32_t*)((gptr)a.v4 + r * cbytes + vc);
      else w = *(const __attribute__((address_space(1))) uint16_t*)((gptr)a.v4 + r * cbytes + vc);
      x.v[i8] = ok ? w : 0;
    }
  };
  auto q4_block = [&](int i0, const Codes& x) __attribute__((always_inline)) {
    const int last = G - 1 - i0;
    int lim[NRB];
#pragma unroll
    for (int rb = 0; rb < NRB; ++rb) lim[rb] = last;
    bf16x8 pf[NRB];
    {
      u32x4 kr[2][NKS];
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int ks = 0; ks < NKS; ++ks) kr[h][ks] = q4_eight(x.k[h][ks], q4_scale(x.ks[h]));
      probabilities(kr, pf, lim, last < BK - 1);
    }
    // each scale byte of the quad's 8 keys to its four lanes
    const uint32_t b0 = x.vs[0] << 23, b1 = x.vs[1] << 23;
    const uint32_t vs[8] = {dpp<0x00>(b0), dpp<0x55>(b0), dpp<0xAA>(b0), dpp<0xFF>(b0),
                            dpp<0x00>(b1), dpp<0x55>(b1), dpp<0xAA>(b1), dpp<0xFF>(b1)};
    vrow_t vr[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float f = __uint_as_float(vs[i]);
      if constexpr (VE == 8) vr[i] = q4_eight(x.v[i], f);
      else vr[i] = vrow_t{q4_pair<0>(x.v[i], f), q4_pair<1>(x.v[i], f)};
    }
    values(vr, pf);
  };

  // ---- the wave's blocks: every NW-th of the part's.  (Loading the next block's codes while one is computed measured
  // the same with 8 waves, 21.3 and 21.8 us on 224 rows over 17.8k keys, and so did two blocks at a time; neither fits
  // 16 waves' registers.  The other waves' loads fill the gap.)
  const int end_g = nb_s + nb_g;
  auto step_to = [&](int b, int to) __attribute__((always_inline)) { return b + (max(to - b, 0) + NW - 1) / NW * NW; };
  const int first_g = step_to(b_lo + wave, nb_s), last_g = min(b_hi, end_g);
  for (int b = b_lo + wave; b < b_hi; b += NW) {
    if (b >= nb_s && b < end_g) {
      b = step_to(b, end_g);
      if (b >= b_hi) break;
    }
    const late_args l = late();
    const bool sink = b < nb_s;
    const int rows = sink ? l->S : l->T, row0 = (sink ? b : b - end_g) * BK;
    int lim[NRB];
#pragma unroll
    for (int rb = 0; rb < NRB; ++rb) lim[rb] = (sink ? rows - 1 : tail0 + tok[rb]) - row0;
    bf16_block(sink ? l->sink_k : l->tail_k, sink ? l->sink_v : l->tail_v, rows, row0, lim,
               row0 + BK - 1 > (sink ? rows - 1 : tail_first), !sink);
  }
  // The waves of a SIMD go by age where they want the same slot: of 224 rows over 17.8k keys the older half ends at
  // 14.5 us of 19, and the younger one goes on alone, at half the issue rate.  Turned round they end closer together:
  // 23.0 -> 22.4 us a call, decode over 262k keys 40.0 -> 39.6.  Turned back after half or three quarters of the blocks:
  // 22.4 and 22.1, but 40.9.
  if (wave >= NW / 2) __builtin_amdgcn_s_setprio(1);
  for (int b = first_g; b < last_g; b += NW) {
    Codes x;
    load_codes((b - nb_s) * BK, x);
    q4_block((b - nb_s) * BK, x);
  }

  // ---- merge of the waves: O^T lane (n, j) holds row n, dims VE*(4j+i) + e
#pragma unroll
  for (int rb = 0; rb < NRB; ++rb) {
    float l = l_run[rb];
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
    if (j == 0) {
      m_s[wave][rb * 16 + n] = m_run[rb];
      l_s[wave][rb * 16 + n] = l;
    }
    float* op = &o_s[wave][rb * 16 + n][VE * 4 * j];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int e = 0; e < VE; e += 4)
        *(f32x4*)(op + i * VE + e) = f32x4{o[rb][e][i], o[rb][e + 1][i], o[rb][e + 2][i], o[rb][e + 3][i]};
  }
  __syncthreads();
  if (odd) odd_s = 1;
  __syncthreads();
  constexpr int NQ = D / 4;
  const int rows = min(RT, NR - rt * RT);
  const late_args l = late();
  for (int it = tid; it < rows * NQ; it += NW * 64) {
    const int r = it / NQ, dq = it % NQ;
    float m = -INFINITY;
#pragma unroll
    for (int w = 0; w < NW; ++w) m = fmaxf(m, m_s[w][r]);
    const float m_use = m == -INFINITY ? 0.f : m;
    float sum = 0.f;
    f32x4 acc{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float f = __builtin_amdgcn_exp2f(m_s[w][r] - m_use);      // 0 for a wave that saw no key of the row
      sum += f * l_s[w][r];
      acc += f * *(const f32x4*)&o_s[w][r][dq * 4];
    }
    acc *= sum > 0.f ? 1.f / sum : sum == sum ? 0.f : sum;                       // an empty row is 0, a NaN stays one
    const float lse2 = sum > 0.f ? m_use + __log2f(sum) : sum == sum ? -INFINITY : sum;
    const int pr = rt * RT + r, t = a.by_g(pr), h = kv * g + pr - t * g;
    if (__builtin_expect(odd_s != 0, 0)) {       // values of the part's tail keys that are not finite, for the rows that see them
      const int k1 = min(max(b_hi - end_g, 0) * BK - 1, tail0 + t);
      for (int k = max(b_lo - end_g, 0) * BK; k <= k1; ++k) {
        const u32x2 w = *(const u32x2*)(l->tail_v + ((int64_t)k * l->Hkv + kv) * D + dq * 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t bits = (i & 1) ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16;
          acc[i] += (bits & 0x7F800000u) == 0x7F800000u ? __uint_as_float(bits) : 0.f;
        }
      }
    }
    if (l->parts > 1) {
      const int64_t prow = ((int64_t)part * l->Hq + h) * l->Lq + t;      // the merge kernel's layout
      *(f32x4*)(l->ws_o + prow * D + dq * 4) = acc;
      if (dq == 0) l->ws_lse[prow] = lse2;
      continue;
    }
    const int64_t oo = ((int64_t)t * l->Hq + h) * D + dq * 4;
    if (l->out_f32) *(f32x4*)((float*)l->out + oo) = acc;
    else *(bf16x4*)((__bf16*)l->out + oo) = bf16x4{(__bf16)acc[0], (__bf16)acc[1], (__bf16)acc[2], (__bf16)acc[3]};
    if (dq == 0 && l->lse) l->lse[(int64_t)h * l->Lq + t] = lse2 * kLn2;
  }
}

template <int D>
hipError_t launch(const RowsQ4Args& a, hipStream_t stream) {
  const dim3 grid(a.n_rt * a.parts * a.Hkv);
  if (a.row_blocks == 1) hipLaunchKernelGGL((attn_rows_q4_kernel<D, 1, 16>), grid, dim3(1024), 0, stream, a);
  else if (a.row_blocks == 2) hipLaunchKernelGGL((attn_rows_q4_kernel<D, 2, 8>), grid, dim3(512), 0, stream, a);
  else return hipErrorInvalidValue;
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rows_q4(const RowsQ4Args& a, hipStream_t stream) {
  if (a.n_segs > kMaxSegments || a.n_rt < 1 || a.parts < 1) return hipErrorInvalidValue;
  return a.D == 128 ? launch<128>(a, stream) : launch<64>(a, stream);
}

}  // namespace vico
