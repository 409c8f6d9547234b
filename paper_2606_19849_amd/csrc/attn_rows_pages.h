// Attention over the cache in pages, few query rows a sequence: decode steps,
// short queries, small chunks of many sequences in one launch (gfx950).
//
//   O_i = softmax_p(scale q_i k_p) v_p over the visible positions p of a
//   sequence, whose rows lie in the pages that its table row lists.
//
// A work-group takes one row tile (16 or 32 packed (token, query head) rows of one KV head) of
// one sequence and one part of its key range; every wave takes 32-key blocks of it
// in turn and keeps a running softmax of its own, and the waves' states are merged
// through LDS at the end: the form of attn_rows.hip, whose products and softmax these
// are.  New here:
//   * Blocks are aligned to positions, so a block lies in one page (16-token pages:
//     two).  The lanes of a wave hold the page numbers of its next 32 blocks, checked
//     once; a block takes its own by a lane read, and no memory latency stands
//     between two blocks.
//   * The part of a ragged batch's sequence is a number of blocks, not a share: short
//     sequences take one part and write their result, long ones up to 64, and work-groups
//     past a sequence's parts end at once.
//   * Positions that no row sees (past the last row, between sink and window, without a
//     page) are zeros in V, whatever the memory holds, and -infinity among the
//     logits.  Positions that some rows see (the causal diagonal) may hold values that
//     are not finite: 0 times those is NaN, so they are zeros in the product and are
//     added at the end for the rows that see them.

#pragma once

#include "attn_common.h"
#include "pages.h"
#include "values.h"

namespace vico {

template <int D, int NRB, int NW>
struct RowsLds {
  __attribute__((aligned(16))) float o[NW][16 * NRB][D + 8];
  float m[NW][16 * NRB], l[NW][16 * NRB];
  int odd;
};

// Work-group `blk` of those that take the sequences of class x: row tiles of 16 * NRB rows.  sequence_at(b): sequence b.
template <int D, int NRB, int NW, class F>
__device__ __forceinline__ void paged_rows(const PagedAttnArgs& a, const RowsClass& x, int blk, RowsLds<D, NRB, NW>& lds,
                                           F&& sequence_at) {
  constexpr int NKS = D / 32;              // k-steps of Q K^T
  constexpr int VE = D / 16;               // dims per lane of a V row
  constexpr int RT = 16 * NRB;             // rows of the work-group
  constexpr int BK = kRowsBlock;           // keys per block
  static_assert(BK == 32, "two 16-key products per block");
  typedef uint32_t vrow_t __attribute__((ext_vector_type(VE / 2)));
  typedef const __attribute__((address_space(1))) char* gptr;

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 15, j = lane >> 4;
  const int g = a.Hq / a.Hkv;

  // ---- work item.  The row tiles and KV heads of one key range lie on one XCD (work-groups go round the XCDs): they
  // share its L2, and the heads of a token its pages of memory.  Parts and sequences go round them, each sequence's
  // parts from another XCD on: short sequences have the first parts only.  (32 sequences of 1000 to 16000 keys in 8
  // parts, us a call: so 122; every sequence's first part on the first XCD 150; the heads of a token on different XCDs
  // 136; a stretch of sequences on each XCD 123.)
  int local = blk / kNumXcd;
  int next = x.by_rt(local);
  const int rt = local - next * x.n_rt;
  local = next;
  next = a.by_kv(local);
  const int kv = local - next * a.Hkv;
  next = next * kNumXcd + blk % kNumXcd;
  if (next >= a.B * x.parts) return;
  const int b = x.by_parts(next), turned = next - b * x.parts + b, part = turned - x.by_parts(turned) * x.parts;

  const Sequence s = sequence_at(b);
  const int NR = g * s.n;
  if (NR > x.most || NR < x.least || rt * RT >= NR) return;
  const KeyBlocks<BK> blocks(s);
  int per;
  const int parts = parts_of(x, blocks.upto(last_position(a, s, s.n - 1)), per);
  if (part >= parts) return;
  if (tid == 0) lds.odd = 0;

  // ---- Q rows as B fragments; rows past the end repeat the last one and are never stored
  bf16x8 qf[NRB][NKS];
  int lim[NRB];                            // the row's last position
#pragma unroll
  for (int rb = 0; rb < NRB; ++rb) {
    const int r = min(rt * RT + rb * 16 + n, NR - 1), tok = a.by_g(r);
    lim[rb] = last_position(a, s, tok);
    const uint16_t* qp = a.q + ((int64_t)(s.q0 + tok) * a.Hq + kv * g + r - tok * g) * D + j * 8;
#pragma unroll
    for (int ks = 0; ks < NKS; ++ks) qf[rb][ks] = __builtin_bit_cast(bf16x8, *(const u32x4*)(qp + ks * 32));
  }
  const int first_lim = last_position(a, s, a.by_g(rt * RT));
  const int last_lim = last_position(a, s, a.by_g(min((rt + 1) * RT, NR) - 1));
  const int n_blocks = blocks.upto(last_lim);
  const int b_lo = min(part * per, n_blocks), b_hi = min(b_lo + per, n_blocks);

  // ---- pages: lane 2i + h has that of keys 16h .. 16h + 15 of the wave's i-th next block, -1 for none
  const int32_t* const row = a.table + (int64_t)b * a.width;
  auto pages_from = [&](int blk) __attribute__((always_inline)) {
    const int at = blk + (lane >> 1) * NW;
    const int e = (blocks.position(min(at, n_blocks - 1)) + (lane & 1) * 16) >> a.page_shift;
    const int p = row[min(e, a.width - 1)];
    return at < n_blocks && (uint32_t)p < (uint32_t)a.N ? p : -1;
  };

  const int rbytes = a.Hkv * D * 2;
  const int64_t pbytes = (int64_t)rbytes << a.page_shift;
  const int ka = 8 * (n >> 2) + (n & 3);                       // this lane's key of the first product; second: + 4
  const int in_page = (1 << a.page_shift) - 1;

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
  bool odd = false;                                // a value on the causal diagonal that is not finite

  struct Block {
    u32x4 k[2][NKS];
    vrow_t v[8];
    int pv;                                        // page of keys 8j .. 8j + 7
    int pos;
  };
  auto load_block = [&](int blk, int held, int i, Block& y) __attribute__((always_inline)) {
    y.pos = blocks.position(blk);
    const int pk = __shfl(held, 2 * i + (n >> 3), 64);
    y.pv = __shfl(held, 2 * i + (j >> 1), 64);
    const gptr kp = (gptr)a.k_pages + (max(pk, 0) * pbytes + (uint32_t)(((y.pos + ka) & in_page) * rbytes + kv * D * 2 + j * 16));
    const gptr vp = (gptr)a.v_pages + (max(y.pv, 0) * pbytes + (uint32_t)(((y.pos + 8 * j) & in_page) * rbytes + kv * D * 2 + n * (VE * 2)));
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int ks = 0; ks < NKS; ++ks)
        y.k[h][ks] = *(const __attribute__((address_space(1))) u32x4*)(kp + h * 4 * rbytes + ks * 64);
#pragma unroll
    for (int r = 0; r < 8; ++r) y.v[r] = *(const __attribute__((address_space(1))) vrow_t*)(vp + r * rbytes);
  };

  auto compute_block = [&](Block& y) __attribute__((always_inline)) {
    const int k0 = y.pos + 8 * j;                  // this lane's eight keys
    const bool gap = y.pos + BK > s.sink && y.pos < s.first;
    // what some lane's row does not see of the block
    const bool cut = y.pos + BK - 1 > first_lim, holes = __builtin_amdgcn_ballot_w64(y.pv < 0) != 0;
    if (__builtin_expect(cut || gap || holes, 0)) {
      u16x2 most{0, 0};
#pragma unroll
      for (int r = 0; r < 8; ++r) {
        const int p = k0 + r;
        const bool none = y.pv < 0 || p > last_lim || (p >= s.sink && p < s.first);
        y.v[r] = none ? vrow_t{} : y.v[r];
        if (cut) {
#pragma unroll
          for (int d = 0; d < VE / 2; ++d) {
            largest_exponents(most, y.v[r][d]);
            y.v[r][d] = finite_or_zero(y.v[r][d]);
          }
        }
      }
      odd |= not_finite(most);
    }
    bf16x8 pf[NRB];
#pragma unroll
    for (int rb = 0; rb < NRB; ++rb) {
      f32x4 sc[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        sc[h] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ks = 0; ks < NKS; ++ks)
          sc[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, y.k[h][ks]), qf[rb][ks], sc[h], 0, 0, 0);
      }
      if (__builtin_expect(cut || gap || holes, 0)) {
#pragma unroll
        for (int v = 0; v < 8; ++v) {
          const int p = k0 + v;
          const bool none = y.pv < 0 || p > lim[rb] || (p >= s.sink && p < s.first);
          sc[v / 4][v % 4] = none ? -INFINITY : sc[v / 4][v % 4];
        }
      }
      // probabilities against the running max; raised when a lane's sum of 8
      // (which bounds each) passes kLaneSumLimit, or there is no max yet
      float e[8], sum;
      auto expo = [&](float nm) __attribute__((always_inline)) {
#pragma unroll
        for (int v = 0; v < 8; ++v) e[v] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[v / 4][v % 4], c, nm));
        sum = ((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7]));
      };
      expo(neg_m[rb]);
      if (__builtin_amdgcn_ballot_w64(!(sum <= kLaneSumLimit))) {
        float mx = fmaxf(fmaxf(fmaxf(sc[0][0], sc[0][1]), fmaxf(sc[0][2], sc[0][3])),
                         fmaxf(fmaxf(sc[1][0], sc[1][1]), fmaxf(sc[1][2], sc[1][3])));
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
      // the sum is of fp32; the product with V takes bf16 operands, so a probability is off by 2^-8 of itself at most there
      // (of all attention calls: the matrix cores' fp32 products run at a sixteenth of the rate)
#pragma unroll
      for (int v = 0; v < 8; ++v) pf[rb][v] = (__bf16)e[v];
    }
#pragma unroll
    for (int e = 0; e < VE; ++e) {
      u32x4 w;           // value e of this lane's 8 keys
#pragma unroll
      for (int p = 0; p < 4; ++p)
        w[p] = __builtin_amdgcn_perm(y.v[2 * p + 1][e / 2], y.v[2 * p][e / 2], (e & 1) ? 0x07060302u : 0x05040100u);
      const bf16x8 vf = __builtin_bit_cast(bf16x8, w);
#pragma unroll
      for (int rb = 0; rb < NRB; ++rb) o[rb][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[rb], o[rb][e], 0, 0, 0);
    }
  };

  // ---- the wave's blocks
  for (int at = b_lo + wave; at < b_hi;) {
    const int held = pages_from(at);
    for (int i = 0; i < 32 && at < b_hi; ++i, at += NW) {
      Block y;
      load_block(at, held, i, y);
      compute_block(y);
    }
  }

  // ---- merge of the waves: O^T lane (n, j) holds row n, dims VE*(4j+i) + e
#pragma unroll
  for (int rb = 0; rb < NRB; ++rb) {
    float l = l_run[rb];
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
    if (j == 0) {
      lds.m[wave][rb * 16 + n] = m_run[rb];
      lds.l[wave][rb * 16 + n] = l;
    }
    float* op = &lds.o[wave][rb * 16 + n][VE * 4 * j];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int e = 0; e < VE; e += 4)
        *(f32x4*)(op + i * VE + e) = f32x4{o[rb][e][i], o[rb][e + 1][i], o[rb][e + 2][i], o[rb][e + 3][i]};
  }
  __syncthreads();
  if (odd) lds.odd = 1;
  __syncthreads();
  constexpr int NQ = D / 4;
  const int rows = min(RT, NR - rt * RT);
  for (int it = tid; it < rows * NQ; it += NW * 64) {
    const int r = it / NQ, dq = it % NQ;
    float m = -INFINITY;
#pragma unroll
    for (int w = 0; w < NW; ++w) m = fmaxf(m, lds.m[w][r]);
    const float m_use = m == -INFINITY ? 0.f : m;
    float l = 0.f;
    f32x4 acc{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float f = __builtin_amdgcn_exp2f(lds.m[w][r] - m_use);      // 0 for a wave that saw no key of the row
      l += f * lds.l[w][r];
      acc += f * *(const f32x4*)&lds.o[w][r][dq * 4];
    }
    acc *= l > 0.f ? 1.f / l : l == l ? 0.f : l;                      // an empty row is 0, a NaN stays one
    const float lse2 = l > 0.f ? m_use + __log2f(l) : l == l ? -INFINITY : l;
    const int pr = rt * RT + r, t = a.by_g(pr), h = kv * g + pr - t * g;
    if (__builtin_expect(lds.odd != 0, 0)) {     // values of the part's blocks on the diagonal, for the rows that see them
      const int upto = last_position(a, s, t);
      for (int blk = max(b_lo, blocks.upto(first_lim) - 1); blk < b_hi; ++blk) {
        const int pos = blocks.position(blk);
        if (pos + BK - 1 <= first_lim) continue;
        for (int p = pos; p <= min(pos + BK - 1, upto); ++p) {
          const int page = row[p >> a.page_shift];
          if ((uint32_t)page >= (uint32_t)a.N || (p >= s.sink && p < s.first)) continue;
          const uint32_t* w = (const uint32_t*)(a.v_pages + ((((int64_t)page << a.page_shift) + (p & in_page)) * a.Hkv + kv) * D + dq * 4);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t bits = (i & 1) ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16;
            acc[i] += (bits & 0x7F800000u) == 0x7F800000u ? __uint_as_float(bits) : 0.f;
          }
        }
      }
    }
    if (parts > 1) {
      const int64_t prow = ((((int64_t)b * x.parts + part) * a.Hkv + kv) * x.n_rt + rt) * RT + r;
      *(f32x4*)(x.ws_o + prow * D + dq * 4) = acc;
      if (dq == 0) x.ws_lse[prow] = lse2;
      continue;
    }
    const int64_t orow = (int64_t)(s.q0 + t) * a.Hq + h;
    if (a.out_f32) *(f32x4*)((float*)a.out + orow * D + dq * 4) = acc;
    else *(bf16x4*)((__bf16*)a.out + orow * D + dq * 4) = bf16x4{(__bf16)acc[0], (__bf16)acc[1], (__bf16)acc[2], (__bf16)acc[3]};
    if (dq == 0 && a.lse) a.lse[(int64_t)h * a.total + s.q0 + t] = lse2 * kLn2;
  }
}

// The parts of a row tile joined: PG groups of threads take every PG-th part, D / 4
// threads four columns each; all loads of a thread are on their way together.
//     lse = log2 sum_s 2^lse_s,   O = sum_s 2^(lse_s - lse) O_s
// A part without a key of the row (lse_s = -inf) is all zeros; a NaN or an
// infinity of a part reaches the row whatever the part's weight, 0 as well.
constexpr int kMergeThreads = 256;
template <int D, int PG>
__device__ __forceinline__ void paged_rows_merge(const PagedAttnArgs& a, const RowsClass& x, int blk) {
  constexpr int NQ = D / 4, RPB = kMergeThreads / (NQ * PG), NP = kPagedParts / PG < 8 ? kPagedParts / PG : 8;
  __shared__ float m_s[PG][RPB][NQ], l_s[PG][RPB][NQ];
  __shared__ f32x4 acc_s[PG][RPB][NQ];
  const int tid = threadIdx.x, dq = tid % NQ, pg = tid / NQ % PG, rr = tid / (NQ * PG);
  const int RT = x.tile_rows, chunks = (x.merge_rows + RPB - 1) / RPB;       // (RPB divides RT)
  const int L = blk / chunks, r = (blk - L * chunks) * RPB + rr;
  int next = x.by_rt(L);
  const int rt = L - next * x.n_rt;
  const int b = a.by_kv(next), kv = next - b * a.Hkv;
  const Sequence s = sequence(a, b);
  const int g = a.Hq / a.Hkv, NR = g * s.n;
  if (NR > x.most || NR < x.least || rt * RT + r - rr >= NR) return;        // the whole work-group
  int per;
  const int parts = parts_of(x, KeyBlocks<kRowsBlock>(s).upto(last_position(a, s, s.n - 1)), per);
  if (parts == 1) return;                                        // written by the attention kernel
  const int64_t row0 = (((int64_t)b * x.parts * a.Hkv + kv) * x.n_rt + rt) * RT + r, step = (int64_t)a.Hkv * x.n_rt * RT;
  float m = -INFINITY, l = 0.f;
  f32x4 acc{0.f, 0.f, 0.f, 0.f};
  for (int p0 = pg; p0 < parts; p0 += PG * NP) {
    float ls[NP];
    f32x4 os[NP];
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int64_t at = row0 + min(p0 + i * PG, parts - 1) * step;
      ls[i] = p0 + i * PG < parts ? x.ws_lse[at] : -INFINITY;
      os[i] = *(const f32x4*)(x.ws_o + at * D + dq * 4);
    }
    float mx = m;
#pragma unroll
    for (int i = 0; i < NP; ++i) mx = fmaxf(mx, ls[i]);
    const float use = mx == -INFINITY ? 0.f : mx, f = __builtin_amdgcn_exp2f(m - use);
    l *= f;
    acc *= f;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const float w = __builtin_amdgcn_exp2f(ls[i] - use);
      l += w;
      acc += w * os[i];
    }
    m = mx;
  }
  if constexpr (PG > 1) {
    m_s[pg][rr][dq] = m;
    l_s[pg][rr][dq] = l;
    acc_s[pg][rr][dq] = acc;
    __syncthreads();
    if (pg != 0) return;
    float mx = m;
#pragma unroll
    for (int i = 1; i < PG; ++i) mx = fmaxf(mx, m_s[i][rr][dq]);
    const float use = mx == -INFINITY ? 0.f : mx;
    l = 0.f;
    acc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < PG; ++i) {
      const float f = __builtin_amdgcn_exp2f(m_s[i][rr][dq] - use);
      l += f * l_s[i][rr][dq];
      acc += f * acc_s[i][rr][dq];
    }
    m = mx;
  }
  const int pr = rt * RT + r;
  if (pr >= NR) return;
  acc *= l > 0.f ? 1.f / l : l == l ? 0.f : l;
  const float lse2 = l > 0.f ? m + __log2f(l) : l == l ? -INFINITY : l;
  const int t = a.by_g(pr), h = kv * g + pr - t * g;
  const int64_t orow = (int64_t)(s.q0 + t) * a.Hq + h;
  if (a.out_f32) *(f32x4*)((float*)a.out + orow * D + dq * 4) = acc;
  else *(bf16x4*)((__bf16*)a.out + orow * D + dq * 4) = bf16x4{(__bf16)acc[0], (__bf16)acc[1], (__bf16)acc[2], (__bf16)acc[3]};
  if (dq == 0 && a.lse) a.lse[(int64_t)h * a.total + s.q0 + t] = lse2 * kLn2;
}

}  // namespace vico
