// Attention over a 4-bit store, many query rows (gfx950): what attn_rows_q4.hip
// computes, for calls whose rows share every key often enough to be bound by
// the matrix cores -- a visual chunk over a window of the store used as a ring, a
// query of some dozens of tokens.
//
// A work-group of 8 waves owns 256 packed (token, query head) rows of one KV
// head, 32 a wave, and walks 64-key tiles; the tile body is PipeTile
// (attn_pipe.h), the software-pipelined one of the chunk prefill.  It wants K and
// V as bf16 in LDS.  Of a tile each thread turns 8 codes of K and 8 of V a load
// (one 16-byte unit each) into bf16, in the layout that PipeTile reads: 64 lanes
// write 1024 consecutive bytes.  So the codes are converted once for 256 rows,
// and the store is read at 34 bytes for 64 values.
//   * One barrier a tile.  After the barrier in the middle of step t the thread
//     converts tile t + 2, whose codes it has in registers, writes it to LDS and
//     sends the loads of tile t + 3, which have a whole step to arrive.  Sink and
//     tail tiles are bf16: their loads go straight to LDS.  Inside a run of tiles
//     in one segment the conversion and the loads are dealt out over the slots of
//     the tile body's second half, in the shadow of its MFMAs.
//   * A tile lies in one region (sink, store, tail); the regions' last tiles may
//     be part-filled, with zeros that the mask hides.
//   * Values that are not finite in a tail tile that the causal mask cuts are
//     zeros in LDS (0 times such a value would reach the rows that do not see it)
//     and are added afterwards for the rows that do: such a row's result is that
//     value whatever its weight.
// It is bound by the matrix cores, as the chunk prefill is, and by what goes
// between their instructions.  1024 tokens over 8192 store keys, 7B heads, 128.7
// GFLOP: 140 to 145 us a call by the box, 885 to 920 TFLOP/s, with the merge of its
// two parts (7 us).  173 with all of the conversion and the loads between two barriers, 156 in the slots;
// a copy for timing that does neither took 149 us traced for 166.  Equal shares of
// the tiles for every CU (224 work-groups leave 32 idle) took 146.6 for 145: a row
// tile's keys then come in more parts.

#include <type_traits>

#include "attn_pipe.h"
#include "q4_common.h"

namespace vico {
namespace {

template <int D>
__global__ __launch_bounds__(kThreads, kWgPerCU) void attn_tile_q4_kernel(RowsQ4Args a) {
  constexpr int RB = 1;
  typedef PipeTile<D, RB> Tile;
  constexpr int BN = kKeyTile, BM = kThreads / 64 * 32, NW = kThreads / 64;
  constexpr int RBY = D * 2;                 // bytes per LDS row
  constexpr uint32_t TBY = BN * RBY;         // bytes of one K (or V) tile
  constexpr int NLD = TBY / 1024 / NW;       // 1 KiB chunks a wave fills, of K and of V
  constexpr int RPL = Tile::RPC;             // rows per chunk
  constexpr int NDB = Tile::NDB, NKS = Tile::NKS;
  constexpr int NB = 4;                      // tile t in buffer t mod NB; steps t - 1 .. t + 2 are in use
  constexpr uint32_t kKBase = NB * TBY, kWrap = NB * TBY - 1;
  static_assert(6 * NLD <= Tile::NSLOT, "a tile's conversion and loads fit a body's slots");
  static_assert(NLD * NW * 1024 == TBY && BN == 64 && (NB & (NB - 1)) == 0, "tile geometry");
  typedef __attribute__((address_space(3))) u32x4* lds_u4;
  typedef const __attribute__((address_space(1))) char* gptr;

  __shared__ __attribute__((aligned(16))) uint8_t lds[2 * NB * TBY];
  __shared__ typename Segments<kThreads>::Lds seg_s;
  __shared__ int odd_s;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_void*)lds;

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, hh = lane >> 5;
  const int g = a.Hq / a.Hkv;
  const int NR = g * a.Lq;

  // ---- work item: the row tiles of one key range side by side, then its KV heads: they share its codes, and the
  // heads the cache lines (a head's codes of a token are 64 or 32 bytes), in an XCD's L2
  const int L = xcd_remap(blockIdx.x, gridDim.x);
  const int group = a.by_rt(L), part = a.by_kv(group);
  const int rt = a.n_rt - 1 - (L - group * a.n_rt);      // longest first
  const int kv = group - part * a.Hkv;

  if (tid == 0) odd_s = 0;
  int incl, shift, win;
  const Segments<kThreads> seg{seg_s, incl, shift, win};
  const int G = seg.build(a.seg_start, a.seg_len, a.n_segs, a.cap);

  // ---- this lane's packed row; rows past the end repeat the last one and are never stored
  const int wrow0 = rt * BM + wave * 32;
  const bool wave_active = wrow0 < NR;
  const int my_row = min(wrow0 + l32, NR - 1);
  const int tok = a.by_g(my_row), head = kv * g + my_row - tok * g;
  bf16x8 qf[RB][NKS];
  WaveTile<D>::load_q(qf[0], a.q + ((int64_t)tok * a.Hq + head) * D + hh * 8);

  // ---- tiles: sink, store, tail up to the row tile's last row
  const int tail0 = a.T - a.Lq;              // tail key `tail0 + t` is row t's last
  const int first_lim = tail0 + a.by_g(min(wrow0, NR - 1)), last_lim = tail0 + a.by_g(min(wrow0 + 31, NR - 1));
  const int nb_s = (a.S + BN - 1) / BN, nb_sg = nb_s + (G + BN - 1) / BN;
  const int n_tiles = nb_sg + (tail0 + a.by_g(min((rt + 1) * BM, NR) - 1)) / BN + 1;
  const int per_part = a.by_parts(n_tiles + a.parts - 1);
  const int t_lo = min(per_part * part, n_tiles), t_hi = min(t_lo + per_part, n_tiles);
  const int t_end = wave_active ? min(t_hi, nb_sg + last_lim / BN + 1) : t_lo;      // the wave's last tile
  // the first tail tile that the causal mask cuts for some row of the work-group
  const int t_cut = nb_sg + (tail0 + a.by_g(rt * BM) + 1) / BN;
  // the lane's last visible key in tile t, and whether some lane of the wave does not see all of the tile
  auto lim_of = [&](int t) __attribute__((always_inline)) {
    return t < nb_s ? a.S - 1 - t * BN : t < nb_sg ? G - 1 - (t - nb_s) * BN : tail0 + tok - (t - nb_sg) * BN;
  };
  auto cut = [&](int t) __attribute__((always_inline)) {
    return (t < nb_s ? a.S - 1 - t * BN : t < nb_sg ? G - 1 - (t - nb_s) * BN : first_lim - (t - nb_sg) * BN) < BN - 1;
  };

  // ---- tile loader: this thread's units.  Chunk wave * NLD + n holds RPL rows; the layout says which row and
  // 16-byte unit of it lane `lane` brings, to lane * 16.  Rows and units are computed anew for each tile: kept,
  // they would take registers that the tile body needs.
  const int rbytes = a.Hkv * D * 2, cbytes = a.Hkv * (D / 2), sbytes = a.Hkv * (D / kQ4Group);
  const uint32_t my_part = (uint32_t)(wave * NLD * 1024);
  auto place = [&](int n, int& rk, int& uk, int& rv, int& uv) __attribute__((always_inline)) {
    int l = lane;
    asm volatile("" : "+v"(l));
    Tile::k_source(wave * NLD + n, l, rk, uk);
    Tile::v_source(l, rv, uv);
    rk += (wave * NLD + n) * RPL;
    rv += (wave * NLD + n) * RPL;
  };
  // 16 bytes a lane of a bf16 tensor straight to LDS address `to` (m0, which the compiler has for itself, is given
  // back; wait states: one after a write of m0, five after a VALU write of a scalar operand)
  auto load_direct = [&](const void* base, int size, uint32_t off, uint32_t to) __attribute__((always_inline)) {
    const uint64_t p = (uint64_t)base;
    const u32x4 r = u32x4{(uint32_t)p, (uint32_t)(p >> 32) & 0xFFFFu, (uint32_t)size, 0x00020000u};
    uint32_t m0;
    asm volatile(
        "s_mov_b32 %0, m0\n\ts_mov_b32 m0, %3\n\ts_nop 4\n\t"
        "buffer_load_dwordx4 %1, %2, 0 offen lds\n\ts_mov_b32 m0, %0"
        : "=&s"(m0)
        : "v"(off), "s"(r), "s"(to)
        : "memory");
  };
  // Codes.  Consecutive tiles in one segment are a run: their loads share the per-lane offsets, and the bases move
  // on.  A wave's chunks differ by RPL rows, and K's units by an exclusive or of the lowest bit.
  struct Codes {
    uint32_t kc[NLD], vc[NLD], ks[NLD], vs[NLD];
  };
  uint32_t k_off[NLD], v_off, ks_off, vs_off;
  {
    int rk, uk, rv, uv;
    place(0, rk, uk, rv, uv);
    v_off = (uint32_t)(rv * cbytes + kv * (D / 2) + uv * 4);
    ks_off = (uint32_t)(rk * sbytes + kv * (D / kQ4Group) + uk / 4);
    vs_off = (uint32_t)(rv * sbytes + kv * (D / kQ4Group) + uv / 4);
#pragma unroll
    for (int n = 0; n < NLD; ++n) k_off[n] = (uint32_t)((rk + n * RPL) * cbytes + kv * (D / 2) + (uk ^ n) * 4);
  }
  static_assert(NLD == 1 || Tile::CPB == 4, "K units of a wave's two chunks");
  const uint8_t *run_k = nullptr, *run_v = nullptr, *run_ks = nullptr, *run_vs = nullptr;
  int run_left = 0;                          // tiles left in the run, all below t_hi
  constexpr int NLOAD = 4 * NLD;
  auto load_run = [&](auto job, Codes& x) __attribute__((always_inline)) {
    constexpr int n = decltype(job)::value / 4, what = decltype(job)::value % 4;
    if constexpr (what == 0) x.kc[n] = __builtin_amdgcn_raw_buffer_load_b32(make_rsrc(run_k, BN * cbytes), k_off[n], 0, 0);
    if constexpr (what == 1) x.vc[n] = __builtin_amdgcn_raw_buffer_load_b32(make_rsrc(run_v, BN * cbytes), v_off + n * RPL * cbytes, 0, 0);
    if constexpr (what == 2) x.ks[n] = __builtin_amdgcn_raw_buffer_load_b8(make_rsrc(run_ks, BN * sbytes), ks_off + n * RPL * sbytes, 0, 0);
    if constexpr (what == 3) x.vs[n] = __builtin_amdgcn_raw_buffer_load_b8(make_rsrc(run_vs, BN * sbytes), vs_off + n * RPL * sbytes, 0, 0);
  };
  auto advance_run = [&]() __attribute__((always_inline)) {
    run_k += BN * cbytes;
    run_v += BN * cbytes;
    run_ks += BN * sbytes;
    run_vs += BN * sbytes;
    --run_left;
  };
  // codes in the registers to the buffers at `boff`: job 2n: K, 2n + 1: V
  constexpr int NCVT = 2 * NLD;
  auto convert = [&](auto job, uint32_t boff, const Codes& x) __attribute__((always_inline)) {
    constexpr int n = decltype(job)::value / 2;
    const uint32_t at = lds0 + boff + my_part + (uint32_t)(lane * 16 + n * 1024);
    if constexpr (decltype(job)::value % 2 == 0) *(lds_u4)(uintptr_t)(at + kKBase) = q4_eight(x.kc[n], q4_scale(x.ks[n]));
    else *(lds_u4)(uintptr_t)at = q4_eight(x.vc[n], q4_scale(x.vs[n]));
  };

  // sends the loads of tile t: codes and scale bytes to registers, bf16 rows to their buffers at `boff`
  auto send = [&](int t, uint32_t boff, Codes& x) __attribute__((always_inline)) {
    if (t >= t_hi) return;
    if (t >= nb_s && t < nb_sg) {
      const int i0 = (t - nb_s) * BN;
      if (run_left == 0) {
        int slot0;
        const int n = seg.straight(i0, slot0);
        run_left = min(n / BN, t_hi - t);
        run_k = a.k4 + (int64_t)slot0 * cbytes;
        run_v = a.v4 + (int64_t)slot0 * cbytes;
        run_ks = a.ks + (int64_t)slot0 * sbytes;
        run_vs = a.vs + (int64_t)slot0 * sbytes;
      }
      if (run_left > 0) {
        unrolled<NLOAD>([&](auto job) __attribute__((always_inline)) { load_run(job, x); });
        advance_run();
      } else {
        bool real;
        const int slot = seg.slot_of_lane(i0, BN, G, real);
#pragma unroll
        for (int n = 0; n < NLD; ++n) {
          int k_row, k_unit, v_row, v_unit;
          place(n, k_row, k_unit, v_row, v_unit);
          const int64_t sk = __shfl(slot, k_row, 64), sv = __shfl(slot, v_row, 64);
          const bool ok = __shfl((int)real, v_row, 64);
          x.kc[n] = *(const __attribute__((address_space(1))) uint32_t*)((gptr)a.k4 + sk * cbytes + kv * (D / 2) + k_unit * 4);
          x.ks[n] = *(const __attribute__((address_space(1))) uint8_t*)((gptr)a.ks + sk * sbytes + kv * (D / kQ4Group) + k_unit / 4);
          const uint32_t w = *(const __attribute__((address_space(1))) uint32_t*)((gptr)a.v4 + sv * cbytes + kv * (D / 2) + v_unit * 4);
          const uint32_t b = *(const __attribute__((address_space(1))) uint8_t*)((gptr)a.vs + sv * sbytes + kv * (D / kQ4Group) + v_unit / 4);
          x.vc[n] = ok ? w : 0;
          x.vs[n] = ok ? b : 127;
        }
      }
      return;
    }
    const late_args l = late();
    const bool sink = t < nb_s;
    const int row0 = (sink ? t : t - nb_sg) * BN, left = min((sink ? l->S : l->T) - row0, BN) * rbytes;
    const char* const bk = (const char*)(sink ? l->sink_k : l->tail_k) + (int64_t)row0 * rbytes;
    const char* const bv = (const char*)(sink ? l->sink_v : l->tail_v) + (int64_t)row0 * rbytes;
#pragma unroll
    for (int n = 0; n < NLD; ++n) {
      int k_row, k_unit, v_row, v_unit;
      place(n, k_row, k_unit, v_row, v_unit);
      const uint32_t to = lds0 + my_part + boff + n * 1024;
      load_direct(bk, left, (uint32_t)(k_row * rbytes + kv * RBY + k_unit * 16), to + kKBase);
      load_direct(bv, left, (uint32_t)(v_row * rbytes + kv * RBY + v_unit * 16), to);
    }
  };
  // tile t into its buffers at `boff`: converted from the registers, or landed
  bool odd = false;                          // a value of the tail that is not finite
  auto finish = [&](int t, uint32_t boff, const Codes& x) __attribute__((always_inline)) {
    if (t >= t_hi) return;
    if (t >= nb_s && t < nb_sg) {
      unrolled<NCVT>([&](auto job) __attribute__((always_inline)) { convert(job, boff, x); });
      return;
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    if (t < t_cut) return;
    const uint32_t at = lds0 + boff + my_part + (uint32_t)(lane * 16);
#pragma unroll
    for (int n = 0; n < NLD; ++n) {
      u32x4 y = *(lds_u4)(uintptr_t)(at + n * 1024);
      u16x2 most{0, 0};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        largest_exponents(most, y[i]);
        y[i] = finite_or_zero(y[i]);
      }
      odd |= not_finite(most);
      *(lds_u4)(uintptr_t)(at + n * 1024) = y;
    }
  };
  // what this wave wrote is there, and every other wave's
  auto meet = [&]() __attribute__((always_inline)) { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); };

  Codes codes;                               // of the tile after the last one in LDS
  f32x16 o[RB][NDB];
  float m_run[RB] = {-INFINITY}, l_run[RB] = {0.f}, neg_m[RB] = {INFINITY};
#pragma unroll
  for (int db = 0; db < NDB; ++db) o[0][db] = f32x16{};
  uint32_t k_rd[2], v_rd, v_nx;
  Tile::start(k_rd, v_nx);
  k_rd[0] += lds0 + kKBase;                  // the part's first tile: buffer 0
  k_rd[1] += lds0 + kKBase;
  v_nx += lds0;
  v_rd = v_nx + (NB - 1) * TBY;
  if (t_lo < t_hi) {
    {
      Codes c0, c1;                          // three tiles on the way together: one memory latency before the first step
      send(t_lo, 0, c0);
      send(t_lo + 1, TBY, c1);
      send(t_lo + 2, 2 * TBY, codes);
      finish(t_lo, 0, c0);
      finish(t_lo + 1, TBY, c1);
    }
    // the pipeline's first P V multiplies zero probabilities with the last 16 rows of the last V buffer (tile t_lo + 3
    // goes there after the first barrier of the loop)
    if (tid < RBY) *(lds_u4)(uintptr_t)(lds0 + (NB - 1) * TBY + 48 * RBY + tid * 16) = u32x4{0, 0, 0, 0};
    meet();
    uint32_t boff = 0;                       // buffer offset of tile t
    int t = t_lo;
    if (t < t_end) {
      bf16x8 vf[NDB] = {};
      Tile wt{qf, k_rd, v_rd, v_nx, o, m_run, l_run, neg_m, vf, a.scale_log2};
      f32x16 s0[RB], s1[RB];
      bf16x8 p0[RB][2] = {}, p1[RB][2] = {};
      wt.first_logits(s0);
      {
        const int lim[RB] = {lim_of(t)};
        if (cut(t)) Tile::mask(0, lim, hh, s0);
      }
      wt.first_max(s0);
      for (; t < t_end; ++t) {
        const bool masked = cut(t);
        const int lim[RB] = {lim_of(t)};
        if (__builtin_expect(masked, 0)) Tile::mask(0, lim, hh, s0);
        uint32_t next = 0;                   // of tile t + 1
        wt.template half<32, 48, 0>(s0, s1, p1, p0, [&](auto slot) __attribute__((always_inline)) {
          constexpr int s = decltype(slot)::value;
          if constexpr (s == Tile::NQK + Tile::NPV) {
            next = (boff + TBY) & kWrap;
            k_rd[0] += next - boff;          // K of tile t + 1
            k_rd[1] += next - boff;
            v_rd = v_nx;                     // V of tile t
          }
        });
        meet();
        if (__builtin_expect(masked, 0)) Tile::mask(32, lim, hh, s1);
        const uint32_t fill = (boff + 2 * TBY) & kWrap;
        // tile t + 2 is codes in the registers and t + 3 the run's next: one piece of that work a slot
        const bool in_run = run_left > 0 && t + 2 >= nb_s;
        if (!in_run) {
          finish(t + 2, fill, codes);
          send(t + 3, (fill + TBY) & kWrap, codes);
        }
        wt.template half<0, 16, 32>(s1, s0, p0, p1, [&](auto slot) __attribute__((always_inline)) {
          constexpr int s = decltype(slot)::value;
          if constexpr (s < NCVT + NLOAD) {
            if (in_run) {
              if constexpr (s < NCVT) convert(slot, fill, codes);
              else load_run(std::integral_constant<int, s - NCVT>{}, codes);
            }
          }
        });
        if (in_run) advance_run();
        v_nx += next - boff;                 // V of tile t + 1
        boff = next;
      }
      wt.template last_values<48>(p1);
    }
    for (; t < t_hi; ++t) {                  // tiles that this wave's rows do not see: it brings its share
      meet();
      finish(t + 2, (boff + 2 * TBY) & kWrap, codes);
      send(t + 3, (boff + 3 * TBY) & kWrap, codes);
      boff = (boff + TBY) & kWrap;
    }
  }

  // ---- values of the tail that are not finite
  if (odd) odd_s = 1;
  __syncthreads();
  if (!wave_active) return;
  if (__builtin_expect(odd_s != 0, 0)) {
    const int k0 = max(t_lo - nb_sg, 0) * BN, k1 = min(max(t_hi - nb_sg, 0) * BN, last_lim + 1);
    for (int k = k0; k < k1; ++k) {
      const uint16_t* p = late()->tail_v + ((int64_t)k * a.Hkv + kv) * D + hh * 4;
#pragma unroll
      for (int db = 0; db < NDB; ++db)
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          const uint32_t bits = (uint32_t)p[db * 32 + (v >> 2) * 8 + (v & 3)] << 16;
          o[0][db][v] += (k <= tail0 + tok && (bits & 0x7F800000u) == 0x7F800000u) ? __uint_as_float(bits) : 0.f;
        }
    }
  }

  const float l_tot = pair_sum(l_run[0]);
  const float inv = l_tot > 0.f ? 1.f / l_tot : l_tot == l_tot ? 0.f : l_tot;        // 0 for an empty row, NaN stays
  const float lse2 = l_tot > 0.f ? m_run[0] + __log2f(l_tot) : l_tot == l_tot ? -INFINITY : l_tot;
  if (wrow0 + l32 >= NR) return;
  const late_args l = late();
  const bool partial = l->parts > 1;
  if (partial || l->out_f32) {
    float* op = partial ? l->ws_o + (((int64_t)part * l->Hq + head) * l->Lq + tok) * D
                        : (float*)l->out + ((int64_t)tok * l->Hq + head) * D;
    op += hh * 4;
#pragma unroll
    for (int db = 0; db < NDB; ++db)
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4) {
        const f32x16& x = o[0][db];
        *(f32x4*)(op + db * 32 + q4 * 8) =
            f32x4{x[q4 * 4] * inv, x[q4 * 4 + 1] * inv, x[q4 * 4 + 2] * inv, x[q4 * 4 + 3] * inv};
      }
  } else {
    __bf16* op = (__bf16*)l->out + ((int64_t)tok * l->Hq + head) * D + hh * 4;
#pragma unroll
    for (int db = 0; db < NDB; ++db)
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4) {
        const f32x16& x = o[0][db];
        *(bf16x4*)(op + db * 32 + q4 * 8) = bf16x4{(__bf16)(x[q4 * 4] * inv), (__bf16)(x[q4 * 4 + 1] * inv),
                                                   (__bf16)(x[q4 * 4 + 2] * inv), (__bf16)(x[q4 * 4 + 3] * inv)};
      }
  }
  if (hh != 0) return;
  if (partial) l->ws_lse[((int64_t)part * l->Hq + head) * l->Lq + tok] = lse2;
  else if (l->lse) l->lse[(int64_t)head * l->Lq + tok] = lse2 * kLn2;
}

}  // namespace

hipError_t launch_tile_q4(const RowsQ4Args& a, hipStream_t stream) {
  if (a.n_segs > kMaxSegments || a.n_rt < 1 || a.parts < 1) return hipErrorInvalidValue;
  const dim3 grid(a.n_rt * a.parts * a.Hkv), block(kThreads);
  if (a.D == 128) hipLaunchKernelGGL(attn_tile_q4_kernel<128>, grid, block, 0, stream, a);
  else hipLaunchKernelGGL(attn_tile_q4_kernel<64>, grid, block, 0, stream, a);
  return hipGetLastError();
}

}  // namespace vico
