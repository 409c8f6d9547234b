// Attention over the cache in pages, many query rows a sequence (gfx950): what
// attn_rows_pages.h computes, for sequences whose rows share every key often
// enough to be bound by the matrix cores -- visual chunks, long queries.
//
// A work-group of 8 waves owns 256 packed (token, query head) rows of one KV head of
// one sequence, 32 a wave, and walks 64-key tiles of its visible positions; the tile
// body is PipeTile (attn_pipe.h), the software-pipelined one of the chunk prefill,
// with K and V loaded straight to LDS three tiles ahead and one barrier a tile.
//   * Tiles are aligned to positions, and a wave's share of a tile is 8 consecutive
//     rows: they lie in one page whatever its size (16 tokens at least).  So a page
//     costs a wave one scalar offset a tile.
//   * The page numbers of the part's tiles are in LDS, checked, two halves in turn: one
//     is filled while the other is read, in the middle of it, so that no wait or
//     barrier of its own is needed.
//   * Between sink and window nothing is walked; what no row of the sequence sees in the
//     two tiles there, behind the sequence's end or for want of a page becomes zero in LDS.
//   * Values that are not finite in tiles that the causal mask cuts are zeros in LDS (0
//     times such a value would reach rows that do not see it) and are added afterwards for
//     the rows that do.  Each wave looks at what it loaded, before the barrier that
//     shows it to the others.
// Which sequences these are stands in device memory, so every work-group counts the
// row tiles of all sequences and finds its own; where they leave CUs idle, key ranges
// are split and joined by the merge kernel.
// It is bound by the matrix cores, 68 % busy in a chunk of 2048 tokens over 16384 keys (7B
// heads, 513 GFLOP): 445 to 500 us a call by the box, 1030 to 1150 TFLOP/s; the chunk prefill
// over a dense ring took 447 to 473 on two boxes where this took 445 to 468.  What stands
// between its matrix instructions counts: with half of the CUs at work a tile takes 1.18 us (the
// chunk prefill's 1.14), 1.24 with a resource for each tile and its questions asked anew at each.
// A work-group's start takes 6 us: 1.6 for the lengths, 2.2 for page numbers and Q, 1.9
// for the first tile.

#pragma once

#include "attn_pipe.h"
#include "pages.h"
#include "values.h"

namespace vico {

typedef const __attribute__((address_space(4))) PagedAttnArgs* late_args;
// the kernel's arguments, read again where they are used: what only the start and the end need takes no registers
// in the loop
__device__ __forceinline__ late_args late() {
  late_args p = (late_args)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  return p;
}

// Row tiles on this kernel of a sequence with so many rows.
__device__ __forceinline__ int row_tiles(const PagedAttnArgs& a, int tokens) {
  const int rows = a.Hq / a.Hkv * min(tokens, a.max_q);
  return rows >= a.tile_least ? (rows + kBlockM - 1) / kBlockM : 0;
}
// The first 64 sequences, one a lane: first row, rows, length.
struct LaneSequences {
  int q0, rows, len;
};
__device__ __forceinline__ LaneSequences lane_sequences(const PagedAttnArgs& a) {
  const int lane = threadIdx.x & 63, b = min(lane, a.B - 1);
  LaneSequences x;
  x.rows = rows_of(a, b, x.q0);
  x.rows = lane < a.B ? x.rows : 0;
  x.len = a.seq_len[b];
  return x;
}
// Sequence b, the same one for all lanes; in scalar registers, whatever the compiler makes of loads whose address it cannot
// prove to be the same in all lanes.
__device__ __forceinline__ Sequence sequence(const PagedAttnArgs& a, const LaneSequences& x, int b) {
  int q0, rows, len;
  if (a.B <= 64) {
    q0 = __builtin_amdgcn_readlane(x.q0, b);
    rows = __builtin_amdgcn_readlane(x.rows, b);
    len = __builtin_amdgcn_readlane(x.len, b);
  } else {
    rows = __builtin_amdgcn_readfirstlane(rows_of(a, b, q0));
    q0 = __builtin_amdgcn_readfirstlane(q0);
    len = __builtin_amdgcn_readfirstlane(a.seq_len[b]);
  }
  return sequence(a, q0, rows, len);
}
// Row tiles of all sequences and heads, and the parts that their key ranges are split into.  Sequences of fewer rows count
// for their keys, once for the first row tile of 16 and half for each more (they meet in L2), if they are in this launch.
__device__ __forceinline__ int all_row_tiles(const PagedAttnArgs& a, const LaneSequences& x, int& parts) {
  const int lane = threadIdx.x & 63;
  int n = 0, keys = 0, beside = 0;           // (beside: half blocks)
  auto add = [&](int q0, int rows, int len) __attribute__((always_inline)) {
    const int m = row_tiles(a, rows);
    const Sequence s = sequence(a, q0, rows, len);
    n += m;
    if (a.tile_parts <= 1 || s.n <= 0) return;
    const int last = last_position(a, s, s.n - 1);
    keys = max(keys, m > 0 ? KeyBlocks<kKeyTile>(s).upto(last) : 0);
    const int tiles16 = (a.Hq / a.Hkv * s.n + 15) / 16;
    beside += m > 0 || a.rows_apart ? 0 : min(KeyBlocks<kRowsBlock>(s).upto(last), 1 << 16) * (1 + tiles16);
  };
  add(x.q0, x.rows, x.len);
  for (int b = lane + 64; b < a.B; b += 64) {
    int q0;
    const int rows = rows_of(a, b, q0);
    add(q0, rows, a.seq_len[b]);
  }
  n = __builtin_amdgcn_readlane(wave_scan(n), 63);
  const int items = n * a.Hkv;
  parts = max(a.tile_splits, 1);
  if (a.tile_parts <= 1 || items == 0) return items;
  // the most keys: lane 63's after the steps of wave_scan
  keys = max(keys, __builtin_amdgcn_update_dpp(0, keys, 0x111, 0xF, 0xF, true));
  keys = max(keys, __builtin_amdgcn_update_dpp(0, keys, 0x112, 0xF, 0xF, true));
  keys = max(keys, __builtin_amdgcn_update_dpp(0, keys, 0x114, 0xF, 0xF, true));
  keys = max(keys, __builtin_amdgcn_update_dpp(0, keys, 0x118, 0xF, 0xF, true));
  keys = max(keys, __builtin_amdgcn_update_dpp(0, keys, 0x142, 0xA, 0xF, false));
  keys = max(keys, __builtin_amdgcn_update_dpp(0, keys, 0x143, 0xC, 0xF, false));
  keys = __builtin_amdgcn_readlane(keys, 63);
  const float others = (float)__builtin_amdgcn_readlane(wave_scan(beside), 63) * (float)a.Hkv * (0.5f * paged_block_cost(a.D));
  // lane p - 1 takes p parts; of equal times the fewest
  static_assert(kPagedTileParts == 16, "one lane of a row for each number of parts");
  const int p = (lane & 15) + 1;
  const bool fits = p <= a.tile_parts && (p == 1 || items <= a.tile_slots / p);
  int best = fits ? (int)fminf(32.f * paged_tile_cost(items, keys, p, others), 16777215.f) : 1 << 24;
  best = best * 64 + p;
  constexpr int kNone = 0x7FFFFFFF;
  best = min(best, __builtin_amdgcn_update_dpp(kNone, best, 0x111, 0xF, 0xF, false));
  best = min(best, __builtin_amdgcn_update_dpp(kNone, best, 0x112, 0xF, 0xF, false));
  best = min(best, __builtin_amdgcn_update_dpp(kNone, best, 0x114, 0xF, 0xF, false));
  best = min(best, __builtin_amdgcn_update_dpp(kNone, best, 0x118, 0xF, 0xF, false));
  parts = __builtin_amdgcn_readlane(best, 15) & 63;
  return items;
}
// The sequence whose row tiles, each `times` times, hold item x; its first item and its row tiles.
__device__ __forceinline__ int sequence_of_item(const PagedAttnArgs& a, const LaneSequences& y, int x, int times, int& first,
                                                int& tiles) {
  const int lane = threadIdx.x & 63;
  int before = 0;
  for (int b0 = 0;; b0 += 64) {
    int q0;
    const int n = b0 == 0 ? row_tiles(a, y.rows) : b0 + lane < a.B ? row_tiles(a, rows_of(a, b0 + lane, q0)) : 0;
    const int upto = before + wave_scan(n) * times;
    const int all = __builtin_amdgcn_readlane(upto, 63);
    if (x < all || b0 + 64 >= a.B) {
      const int i = min(__builtin_popcountll(__builtin_amdgcn_ballot_w64(upto <= x)), 63);
      tiles = __builtin_amdgcn_readlane(n, i);
      first = __builtin_amdgcn_readlane(upto, i) - tiles * times;
      return b0 + i;
    }
    before = all;
  }
}

constexpr int kTabHalf = 1024;             // page numbers of a half of the table in LDS

template <int D>
struct TileLds {
  __attribute__((aligned(16))) uint8_t kv[2 * kBuffers * kKeyTile * D * 2];
  int32_t tab[2 * kTabHalf];
  int odd;
};

// Work-group `blk` of n_work: the row tiles times `parts`.
template <int D>
__device__ __forceinline__ void paged_tile(const PagedAttnArgs& a, const LaneSequences& y, int blk, int n_work, int parts,
                                           TileLds<D>& sh) {
  constexpr int RB = 1;
  typedef PipeTile<D, RB> Tile;
  constexpr int BN = kKeyTile, BM = kBlockM, NW = kThreads / 64;
  constexpr int RBY = D * 2;                 // bytes per LDS row
  constexpr uint32_t TBY = BN * RBY;         // bytes of one K (or V) tile
  constexpr int NLD = TBY / 1024 / NW;       // direct 1 KiB loads a wave and tile, of K and of V
  constexpr int RPL = Tile::RPC;             // rows of one
  constexpr int NDB = Tile::NDB, NKS = Tile::NKS;
  constexpr int NB = kBuffers, AHEAD = NB - 1;
  constexpr uint32_t kKBase = NB * TBY, kWrap = NB * TBY - 1;
  constexpr int NL = 2 * NLD, LSTEP = (Tile::NSLOT - 2) / (NL + 1);
  static_assert(NLD * NW * 1024 == TBY && BN == 64 && NLD * RPL == 8, "a wave loads 8 rows of a tile");
  static_assert(BM == NW * 32 && RB == kRowBlocks && (NB & (NB - 1)) == 0 && LSTEP >= 1, "tile geometry");
  typedef __attribute__((address_space(3))) u32x4* lds_u4;

  int32_t (&tab)[2 * kTabHalf] = sh.tab;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_void*)sh.kv;

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, hh = lane >> 5;
  const int g = a.Hq / a.Hkv;

  // ---- work item: the row tiles of one key range side by side (they share its K/V in an XCD's L2), longest first
  const int L = xcd_remap(blk, n_work);
  int first_item, cnt;
  const int b = __builtin_amdgcn_readfirstlane(sequence_of_item(a, y, L, a.Hkv * parts, first_item, cnt));
  // (in scalar registers, whatever the compiler makes of divisions: no branch of the key loop may be on lanes)
  const int kp = __builtin_amdgcn_readfirstlane((L - first_item) / cnt), rt = cnt - 1 - (L - first_item - kp * cnt);
  const int kv = __builtin_amdgcn_readfirstlane(kp / parts), part = kp - kv * parts;
  if (tid == 0) sh.odd = 0;
  const Sequence s = sequence(a, y, b);
  const int NR = g * s.n;
  if (parts > 1 && part == 0 && tid == 0)
    a.ws_items->item[(unsigned)first_item / (unsigned)parts + kv * cnt + cnt - 1 - rt] = TileItem{s.q0, NR, kv, rt, L, cnt};
  const KeyBlocks<BN> tiles(s);
  auto lim_of_row = [&](int r) __attribute__((always_inline)) { return last_position(a, s, a.by_g(min(r, NR - 1))); };

  // ---- this lane's packed row; rows past the end repeat the last one and are never stored
  const int wrow0 = rt * BM + wave * 32;
  const bool wave_active = wrow0 < NR;
  const int my_row = min(wrow0 + l32, NR - 1);
  const int tok = a.by_g(my_row), head = kv * g + my_row - tok * g;
  const int lim = last_position(a, s, tok);                        // the row's last position
  bf16x8 qf[RB][NKS];
  WaveTile<D>::load_q(qf[0], a.q + ((int64_t)(s.q0 + tok) * a.Hq + head) * D + hh * 8);

  // ---- tiles
  const int first_lim = __builtin_amdgcn_readfirstlane(lim_of_row(wrow0)), last_lim = __builtin_amdgcn_readfirstlane(lim_of_row(wrow0 + 31));
  const int n_tiles = __builtin_amdgcn_readfirstlane(tiles.upto(lim_of_row((rt + 1) * BM - 1)));
  const int t_lo = __builtin_amdgcn_readfirstlane((int)((int64_t)n_tiles * part / parts));
  const int t_hi = __builtin_amdgcn_readfirstlane((int)((int64_t)n_tiles * (part + 1) / parts));
  const int t_end = wave_active ? min(t_hi, tiles.upto(last_lim)) : t_lo;          // past the wave's last tile
  const int kv_end = __builtin_amdgcn_readfirstlane(lim_of_row(NR - 1) + 1);                       // rows of the sequence that exist
  const int cut_from = __builtin_amdgcn_readfirstlane(lim_of_row(rt * BM) + 1);                    // from here on some row of the work-group sees not all
  const int sink = s.sink, first = s.first;
  // Tiles [t_plain, t_plain + n_plain) need no mask for this wave, and [t_plain, t_plain + n_whole) none for any row of
  // the work-group: behind those that hold positions between sink and window, before the causal diagonal.  A page that
  // is none makes all tiles from there on masked ones.  (The sink's own tiles are masked ones: no matter at 64 tokens of it,
  // 10 % of a 2048-token chunk over 16448 keys of which 4096 are the sink's, 7B heads: 520 us for 472.)
  const int t_plain = sink < first ? tiles.of_sink + 1 : 0;
  auto upto_whole = [&](int lim_) __attribute__((always_inline)) {      // tiles that lie wholly in positions <= lim_
    const int n = (lim_ + 1) / BN;
    return min(n, tiles.of_sink) + max(n - tiles.from, 0);
  };
  int n_plain = max(upto_whole(first_lim) - t_plain, 0);
  const int n_whole = max(upto_whole(cut_from - 1) - t_plain, 0);

  // ---- page numbers: entry (t - t_lo) * EPT + e of the part's tile t, in tab at that number mod 2 * kTabHalf
  const int shift = a.page_shift;
  const int ept_shift = shift < 6 ? 6 - shift : 0;                 // 64 / page_size pages a tile, or one
  const int32_t* const row = a.table + (int64_t)b * a.width;
  const int n_entries = (t_hi - t_lo) << ept_shift;
  auto fill_tab = [&](int e0) __attribute__((always_inline)) {     // entries e0 .. e0 + kTabHalf - 1, without a branch
#pragma unroll
    for (int i = 0; i < kTabHalf / kThreads; ++i) {                // on lanes (past the last one: anything)
      const int e = e0 + i * kThreads + tid, in = min(e, n_entries - 1);
      const int p0 = tiles.position(t_lo + (in >> ept_shift)) + ((in & ((1 << ept_shift) - 1)) << (shift < 6 ? shift : 0));
      const int at = p0 >> shift;
      const int p = row[min(at, a.width - 1)];
      tab[e & (2 * kTabHalf - 1)] = ((at < a.width) & ((uint32_t)p < (uint32_t)a.N)) ? p : -1;
    }
  };

  // ---- tile loader
  const int rbytes = a.Hkv * D * 2;
  const uint32_t my_part = (uint32_t)(wave * NLD * 1024);
  uint32_t ld_k[NLD], ld_v;                                        // byte offsets from the wave's first row
  {
    int r, u;
#pragma unroll
    for (int n = 0; n < NLD; ++n) {
      Tile::k_source(wave * NLD + n, lane, r, u);
      ld_k[n] = (uint32_t)((n * RPL + r) * rbytes + u * 16);
    }
    Tile::v_source(lane, r, u);
    ld_v = (uint32_t)(r * rbytes + u * 16);
  }
  // Where the wave's rows of a tile lie in the pools, the same in both: lane i of `run` has it for the i-th of 64 tiles,
  // computed for all of them at once; a tile takes its own by lane reads.  It is the loads' scalar offset, below 2^31,
  // from a resource that holds for 2 GiB of the pool; for rows without a page, page 0 is read, and look() makes them
  // zeros.  (A resource of its own for each tile took 4 % longer: each scalar instruction between MFMAs counts.)
  const int my_page = shift < 6 ? (8 * wave) >> shift : 0, in_page = (1 << shift) - 1;
  uint32_t run_lo = 0, run_hi = 0;
  // the resources, `window` 2 GiB pieces into the pools (addresses are below 2^48)
  auto resource = [&](const uint16_t* pool, uint32_t window) __attribute__((always_inline)) {
    const late_args l = late();
    const uint64_t before = ((uint64_t)window << 31) + (uint32_t)(kv * RBY), p = (uint64_t)pool + before;
    const uint64_t left = ((uint64_t)(uint32_t)l->N << l->page_shift) * (uint32_t)(l->Hkv * RBY) - before;
    const uint32_t bytes = left > 0xFFFFFFFFull ? 0xFFFFFFFFu : (uint32_t)left;
    return u32x4{(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)p), (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(p >> 32)),
                 (uint32_t)__builtin_amdgcn_readfirstlane(bytes), 0x00020000u};
  };
  u32x4 run_k = resource(late()->k_pages, 0), run_v = resource(late()->v_pages, 0);
  uint32_t run_at = 0, run_window = 0;       // of the tile to be loaded
  // the 64 tiles lie in several windows: moved at each of them (2048 tokens over 16384 keys, 7B heads, pages all over a pool
  // of 2, 5 and 10 GB: 464, 487 and 487 us; 455 in one of 19 MB)
  bool far = false;
  auto start_tile = [&](int t) __attribute__((always_inline)) { run_at = __builtin_amdgcn_readlane(run_lo, (t - t_lo) & 63); };
  auto move_window = [&](uint32_t window) __attribute__((always_inline)) {
    if (window == run_window) return;
    run_window = window;
    run_k = resource(late()->k_pages, window);
    run_v = resource(late()->v_pages, window);
  };
  auto find_tiles = [&](int t) __attribute__((always_inline)) {                     // of tiles t .. t + 63
    const int tl = t + lane, e0 = (tl - t_lo) << ept_shift;
    const int pos = tiles.position(tl), size = min(1 << shift, BN);
    bool bad = false;                        // no page where some row sees a position
    for (int e = 0; e < 1 << ept_shift; ++e) {
      const int at = pos + e * size;
      bad |= (tab[(e0 + e) & (2 * kTabHalf - 1)] < 0) & (at < kv_end) & !((at >= sink) & (at + size <= first));
    }
    const bool some = tl < t_hi;             // past the part's last tile: nothing
    n_plain = __builtin_amdgcn_ballot_w64(some & bad) != 0 ? 0 : n_plain;
    const int page = tab[(e0 + my_page) & (2 * kTabHalf - 1)], p0 = pos + 8 * wave;
    const int there = (some & (page >= 0)) ? page : 0;
    const uint64_t at = (uint64_t)(((uint32_t)there << shift) + (uint32_t)(p0 & in_page)) * (uint32_t)rbytes;
    run_lo = (uint32_t)at & 0x7FFFFFFFu;
    run_hi = (uint32_t)(at >> 31);
    const uint32_t window = __builtin_amdgcn_readlane(run_hi, 0);
    far = __builtin_amdgcn_ballot_w64(some & (run_hi != window)) != 0;
    if (!far) move_window(window);
  };
  // direct load i (0 .. NLD-1: K, NLD .. 2*NLD-1: V) to the buffers at byte offset `boff`.  m0, which holds a load's
  // LDS address, is the compiler's own: every load sets it and gives it back.  Wait states that the compiler does not
  // know assembly to need: one after a write of m0, five after a VALU write of a scalar operand.
  auto load_direct = [&](auto idx, uint32_t boff) __attribute__((always_inline)) {
    constexpr int i = decltype(idx)::value, n = i % NLD;
    const uint32_t off = i < NLD ? ld_k[n] : ld_v + n * RPL * rbytes;
    const uint32_t to = lds0 + my_part + boff + (i < NLD ? kKBase : 0u) + n * 1024;
    const u32x4 rs = i < NLD ? run_k : run_v;
    const uint32_t so = run_at;
    uint32_t m0;
    asm volatile(
        "s_mov_b32 %0, m0\n\ts_mov_b32 m0, %3\n\ts_nop 4\n\t"
        "buffer_load_dwordx4 %1, %2, %4 offen lds\n\ts_mov_b32 m0, %0"
        : "=&s"(m0)
        : "v"(off), "s"(rs), "s"(to), "s"(so)
        : "memory");
  };
  auto load_whole = [&](uint32_t boff, int t) __attribute__((always_inline)) {
    start_tile(t);
    move_window(__builtin_amdgcn_readlane(run_hi, (t - t_lo) & 63));
    unrolled<NL>([&](auto i) __attribute__((always_inline)) { load_direct(i, boff); });
  };

  // ---- the wave's share of V of tile t, landed at `boff`: zeros for what no row sees (the sequence's last tile is cut by
  // the mask, so its end is among them), and for what is not finite where the mask cuts
  uint32_t odd = 0;
  auto look = [&](int t, uint32_t boff) __attribute__((always_inline)) {
    if (__builtin_expect((uint32_t)(t - t_plain) >= (uint32_t)n_whole || n_plain == 0, 0)) {
      const int pos = tiles.position(t);
      const bool none = tab[(((t - t_lo) << ept_shift) + my_page) & (2 * kTabHalf - 1)] < 0;
      const uint32_t at = lds0 + boff + my_part + (uint32_t)(lane * 16);
      int r, u;
      Tile::v_source(lane, r, u);
#pragma unroll
      for (int n = 0; n < NLD; ++n) {
        u32x4 y = *(lds_u4)(uintptr_t)(at + n * 1024);
        const int p = pos + 8 * wave + n * RPL + r;
        const uint32_t keep = (none | ((p >= sink) & (p < first)) | (p >= kv_end)) ? 0u : ~0u;
        u16x2 most{0, 0};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          y[i] &= keep;
          largest_exponents(most, pos + BN > cut_from ? y[i] : 0u);
          y[i] = pos + BN > cut_from ? finite_or_zero(y[i]) : y[i];
        }
        odd |= not_finite(most) ? 1u : 0u;
        *(lds_u4)(uintptr_t)(at + n * 1024) = y;
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }
  };
  // what the mask takes from a half of tile t, whose keys start at position p0
  auto mask = [&](int t, int p0, f32x16& x) __attribute__((always_inline)) {
    const int e0 = (t - t_lo) << ept_shift, per = shift < 6 ? shift : 6;
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      const int at = 8 * (v >> 2) + hh * 4 + (v & 3), p = p0 + at;
      const bool none = p > lim || (p >= sink && p < first);
      x[v] = none ? -INFINITY : x[v];
    }
    if (n_plain == 0) {
#pragma unroll
      for (int q = 0; q < 4; ++q) {          // eight keys lie in one page
        const int in_tile = ((p0 & 32) | (8 * q)) >> per;
        const bool none = tab[(e0 + in_tile) & (2 * kTabHalf - 1)] < 0;
#pragma unroll
        for (int v = 4 * q; v < 4 * q + 4; ++v) x[v] = none ? -INFINITY : x[v];
      }
    }
  };

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
    fill_tab(0);
    fill_tab(kTabHalf);
    // the pipeline's first P V multiplies zero probabilities with the last 16 rows of the last V buffer: any bits
    // there must be finite
    if (tid < RBY) *(lds_u4)(uintptr_t)(lds0 + (NB - 1) * TBY + 48 * RBY + tid * 16) = u32x4{0, 0, 0, 0};
    __syncthreads();
    find_tiles(t_lo);
#pragma unroll 1
    for (int i = 0; i < AHEAD; ++i) load_whole(i * TBY, t_lo + i);
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"((AHEAD - 1) * NL) : "memory");      // tile t_lo
    look(t_lo, 0);
    barrier_keep_loads();
    // the half of the table that is not in use is filled for its next turn as the loads pass the middle of the other
    // (t: the last tile that has been sent)
    auto more_tab = [&](int t) __attribute__((always_inline)) {
      if (__builtin_expect(((t + 1 - t_lo) & 63) != 0, 1)) return;
      const int e = (t + 1 - t_lo) << ept_shift;
      if ((e & (kTabHalf - 1)) == kTabHalf / 2 && e > kTabHalf) fill_tab(e - kTabHalf / 2 + kTabHalf);
      find_tiles(t + 1);
    };
    uint32_t boff = 0;                       // buffer offset of tile t
    int t = t_lo;
    if (t < t_end) {
      bf16x8 vf[NDB] = {};
      Tile wt{qf, k_rd, v_rd, v_nx, o, m_run, l_run, neg_m, vf, a.scale_log2};
      f32x16 s0[RB], s1[RB];
      bf16x8 p0[RB][2] = {}, p1[RB][2] = {};
      // How many tiles from t on need no mask, have none to look at behind them, no page numbers to be found and no
      // window to move: their steps ask for nothing but this, once between the halves and once at the end (no MFMA's shadow lies on either).
      auto quiet_from = [&](int t) __attribute__((always_inline)) {
        const int plain = (uint32_t)(t - t_plain) < (uint32_t)n_plain ? t_plain + n_plain - t : 0;
        const int whole = (uint32_t)(t + 1 - t_plain) < (uint32_t)n_whole ? t_plain + n_whole - t - 1 : 0;
        return far ? 0 : __builtin_amdgcn_readfirstlane(min(min(plain, whole), -(t + AHEAD + 1 - t_lo) & 63));
      };
      auto cut = [&](int t) __attribute__((always_inline)) { return (uint32_t)(t - t_plain) >= (uint32_t)n_plain; };
      wt.first_logits(s0);
      if (cut(t)) mask(t, tiles.position(t), s0[0]);
      wt.first_max(s0);
      int quiet = quiet_from(t);
      for (; t < t_end; ++t) {
        uint32_t next = 0;                   // of tile t + 1
        wt.template half<32, 48, 0>(s0, s1, p1, p0, [&](auto slot) __attribute__((always_inline)) {
          constexpr int i = decltype(slot)::value;
          if constexpr (i == Tile::NPV + 2) start_tile(t + AHEAD);
          if constexpr (i == Tile::NQK + Tile::NPV) {
            next = (boff + TBY) & kWrap;
            k_rd[0] += next - boff;          // K of tile t + 1
            k_rd[1] += next - boff;
            v_rd = v_nx;                     // V of tile t
          }
        });
        // tile t + 1 has landed (the loads of the AHEAD - 2 tiles after it may be in flight), for this wave ...
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"((AHEAD - 2) * NL) : "memory");
        if (__builtin_expect(quiet <= 0, 0)) {
          move_window(__builtin_amdgcn_readlane(run_hi, (t + AHEAD - t_lo) & 63));
          look(t + 1, next);
          if (cut(t)) mask(t, tiles.position(t) + 32, s1[0]);
        }
        barrier_keep_loads();                // ... and every other
        const uint32_t fill = (boff + AHEAD * TBY) & kWrap;
        wt.template half<0, 16, 32>(s1, s0, p0, p1, [&](auto slot) __attribute__((always_inline)) {
          constexpr int j = decltype(slot)::value, i = j / LSTEP - 1;
          if constexpr (j % LSTEP == 0 && i >= 0 && i < NL) load_direct(std::integral_constant<int, i>{}, fill);
        });
        v_nx += next - boff;                 // V of tile t + 1
        boff = next;
        if (__builtin_expect(--quiet <= 0, 0)) {
          more_tab(t + AHEAD);
          quiet = quiet_from(t + 1);
          if (cut(t + 1)) mask(t + 1, tiles.position(t + 1), s0[0]);
        }
      }
      wt.template last_values<48>(p1);
    }
    for (; t < t_hi; ++t) {                  // tiles that this wave's rows do not see: it brings its share
      const uint32_t next = (boff + TBY) & kWrap;
      asm volatile("s_waitcnt vmcnt(%0)" ::"n"((AHEAD - 2) * NL) : "memory");
      look(t + 1, next);
      barrier_keep_loads();
      load_whole((boff + AHEAD * TBY) & kWrap, t + AHEAD);
      boff = next;
      more_tab(t + AHEAD);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");     // the empty loads past the last tile
  }

  // ---- values of the cut tiles that are not finite
  if (odd != 0) sh.odd = 1;
  __syncthreads();
  if (!wave_active) return;
  const late_args l = late();
  if (__builtin_expect(sh.odd != 0, 0)) {
    for (int t = t_lo; t < t_hi; ++t) {
      const int pos = tiles.position(t);
      if (pos + BN <= cut_from) continue;
      for (int p = pos; p <= min(pos + BN - 1, last_lim); ++p) {
        const int page = row[p >> shift];
        if ((uint32_t)page >= (uint32_t)a.N || (p >= sink && p < first)) continue;
        const uint16_t* v0 = l->v_pages + ((((int64_t)page << shift) + (p & ((1 << shift) - 1))) * a.Hkv + kv) * D + hh * 4;
#pragma unroll
        for (int db = 0; db < NDB; ++db)
#pragma unroll
          for (int v = 0; v < 16; ++v) {
            const uint32_t bits = (uint32_t)v0[db * 32 + (v >> 2) * 8 + (v & 3)] << 16;
            o[0][db][v] += (p <= lim && (bits & 0x7F800000u) == 0x7F800000u) ? __uint_as_float(bits) : 0.f;
          }
      }
    }
  }

  const float l_tot = pair_sum(l_run[0]);
  const float inv = l_tot > 0.f ? 1.f / l_tot : l_tot == l_tot ? 0.f : l_tot;        // 0 for an empty row, NaN stays
  const float lse2 = l_tot > 0.f ? m_run[0] + __log2f(l_tot) : l_tot == l_tot ? -INFINITY : l_tot;
  if (wrow0 + l32 >= NR) return;
  const bool partial = parts > 1;
  const int64_t prow = (int64_t)L * BM + wave * 32 + l32;
  if (partial || l->out_f32) {
    float* op = partial ? l->ws_o + prow * D : (float*)l->out + ((int64_t)(s.q0 + tok) * l->Hq + head) * D;
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
    __bf16* op = (__bf16*)l->out + ((int64_t)(s.q0 + tok) * l->Hq + head) * D + hh * 4;
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
  if (partial) l->ws_lse[prow] = lse2;
  else if (l->lse) l->lse[(int64_t)head * l->total + s.q0 + tok] = lse2 * kLn2;
}

// The parts of a row tile joined, as in attn_rows_pages.h: one thread takes four columns of a row, all parts' loads
// together.
template <int D, int NP>
__device__ __forceinline__ f32x4 joined(const PagedAttnArgs& a, int64_t row0, int64_t step, int parts, int dq, float& lse2) {
  float ls[NP];
  f32x4 os[NP];
#pragma unroll
  for (int i = 0; i < NP; ++i) {             // past the last part: the last one again, with a weight of 0
    const int64_t at = row0 + min(i, parts - 1) * step;
    ls[i] = i < parts ? a.ws_lse[at] : -INFINITY;
    os[i] = *(const f32x4*)(a.ws_o + at * D + dq * 4);
  }
  float m = -INFINITY;
#pragma unroll
  for (int i = 0; i < NP; ++i) m = fmaxf(m, ls[i]);
  const float use = m == -INFINITY ? 0.f : m;
  float sum = 0.f;
  f32x4 acc{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    const float w = __builtin_amdgcn_exp2f(ls[i] - use);
    sum += w;
    acc += w * os[i];
  }
  acc *= sum > 0.f ? 1.f / sum : sum == sum ? 0.f : sum;
  lse2 = sum > 0.f ? use + __log2f(sum) : sum == sum ? -INFINITY : sum;
  return acc;
}

constexpr int kTileMergeRows = 32;         // rows of a work-group
template <int D>
__device__ __forceinline__ void paged_tile_merge(const PagedAttnArgs& a, int blk) {
  constexpr int NQ = D / 4, RPB = kMergeThreads / NQ, CH = kBlockM / kTileMergeRows;
  const int it = blk / CH;
  const TileItem x = a.ws_items->item[it];       // (whatever stands there past the last one)
  const int parts = a.ws_items->parts;
  if (it >= a.ws_items->items) return;
  const int g = a.Hq / a.Hkv, dq = threadIdx.x % NQ;
  const int64_t item0 = (int64_t)x.slot * kBlockM, step = (int64_t)x.step * kBlockM;
#pragma unroll
  for (int i = 0; i < kTileMergeRows / RPB; ++i) {
    const int r = (blk - it * CH) * kTileMergeRows + i * RPB + threadIdx.x / NQ, pr = x.rt * kBlockM + r;
    if (pr >= x.rows) return;
    float lse2;
    f32x4 acc;
    if (parts <= 2) acc = joined<D, 2>(a, item0 + r, step, parts, dq, lse2);
    else if (parts <= 4) acc = joined<D, 4>(a, item0 + r, step, parts, dq, lse2);
    else if (parts <= 8) acc = joined<D, 8>(a, item0 + r, step, parts, dq, lse2);
    else acc = joined<D, 16>(a, item0 + r, step, parts, dq, lse2);
    const int t = a.by_g(pr), h = x.kv * g + pr - t * g;
    const int64_t orow = (int64_t)(x.q0 + t) * a.Hq + h;
    if (a.out_f32) *(f32x4*)((float*)a.out + orow * D + dq * 4) = acc;
    else *(bf16x4*)((__bf16*)a.out + orow * D + dq * 4) = bf16x4{(__bf16)acc[0], (__bf16)acc[1], (__bf16)acc[2], (__bf16)acc[3]};
    if (dq == 0 && a.lse) a.lse[(int64_t)h * a.total + x.q0 + t] = lse2 * kLn2;
  }
}

}  // namespace vico
