// Host side of include/vico_pages.h: argument validation, launch planning and
// error mapping, as vico_api.hip does it for vico.h.

#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "vico_pages.h"
#include "pages.h"
#include "host_util.h"

using namespace vico;

namespace {

struct Region {
  const void* p;
  int64_t bytes;
};

// Whether a written region meets any other region, written or read.
template <int NW, int NR>
bool collide(const Region (&w)[NW], const Region (&r)[NR]) {
  for (int i = 0; i < NW; ++i) {
    if (!w[i].p) continue;
    for (int k = 0; k < NR; ++k)
      if (r[k].p && overlaps(w[i].p, w[i].bytes, r[k].p, r[k].bytes)) return true;
    for (int k = i + 1; k < NW; ++k)
      if (w[k].p && overlaps(w[i].p, w[i].bytes, w[k].p, w[k].bytes)) return true;
  }
  return false;
}

bool heads_ok(int32_t Hq, int32_t Hkv) { return Hq >= 1 && Hkv >= 1 && Hq <= kMaxHeads && Hkv <= kMaxHeads; }

// The table's sizes; page_size 0: the call has none.
bool table_ok(int32_t B, int32_t width, int32_t N, int32_t page_size) {
  if (B < 0 || B > kMaxSeqs || width < 0 || N < 0 || N > kMaxPages) return false;
  if (int64_t(B) * width > kMaxKeys || width > kMaxKeys / 16) return false;
  if (page_size == 0) return true;
  return page_size >= 16 && page_size <= 1024 && (page_size & (page_size - 1)) == 0 && int64_t(width) * page_size <= kMaxKeys;
}
int shift_of(int32_t page_size) { return __builtin_ctz((unsigned)page_size); }
int64_t pool_bytes(int64_t N, int64_t page_size, int64_t Hkv, int64_t D) { return N * page_size * Hkv * D * 2; }

int status_of(hipError_t e) { return e == hipSuccess ? VICO_OK : record_hip_failure(e); }

int page_blocks(int32_t N) { return (N + kPageBlock - 1) / kPageBlock; }
int64_t table_workspace(int32_t B, int32_t N) {
  const int64_t words = int64_t(page_blocks(N)) * (kPageBlock / 64);
  return 2 * align256(words * 8) + align256(int64_t(page_blocks(N)) * 4) + align256(int64_t(B) * 4);
}
void use_workspace(PagesArgs* a, void* workspace) {
  const int64_t words = int64_t(a->n_blocks) * (kPageBlock / 64);
  char* p = (char*)workspace;
  a->flags = (uint64_t*)p;
  p += align256(words * 8);
  a->flags1 = (uint64_t*)p;
  p += align256(words * 8);
  a->blocks = (int32_t*)p;
  p += align256(int64_t(a->n_blocks) * 4);
  a->need = (int32_t*)p;
}

// ---- attention: the classes of sequences that a call may have, and how their keys are split.
constexpr int kFewRows = 16;
constexpr int64_t kMaxGroups = int64_t(1) << 23;                           // work-groups of a launch: fewer
constexpr int kSomeRows = 64;                                              // more: 256-row tiles, in a launch that has them
constexpr int kRowsOnly = 1024;                                            // a launch may do without them up to here (rows_alone)
constexpr int64_t kPagedWorkspace = int64_t(64) << 20;                     // most bytes of a split picked by the library

int64_t items_bytes(int64_t items) { return align256(sizeof(TileItems) + items * sizeof(TileItem)); }

struct PagedPlan {
  RowsClass few, some;
  bool apart;                // 256-row tiles and the others in a launch each
  int some_most, tile_grid, tile_items, tile_slots, tile_parts, tile_splits;
  int64_t few_ws, some_ws, ws_bytes;
};
int64_t partial_bytes(int64_t slots, int64_t rows, int64_t D) { return align256(slots * rows * D * 4) + align256(slots * rows * 4); }

// A class of sequences with up to `rows` rows over `keys` keys, in work-groups of which `target` are wanted.
// A part has two steps of each wave at least, 1.1 us each, where the merge's launch costs 3.3: eight 32-key blocks on the
// kernels of four waves, sixteen beside 256-row tiles.  (Four waves, least blocks of a part 4 / 8 / 16 / all in one, us: 7B heads, 35 rows over 500 keys 12.0 / 13.4 / 12.6 / 12.5,
// over 1000 12.4 / 13.4 / 15.8 / 17.0, over 2000 12.3 / 14.6 / 17.9 / 25.8; four sequences of 70 rows over 1000 15.3 / 14.2 /
// 16.4 / 17.7, over 2000 24.9 / 18.6 / 18.9 / 26.4; 3B heads, 144 rows over 1000 12.5 / 13.5 / 16.3 / 17.8; one token of 7B
// heads over 500 9.5 / 10.5 / 9.6 / 9.6, over 2000 9.6 / 11.5 / 14.3 / 22.6, of 16 sequences over 2000 20.1 / 19.0 / 19.3 / 24.1.)
bool plan_rows(RowsClass* x, int64_t least, int64_t rows, int tile_rows, int waves, int64_t B, int64_t Hkv, int64_t keys,
               int64_t target, int splits) {
  x->least = (int)least;
  x->most = (int)rows;
  x->tile_rows = tile_rows;
  x->n_rt = (int)((rows + tile_rows - 1) / tile_rows);
  x->merge_rows = (int)std::min<int64_t>(rows, tile_rows);
  const int64_t groups = B * Hkv * x->n_rt, blocks = keys / kRowsBlock + 1;
  x->parts = splits > 0 ? std::min(splits, kPagedParts)
                        : (int)std::max<int64_t>(std::min(std::min<int64_t>(kPagedParts, target / groups), blocks / (2 * waves)), 1);
  x->per_part = splits > 0 ? 1 : (int)((blocks + x->parts - 1) / x->parts);
  // (a launch has fewer than 2^32 threads: 512 a work-group, and 256 in the merge, with a row or more)
  const int64_t launched = (B * x->parts + 7) / 8 * 8 * Hkv * x->n_rt;
  if (launched >= kMaxGroups / 2 || (x->parts > 1 && groups * tile_rows >= kMaxGroups / 2)) return false;
  x->slots = (int)(groups * x->parts);
  x->groups = (int)launched;
  x->by_rt = FastDiv::by(x->n_rt);
  x->by_parts = FastDiv::by(x->parts);
  return true;
}

// Whether the call does without 256-row tiles: its time on row tiles of 32 against theirs, from the rows that its sequences
// have on average.  Each row tile of 32 streams its keys for itself, 1.6 ns for a 32-key block with all CUs at work (1.1
// with heads of size 64); 256 rows read them once, but a launch with such tiles starts slowly and has few of them.
// Measured, us, 32-row tiles / 256-row tiles, 7B heads: one sequence of 126 rows over 8000 keys 20.5 / 30.9, 252 rows
// 25.9 / 36.6, 511 rows 34.0 / 42.2, over 40000 keys 108.5 / 83.6; eight of 35 rows over 8000 keys 42.3 / 39.9, of 70
// rows 55.7 / 41.1, of 252 rows over 1000 keys 32.2 / 37.7, over 8000 keys 93.9 / 60.2; 3B heads, eight of 144 rows over
// 8000 keys 50.1 / 41.5; small heads, one of 292 rows over 8000 keys 14.7 / 25.5, eight 47.9 / 37.9.
// Past kRowsOnly the 256-row tiles win nearly everywhere, and these formulas, which know no more than the streams, do not
// see it: one sequence over 300 keys, 7B heads, 1050 rows 36.3 / 22.9, 2100 rows 67.3 / 26.7; 3B heads, 1200 rows 25.2 / 22.8,
// over 1000 keys 26.4 / 30.6, 2400 rows 37.2 / 26.2; small heads, 1200 rows 15.3 / 18.8, over 1000 keys 15.2 / 23.6, four of
// them 28.4 / 26.9, 2800 rows 30.5 / 24.9.
bool rows_alone(int64_t B, int64_t rows, int64_t all, int64_t Hkv, int64_t keys, int D) {
  if (rows > kRowsOnly) return false;
  const double tiles32 = double(Hkv) * (double(all) / 32 + double(B));
  const double t_rows = (D == 128 ? 12.0 : 8.0) + (D == 128 ? 1.6e-3 : 1.1e-3) * tiles32 * double(keys) / kRowsBlock;
  const int64_t each = std::max<int64_t>((all / B + kBlockM - 1) / kBlockM, 1), items = Hkv * B * each;
  if (items > (1 << 20)) return false;
  const int tiles = (int)(keys / kKeyTile) + 1;
  const int p = paged_tile_parts((int)items, tiles, std::max(std::min(tiles / kMinSplitTiles, kPagedTileParts), 1), 450);
  const double t_tile = 6.5 + (D == 128 ? 1.2 : 0.8) * double(paged_tile_cost((int)items, tiles, p, 0.f));     // (short: no power limit)
  return t_rows <= t_tile;
}

// Whether sequences of few rows get a launch of their own where the call has 256-row tiles.  Beside those, each of their
// work-groups (five for a sequence and KV head, most of them of another class) starts with all lengths, about B / 160 us,
// one work-group a CU; apart, the two kinds wait for each other.
// Measured, us, one launch / two, 7B heads, a chunk of 1024 tokens over 4000 keys beside decode steps over 200 each: 255
// of them 165 / 118, 330 204 / 124, 511 288 / 141, 1023 756 / 222, 4095 8578 / 769; over 8000 beside 2000: 255 341 / 395,
// 330 436 / 427, 511 658 / 546; over 8192 beside 8192: 200 750 / 876; 3B heads, 512 over 4000 beside 1000: 255 136 / 130,
// 463 179 / 153, 1023 490 / 267, 4095 5093 / 986; small heads, 512 over 2000 beside 1000: 255 81 / 71, 463 118 / 71, 1023
// 377 / 145, 4095 4603 / 522.
bool rows_apart(int64_t B, int64_t Hkv, int splits) {
  const int64_t groups = 5 * B * Hkv * std::max(std::min(splits, kPagedParts), 1);
  return groups * B > (1 << 21);             // 50 us of all CUs
}

int check_paged_shape(int32_t B, int32_t total, int32_t max_q, int32_t page_size, int32_t width, int32_t S, int64_t W,
                      int64_t hint, int32_t Hq, int32_t Hkv, int32_t D, int32_t splits, PagedPlan* pl) {
  if (total < 0 || max_q < 0 || S < 0 || W < VICO_FULL_HISTORY || hint < 0 || splits < 0) return VICO_ERR_INVALID_ARG;
  if (!heads_ok(Hq, Hkv) || Hq % Hkv != 0) return VICO_ERR_INVALID_ARG;
  if (D != 64 && D != 128) return VICO_ERR_UNSUPPORTED;
  if (page_size == 0 || !table_ok(B, width, 0, page_size)) return VICO_ERR_INVALID_ARG;
  if (total > kMaxChunk || int64_t(total) * Hq * D * 4 >= kMaxTensorBytes) return VICO_ERR_INVALID_ARG;
  *pl = PagedPlan{};
  const int n = std::min(max_q, total), g = Hq / Hkv;
  if (n == 0 || B == 0) return VICO_OK;
  const int64_t cap = int64_t(width) * page_size, rows = int64_t(g) * n;
  int64_t keys = std::min(hint > 0 ? hint : cap, cap);
  if (W != VICO_FULL_HISTORY && W < keys) keys = std::min(keys, S + W + n);
  // work-groups: some rounds of them where sequences differ (answer tokens of 32 sequences of 1000 to 16000 keys, us
  // with 4, 8, 12, 16 a CU: 123.0, 124.1, 120.7, 120.2); in a launch with 256-row tiles as many as leave those
  // room for their partial results.  One sequence is no exception: how many of the call's rows are its own stands in
  // device memory.  (7B heads, room for 2048 rows, us with all of them taken for the sequence's / as here: one token over
  // 8000 keys 77 / 13, over 262144 keys 3195 / 106, 300 tokens over 8000 keys 169 / 58; all 2048 over 16384 keys
  // 449 to 453 / 450; 3B heads, 500 of 500 over 500 keys 33.2 / 35.2, the merge's launch.)
  const int64_t all = int64_t(total) * g;
  const bool tile = rows > kSomeRows && !rows_alone(B, rows, all, Hkv, keys, D);
  const int64_t some_most = tile ? kSomeRows : rows;
  const int64_t groups = int64_t(B) * Hkv;
  pl->apart = tile && rows_apart(B, Hkv, splits);
  const bool beside = tile && !pl->apart;
  const int waves = beside ? 8 : 4;
  const int64_t target = beside ? std::min<int64_t>(std::max<int64_t>(8 * groups, kNumCUs), 4 * kNumCUs)
                                : (B == 1 ? 2 : rows > kFewRows ? 4 : 12) * kNumCUs;
  if (!plan_rows(&pl->few, 1, std::min<int64_t>(rows, kFewRows), 16, waves, B, Hkv, keys, target, splits)) return VICO_ERR_INVALID_ARG;
  if (pl->few.parts > 1) pl->few_ws = partial_bytes(pl->few.slots, 16, D);
  if (rows > kFewRows) {
    if (!plan_rows(&pl->some, kFewRows + 1, some_most, beside ? 16 : 32, waves, B, Hkv, keys,
                   beside ? std::min<int64_t>(target, kNumCUs / 4) : target, splits))
      return VICO_ERR_INVALID_ARG;
    if (pl->some.parts > 1) pl->some_ws = partial_bytes(pl->some.slots, pl->some.tile_rows, D);
  }
  pl->some_most = (int)some_most;
  pl->ws_bytes = pl->few_ws + pl->some_ws;
  if (!tile) return VICO_OK;
  // row tiles of 256: of a sequence its rows rounded up, and such a sequence has more than kSomeRows
  const int64_t items = Hkv * (all / kBlockM + std::min<int64_t>(B, all / (kSomeRows + 1)));
  pl->tile_splits = std::min(splits, kPagedTileParts);
  if (items * std::max(pl->tile_splits, 8) >= kMaxGroups / 2) return VICO_ERR_INVALID_ARG;
  pl->tile_items = (int)items;
  if (splits > 0) {
    pl->tile_slots = pl->tile_grid = (int)items * pl->tile_splits;
  } else {
    pl->tile_parts = (int)std::max<int64_t>(std::min<int64_t>(kPagedTileParts, keys / kKeyTile / kMinSplitTiles), 1);
    pl->tile_slots = (int)std::min((kPagedWorkspace - pl->ws_bytes - items_bytes(1024) - 512) / (kBlockM * (D + 1) * 4), items * pl->tile_parts);
    pl->tile_grid = (int)std::max<int64_t>(items, pl->tile_slots);
    pl->tile_items = (int)std::min<int64_t>(items, pl->tile_slots / 2);
    if (pl->tile_items == 0) pl->tile_parts = 1;
  }
  if (std::max(pl->tile_splits, pl->tile_parts) > 1)
    pl->ws_bytes += items_bytes(pl->tile_items) + partial_bytes(pl->tile_slots, kBlockM, D);
  return VICO_OK;
}

}  // namespace

extern "C" {

int vico_paged_append(const void* k, const void* v, int32_t total_tokens, const int32_t* q_start,
                      const int32_t* seq_len, int32_t num_seqs, void* k_pages, void* v_pages, int32_t num_pages,
                      int32_t page_size, const int32_t* page_table, int32_t max_pages, int32_t num_kv_heads,
                      int32_t head_dim, void* stream) {
  if (total_tokens < 0 || total_tokens > kMaxChunk || !heads_ok(num_kv_heads, num_kv_heads)) return VICO_ERR_INVALID_ARG;
  if (head_dim != 64 && head_dim != 128) return VICO_ERR_UNSUPPORTED;
  if (page_size == 0 || !table_ok(num_seqs, max_pages, num_pages, page_size)) return VICO_ERR_INVALID_ARG;
  const int64_t row = int64_t(num_kv_heads) * head_dim * 2, bytes = row * total_tokens;
  if (bytes >= kMaxTensorBytes) return VICO_ERR_INVALID_ARG;
  if (total_tokens == 0 || num_seqs == 0 || max_pages == 0 || num_pages == 0) return VICO_OK;
  if (!k || !v || !q_start || !seq_len || !k_pages || !v_pages || !page_table) return VICO_ERR_INVALID_ARG;
  if (!aligned16(k) || !aligned16(v) || !aligned16(k_pages) || !aligned16(v_pages) || !aligned_to(q_start, 4) ||
      !aligned_to(seq_len, 4) || !aligned_to(page_table, 4))
    return VICO_ERR_MISALIGNED;
  const int64_t pool = pool_bytes(num_pages, page_size, num_kv_heads, head_dim);
  const Region w[] = {{k_pages, pool}, {v_pages, pool}};
  const Region r[] = {{k, bytes}, {v, bytes}, {q_start, int64_t(num_seqs + 1) * 4}, {seq_len, int64_t(num_seqs) * 4},
                      {page_table, int64_t(num_seqs) * max_pages * 4}};
  if (collide(w, r)) return VICO_ERR_INVALID_ARG;
  PagedAppendArgs a{};
  a.k = (const uint16_t*)k; a.v = (const uint16_t*)v;
  a.k_pages = (uint16_t*)k_pages; a.v_pages = (uint16_t*)v_pages;
  a.q_start = q_start; a.seq_len = seq_len; a.table = page_table;
  a.B = num_seqs; a.total = total_tokens; a.N = num_pages; a.width = max_pages; a.page_shift = shift_of(page_size);
  a.row_units = (int)(row / 16);
  a.by_units = FastDiv::by(a.row_units);
  return status_of(launch_paged_append(a, (hipStream_t)stream));
}

int vico_paged_attn_plan(int32_t num_seqs, int32_t total_q, int32_t max_q_len, int32_t page_size, int32_t max_pages,
                         int32_t sink_len, int64_t window, int64_t keys_hint, int32_t num_q_heads,
                         int32_t num_kv_heads, int32_t head_dim, int32_t num_splits, int32_t* num_splits_out,
                         int64_t* workspace_bytes_out) {
  PagedPlan pl;
  const int st = check_paged_shape(num_seqs, total_q, max_q_len, page_size, max_pages, sink_len, window, keys_hint,
                                   num_q_heads, num_kv_heads, head_dim, num_splits, &pl);
  if (st != VICO_OK) return st;
  if (num_splits_out) *num_splits_out = std::max(std::max(std::max(pl.few.parts, pl.some.parts), std::max(pl.tile_splits, pl.tile_parts)), 1);
  if (workspace_bytes_out) *workspace_bytes_out = pl.ws_bytes;
  return VICO_OK;
}

int vico_paged_route(int32_t num_seqs, int32_t total_q, int32_t max_q_len, int32_t page_size, int32_t max_pages,
                     int32_t sink_len, int64_t window, int64_t keys_hint, int32_t num_q_heads, int32_t num_kv_heads,
                     int32_t head_dim, int32_t num_splits, int32_t* route_out) {
  PagedPlan pl;
  const int st = check_paged_shape(num_seqs, total_q, max_q_len, page_size, max_pages, sink_len, window, keys_hint,
                                   num_q_heads, num_kv_heads, head_dim, num_splits, &pl);
  if (st != VICO_OK) return st;
  const int rows = pl.few.groups + pl.some.groups;
  const bool beside = pl.tile_grid > 0 && !pl.apart;
  route_out[0] = pl.tile_grid;
  route_out[1] = beside ? rows : 0;
  route_out[2] = beside ? 0 : rows;
  route_out[3] = pl.few.parts;
  route_out[4] = pl.some.parts;
  return VICO_OK;
}

int vico_paged_attn(const void* q, const int32_t* q_start, const int32_t* seq_len, int32_t num_seqs, int32_t total_q,
                    int32_t max_q_len, const void* k_pages, const void* v_pages, int32_t num_pages, int32_t page_size,
                    const int32_t* page_table, int32_t max_pages, int32_t sink_len, int64_t window, int64_t keys_hint,
                    int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim, float softmax_scale, int32_t flags,
                    void* out, int32_t out_dtype, float* lse_out, int32_t num_splits, void* workspace,
                    int64_t workspace_bytes, void* stream) {
  PagedPlan pl;
  const int st = check_paged_shape(num_seqs, total_q, max_q_len, page_size, max_pages, sink_len, window, keys_hint,
                                   num_q_heads, num_kv_heads, head_dim, num_splits, &pl);
  if (st != VICO_OK) return st;
  if (out_dtype != VICO_DTYPE_BF16 && out_dtype != VICO_DTYPE_F32) return VICO_ERR_UNSUPPORTED;
  if (flags & ~VICO_ATTN_BIDIRECTIONAL) return VICO_ERR_INVALID_ARG;
  if (isnan(softmax_scale) || isinf(softmax_scale) || workspace_bytes < 0) return VICO_ERR_INVALID_ARG;
  if (num_pages < 0 || num_pages > kMaxPages) return VICO_ERR_INVALID_ARG;
  if (num_seqs == 0 || total_q == 0 || max_q_len == 0) return VICO_OK;
  // a pool or a table without an entry leaves every row without keys, and the kernels without an address to read
  if (num_pages == 0 || max_pages == 0) return VICO_ERR_CAPACITY;
  if (!q || !q_start || !seq_len || !k_pages || !v_pages || !page_table || !out) return VICO_ERR_INVALID_ARG;
  if (!aligned16(q) || !aligned16(k_pages) || !aligned16(v_pages) || !aligned16(out) || (workspace && !aligned16(workspace)) ||
      !aligned_to(q_start, 4) || !aligned_to(seq_len, 4) || !aligned_to(page_table, 4) || !aligned_to(lse_out, 4))
    return VICO_ERR_MISALIGNED;
  if (pl.ws_bytes > 0 && (!workspace || workspace_bytes < pl.ws_bytes)) return VICO_ERR_WORKSPACE;
  const int64_t rows = int64_t(total_q) * num_q_heads, pool = pool_bytes(num_pages, page_size, num_kv_heads, head_dim);
  const Region w[] = {{out, rows * head_dim * (out_dtype == VICO_DTYPE_F32 ? 4 : 2)}, {lse_out, rows * 4},
                      {pl.ws_bytes > 0 ? workspace : nullptr, pl.ws_bytes}};
  const Region r[] = {{q, rows * head_dim * 2}, {k_pages, pool}, {v_pages, pool}, {q_start, int64_t(num_seqs + 1) * 4},
                      {seq_len, int64_t(num_seqs) * 4}, {page_table, int64_t(num_seqs) * max_pages * 4}};
  if (collide(w, r)) return VICO_ERR_INVALID_ARG;

  PagedAttnArgs a{};
  a.q = (const uint16_t*)q; a.q_start = q_start; a.seq_len = seq_len;
  a.k_pages = (const uint16_t*)k_pages; a.v_pages = (const uint16_t*)v_pages; a.table = page_table;
  a.out = out; a.lse = lse_out;
  a.B = num_seqs; a.total = total_q; a.max_q = max_q_len; a.N = num_pages; a.width = max_pages;
  a.page_shift = shift_of(page_size);
  a.S = sink_len; a.W = window;
  a.Hq = num_q_heads; a.Hkv = num_kv_heads; a.D = head_dim;
  a.bidir = (flags & VICO_ATTN_BIDIRECTIONAL) != 0;
  a.out_f32 = out_dtype == VICO_DTYPE_F32;
  const double scale = softmax_scale > 0.f ? double(softmax_scale) : 1.0 / sqrt(double(head_dim));
  a.scale_log2 = (float)(scale * 1.4426950408889634);
  a.by_g = FastDiv::by(a.Hq / a.Hkv);
  a.by_kv = FastDiv::by(a.Hkv);
  a.few = pl.few;
  a.some = pl.some;
  a.rows_apart = pl.apart;
  a.tile_least = pl.some_most + 1;
  a.tile_grid = pl.tile_grid; a.tile_items = pl.tile_items; a.tile_slots = pl.tile_slots;
  a.tile_parts = pl.tile_parts; a.tile_splits = pl.tile_splits;
  char* ws = (char*)workspace;
  auto room = [&](int64_t slots, int64_t rows_of_slot, int64_t bytes, float** o, float** lse) {
    if (bytes == 0) return;
    *o = (float*)ws;
    *lse = (float*)(ws + align256(slots * rows_of_slot * a.D * 4));
    ws += bytes;
  };
  room(pl.few.slots, 16, pl.few_ws, &a.few.ws_o, &a.few.ws_lse);
  room(pl.some.slots, pl.some.tile_rows, pl.some_ws, &a.some.ws_o, &a.some.ws_lse);
  if (pl.ws_bytes > pl.few_ws + pl.some_ws) {
    a.ws_items = (TileItems*)ws;
    ws += items_bytes(pl.tile_items);
    room(pl.tile_slots, kBlockM, partial_bytes(pl.tile_slots, kBlockM, a.D), &a.ws_o, &a.ws_lse);
  }
  const hipError_t e = launch_paged_attention(a, (hipStream_t)stream);
  return status_of(e);
}

int64_t vico_pages_workspace_bytes(int32_t num_seqs, int32_t num_pages) {
  if (!table_ok(num_seqs, 0, num_pages, 0)) return VICO_ERR_INVALID_ARG;
  return table_workspace(num_seqs, num_pages);
}

int vico_pages_fork(int32_t* page_table, int32_t num_seqs, int32_t max_pages, int32_t* page_refs, int32_t num_pages,
                    int32_t page_size, int32_t* seq_len, const int32_t* parent, void* stream) {
  if (page_size == 0 || !table_ok(num_seqs, max_pages, num_pages, page_size)) return VICO_ERR_INVALID_ARG;
  if (num_seqs == 0) return VICO_OK;
  if (max_pages == 0 || num_pages == 0) return VICO_ERR_CAPACITY;
  if (!page_table || !page_refs || !seq_len || !parent) return VICO_ERR_INVALID_ARG;
  if (!aligned_to(page_table, 4) || !aligned_to(page_refs, 4) || !aligned_to(seq_len, 4) || !aligned_to(parent, 4))
    return VICO_ERR_MISALIGNED;
  const Region w[] = {{page_table, int64_t(num_seqs) * max_pages * 4}, {page_refs, int64_t(num_pages) * 4},
                      {seq_len, int64_t(num_seqs) * 4}};
  const Region r[] = {{parent, int64_t(num_seqs) * 4}};
  if (collide(w, r)) return VICO_ERR_INVALID_ARG;
  PagesArgs a{};
  a.table = page_table; a.refs = page_refs; a.seq_len = seq_len; a.parent = parent;
  a.B = num_seqs; a.width = max_pages; a.N = num_pages; a.page_shift = shift_of(page_size);
  return status_of(launch_pages_fork(a, (hipStream_t)stream));
}

int vico_pages_free(int32_t* page_table, int32_t num_seqs, int32_t max_pages, int32_t* page_refs, int32_t num_pages,
                    int32_t page_size, const int32_t* first, const int32_t* last, void* stream) {
  if (page_size == 0 || !table_ok(num_seqs, max_pages, num_pages, page_size)) return VICO_ERR_INVALID_ARG;
  if (num_seqs == 0 || max_pages == 0) return VICO_OK;
  if (num_pages == 0) return VICO_ERR_CAPACITY;
  if (!page_table || !page_refs || !first || !last) return VICO_ERR_INVALID_ARG;
  if (!aligned_to(page_table, 4) || !aligned_to(page_refs, 4) || !aligned_to(first, 4) || !aligned_to(last, 4))
    return VICO_ERR_MISALIGNED;
  const Region w[] = {{page_table, int64_t(num_seqs) * max_pages * 4}, {page_refs, int64_t(num_pages) * 4}};
  const Region r[] = {{first, int64_t(num_seqs) * 4}, {last, int64_t(num_seqs) * 4}};
  if (collide(w, r)) return VICO_ERR_INVALID_ARG;
  PagesArgs a{};
  a.table = page_table; a.refs = page_refs; a.first = first; a.last = last;
  a.B = num_seqs; a.width = max_pages; a.N = num_pages; a.page_shift = shift_of(page_size);
  return status_of(launch_pages_free(a, (hipStream_t)stream));
}

int vico_pages_reserve(int32_t* page_table, int32_t num_seqs, int32_t max_pages, int32_t* page_refs,
                       int32_t num_pages, int32_t page_size, const int32_t* seq_len, const int32_t* q_start,
                       int32_t* moves, int32_t* granted, void* workspace, int64_t workspace_bytes, void* stream) {
  if (page_size == 0 || !table_ok(num_seqs, max_pages, num_pages, page_size) || workspace_bytes < 0) return VICO_ERR_INVALID_ARG;
  if (num_seqs == 0) return VICO_OK;
  if (max_pages == 0 || num_pages == 0) return VICO_ERR_CAPACITY;
  if (!page_table || !page_refs || !seq_len || !q_start || !moves || !granted) return VICO_ERR_INVALID_ARG;
  if (!aligned_to(page_table, 4) || !aligned_to(page_refs, 4) || !aligned_to(seq_len, 4) || !aligned_to(q_start, 4) ||
      !aligned_to(moves, 8) || !aligned_to(granted, 4) || (workspace && !aligned16(workspace)))
    return VICO_ERR_MISALIGNED;
  const int64_t ws = table_workspace(num_seqs, num_pages);
  if (!workspace || workspace_bytes < ws) return VICO_ERR_WORKSPACE;
  const Region w[] = {{page_table, int64_t(num_seqs) * max_pages * 4}, {page_refs, int64_t(num_pages) * 4},
                      {moves, int64_t(num_seqs) * 8}, {granted, int64_t(num_seqs) * 4}, {workspace, ws}};
  const Region r[] = {{seq_len, int64_t(num_seqs) * 4}, {q_start, int64_t(num_seqs + 1) * 4}};
  if (collide(w, r)) return VICO_ERR_INVALID_ARG;
  PagesArgs a{};
  a.table = page_table; a.refs = page_refs; a.seq_len = const_cast<int32_t*>(seq_len); a.q_start = q_start;
  a.moves = moves; a.granted = granted;
  a.B = num_seqs; a.width = max_pages; a.N = num_pages; a.page_shift = shift_of(page_size); a.n_blocks = page_blocks(num_pages);
  use_workspace(&a, workspace);
  return status_of(launch_pages_reserve(a, (hipStream_t)stream));
}

int vico_pages_compact(int32_t* page_table, int32_t num_seqs, int32_t max_pages, int32_t* page_refs,
                       int32_t num_pages, int32_t* moves, int32_t max_moves, int32_t* count, void* workspace,
                       int64_t workspace_bytes, void* stream) {
  if (!table_ok(num_seqs, max_pages, num_pages, 0) || max_moves < 0 || max_moves > kMaxMoves || workspace_bytes < 0)
    return VICO_ERR_INVALID_ARG;
  if (max_moves < num_pages / 2) return VICO_ERR_CAPACITY;
  if (num_pages == 0) return VICO_ERR_CAPACITY;
  if (!page_refs || !count || (max_moves > 0 && !moves) || (int64_t(num_seqs) * max_pages > 0 && !page_table)) return VICO_ERR_INVALID_ARG;
  if (!aligned_to(page_table, 4) || !aligned_to(page_refs, 4) || !aligned_to(moves, 8) || !aligned_to(count, 4) ||
      (workspace && !aligned16(workspace)))
    return VICO_ERR_MISALIGNED;
  const int64_t ws = table_workspace(num_seqs, num_pages);
  if (!workspace || workspace_bytes < ws) return VICO_ERR_WORKSPACE;
  const Region w[] = {{page_table, int64_t(num_seqs) * max_pages * 4}, {page_refs, int64_t(num_pages) * 4},
                      {moves, int64_t(max_moves) * 8}, {count, 4}, {workspace, ws}};
  const Region r[] = {{nullptr, 0}};
  if (collide(w, r)) return VICO_ERR_INVALID_ARG;
  PagesArgs a{};
  a.table = page_table; a.refs = page_refs; a.moves = moves; a.count = count;
  a.B = num_seqs; a.width = max_pages; a.N = num_pages; a.n_blocks = page_blocks(num_pages); a.max_moves = max_moves;
  use_workspace(&a, workspace);
  return status_of(launch_pages_compact(a, (hipStream_t)stream));
}

int vico_pages_copy(void* k_pages, void* v_pages, int32_t num_layers, int32_t num_pages, int32_t page_size,
                    int32_t num_kv_heads, int32_t head_dim, const int32_t* moves, int32_t num_moves,
                    const int32_t* count, void* stream) {
  if (num_layers < 0 || num_layers > 4096 || num_moves < 0 || num_moves > kMaxMoves || !heads_ok(num_kv_heads, num_kv_heads))
    return VICO_ERR_INVALID_ARG;
  if (head_dim != 64 && head_dim != 128) return VICO_ERR_UNSUPPORTED;
  if (page_size == 0 || !table_ok(0, 0, num_pages, page_size)) return VICO_ERR_INVALID_ARG;
  if (num_layers == 0 || num_pages == 0 || num_moves == 0) return VICO_OK;
  if (!k_pages || !v_pages || !moves) return VICO_ERR_INVALID_ARG;
  if (!aligned16(k_pages) || !aligned16(v_pages) || !aligned_to(moves, 8) || !aligned_to(count, 4)) return VICO_ERR_MISALIGNED;
  const int64_t pool = pool_bytes(num_pages, page_size, num_kv_heads, head_dim);
  const Region w[] = {{k_pages, pool * num_layers}, {v_pages, pool * num_layers}};
  const Region r[] = {{moves, int64_t(num_moves) * 8}, {count, 4}};
  if (collide(w, r)) return VICO_ERR_INVALID_ARG;
  PagesCopyArgs a{};
  a.k = (uint16_t*)k_pages; a.v = (uint16_t*)v_pages; a.moves = moves; a.count = count;
  a.n_moves = num_moves; a.layers = num_layers; a.N = num_pages;
  a.page_units = page_size * num_kv_heads * (head_dim / 8);
  return status_of(launch_pages_copy(a, (hipStream_t)stream));
}

}  // extern "C"
