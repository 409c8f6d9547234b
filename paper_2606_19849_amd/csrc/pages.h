// The cache in pages (include/vico_pages.h): arguments and device helpers that
// its kernels share.
#pragma once

#include "vico_internal.h"

namespace vico {

constexpr int kMaxPages = 1 << 21;
constexpr int kMaxSeqs = 4096;
constexpr int kMaxMoves = 1 << 24;
constexpr int kPageBlock = 512;                       // pages that one count covers: eight words of 64 flags
constexpr int kMaxPageBlocks = kMaxPages / kPageBlock;

// ---- tables
struct PagesArgs {
  int32_t* table;           // [B][width]
  int32_t* refs;            // [N]
  int32_t* seq_len;         // [B]
  const int32_t* parent;    // fork
  const int32_t* first;     // free
  const int32_t* last;
  const int32_t* q_start;   // reserve
  int32_t* moves;           // reserve, compact
  int32_t* granted;         // reserve
  int32_t* count;           // compact
  uint64_t* flags;          // workspace: a bit for each page; reserve: free, compact: in use
  uint64_t* flags1;         // workspace: pages held once (reserve)
  int32_t* blocks;          // workspace: flags counted, kPageBlock pages each
  int32_t* need;            // workspace: pages that each row wants (reserve)
  int B, width, N, n_blocks, page_shift, max_moves;
};
hipError_t launch_pages_fork(const PagesArgs& a, hipStream_t stream);
hipError_t launch_pages_free(const PagesArgs& a, hipStream_t stream);
hipError_t launch_pages_reserve(const PagesArgs& a, hipStream_t stream);
hipError_t launch_pages_compact(const PagesArgs& a, hipStream_t stream);

// ---- contents
struct PagesCopyArgs {
  uint16_t* k;              // [layers][N][page_units * 8 elements]
  uint16_t* v;
  const int32_t* moves;     // [n_moves][2]
  const int32_t* count;     // may be null
  int n_moves, layers, N;
  int page_units;           // 16-byte units of a page
  int pieces;               // pieces that a page is copied in: set by the launch
};
hipError_t launch_pages_copy(const PagesCopyArgs& a, hipStream_t stream);

struct PagedAppendArgs {
  const uint16_t* k;        // [total][row_units * 8 elements]
  const uint16_t* v;
  uint16_t* k_pages;
  uint16_t* v_pages;
  const int32_t* q_start;
  const int32_t* seq_len;
  const int32_t* table;
  int B, total, N, width, page_shift;
  int row_units;            // 16-byte units of a token's row
  FastDiv by_units;
  int per_wave;             // tokens of a wave: set by the launch
};
hipError_t launch_paged_append(const PagedAppendArgs& a, hipStream_t stream);

// ---- attention
constexpr int kPagedParts = 64;       // most key-range parts of a row tile of the classes below
constexpr int kPagedTileParts = 16;   // and of a 256-row tile
// Sequences of `least` to `most` packed rows, on row tiles of tile_rows rows.
struct RowsClass {
  int least, most, tile_rows;
  int merge_rows;           // of a row tile, rows that a sequence may have there
  int n_rt;                 // row tiles of a sequence at most
  int parts, per_part;      // parts of its key range at most, 32-key blocks of one at least
  int groups, merge;        // work-groups: Hkv * n_rt for each of B * parts key ranges, in eights; of the merge
  int slots;                // partial results: B * parts * Hkv * n_rt
  float* ws_o;              // partial results [B][parts][Hkv][n_rt][tile_rows][D], and their log2-sum-exps
  float* ws_lse;
  FastDiv by_rt, by_parts;
};
struct PagedAttnArgs {
  const uint16_t* q;
  const int32_t* q_start;
  const int32_t* seq_len;
  const uint16_t* k_pages;
  const uint16_t* v_pages;
  const int32_t* table;
  void* out;
  float* lse;               // may be null
  int B, total, max_q, N, width, page_shift;
  int S;
  int64_t W;                // < 0: the whole history
  int Hq, Hkv, D;
  int bidir, out_f32;
  float scale_log2;
  FastDiv by_g, by_kv;
  RowsClass few, some;      // up to 16 rows, up to tile_least - 1 (groups 0: none)
  int rows_apart;           // these are not in the launch of the 256-row tiles
  // sequences of tile_least rows and more, on 256-row tiles: work-groups (0: none) and those of the merge, the row
  // tiles of all heads that may be split, room for partial results, the parts that the caller asked for (0: the
  // kernel's choice, of tile_parts at most)
  int tile_least, tile_grid, tile_merge, tile_items, tile_slots, tile_splits, tile_parts;
  float* ws_o;              // partial results of 256-row tiles [slot][256][D], and their log2-sum-exps (null: no parts)
  float* ws_lse;
  struct TileItems* ws_items;
};
// What the 256-row kernel leaves for the merge: the row tiles that it has split, found by no search of their sequences.
struct TileItem {
  int q0, rows, kv, rt;     // the sequence's first row and packed rows, the head, the row tile
  int slot, step;           // of the first part's result, and on to the next part's
};
struct TileItems {
  int items, parts;         // (items: 0 where nothing is split)
  TileItem item[1];         // tile_items of them
};
// The time of `items` row tiles over `tiles` 64-key tiles in p parts, beside sequences of few rows whose keys alone
// take `beside`, counted in such tiles (1.35 us with heads of size 128, 0.9 of size 64).  Rounds of work-groups over
// the CUs, each a start, an end and its keys, which take longer where more than half of the CUs are at it (the power
// limit); the CUs that the last round leaves stream the others' keys, 1.3 times their share; what is left of those comes
// after; then the merge and the partial results' way to memory and back.
// (Us measured / this, in 1, 2, 3, 4, 6, 8 parts.  7B heads, 1024 tokens over 8192 keys 196, 139, 166, 146, 160, 175 / 196,
// 134, 179, 157, 179, 202; beside 31 answer tokens 203, 218, 217, 233, 249, 267 / 196, 205, 206, 227, 249, 271; beside 100
// of them 337, 420, 430, 445, 474, 490 / 343, 405, 406, 427, 449, 471; 256 tokens beside 31 185, 117, 119, 118, 130, 146 /
// 180, 100, 105, 113, 124, 134; 3B heads, 1024 beside 31 197, 116, 108, 123, 126, 143 / 196, 112, 111, 130, 131, 154.)
__host__ __device__ inline float paged_tile_cost(int items, int tiles, int p, float beside) {
  const int64_t n = (int64_t)items * p, full = n > 0 ? (n - 1) / kNumCUs : 0;                // rounds before the last one
  const float busy = (float)(n - full * kNumCUs) / kNumCUs, each = (float)(6 + (tiles + p - 1) / p);
  const float last = each * (0.96f + 0.22f * fmaxf(2 * busy - 1, 0.f));
  return each * 1.18f * (float)full + last + fmaxf(beside - fminf(1.3f * (1 - busy), 1.f) * last, 0.f) +
         (p > 1 ? 2.f + 0.039f * (float)n : 0.f);
}
// 32-key blocks of one KV head at the memory's rate, in the same unit.
__host__ __device__ constexpr float paged_block_cost(int D) { return D == 128 ? 2.4e-3f : 1.8e-3f; }
inline int paged_tile_parts(int items, int tiles, int most, int slots) {
  int parts = 1;
  for (int p = 2; p <= most && items * p <= slots; ++p)
    if (paged_tile_cost(items, tiles, p, 0.f) < paged_tile_cost(items, tiles, parts, 0.f)) parts = p;
  return parts;
}
hipError_t launch_paged_attention(const PagedAttnArgs& a, hipStream_t stream);

// What a sequence's rows are and see.  Numbers from device memory are brought
// into range here: whatever the arrays hold, rows lie in [0, total) and positions in
// [0, width * page_size).
struct Sequence {
  int q0, n, all;           // its first row, its rows that are computed, its rows
  int H;                    // tokens before them
  int sink, first;          // visible before the new tokens: [0, sink) and [first, H), sink <= first
};
template <class A>
__device__ __forceinline__ int rows_of(const A& a, int b, int& q0) {
  q0 = min(max(a.q_start[b], 0), a.total);
  return min(max(a.q_start[b + 1], q0), a.total) - q0;
}
__device__ __forceinline__ Sequence sequence(const PagedAttnArgs& a, int q0, int rows, int len) {
  Sequence s;
  s.q0 = q0;
  s.all = rows;
  s.n = min(s.all, a.max_q);
  s.H = min(max(len, 0), a.width << a.page_shift);
  s.first = a.W < 0 || a.W >= s.H ? 0 : s.H - (int)a.W;
  s.sink = min(a.S, s.first);
  return s;
}
__device__ __forceinline__ Sequence sequence(const PagedAttnArgs& a, int b) {
  int q0;
  const int rows = rows_of(a, b, q0);
  return sequence(a, q0, rows, a.seq_len[b]);
}
// A row's last position: token t of the sequence's chunk.
__device__ __forceinline__ int last_position(const PagedAttnArgs& a, const Sequence& s, int t) {
  return min(s.H + (a.bidir ? s.all - 1 : t), (a.width << a.page_shift) - 1);
}
// Blocks of BN positions (a power of two): those of the sink, then those from the window on; the first block after the
// sink's, and how many there are up to position `last`.
template <int BN>
struct KeyBlocks {
  int of_sink, from;
  __device__ __forceinline__ explicit KeyBlocks(const Sequence& s)
      : of_sink((s.sink + BN - 1) / BN), from(max(s.first / BN, (s.sink + BN - 1) / BN)) {}
  __device__ __forceinline__ int upto(int last) const { return max(last / BN + 1 - from, 0) + of_sink; }
  __device__ __forceinline__ int position(int i) const { return (i < of_sink ? i : i - of_sink + from) * BN; }
};
// Parts of a sequence's key range, and 32-key blocks of one.
__device__ __forceinline__ int parts_of(const RowsClass& x, int blocks, int& per) {
  per = max(x.per_part, x.by_parts(blocks + x.parts - 1));
  return max((blocks + per - 1) / per, 1);
}

// The sequence that row t of the calls' tensors belongs to (every lane of a wave
// asks for the same t), B where none does: the number of entries q_start[1 .. B]
// that are <= t, 64 at a time.
__device__ __forceinline__ int sequence_of(const int32_t* q_start, int B, int t, int lane) {
  int lo = 0, step = 1;
  while (step * 64 < B) step *= 64;
  for (; step > 0; step /= 64) {
    const int i = lo + (lane + 1) * step;
    const bool passed = i <= B && q_start[i] <= t;
    lo += step * __builtin_popcountll(__builtin_amdgcn_ballot_w64(passed));
  }
  return lo;
}

}  // namespace vico
