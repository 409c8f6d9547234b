// The page table of the cache in pages (gfx950): forks, frees, reserves and
// compaction (include/vico_pages.h).  The stream's history is what grows (ViCoStream,
// Sec. 3); in pages, a question's branch of it holds the stream's own pages, and a
// window's old pages serve other streams.
//
// All of it is counting: a page's reference count, the r-th free page, how many
// pages are in use below one.  Counts are integers and change by integer atomics,
// whose order does not show.  Reserve and compact ask for ranks over the whole
// pool, in two launches: the first sets a flag for each page (a ballot of 64 counts
// of references a word) and counts the flags of 512 pages; in the second, every
// work-group sums the counts into LDS (at most 4096), after which a rank or the
// r-th flag is a search there and the population counts of at most eight words.
// The second launch changes reference counts, so it decides by the flags alone.
// The tables are small (a 2048-page pool: 8 KB of counts): launches and memory
// latencies bound these calls, so where one work-group can hold the flags it does all in
// one launch.  Alone, us: 16 of 32 rows of 186 entries forked 4.3, new tokens of 16 rows
// in a pool of 1678 pages reserved 5.0; of a pool of 3751 pages a part freed 3.9 to 4.6,
// flags 2.7 to 4.6, compacted 5.1 to 5.9.

#include <algorithm>

#include "attn_common.h"
#include "pages.h"

namespace vico {
namespace {

constexpr int kTableThreads = 256;

__device__ __forceinline__ bool is_page(int e, int n) { return (uint32_t)e < (uint32_t)n; }

// ---- fork.  A work-group owns columns of the table for all rows: its threads hold what the changed rows' entries
// become, and were, in registers before any of them is written, so rows may be taken from each other in any way.
// Few entries: one work-group takes all columns, slice after slice, and the lengths; of a large table each takes slices
// of its own, and the lengths, which all of them read, are another launch's.  (16 of 32 rows of 186 entries 4.4 us;
// 6.4 with the new entries in LDS and their old values read after the barrier.)
constexpr int kForkThreads = 1024, kForkPer = 8, kForkEntries = kForkThreads * kForkPer;

__global__ __launch_bounds__(kForkThreads) void pages_fork_kernel(PagesArgs a) {
  __shared__ int32_t row_s[kMaxSeqs], from_s[kMaxSeqs], len_s[kMaxSeqs], keep_s[kMaxSeqs], rows_s;
  if (threadIdx.x == 0) rows_s = 0;
  __syncthreads();
  for (int b = threadIdx.x; b < a.B; b += kForkThreads) {
    const int p = a.parent[b];
    if (p == b || p < -1 || p >= a.B) continue;
    const int len = p < 0 ? 0 : a.seq_len[p], i = atomicAdd(&rows_s, 1);       // (any order)
    row_s[i] = b;
    from_s[i] = p;
    len_s[i] = len;
    keep_s[i] = len > 0 ? min(((len - 1) >> a.page_shift) + 1, a.width) : 0;
  }
  __syncthreads();
  const int rows = rows_s;
  if (rows == 0) return;
  const int cols = min(kForkEntries / rows, a.width);
  for (int c0 = blockIdx.x * cols; c0 < a.width; c0 += gridDim.x * cols) {
    int old[kForkPer], e[kForkPer];
    int32_t* at[kForkPer];
#pragma unroll
    for (int u = 0; u < kForkPer; ++u) {
      const int i = u * kForkThreads + threadIdx.x, r = i / cols, c = c0 + i - r * cols;
      at[u] = nullptr;
      e[u] = old[u] = -1;
      if (r >= rows || c >= a.width) continue;
      at[u] = a.table + (int64_t)row_s[r] * a.width + c;
      old[u] = *at[u];
      if (c < keep_s[r]) e[u] = a.table[(int64_t)from_s[r] * a.width + c];
    }
    __syncthreads();                      // every row of these columns is read
#pragma unroll
    for (int u = 0; u < kForkPer; ++u) {
      if (!at[u]) continue;
      const int to = is_page(e[u], a.N) ? e[u] : -1;
      if (old[u] == to) continue;
      *at[u] = to;
      if (is_page(old[u], a.N)) atomicSub(a.refs + old[u], 1);
      if (to >= 0) atomicAdd(a.refs + to, 1);
    }
  }
  if (gridDim.x > 1) return;
  for (int i = threadIdx.x; i < rows; i += kForkThreads) a.seq_len[row_s[i]] = len_s[i];
}

__global__ __launch_bounds__(kForkThreads) void pages_fork_lengths_kernel(PagesArgs a) {
  __shared__ int32_t len_s[kMaxSeqs];
  for (int b = threadIdx.x; b < a.B; b += kForkThreads) {
    const int p = a.parent[b];
    len_s[b] = p < 0 ? 0 : a.seq_len[p < a.B ? p : 0];
  }
  __syncthreads();
  for (int b = threadIdx.x; b < a.B; b += kForkThreads) {
    const int p = a.parent[b];
    if (p != b && p >= -1 && p < a.B) a.seq_len[b] = len_s[b];
  }
}

// ---- free
__global__ __launch_bounds__(kTableThreads) void pages_free_kernel(PagesArgs a) {
  const int b = blockIdx.x;
  const int first = max(a.first[b], 0), last = max(a.last[b], 0);
  const int j0 = (int)(((int64_t)first + (1 << a.page_shift) - 1) >> a.page_shift);
  const int j1 = min(last >> a.page_shift, a.width);
  for (int j = j0 + blockIdx.y * kTableThreads + threadIdx.x; j < j1; j += gridDim.y * kTableThreads) {
    int32_t* const at = a.table + (int64_t)b * a.width + j;
    const int e = *at;
    if (is_page(e, a.N)) atomicSub(a.refs + e, 1);
    *at = -1;
  }
}

// ---- flags of pages, and their counts
template <bool IN_USE>
__device__ __forceinline__ void flag_pages(const PagesArgs& a, int block, int32_t* wave_count) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  int n = 0;
#pragma unroll
  for (int r = 0; r < kPageBlock / kTableThreads; ++r) {
    const int p = block * kPageBlock + r * kTableThreads + threadIdx.x;
    const int c = p < a.N ? a.refs[p] : 2;
    const uint64_t set = __builtin_amdgcn_ballot_w64(p < a.N && (c > 0) == IN_USE);
    const uint64_t once = __builtin_amdgcn_ballot_w64(c == 1);
    n += __builtin_popcountll(set);
    if (lane == 0) {
      const int w = block * (kPageBlock / 64) + r * (kTableThreads / 64) + wave;
      a.flags[w] = set;
      if (!IN_USE) a.flags1[w] = once;
    }
  }
  if (lane == 0) wave_count[wave] = n;
  __syncthreads();
  if (threadIdx.x == 0) a.blocks[block] = wave_count[0] + wave_count[1] + wave_count[2] + wave_count[3];
}

// Sums over the work-group: inclusive sum of x over the threads up to this one; `total` of all.
template <int NT = kTableThreads>
__device__ __forceinline__ int group_scan(int x, int& total, int32_t* wave_sum) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  x = wave_scan(x);
  __syncthreads();                        // wave_sum is free
  if (lane == 63) wave_sum[wave] = x;
  __syncthreads();
  int before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) {
    before += w < wave ? wave_sum[w] : 0;
    total += wave_sum[w];
  }
  return x + before;
}

// Position of the r-th bit that is set in x (r counts from 0, and there is one).
__device__ __forceinline__ int nth_bit(uint64_t x, int r) {
  int at = 0;
#pragma unroll
  for (int half = 32; half > 0; half >>= 1) {
    const int n = __builtin_popcountll(x & ((uint64_t(1) << half) - 1));
    const bool upper = n <= r;
    r -= upper ? n : 0;
    x = upper ? x >> half : x;
    at += upper ? half : 0;
  }
  return at;
}

// The flags counted up to each block, in LDS; ranks and r-th flags from it.
struct Ranks {
  const PagesArgs& a;
  int32_t* upto;                          // flags in blocks 0 .. i - 1
  int total;

  __device__ __forceinline__ Ranks(const PagesArgs& a_, int32_t* upto_, int32_t* wave_sum) : a(a_), upto(upto_), total(0) {
    for (int i0 = 0; i0 < a.n_blocks; i0 += kTableThreads) {
      const int i = i0 + threadIdx.x, x = i < a.n_blocks ? a.blocks[i] : 0;
      int sum;
      const int incl = group_scan(x, sum, wave_sum);
      if (i < a.n_blocks) upto[i] = total + incl - x;
      total += sum;
    }
    __syncthreads();
  }
  __device__ __forceinline__ bool set(int p) const { return (a.flags[p >> 6] >> (p & 63)) & 1; }
  // flagged pages below p
  __device__ __forceinline__ int below(int p) const {
    const int block = p / kPageBlock;
    if (block >= a.n_blocks) return total;
    uint64_t x[kPageBlock / 64];
    words(block, x);
    int n = upto[block];
#pragma unroll
    for (int w = 0; w < kPageBlock / 64; ++w) {
      const int bits = min(max(p - block * kPageBlock - 64 * w, 0), 64);         // of this word, those below p
      n += __builtin_popcountll(bits == 64 ? x[w] : x[w] & ((uint64_t(1) << bits) - 1));
    }
    return n;
  }
  // the words of a block, all loads together
  __device__ __forceinline__ void words(int block, uint64_t (&x)[kPageBlock / 64]) const {
#pragma unroll
    for (int w = 0; w < kPageBlock / 64; ++w) x[w] = a.flags[block * (kPageBlock / 64) + w];
  }
  // page of the r-th flag that is set (FLAG) or not (r counts from 0, and there is one)
  template <bool FLAG>
  __device__ __forceinline__ int nth(int r) const {
    auto before = [&](int block) { return FLAG ? upto[block] : block * kPageBlock - upto[block]; };
    int lo = 0, hi = a.n_blocks;          // the last block with before(block) <= r
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (before(mid) <= r) lo = mid;
      else hi = mid;
    }
    r -= before(lo);
    uint64_t y[kPageBlock / 64];
    words(lo, y);
    uint64_t x = 0;
    int w = 0;
    bool found = false;
#pragma unroll
    for (int i = 0; i < kPageBlock / 64; ++i) {
      const uint64_t z = FLAG ? y[i] : ~y[i];
      const int n = __builtin_popcountll(z);
      const bool here = !found & (r < n);
      x = here ? z : x;
      w = here ? lo * (kPageBlock / 64) + i : w;
      found |= here;
      r -= found ? 0 : n;
    }
    return w * 64 + nth_bit(x, r);
  }
};

// ---- reserve.  The entries that a row's new tokens go to, [j0, j1), and whether there is room for them.
__device__ __forceinline__ bool new_entries(const PagesArgs& a, int b, int& H, int& j0, int& j1) {
  H = max(a.seq_len[b], 0);
  const int64_t n = (int64_t)a.q_start[b + 1] - a.q_start[b];
  j0 = j1 = 0;
  if (n <= 0) return true;
  const int64_t end = ((int64_t)H + n + (1 << a.page_shift) - 1) >> a.page_shift;
  if (end > a.width) return false;
  j0 = H >> a.page_shift;
  j1 = (int)end;
  return true;
}

__global__ __launch_bounds__(kTableThreads) void pages_count_kernel(PagesArgs a) {
  __shared__ int32_t wave_count[kTableThreads / 64];
  if ((int)blockIdx.x < a.n_blocks) {
    flag_pages<false>(a, blockIdx.x, wave_count);
    return;
  }
  const int b = (blockIdx.x - a.n_blocks) * (kTableThreads / 64) + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (b >= a.B) return;
  int H, j0, j1, n = 0;
  new_entries(a, b, H, j0, j1);
  for (int j = j0 + lane; j < j1; j += 64) {
    const int e = a.table[(int64_t)b * a.width + j];
    n += !(is_page(e, a.N) && a.refs[e] == 1);
  }
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) n += __shfl_xor(n, o, 64);
  if (lane == 0) a.need[b] = n;
}

__global__ __launch_bounds__(kTableThreads) void pages_reserve_kernel(PagesArgs a) {
  __shared__ int32_t upto[kMaxPageBlocks], wave_sum[kTableThreads / 64];
  const int b = blockIdx.x;
  const int want = a.need[b];
  int H, j0, j1;
  bool ok = new_entries(a, b, H, j0, j1);
  if (threadIdx.x == 0) {
    a.moves[2 * b] = -1;
    a.moves[2 * b + 1] = -1;
  }
  if (want == 0) {                        // the same for the whole work-group
    if (threadIdx.x == 0) a.granted[b] = ok;
    return;
  }
  int before = 0, x = 0;
  for (int i = threadIdx.x; i < b; i += kTableThreads) x = min(x + a.need[i], kMaxPages);
  group_scan(x, before, wave_sum);        // pages that the rows before this one want
  const Ranks free(a, upto, wave_sum);
  ok = before <= free.total - want;
  if (threadIdx.x == 0) a.granted[b] = ok;
  if (!ok) return;
  for (int at = j0; at < j1; at += kTableThreads) {
    const int j = at + threadIdx.x;
    int32_t* const entry = a.table + (int64_t)b * a.width + j;
    const int e = j < j1 ? *entry : -1;
    const bool page = is_page(e, a.N);
    const bool wants = j < j1 && !(page && ((a.flags1[e >> 6] >> (e & 63)) & 1));
    int sum;
    const int rank = before + group_scan(wants, sum, wave_sum) - 1;
    before += sum;
    if (!wants) continue;
    const int p = free.nth<true>(rank);
    *entry = p;
    a.refs[p] = 1;
    if (!page || free.set(e)) continue;   // (a page that the counts call free is not held)
    atomicSub(a.refs + e, 1);
    if (j == j0 && (H & ((1 << a.page_shift) - 1)) != 0) {
      a.moves[2 * b] = e;
      a.moves[2 * b + 1] = p;
    }
  }
}

// ---- compact
__global__ __launch_bounds__(kTableThreads) void pages_in_use_kernel(PagesArgs a) {
  __shared__ int32_t wave_count[kTableThreads / 64];
  flag_pages<true>(a, blockIdx.x, wave_count);
}

// Work-groups 0 .. n_blocks - 1 take a block of pages each, the others the table and the rest of the moves.
__global__ __launch_bounds__(kTableThreads) void pages_compact_kernel(PagesArgs a) {
  __shared__ int32_t upto[kMaxPageBlocks], wave_sum[kTableThreads / 64];
  const Ranks used(a, upto, wave_sum);
  const int U = used.total, low = used.below(U), moved = U - low;
  if ((int)blockIdx.x < a.n_blocks) {
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.count = moved;
#pragma unroll
    for (int r = 0; r < kPageBlock / kTableThreads; ++r) {
      const int p = blockIdx.x * kPageBlock + r * kTableThreads + threadIdx.x;
      if (p >= a.N || p < U || !used.set(p)) continue;
      const int i = used.below(p) - low, to = used.nth<false>(i);
      a.moves[2 * i] = p;
      a.moves[2 * i + 1] = to;
      a.refs[to] = a.refs[p];
      a.refs[p] = 0;
    }
    return;
  }
  const int64_t n = (int64_t)(gridDim.x - a.n_blocks) * kTableThreads;
  const int64_t at = (int64_t)(blockIdx.x - a.n_blocks) * kTableThreads + threadIdx.x;
  const int64_t entries = (int64_t)a.B * a.width;
  for (int64_t i = at; i < entries; i += n) {
    const int e = a.table[i];
    if (e >= U && e < a.N && used.set(e)) a.table[i] = used.nth<false>(used.below(e) - low);
  }
  for (int64_t i = moved + at; i < a.max_moves; i += n) {
    a.moves[2 * i] = -1;
    a.moves[2 * i + 1] = -1;
  }
}

// ---- small pools: one work-group, one launch, flags and counts in LDS.  (2300 pages, 32 rows, 16 of them with new
// tokens: 9 us in two launches.)
constexpr int kSmallThreads = 1024;
constexpr int kSmallPages = 65536;         // reserve: a count for each word of flags is one a thread
constexpr int kSmallEntries = 65536;       // of the table

struct SmallRanks {                        // as Ranks, from words of flags in LDS
  uint64_t flags[kSmallPages / 64];
  int32_t upto[kSmallPages / 64];          // flags in the words before
  int32_t wave_sum[kSmallThreads / 64];
  // every thread: after the flags have been written; returns their number
  __device__ __forceinline__ int count(int words) {
    __syncthreads();
    const int n = (int)threadIdx.x < words ? __builtin_popcountll(flags[threadIdx.x]) : 0;
    int total;
    const int incl = group_scan<kSmallThreads>(n, total, wave_sum);
    if ((int)threadIdx.x < words) upto[threadIdx.x] = incl - n;
    __syncthreads();
    return total;
  }
  __device__ __forceinline__ bool set(int p) const { return (flags[p >> 6] >> (p & 63)) & 1; }
  __device__ __forceinline__ int below(int p) const {
    return upto[p >> 6] + __builtin_popcountll(flags[p >> 6] & ((uint64_t(1) << (p & 63)) - 1));
  }
  template <bool FLAG>
  __device__ __forceinline__ int nth(int r, int words) const {
    auto before = [&](int w) { return FLAG ? upto[w] : w * 64 - upto[w]; };
    int lo = 0, hi = words;                // the last word with before(w) <= r
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (before(mid) <= r) lo = mid;
      else hi = mid;
    }
    return lo * 64 + nth_bit(FLAG ? flags[lo] : ~flags[lo], r - before(lo));
  }
};

// The new tokens' entries of all rows are numbered one after the other, which is the order that free pages are given
// out in; a thread takes every 1024th.
__global__ __launch_bounds__(kSmallThreads) void pages_reserve_small_kernel(PagesArgs a) {
  __shared__ SmallRanks free;
  __shared__ uint64_t once[kSmallPages / 64];
  // of each row: entries up to its end, its length, its wants, and those up to its end
  __shared__ int32_t end_s[kMaxSeqs], len_s[kMaxSeqs], need_s[kMaxSeqs], upto_s[kMaxSeqs];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int words = (a.N + 63) / 64;
  int H = 0, j0 = 0, j1 = 0;              // of row tid, on the way together with the counts
  bool ok = true;
  if (tid < a.B) ok = new_entries(a, tid, H, j0, j1);
  for (int i0 = 0; i0 < a.N; i0 += 4 * kSmallThreads) {
    int c[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int p = i0 + u * kSmallThreads + tid;
      c[u] = p < a.N ? a.refs[p] : 2;
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const uint64_t none = __builtin_amdgcn_ballot_w64(c[u] <= 0), one = __builtin_amdgcn_ballot_w64(c[u] == 1);
      const int w = (i0 + u * kSmallThreads) / 64 + wave;
      if (lane == 0 && w < words) {
        free.flags[w] = none;
        once[w] = one;
      }
    }
  }
  int entries = 0;
  for (int b0 = 0; b0 < a.B; b0 += kSmallThreads) {
    const int b = b0 + tid;
    if (b0 > 0) {
      j0 = j1 = 0;
      if (b < a.B) ok = new_entries(a, b, H, j0, j1);
    }
    int sum;
    const int incl = group_scan<kSmallThreads>(j1 - j0, sum, free.wave_sum);
    if (b < a.B) {
      need_s[b] = 0;
      end_s[b] = entries + incl;
      len_s[b] = H;
      if (j1 == j0) {                     // nothing new, or no room in the table
        a.granted[b] = ok;
        a.moves[2 * b] = -1;
        a.moves[2 * b + 1] = -1;
      }
    }
    entries += sum;
  }
  const int n_free = free.count(words);
  // the wants of each row, and up to its end
  int j = 0, e = -1, row = 0, rank = 0;
  bool wants = false;
  auto look_at = [&](int i) {
    int lo = -1, hi = a.B - 1;            // the first row whose end is past i
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (end_s[mid] > i) hi = mid;
      else lo = mid;
    }
    row = hi;
    H = len_s[row];
    j0 = H >> a.page_shift;
    j = j0 + i - (row > 0 ? end_s[row - 1] : 0);
    e = a.table[(int64_t)row * a.width + j];
    wants = !(is_page(e, a.N) && ((once[e >> 6] >> (e & 63)) & 1));
  };
  int wanted = 0;
  for (int i0 = 0; i0 < entries; i0 += kSmallThreads) {
    const int i = i0 + tid;
    wants = false;
    if (i < entries) look_at(i);
    int sum;
    rank = wanted + group_scan<kSmallThreads>(wants, sum, free.wave_sum);
    if (i < entries) {
      if (wants) atomicAdd(&need_s[row], 1);
      if (i == end_s[row] - 1) upto_s[row] = rank;
    }
    wanted += sum;
  }
  __syncthreads();
  int given = 0;
  for (int i0 = 0; i0 < entries; i0 += kSmallThreads) {
    const int i = i0 + tid;
    if (entries > kSmallThreads) {        // (a single round has its entries still)
      wants = false;
      if (i < entries) look_at(i);
      int sum;
      rank = given + group_scan<kSmallThreads>(wants, sum, free.wave_sum);
      given += sum;
    }
    if (i >= entries) continue;
    ok = need_s[row] == 0 || upto_s[row] <= n_free;
    const int p = wants && ok ? free.nth<true>(rank - 1, words) : -1;
    const bool held = p >= 0 && is_page(e, a.N) && !free.set(e);
    if (j == j0) {
      const bool moves = held && (H & ((1 << a.page_shift) - 1)) != 0;
      a.granted[row] = ok;
      a.moves[2 * row] = moves ? e : -1;
      a.moves[2 * row + 1] = moves ? p : -1;
    }
    if (p < 0) continue;
    a.table[(int64_t)row * a.width + j] = p;
    a.refs[p] = 1;
    if (held) atomicSub(a.refs + e, 1);
  }
}

// Pages, and entries: those of a thread stay in its registers.  (4700 pages, 24 rows of 250 entries: 11.1 us with sixteen a
// thread, 7.1 in two launches; 260 pages 4 us and 6.1.)
constexpr int kSmallCompact = 2 * kSmallThreads;
__global__ __launch_bounds__(kSmallThreads) void pages_compact_small_kernel(PagesArgs a) {
  __shared__ SmallRanks used;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int words = (a.N + 63) / 64, entries = a.B * a.width;
  int c[kSmallCompact / kSmallThreads], e[kSmallCompact / kSmallThreads];
#pragma unroll
  for (int u = 0; u < kSmallCompact / kSmallThreads; ++u) {
    const int i = u * kSmallThreads + tid;
    c[u] = i < a.N ? a.refs[i] : 0;
    e[u] = i < entries ? a.table[i] : -1;
  }
#pragma unroll
  for (int u = 0; u < kSmallCompact / kSmallThreads; ++u) {
    const uint64_t set = __builtin_amdgcn_ballot_w64(c[u] > 0);
    const int w = u * (kSmallThreads / 64) + wave;
    if (lane == 0 && w < words) used.flags[w] = set;
  }
  const int U = used.count(words), low = U < a.N ? used.below(U) : U, moved = U - low;
  if (tid == 0) *a.count = moved;
#pragma unroll
  for (int u = 0; u < kSmallCompact / kSmallThreads; ++u) {
    const int i = u * kSmallThreads + tid;
    if (i < a.N && i >= U && c[u] > 0) {
      const int m = used.below(i) - low, to = used.nth<false>(m, words);
      a.moves[2 * m] = i;
      a.moves[2 * m + 1] = to;
      a.refs[to] = c[u];
      a.refs[i] = 0;
    }
    if (e[u] >= U && e[u] < a.N && used.set(e[u])) a.table[i] = used.nth<false>(used.below(e[u]) - low, words);
  }
  for (int i = moved + tid; i < a.max_moves; i += kSmallThreads) {
    a.moves[2 * i] = -1;
    a.moves[2 * i + 1] = -1;
  }
}

}  // namespace

hipError_t launch_pages_fork(const PagesArgs& a, hipStream_t stream) {
  const int cols = std::max(kForkEntries / a.B, 1), slices = (a.width + cols - 1) / cols;
  const int groups = (int64_t)a.B * a.width <= kSmallEntries ? 1 : std::min(slices, 1024);
  hipLaunchKernelGGL(pages_fork_kernel, dim3(groups), dim3(kForkThreads), 0, stream, a);
  if (groups > 1) hipLaunchKernelGGL(pages_fork_lengths_kernel, dim3(1), dim3(kForkThreads), 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_pages_free(const PagesArgs& a, hipStream_t stream) {
  const int y = std::min((a.width + kTableThreads - 1) / kTableThreads, std::max(2048 / a.B, 1));
  hipLaunchKernelGGL(pages_free_kernel, dim3(a.B, y), dim3(kTableThreads), 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_pages_reserve(const PagesArgs& a, hipStream_t stream) {
  if (a.N <= kSmallPages && (int64_t)a.B * a.width <= kSmallEntries) {
    hipLaunchKernelGGL(pages_reserve_small_kernel, dim3(1), dim3(kSmallThreads), 0, stream, a);
    return hipGetLastError();
  }
  constexpr int rows = kTableThreads / 64;
  hipLaunchKernelGGL(pages_count_kernel, dim3(a.n_blocks + (a.B + rows - 1) / rows), dim3(kTableThreads), 0, stream, a);
  hipLaunchKernelGGL(pages_reserve_kernel, dim3(a.B), dim3(kTableThreads), 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_pages_compact(const PagesArgs& a, hipStream_t stream) {
  if (a.N <= kSmallCompact && (int64_t)a.B * a.width <= kSmallCompact) {
    hipLaunchKernelGGL(pages_compact_small_kernel, dim3(1), dim3(kSmallThreads), 0, stream, a);
    return hipGetLastError();
  }
  const int64_t work = std::max<int64_t>((int64_t)a.B * a.width, a.max_moves);
  const int groups = (int)std::min<int64_t>((work + kTableThreads - 1) / kTableThreads, 1024);
  hipLaunchKernelGGL(pages_in_use_kernel, dim3(a.n_blocks), dim3(kTableThreads), 0, stream, a);
  hipLaunchKernelGGL(pages_compact_kernel, dim3(a.n_blocks + groups), dim3(kTableThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace vico
