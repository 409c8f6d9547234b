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
// The tables are small (a 2048-page pool: 8 KB of counts): the launches bound
// these calls.

#include <algorithm>

#include "pages.h"

namespace vico {
namespace {

constexpr int kTableThreads = 256;

__device__ __forceinline__ bool is_page(int e, int n) { return (uint32_t)e < (uint32_t)n; }

// ---- fork.  A work-group owns columns of the table for all rows: it reads what the
// changed rows become into LDS before any of them is written, so rows may be taken
// from each other in any way.
constexpr int kForkThreads = 512;
constexpr int kForkEntries = 32768;        // of a work-group: 128 KB of LDS

__device__ __forceinline__ int parent_of(const PagesArgs& a, int b) {
  const int p = a.parent[b];
  return p == b || p < -1 || p >= a.B ? b : p;
}
__device__ __forceinline__ void fork_lengths(const PagesArgs& a, int32_t* lds) {
  for (int b = threadIdx.x; b < a.B; b += kForkThreads) {
    const int p = parent_of(a, b);
    lds[b] = p < 0 ? 0 : a.seq_len[p];
  }
  __syncthreads();
  for (int b = threadIdx.x; b < a.B; b += kForkThreads)
    if (parent_of(a, b) != b) a.seq_len[b] = lds[b];
}

// cols: columns of a slice (a power of two).  One work-group takes all slices and the lengths; several take one each,
// and the lengths, which all of them read, are another launch's.
__global__ __launch_bounds__(kForkThreads) void pages_fork_kernel(PagesArgs a, int cols, int slices) {
  __shared__ int32_t becomes[kForkEntries];
  const int shift = 31 - __builtin_clz(cols);
  for (int s = blockIdx.x; s < slices; s += gridDim.x) {
    const int c0 = s * cols;
    for (int i = threadIdx.x; i < a.B * cols; i += kForkThreads) {
      const int b = i >> shift, c = c0 + (i & (cols - 1)), p = parent_of(a, b);
      if (p == b || c >= a.width) continue;
      int e = -1;
      if (p >= 0) {
        const int len = a.seq_len[p];
        if (len > 0 && c <= (len - 1) >> a.page_shift) e = a.table[(int64_t)p * a.width + c];
      }
      becomes[i] = is_page(e, a.N) ? e : -1;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < a.B * cols; i += kForkThreads) {
      const int b = i >> shift, c = c0 + (i & (cols - 1));
      if (parent_of(a, b) == b || c >= a.width) continue;
      int32_t* const at = a.table + (int64_t)b * a.width + c;
      const int old = *at, e = becomes[i];
      if (old == e) continue;
      *at = e;
      if (is_page(old, a.N)) atomicSub(a.refs + old, 1);
      if (e >= 0) atomicAdd(a.refs + e, 1);
    }
    __syncthreads();
  }
  if (gridDim.x == 1) fork_lengths(a, becomes);
}

__global__ __launch_bounds__(kForkThreads) void pages_fork_lengths_kernel(PagesArgs a) {
  __shared__ int32_t becomes[kMaxSeqs];
  fork_lengths(a, becomes);
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
__device__ __forceinline__ int group_scan(int x, int& total, int32_t* wave_sum) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(x, o, 64);
    x += lane >= o ? y : 0;
  }
  __syncthreads();                        // wave_sum is free
  if (lane == 63) wave_sum[wave] = x;
  __syncthreads();
  int before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < kTableThreads / 64; ++w) {
    before += w < wave ? wave_sum[w] : 0;
    total += wave_sum[w];
  }
  return x + before;
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
    int n = upto[block];
    for (int w = block * (kPageBlock / 64); w < (p >> 6); ++w) n += __builtin_popcountll(a.flags[w]);
    const int bit = p & 63;
    return bit == 0 ? n : n + __builtin_popcountll(a.flags[p >> 6] & ((uint64_t(1) << bit) - 1));
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
    int w = lo * (kPageBlock / 64);
    const int last = w + kPageBlock / 64 - 1;
    uint64_t x = FLAG ? a.flags[w] : ~a.flags[w];
    while (w < last && __builtin_popcountll(x) <= r) {
      r -= __builtin_popcountll(x);
      ++w;
      x = FLAG ? a.flags[w] : ~a.flags[w];
    }
    int at = 0;                           // the r-th bit of x
#pragma unroll
    for (int half = 32; half > 0; half >>= 1) {
      const int n = __builtin_popcountll(x & ((uint64_t(1) << half) - 1));
      const bool upper = n <= r;
      r -= upper ? n : 0;
      x = upper ? x >> half : x;
      at += upper ? half : 0;
    }
    return w * 64 + at;
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

}  // namespace

hipError_t launch_pages_fork(const PagesArgs& a, hipStream_t stream) {
  int cols = 64;
  while (cols * a.B > kForkEntries) cols /= 2;          // B <= 4096: eight at least
  const int slices = (a.width + cols - 1) / cols;
  // few entries: one work-group, one launch
  const int groups = (int64_t)a.B * a.width <= 16384 ? 1 : slices;
  hipLaunchKernelGGL(pages_fork_kernel, dim3(groups), dim3(kForkThreads), 0, stream, a, cols, slices);
  if (groups > 1) hipLaunchKernelGGL(pages_fork_lengths_kernel, dim3(1), dim3(kForkThreads), 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_pages_free(const PagesArgs& a, hipStream_t stream) {
  const int y = std::min((a.width + kTableThreads - 1) / kTableThreads, std::max(2048 / a.B, 1));
  hipLaunchKernelGGL(pages_free_kernel, dim3(a.B, y), dim3(kTableThreads), 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_pages_reserve(const PagesArgs& a, hipStream_t stream) {
  constexpr int rows = kTableThreads / 64;
  hipLaunchKernelGGL(pages_count_kernel, dim3(a.n_blocks + (a.B + rows - 1) / rows), dim3(kTableThreads), 0, stream, a);
  hipLaunchKernelGGL(pages_reserve_kernel, dim3(a.B), dim3(kTableThreads), 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_pages_compact(const PagesArgs& a, hipStream_t stream) {
  const int64_t work = std::max<int64_t>((int64_t)a.B * a.width, a.max_moves);
  const int groups = (int)std::min<int64_t>((work + kTableThreads - 1) / kTableThreads, 1024);
  hipLaunchKernelGGL(pages_in_use_kernel, dim3(a.n_blocks), dim3(kTableThreads), 0, stream, a);
  hipLaunchKernelGGL(pages_compact_kernel, dim3(a.n_blocks + groups), dim3(kTableThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace vico
