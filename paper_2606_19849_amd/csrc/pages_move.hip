// The contents of the cache in pages (gfx950): new tokens into their pages, and
// pages copied as the table's calls have decided (include/vico_pages.h).
//
// Both move bytes and compute nothing.  Append: a wave takes a few tokens, its
// lanes find the tokens' sequences (64 entries of q_start at a time) and slots
// together, then the wave copies their rows of K and V in 16-byte units: three
// memory latencies whatever the number of sequences up to 64, four up to 4096.
// Copy: a page of one layer is cut into pieces of 16 KB, four units a thread, all of a
// piece's loads on their way together.
// Alone: append of 32 tokens (7B heads) 2.7 us, of 18.5k tokens in 16 chunks (3B heads, 38 MB)
// 7.0 to 7.4, 5.1 to 5.4 TB/s; copy of 905 pages (237 MB) 36.6, 6.5 TB/s (some of it from the caches).

#include <algorithm>

#include "pages.h"

namespace vico {
namespace {

typedef uint32_t unit_t __attribute__((ext_vector_type(4)));
constexpr int kMoveThreads = 256;

__global__ __launch_bounds__(kMoveThreads) void paged_append_kernel(PagedAppendArgs a) {
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(blockIdx.x * (kMoveThreads / 64) + (threadIdx.x >> 6));
  const int t0 = wave * a.per_wave;
  const int n = min(a.per_wave, a.total - t0);
  if (n <= 0) return;
  int b = a.B;                                   // of token t0 + lane
  for (int i = 0; i < n; ++i) {
    const int s = sequence_of(a.q_start, a.B, t0 + i, lane);
    b = lane == i ? s : b;
  }
  int64_t slot = -1;
  if (lane < n && b < a.B) {
    int q0;
    const int rows = rows_of(a, b, q0), j = t0 + lane - q0;
    const int64_t pos = (int64_t)max(a.seq_len[b], 0) + j;
    if (j >= 0 && j < rows && (pos >> a.page_shift) < a.width) {
      const int page = a.table[(int64_t)b * a.width + (pos >> a.page_shift)];
      if ((uint32_t)page < (uint32_t)a.N) slot = ((int64_t)page << a.page_shift) + (pos & ((1 << a.page_shift) - 1));
    }
  }
  const unit_t* const k = (const unit_t*)a.k + (int64_t)t0 * a.row_units;
  const unit_t* const v = (const unit_t*)a.v + (int64_t)t0 * a.row_units;
  const int units = n * a.row_units;
  for (int u = lane; u - lane < units; u += 64) {        // every lane goes along: __shfl reads from all of them
    const int i = min(a.by_units(u), n - 1);
    const int64_t s = __shfl(slot, i, 64);
    if (u >= units || s < 0) continue;
    const unit_t x = k[u], y = v[u];
    const int64_t to = s * a.row_units + (u - i * a.row_units);
    ((unit_t*)a.k_pages)[to] = x;
    ((unit_t*)a.v_pages)[to] = y;
  }
}

constexpr int kPiece = 4 * kMoveThreads;         // 16-byte units

// work item: (move, layer, K or V, piece), pieces fastest
__global__ __launch_bounds__(kMoveThreads) void pages_copy_kernel(PagesCopyArgs a) {
  const int n = a.count ? min(max(*a.count, 0), a.n_moves) : a.n_moves;
  const int per_move = a.layers * 2 * a.pieces;
  const int64_t items = (int64_t)n * per_move;
  for (int64_t it = blockIdx.x; it < items; it += gridDim.x) {
    const int m = (int)(it / per_move), r = (int)(it - (int64_t)m * per_move);
    const int from = a.moves[2 * m], to = a.moves[2 * m + 1];
    if ((uint32_t)from >= (uint32_t)a.N || (uint32_t)to >= (uint32_t)a.N || from == to) continue;
    const int piece = r % a.pieces, lv = r / a.pieces;
    unit_t* const pool = (unit_t*)((lv & 1) ? a.v : a.k) + (int64_t)(lv >> 1) * a.N * a.page_units;
    const unit_t* const src = pool + (int64_t)from * a.page_units;
    unit_t* const dst = pool + (int64_t)to * a.page_units;
    const int u = piece * kPiece + threadIdx.x;
    unit_t x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (u + i * kMoveThreads < a.page_units) x[i] = src[u + i * kMoveThreads];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (u + i * kMoveThreads < a.page_units) dst[u + i * kMoveThreads] = x[i];
  }
}

}  // namespace

hipError_t launch_paged_append(const PagedAppendArgs& args, hipStream_t stream) {
  PagedAppendArgs a = args;
  constexpr int waves = kMoveThreads / 64;
  // as many tokens a wave as leave every CU four work-groups, eight at most
  a.per_wave = std::min(std::max(a.total / (kNumCUs * 4 * waves), 1), 8);
  const int groups = (a.total + a.per_wave * waves - 1) / (a.per_wave * waves);
  hipLaunchKernelGGL(paged_append_kernel, dim3(groups), dim3(kMoveThreads), 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_pages_copy(const PagesCopyArgs& args, hipStream_t stream) {
  PagesCopyArgs a = args;
  a.pieces = (a.page_units + kPiece - 1) / kPiece;
  const int64_t items = (int64_t)a.n_moves * a.layers * 2 * a.pieces;
  hipLaunchKernelGGL(pages_copy_kernel, dim3((unsigned)std::min<int64_t>(items, kNumCUs * 32)), dim3(kMoveThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace vico
