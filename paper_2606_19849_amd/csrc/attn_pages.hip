// The kernels of attention over the cache in pages (gfx950): which work-group does
// what.  Sequences are of three classes by their packed rows (tokens times query heads
// of a KV head): up to 16, decode steps and the shortest queries; up to 64 rows (more where a
// launch has no 256-row tiles); more.  Which sequence is of which class stands in device memory: a launch
// has work-groups for every sequence in every class that max_q_len allows, and those
// that find another class end.  What is left of a call in which a class has no
// sequence is the time of that, about 1 us a 256 work-groups (up to 64 sequences).
//
// Calls of one class, or of the first two, have kernels of four waves of which a CU
// holds several, so that one's start is hidden behind another's keys.  With
// the third, one launch does all: work-groups of the matrix cores first, which are
// long, then those that stream keys, in parts that count both (paged_tile_cost).  Every
// work-group reads all lengths, a sequence a lane, and takes its own from the lanes.
// (A chunk of 1024 tokens beside 31 answer tokens, 7B heads, windows of 8192 keys: 206 us, 141
// and 99 each alone; 220 to 228 in parts for the chunk alone; 362 in two launches and
// two merges, row tiles of 32 for the answer tokens.)  Of hundreds of sequences the
// lengths take longer than the streams gain, and there are two launches (rows_apart).

#include "attn_rows_pages.h"
#include "attn_tile_pages.h"

namespace vico {
namespace {

template <int D>
__global__ __launch_bounds__(256, 2) void paged_decode_kernel(PagedAttnArgs a) {
  __shared__ RowsLds<D, 1, 4> lds;
  paged_rows<D, 1, 4>(a, a.few, blockIdx.x, lds, [&](int b) { return sequence(a, b); });
}

template <int D>
__global__ __launch_bounds__(256, 2) void paged_rows_kernel(PagedAttnArgs a) {
  __shared__ union { RowsLds<D, 1, 4> few; RowsLds<D, 2, 4> some; } lds;
  const int blk = blockIdx.x;
  auto at = [&](int b) { return sequence(a, b); };
  if (blk < a.some.groups) paged_rows<D, 2, 4>(a, a.some, blk, lds.some, at);
  else paged_rows<D, 1, 4>(a, a.few, blk - a.some.groups, lds.few, at);
}

template <int D>
__global__ __launch_bounds__(kThreads, 1) void paged_mixed_kernel(PagedAttnArgs a) {
  __shared__ union { TileLds<D> tile; RowsLds<D, 1, 8> rows; } lds;
  const LaneSequences y = lane_sequences(a);
  int blk = blockIdx.x, parts;
  const int items = all_row_tiles(a, y, parts);
  // (starts that decrease may count rows twice: more partial results than there is room for)
  const bool fits = parts == 1 || (items <= a.tile_items && items <= a.tile_slots / parts);
  const int n_work = fits ? items * parts : 0;
  if (blk == 0 && threadIdx.x == 0 && a.ws_items) {
    a.ws_items->items = fits && parts > 1 ? items : 0;
    a.ws_items->parts = parts;
  }
  if (blk < n_work) return paged_tile<D>(a, y, blk, n_work, parts, lds.tile);
  blk -= n_work;
  if (blk >= a.some.groups + a.few.groups) return;
  // 16-row tiles for both: the 256-row kernel's accumulation registers leave 128 others, and 32 rows do not fit those
  const bool some = blk < a.some.groups;
  paged_rows<D, 1, 8>(a, some ? a.some : a.few, blk - (some ? 0 : a.some.groups), lds.rows, [&](int b) { return sequence(a, y, b); });
}

template <int D>
__global__ __launch_bounds__(kMergeThreads) void paged_merge_kernel(PagedAttnArgs a) {
  int blk = blockIdx.x;
  if (blk < a.tile_merge) return paged_tile_merge<D>(a, blk);
  blk -= a.tile_merge;
  if (blk < a.some.merge) {
    if (a.some.parts <= 8) paged_rows_merge<D, 1>(a, a.some, blk);
    else paged_rows_merge<D, 8>(a, a.some, blk);
    return;
  }
  blk -= a.some.merge;
  if (a.few.parts <= 8) paged_rows_merge<D, 1>(a, a.few, blk);
  else paged_rows_merge<D, 8>(a, a.few, blk);
}

// Work-groups of the merge for a class: none for a single part.
template <int D>
int merge_groups(const RowsClass& x, int B, int Hkv) {
  const int per = kMergeThreads / (D / 4) / (x.parts <= 8 ? 1 : 8);      // rows of a work-group
  return x.parts <= 1 ? 0 : B * Hkv * x.n_rt * ((x.merge_rows + per - 1) / per);
}

template <int D>
hipError_t launch(const PagedAttnArgs& args, hipStream_t stream) {
  PagedAttnArgs a = args;
  if (a.tile_grid > 0) {
    PagedAttnArgs t = a;
    if (a.rows_apart) t.some.groups = t.few.groups = 0;
    hipLaunchKernelGGL(paged_mixed_kernel<D>, dim3((unsigned)(t.tile_grid + t.some.groups + t.few.groups)), dim3(kThreads), 0, stream, t);
  }
  if (a.tile_grid == 0 || a.rows_apart) {
    if (a.some.groups > 0) hipLaunchKernelGGL(paged_rows_kernel<D>, dim3((unsigned)(a.some.groups + a.few.groups)), dim3(256), 0, stream, a);
    else hipLaunchKernelGGL(paged_decode_kernel<D>, dim3((unsigned)a.few.groups), dim3(256), 0, stream, a);
  }
  const hipError_t e = hipGetLastError();
  a.few.merge = merge_groups<D>(a.few, a.B, a.Hkv);
  a.some.merge = merge_groups<D>(a.some, a.B, a.Hkv);
  a.tile_merge = a.ws_o ? a.tile_items * (kBlockM / kTileMergeRows) : 0;
  const int groups = a.few.merge + a.some.merge + a.tile_merge;
  if (e != hipSuccess || groups == 0) return e;
  hipLaunchKernelGGL(paged_merge_kernel<D>, dim3((unsigned)groups), dim3(kMergeThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_attention(const PagedAttnArgs& a, hipStream_t stream) {
  if (a.few.groups < 1 || a.few.parts > kPagedParts || a.some.parts > kPagedParts || a.tile_splits > kPagedTileParts)
    return hipErrorInvalidValue;
  return a.D == 128 ? launch<128>(a, stream) : launch<64>(a, stream);
}

}  // namespace vico
