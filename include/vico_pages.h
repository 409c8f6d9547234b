/*
 * vico_pages.h -- a cache in pages: many sequences of ragged length in one pool
 * of keys and values, attention over it, and its page table (C ABI of libvico,
 * with vico.h).
 *
 * A GPU that serves several video streams, and the questions asked of them,
 * holds many histories at once; a question branches off a stream that goes on.
 * The calls, in the order of a step:
 *
 *   vico_pages_fork      rows of the page table become branches of others, or empty
 *   vico_pages_free      pages that a stream's window has left go back to the pool
 *   vico_pages_reserve   every sequence gets pages of its own for its new tokens
 *   vico_pages_copy      the pages that it replaced are copied, in every layer
 *   vico_paged_append    per layer: the new tokens' keys and values into the pages
 *   vico_paged_attn      per layer: the new tokens' attention over sink, window, chunk
 *   vico_pages_compact   now and then: the pages in use to the pool's low end
 *
 * The conventions of vico.h hold: tensors are dense, row-major and in the
 * caller's device memory, nothing is allocated or kept between calls, work is
 * enqueued on `stream`, host-detectable errors come back as a vico_status
 * before anything is enqueued, head_dim is 64 or 128.  Pointers to int32 arrays
 * are 4-byte aligned (moves 8-byte), the others 16-byte.  Every call
 * may be captured into a HIP graph; results repeat bit for bit.  Calls that
 * share a workspace must be ordered (same stream, or synchronised).
 *
 * The cache.
 *   k_pages, v_pages  [num_pages][page_size][num_kv_heads][head_dim] bf16; a
 *                     pool may be longer than 2^32 bytes.  page_size is a power
 *                     of two, 16 .. 1024; num_pages <= 2^21
 *   page_table        [num_seqs][max_pages] int32: entry j of row b is the page
 *                     that holds positions [j * page_size, (j + 1) * page_size)
 *                     of sequence b; a number outside [0, num_pages) is no page
 *                     (the calls write -1).  num_seqs <= 4096,
 *                     max_pages * page_size <= 2^30
 *   page_refs         [num_pages] int32: how many table entries hold the page;
 *                     0: it is free
 *   seq_len           [num_seqs] int32: tokens of the sequence in the cache
 *   q_start           [num_seqs + 1] int32, not decreasing: the new tokens of
 *                     sequence b are rows q_start[b] .. q_start[b + 1] - 1 of the
 *                     calls' q, k, v and out, and take positions seq_len[b] ...
 * The caller moves seq_len on after the last layer.  All of these live in device
 * memory, so the device checks them: a position without a page is neither
 * written nor attended to, rows outside [0, total) do not exist.
 *
 * A table or pool without an entry is VICO_ERR_CAPACITY to attention, fork and
 * reserve where they have a sequence to work for, a pool without one also to
 * compaction, and to free where the table has entries.  It is no error to append
 * (no position has a page), to copy (no pair names one) and, for the table, to
 * free: those have nothing to do and return VICO_OK.
 */
#ifndef VICO_PAGES_H
#define VICO_PAGES_H

#include "vico.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * vico_paged_append -- the new tokens' keys and values into their pages: row
 * q_start[b] + j goes to position seq_len[b] + j of sequence b, as a bit copy.
 *
 *   k, v           [total_tokens][num_kv_heads][head_dim] bf16
 *   k_pages, v_pages  written; rows without a page, rows before q_start[0] and
 *                  rows from q_start[num_seqs] on go nowhere
 * No two written positions may be the same (pages that several rows hold are
 * replaced by vico_pages_reserve).  total_tokens <= 2^20, k below 2^31 bytes.
 */
int vico_paged_append(const void* k, const void* v, int32_t total_tokens, const int32_t* q_start,
                      const int32_t* seq_len, int32_t num_seqs, void* k_pages, void* v_pages, int32_t num_pages,
                      int32_t page_size, const int32_t* page_table, int32_t max_pages, int32_t num_kv_heads,
                      int32_t head_dim, void* stream);

/*
 * vico_paged_attn -- attention of every sequence's new tokens over its pages.
 *
 * With H = seq_len[b], n = q_start[b + 1] - q_start[b] and g = num_q_heads /
 * num_kv_heads, the i-th new token of sequence b attends in query head h to the
 * keys of KV head h / g at the positions
 *     p <= H + i  (p < H + n with VICO_ATTN_BIDIRECTIONAL)  and
 *     p < sink_len  or  p >= H - window
 * that have a page: [sink | the window's newest history tokens | the chunk so
 * far], as vico_chunk_prefill_attn.  The new tokens' keys and values are in
 * the cache already (vico_paged_append).  n = 1 is a decode step; decode steps,
 * short queries and chunks may stand in one call.
 *
 *   q              [total_q][num_q_heads][head_dim] bf16
 *   max_q_len      at least every n: of a sequence with more new tokens the
 *                  first max_q_len rows are computed
 *   window         visible history tokens (>= 0) or VICO_FULL_HISTORY
 *   keys_hint      the longest H + n to be expected (0: not known); sets how the
 *                  work is split, any value gives the same result up to rounding
 *   flags          0 or VICO_ATTN_BIDIRECTIONAL
 *   out, out_dtype, lse_out, softmax_scale: as for vico_chunk_prefill_attn
 *                  ([total_q][num_q_heads][head_dim], [num_q_heads][total_q]);
 *                  rows of no sequence stay as they were; a row that sees no
 *                  key is 0, with lse_out -infinity
 *   num_splits     0: the library's choice; n > 0: key ranges in up to n parts
 *                  (<= 64)
 *   workspace      at least the bytes that vico_paged_attn_plan reports for the
 *                  same arguments (at most 64 MiB with num_splits = 0)
 * total_q <= 2^20; out is below 2^31 bytes as fp32; calls that would take 2^22
 * work-groups or more (num_seqs * num_kv_heads past some hundred thousand) are
 * VICO_ERR_INVALID_ARG.
 *
 * Arithmetic: as for vico_chunk_prefill_attn.  A NaN or an infinity in the value
 * of a key reaches the rows that see the key, as one or the other and whatever
 * its weight, and no other row; lse_out of a row with a NaN or +infinity among
 * its logits is NaN.
 */
int vico_paged_attn(const void* q, const int32_t* q_start, const int32_t* seq_len, int32_t num_seqs, int32_t total_q,
                    int32_t max_q_len, const void* k_pages, const void* v_pages, int32_t num_pages, int32_t page_size,
                    const int32_t* page_table, int32_t max_pages, int32_t sink_len, int64_t window, int64_t keys_hint,
                    int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim, float softmax_scale, int32_t flags,
                    void* out, int32_t out_dtype, float* lse_out, int32_t num_splits, void* workspace,
                    int64_t workspace_bytes, void* stream);

/*
 * vico_paged_attn_plan -- most key-range parts that vico_paged_attn takes with
 * these arguments and the workspace that it requires (host-only; validates the
 * arguments as the call does).
 */
int vico_paged_attn_plan(int32_t num_seqs, int32_t total_q, int32_t max_q_len, int32_t page_size, int32_t max_pages,
                         int32_t sink_len, int64_t window, int64_t keys_hint, int32_t num_q_heads,
                         int32_t num_kv_heads, int32_t head_dim, int32_t num_splits, int32_t* num_splits_out,
                         int64_t* workspace_bytes_out);

/*
 * vico_pages_fork -- rows of the page table taken from others, all at once.
 *
 * Row b becomes the branch of row parent[b] as that was before the call: it
 * holds the same pages for the parent's seq_len tokens (entries past them are
 * none), and has its seq_len.  parent[b] == b, or a number that is neither -1
 * nor a row: the row stays as it is.  -1: the row is empty, with seq_len 0.
 * What the row held before is given back.
 *
 *   page_table, page_refs, seq_len   read and written
 *   parent         [num_seqs] int32
 * Pages held by several rows are not to be written: vico_pages_reserve replaces
 * those that a row's new tokens would go to, the parent's too.
 */
int vico_pages_fork(int32_t* page_table, int32_t num_seqs, int32_t max_pages, int32_t* page_refs, int32_t num_pages,
                    int32_t page_size, int32_t* seq_len, const int32_t* parent, void* stream);

/*
 * vico_pages_free -- pages that lie wholly in positions [first[b], last[b]) of
 * their sequence are given back: their entries become -1.  A stream with a sink
 * and a window frees [sink_len, seq_len - window); [0, 2^31 - 1) is all of it.
 *
 *   page_table, page_refs   read and written
 *   first, last    [num_seqs] int32; first >= last: nothing of that row
 */
int vico_pages_free(int32_t* page_table, int32_t num_seqs, int32_t max_pages, int32_t* page_refs, int32_t num_pages,
                    int32_t page_size, const int32_t* first, const int32_t* last, void* stream);

/*
 * vico_pages_reserve -- pages of its own for every sequence's new tokens.
 *
 * With H = seq_len[b] and n = q_start[b + 1] - q_start[b], every entry that
 * holds one of the positions [H, H + n) and has no page, or one that other
 * entries hold too (page_refs != 1), gets a free page.  The free pages are taken
 * in rising order, for the rows in order and each row's entries in order, as
 * long as they last: a row that needs more of them than the rows before it left
 * gets none, nor does any row after it that needs one.  Nor does a row whose new
 * tokens pass max_pages.  Replaced pages are given back.
 *
 *   page_table, page_refs   read and written
 *   moves          [num_seqs][2] int32, written: {page, new page} where the
 *                  replaced page holds tokens before H (to be copied by
 *                  vico_pages_copy before anything else changes the pages), else
 *                  {-1, -1}
 *   granted        [num_seqs] int32, written: 1, or 0 for a row that got no pages
 *                  and is as it was
 *   workspace      at least vico_pages_workspace_bytes bytes
 */
int vico_pages_reserve(int32_t* page_table, int32_t num_seqs, int32_t max_pages, int32_t* page_refs,
                       int32_t num_pages, int32_t page_size, const int32_t* seq_len, const int32_t* q_start,
                       int32_t* moves, int32_t* granted, void* workspace, int64_t workspace_bytes, void* stream);

/*
 * vico_pages_compact -- the pages in use to the pool's low end.  With U pages in
 * use, those from U on move, in rising order, to the free pages below U, in
 * rising order.
 *
 *   page_table, page_refs   read and written: entries and counts of moved pages
 *   moves          [max_moves][2] int32, written: {from, to} of each move, then
 *                  {-1, -1}; max_moves at least num_pages / 2
 *   count          [1] int32, written: the moves
 *   workspace      at least vico_pages_workspace_bytes bytes
 * The pages' contents are moved by vico_pages_copy.
 */
int vico_pages_compact(int32_t* page_table, int32_t num_seqs, int32_t max_pages, int32_t* page_refs,
                       int32_t num_pages, int32_t* moves, int32_t max_moves, int32_t* count, void* workspace,
                       int64_t workspace_bytes, void* stream);

/* Workspace bytes of vico_pages_reserve and vico_pages_compact, or VICO_ERR_INVALID_ARG. */
int64_t vico_pages_workspace_bytes(int32_t num_seqs, int32_t num_pages);

/*
 * vico_pages_copy -- whole pages of keys and values copied, in every layer.
 *
 *   k_pages, v_pages  [num_layers][num_pages][page_size][num_kv_heads][head_dim]
 *                  bf16, read and written
 *   moves          [num_moves][2] int32: {from, to}; a pair with a number that is
 *                  no page is left out.  No page may be written twice, or both
 *                  written and read
 *   count          NULL or [1] int32 in device memory: only that many of the pairs
 */
int vico_pages_copy(void* k_pages, void* v_pages, int32_t num_layers, int32_t num_pages, int32_t page_size,
                    int32_t num_kv_heads, int32_t head_dim, const int32_t* moves, int32_t num_moves,
                    const int32_t* count, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* VICO_PAGES_H */
