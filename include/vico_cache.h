/*
 * vico_cache.h -- from a decoder layer's projection to a 4-bit store of keys
 * and values, and attention over it (C ABI of libvico, with vico.h).
 *
 * A streaming video LLM keeps the K/V of every past chunk for query-time
 * retrieval (ViCoStream, Sec. 3): the store grows with the stream, and every
 * answer token reads the retrieved chunks of it.  Held in 4 bits it takes 34
 * bytes for 64 values instead of 128.  The calls, in the order of a layer:
 *
 *   vico_qk_norm_rope     the projection's q, k, v -> normed and rotated q, k
 *                         and dense v, as the attention calls take them
 *   vico_gather_attn_q4   attention over [sink | segments of the store | tail]
 *   vico_kv_append_q4     the chunk's k, v into the store
 *   vico_kv_load_q4       segments of the store back as bf16
 *
 * The conventions of vico.h hold: tensors are dense, row-major and in the
 * caller's device memory, nothing is allocated or kept between calls, work is
 * enqueued on `stream`, host-detectable errors come back as a vico_status
 * before anything is enqueued, device pointers are 16-byte aligned unless
 * stated otherwise, head_dim is 64 or 128.  No call uses atomics: results
 * repeat bit for bit.  Every call may be captured into a HIP graph.
 *
 * The 4-bit store.  Four arrays, token-major; R = store_slots:
 *   store_k, store_v  [R][num_kv_heads][head_dim / 2]  uint8: element 2i in the
 *                     low four bits of byte i, element 2i + 1 in the high four
 *   scale_k, scale_v  [R][num_kv_heads][head_dim / 32] uint8
 * A code's highest bit is the sign, the others select 0, .5, 1, 1.5, 2, 3, 4,
 * 6.  Every 32 elements of a head share a scale byte b: the values are
 * code * 2^(b - 127), or all NaN for b = 255.  The calls write b in [4, 252],
 * and 255.  Other bytes are read as well (an array of zeros reads as zeros):
 * subnormal values are exact too, and values from 2^128 on (b = 253: 4 and 6;
 * b = 254: 2 and more) are infinities.  Writing a group with largest
 * magnitude m takes the smallest power of two s with m <= 7 s (the largest
 * element, if it becomes 6 s, is then no further off than half a step), kept
 * in [2^-123, 2^125]; values become x / s to the nearest code, ties to the
 * even one, at most 6 in size.  A group with a NaN or an infinity gets b = 255
 * and zero codes.  So groups below 2^-125 in size become zeros, and values
 * above 6 * 2^125 that.
 */
#ifndef VICO_CACHE_H
#define VICO_CACHE_H

#include "vico.h"

#ifdef __cplusplus
extern "C" {
#endif

/* flags of vico_qk_norm_rope */
#define VICO_ROPE_ADJACENT 1      /* pairs (2i, 2i + 1); else (i, i + rotary_dim / 2) */
#define VICO_ROPE_STRIDED_AXES 2  /* three axes: pairs dealt out in turn; else in sections */

/*
 * vico_qk_norm_rope -- norms of queries and keys for each head, with the
 * position rotation in the same pass; optionally the values' copy.
 *
 * For token t and each head, in fp32 (the norm of finite inputs of any size),
 * rounded to bf16 once at the end:
 *     x' = x * weight / sqrt(mean(x^2) + eps)        (x' = x where the weight is NULL)
 *     y0 = x0' cos a - x1' sin a,  y1 = x1' cos a + x0' sin a
 * for the rotary_dim / 2 pairs (x0, x1) of the head's first rotary_dim
 * elements; elements past rotary_dim are x'.  Pair i turns by
 *     a = positions[axis(i)][t] * inv_freq[i],
 * a product in fp64 (far positions keep their angle).
 *
 *   q, k, v        token t's heads at q + t * q_stride (elements; at least
 *                  heads * head_dim and a multiple of 8): slices of the packed
 *                  projection, or dense tensors.  bf16, num_q_heads heads for
 *                  q, num_kv_heads for k and v.  v may be NULL (with v_out).
 *   q_weight, k_weight  [head_dim] weight_dtype (BF16 or F32); NULL: that
 *                  tensor is not normed
 *   eps            >= 0
 *   positions      [num_axes][num_tokens] int32 (4-byte aligned), any value
 *   num_axes       1 (text, time) or 3 (time, row, column)
 *   inv_freq       [rotary_dim / 2] fp32 (4-byte aligned)
 *   rotary_dim     a multiple of 16, 16 .. head_dim
 *   sections       HOST array of num_axes pair counts, sum rotary_dim / 2; NULL
 *                  with one axis.  In sections, pairs [0, s0) turn with axis
 *                  0, [s0, s0 + s1) with axis 1, the rest with axis 2.  With
 *                  VICO_ROPE_STRIDED_AXES pair i turns with axis 1 if i % 3 == 1
 *                  and i < 3 s1, with axis 2 if i % 3 == 2 and i < 3 s2, else
 *                  with axis 0 (3 s1 - 2 and 3 s2 - 1 must be below
 *                  rotary_dim / 2, so that the counts hold).
 *   q_out          [num_tokens][num_q_heads][head_dim] bf16
 *   k_out, v_out   [num_tokens][num_kv_heads][head_dim] bf16
 *
 * An output may be its own input where that is dense (q_out == q with q_stride
 * == num_q_heads * head_dim); apart from that no output overlaps another
 * argument.  num_tokens == 0 is a no-op.  Each output is below 2^31 bytes.
 */
int vico_qk_norm_rope(const void* q, int64_t q_stride, const void* k, int64_t k_stride, const void* v,
                      int64_t v_stride, int32_t num_tokens, int32_t num_q_heads, int32_t num_kv_heads,
                      int32_t head_dim, const void* q_weight, const void* k_weight, int32_t weight_dtype, float eps,
                      const int32_t* positions, int32_t num_axes, const float* inv_freq, int32_t rotary_dim,
                      const int32_t* sections, int32_t flags, void* q_out, void* k_out, void* v_out, void* stream);

/*
 * vico_kv_append_q4 -- vico_kv_append into the 4-bit store: for j in
 * [0, chunk_len), slot (hist_len + j) % store_slots <- k_chunk[j], v_chunk[j].
 *
 *   k_chunk, v_chunk  [chunk_len][num_kv_heads][head_dim] bf16, read
 *   store_*, scale_*  written (see above); other slots stay as they are
 *
 * chunk_len == 0 is a no-op; chunk_len > store_slots -> VICO_ERR_CAPACITY.  No
 * written array overlaps another argument.  The chunk is below 2^31 bytes; the
 * store may be longer.
 */
int vico_kv_append_q4(const void* k_chunk, const void* v_chunk, int32_t chunk_len, void* store_k, void* store_v,
                      void* scale_k, void* scale_v, int32_t store_slots, int64_t hist_len, int32_t num_kv_heads,
                      int32_t head_dim, void* stream);

/*
 * vico_kv_load_q4 -- segments of the 4-bit store as bf16 (exactly: a value has
 * two significant bits; from 2^128 on an infinity), one after the other in
 * table order.
 *
 *   seg_start, seg_len  the table as for vico_gather_attn: int64 / int32 device
 *                  arrays of num_segments <= 2048 entries, clipped to [0, store_slots)
 *   out_k, out_v   [out_rows][num_kv_heads][head_dim] bf16, written: rows
 *                  0 .. min(G, out_rows) - 1, where G is the total length of the
 *                  clipped segments; further rows stay as they are
 *   out_count      NULL or [1] int32 (4-byte aligned), written: G, which may be
 *                  above out_rows
 *
 * num_segments * store_slots <= 2^30; an output is below 2^31 bytes and
 * overlaps no other argument.
 */
int vico_kv_load_q4(const void* store_k, const void* store_v, const void* scale_k, const void* scale_v,
                    int32_t store_slots, const int64_t* seg_start, const int32_t* seg_len, int32_t num_segments,
                    void* out_k, void* out_v, int32_t out_rows, int32_t* out_count, int32_t num_kv_heads,
                    int32_t head_dim, void* stream);

/*
 * vico_gather_attn_q4 -- vico_gather_attn with the store in 4 bits.
 *
 * Row i of the q_len query rows (the last q_len of tail_len tail tokens)
 * attends to
 *     sink[0 .. sink_len) ++ store[segment 0] ++ ... ++ store[segment n-1]
 *                         ++ tail[0 .. tail_len - q_len + i]
 * with the store's rows as the values they stand for.  q_len = 1 is a decode
 * step; a chunk over a window of the store used as a ring is q_len = tail_len
 * = chunk_len with the window as one or two segments.
 *
 * Arguments, plan and result as for vico_gather_attn, with
 *   store_k, store_v, scale_k, scale_v   the 4-bit store; NULL iff store_slots == 0
 *   keys_hint      expected total segment length (0: not known); sets how the
 *                  work is split and which kernel runs
 *   workspace      at least the bytes that vico_gather_plan_q4 reports for the
 *                  same arguments (at most 48 MiB with num_splits = 0)
 * num_segments * store_slots + sink_len + tail_len <= 2^30; q, sink, tail and
 * out are below 2^31 bytes, the store may be longer.  The table is
 * clipped to the store on the device as for vico_gather_attn.
 *
 * Arithmetic: the store's values as bf16 (exact), bf16 MFMA products with fp32
 * accumulation, fp32 online softmax, probabilities rounded to bf16 for the P.V
 * product.  A NaN or an infinity in a tail key or value reaches the rows that
 * see it, as one or the other and whatever its weight, and no other row.  (An
 * infinite key whose logit is -infinity has none.)  lse_out is NaN for a row
 * with a NaN or +infinity among its logits, where vico_gather_attn writes
 * -infinity: who merges both must take such a row from its output.
 */
int vico_gather_attn_q4(const void* q, int32_t q_len, const void* tail_k, const void* tail_v, int32_t tail_len,
                        const void* sink_k, const void* sink_v, int32_t sink_len, const void* store_k,
                        const void* store_v, const void* scale_k, const void* scale_v, int32_t store_slots,
                        const int64_t* seg_start, const int32_t* seg_len, int32_t num_segments, int64_t keys_hint,
                        int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim, float softmax_scale, void* out,
                        int32_t out_dtype, float* lse_out, int32_t num_splits, void* workspace,
                        int64_t workspace_bytes, void* stream);

/* vico_gather_plan for vico_gather_attn_q4. */
int vico_gather_plan_q4(int32_t q_len, int32_t tail_len, int32_t sink_len, int32_t store_slots,
                        int32_t num_segments, int64_t keys_hint, int32_t num_q_heads, int32_t num_kv_heads,
                        int32_t head_dim, int32_t num_splits, int32_t* num_splits_out, int64_t* workspace_bytes_out);

#ifdef __cplusplus
}
#endif
#endif /* VICO_CACHE_H */
