// Host side of include/vico_cache.h: argument validation, launch planning and
// error mapping, as vico_api.hip does it for vico.h.

#include <math.h>

#include <algorithm>
#include <stdint.h>

#include "vico_cache.h"
#include "vico_internal.h"
#include "host_util.h"

using namespace vico;

namespace {

bool heads_ok(int32_t Hq, int32_t Hkv) { return Hq >= 1 && Hkv >= 1 && Hq <= kMaxHeads && Hkv <= kMaxHeads; }

// Bytes of one code array and one scale array of the store.
int64_t code_bytes(int64_t slots, int32_t Hkv, int32_t D) { return slots * Hkv * (D / 2); }
int64_t scale_bytes(int64_t slots, int32_t Hkv, int32_t D) { return slots * Hkv * (D / 32); }

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

struct GatherQ4Shape {
  int Lq, T, S, cap, n_segs, Hq, Hkv, D;
  int tile, row_blocks, n_rt, parts;     // tile: 256-row tiles; else 16 * row_blocks rows
  int64_t ws_bytes;
};

constexpr int64_t kAutoWorkspace = int64_t(48) << 20;     // most bytes that a split picked by the library needs
constexpr int64_t kTileMinRows = 128;                     // fewer packed rows of a KV head never take the 256-row kernel

// One way to run a call: kernel, row tiles, key-range parts, and its time in ns:
// rounds of work-groups over the CUs, each a start (launch, table, first keys, the
// waves' merge or the output) and its keys, 32 or 64 at a time; then the merge of
// the parts (another launch, and more work above 16 parts) with the partial
// results' way to memory and back (2 MB a us).
//
// The rates, fitted to calls on otherwise idle CUs, all keys in one part, us for
// 64 / 1024 / 8192 / 65536 keys: 16-row tiles, one row of the 7B heads 6.1 / 9.6 /
// 41.4 / 319, of heads of size 64 (2048, 32768 keys) 8.6 / 80; 32-row tiles, 28 rows
// (256, 1024, 16384 keys) 9.0 / 12.5 / 91, heads of size 64 6.4 / 8.6 / 61; 256-row
// tiles 101.6 for 64 tiles more.
//
// Rows against 256-row kernel, each at its best, us: 7B heads, 224 rows, 2048 /
// 20000 keys 13 / 21 and 23 / 34; 700 rows, 8192 / 20000 keys 32 / 36 and 62 / 50;
// 1050 rows, 2048 / 8192 keys 20 / 31 and 51 / 41; 3B heads, 1600 rows, 8192 / 20000
// keys 32 / 38 and 62 / 53; small heads, 1024 rows, 20000 keys 26 / 32.  Both are
// far from a matrix product's rate there (8.5 us of work for 700 rows over 8192 keys): the
// rows kernel converts the codes for every 32 rows, the other has few row tiles.
struct Q4Plan {
  int tile, row_blocks, n_rt, parts;
  int64_t cost;
};

struct Q4Cost {
  int64_t groups, blocks, start, block, part_bytes;      // work-groups of one part, 32- or 64-key blocks
  int64_t operator()(int64_t parts) const {
    const int64_t rounds = (groups * parts + kNumCUs - 1) / kNumCUs;
    return rounds * (start + block * ((blocks + parts - 1) / parts)) +
           (parts > 1 ? (parts > 16 ? 4200 : 3500) + parts * part_bytes / 2000 : 0);
  }
};

// The parts with the least time: those that fill the CUs once, or fewer by halves.
Q4Plan best_parts(const Q4Cost& cost, int tile, int row_blocks, int n_rt, int splits) {
  if (splits > 0) {
    const int p = std::min(splits, kMaxGatherParts);
    return Q4Plan{tile, row_blocks, n_rt, p, cost(p)};
  }
  Q4Plan best{tile, row_blocks, n_rt, 1, cost(1)};
  const int64_t most = std::min(std::min<int64_t>(kNumCUs / cost.groups, kMaxGatherParts),
                                std::min(cost.blocks, (kAutoWorkspace - 256) / cost.part_bytes));
  for (int64_t p = most; p > 1; p /= 2) {
    const int64_t c = cost(p);
    if (c < best.cost) {
      best.parts = (int)p;
      best.cost = c;
    }
  }
  return best;
}

// Validates the shape arguments and plans.
int check_gather_q4_shape(int32_t Lq, int32_t T, int32_t S, int32_t cap, int32_t n_segs, int64_t hint, int32_t Hq,
                          int32_t Hkv, int32_t D, int32_t splits, GatherQ4Shape* sh) {
  if (Lq < 0 || T < Lq || S < 0 || cap < 0 || n_segs < 0 || n_segs > kMaxSegments || hint < 0 || splits < 0)
    return VICO_ERR_INVALID_ARG;
  if (!heads_ok(Hq, Hkv) || Hq % Hkv != 0) return VICO_ERR_INVALID_ARG;
  if (D != 64 && D != 128) return VICO_ERR_UNSUPPORTED;
  if (T > kMaxChunk || S > kMaxChunk || cap > kMaxKeys) return VICO_ERR_INVALID_ARG;
  if (int64_t(n_segs) * cap + S + T > kMaxKeys) return VICO_ERR_INVALID_ARG;
  const int64_t row_bytes = int64_t(Hkv) * D * 2;
  if (row_bytes * T >= kMaxTensorBytes || row_bytes * S >= kMaxTensorBytes ||
      int64_t(Lq) * Hq * D * 4 >= kMaxTensorBytes)
    return VICO_ERR_INVALID_ARG;
  *sh = GatherQ4Shape{Lq, T, S, cap, n_segs, Hq, Hkv, D, 0, 1, 0, 1, 0};
  if (Lq == 0) return VICO_OK;
  const int64_t rows = int64_t(Hq / Hkv) * Lq;
  const int64_t gathered = n_segs == 0 ? 0 : std::min<int64_t>(hint > 0 ? hint : cap, int64_t(n_segs) * cap);
  const int64_t keys = S + gathered + T, part_o = int64_t(4) * Hq * Lq * D, part_lse = int64_t(4) * Hq * Lq;
  const int64_t blocks = (keys + kRowsBlock - 1) / kRowsBlock, tiles = (keys + kKeyTile - 1) / kKeyTile;
  const bool d128 = D == 128;
  const int rb = rows > 16 ? 2 : 1, n_rt = (int)((rows + 16 * rb - 1) / (16 * rb));
  Q4Cost c{int64_t(Hkv) * n_rt, blocks, rb == 1 ? 3800 : d128 ? 6000 : 4800,
           rb == 1 ? (d128 ? 140 : 75) : (d128 ? 163 : 113), part_o + part_lse};
  Q4Plan best = best_parts(c, 0, rb, n_rt, splits);
  if (rows >= kTileMinRows) {
    const int n256 = (int)((rows + kBlockM - 1) / kBlockM);
    c.groups = int64_t(Hkv) * n256;
    c.blocks = tiles;
    c.start = 5000;
    c.block = d128 ? 1600 : 1200;
    const Q4Plan p = best_parts(c, 1, 0, n256, splits);
    if (p.cost < best.cost) best = p;
  }
  sh->tile = best.tile; sh->row_blocks = best.row_blocks; sh->n_rt = best.n_rt; sh->parts = best.parts;
  if (sh->parts > 1) sh->ws_bytes = align256(sh->parts * part_o) + sh->parts * part_lse;
  return VICO_OK;
}

int status_of(hipError_t e) { return e == hipSuccess ? VICO_OK : record_hip_failure(e); }

}  // namespace

extern "C" {

int vico_qk_norm_rope(const void* q, int64_t q_stride, const void* k, int64_t k_stride, const void* v,
                      int64_t v_stride, int32_t num_tokens, int32_t num_q_heads, int32_t num_kv_heads,
                      int32_t head_dim, const void* q_weight, const void* k_weight, int32_t weight_dtype, float eps,
                      const int32_t* positions, int32_t num_axes, const float* inv_freq, int32_t rotary_dim,
                      const int32_t* sections, int32_t flags, void* q_out, void* k_out, void* v_out, void* stream) {
  const int64_t T = num_tokens, D = head_dim;
  if (T < 0 || !heads_ok(num_q_heads, num_kv_heads)) return VICO_ERR_INVALID_ARG;
  if (D != 64 && D != 128) return VICO_ERR_UNSUPPORTED;
  if (weight_dtype != VICO_DTYPE_BF16 && weight_dtype != VICO_DTYPE_F32) return VICO_ERR_UNSUPPORTED;
  if (flags & ~(VICO_ROPE_ADJACENT | VICO_ROPE_STRIDED_AXES)) return VICO_ERR_INVALID_ARG;
  if (!(eps >= 0.f) || isinf(eps)) return VICO_ERR_INVALID_ARG;
  if (num_axes != 1 && num_axes != 3) return VICO_ERR_INVALID_ARG;
  if (rotary_dim < 16 || rotary_dim > D || rotary_dim % 16 != 0) return VICO_ERR_INVALID_ARG;
  const int half = rotary_dim / 2;
  int32_t s[3] = {half, 0, 0};
  if (num_axes == 3) {
    if (!sections) return VICO_ERR_INVALID_ARG;
    int64_t sum = 0;
    for (int i = 0; i < 3; ++i) {
      s[i] = sections[i];
      if (s[i] < 0) return VICO_ERR_INVALID_ARG;
      sum += s[i];
    }
    if (sum != half) return VICO_ERR_INVALID_ARG;
  } else if (sections && sections[0] != half) {
    return VICO_ERR_INVALID_ARG;
  }
  if (flags & VICO_ROPE_STRIDED_AXES) {
    if (num_axes != 3 || (s[1] > 0 && 3 * s[1] - 2 >= half) || (s[2] > 0 && 3 * s[2] - 1 >= half)) return VICO_ERR_INVALID_ARG;
  }
  const int64_t qrow = num_q_heads * D, krow = num_kv_heads * D;
  const int64_t qb = T * qrow * 2, kb = T * krow * 2;
  if (qb >= kMaxTensorBytes || kb >= kMaxTensorBytes) return VICO_ERR_INVALID_ARG;
  if (!v != !v_out) return VICO_ERR_INVALID_ARG;
  constexpr int64_t kMaxStride = int64_t(1) << 31;
  if (q_stride < qrow || k_stride < krow || (v && v_stride < krow) || q_stride % 8 || k_stride % 8 ||
      (v && v_stride % 8) || q_stride >= kMaxStride || k_stride >= kMaxStride || (v && v_stride >= kMaxStride))
    return VICO_ERR_INVALID_ARG;
  if (T == 0) return VICO_OK;
  if (!q || !k || !positions || !inv_freq || !q_out || !k_out) return VICO_ERR_INVALID_ARG;
  const void* ptrs[] = {q, k, v, q_weight, k_weight, q_out, k_out, v_out};
  for (const void* p : ptrs)
    if (p && !aligned16(p)) return VICO_ERR_MISALIGNED;
  if (!aligned_to(positions, 4) || !aligned_to(inv_freq, 4)) return VICO_ERR_MISALIGNED;

  const int64_t wb = D * (weight_dtype == VICO_DTYPE_F32 ? 4 : 2);
  // an output that is its own dense input is left out of that comparison
  const Region in[3] = {{q, ((T - 1) * q_stride + qrow) * 2}, {k, ((T - 1) * k_stride + krow) * 2},
                        {v, ((T - 1) * v_stride + krow) * 2}};
  const Region out[3] = {{q_out, qb}, {k_out, kb}, {v_out, kb}};
  const int64_t dense[3] = {qrow, krow, krow}, strides[3] = {q_stride, k_stride, v_stride};
  for (int o = 0; o < 3; ++o)
    for (int i = 0; i < 3; ++i) {
      if (!out[o].p || !in[i].p) continue;
      if (o == i && out[o].p == in[i].p && (strides[i] == dense[i] || T == 1)) continue;
      if (overlaps(out[o].p, out[o].bytes, in[i].p, in[i].bytes)) return VICO_ERR_INVALID_ARG;
    }
  const Region rest[] = {{q_weight, wb}, {k_weight, wb}, {positions, int64_t(num_axes) * T * 4}, {inv_freq, int64_t(half) * 4}};
  if (collide(out, rest)) return VICO_ERR_INVALID_ARG;

  RopeArgs a{};
  a.q = (const uint16_t*)q; a.k = (const uint16_t*)k; a.v = (const uint16_t*)v;
  a.q_out = (uint16_t*)q_out; a.k_out = (uint16_t*)k_out; a.v_out = (uint16_t*)v_out;
  a.q_weight = q_weight; a.k_weight = k_weight;
  a.positions = positions; a.inv_freq = inv_freq;
  a.q_stride = q_stride; a.k_stride = k_stride; a.v_stride = v_stride;
  a.T = num_tokens; a.Hq = num_q_heads; a.Hkv = num_kv_heads; a.D = head_dim;
  a.axes = num_axes; a.rot = rotary_dim; a.s0 = s[0]; a.s1 = s[1]; a.s2 = s[2];
  a.adjacent = (flags & VICO_ROPE_ADJACENT) != 0;
  a.strided = (flags & VICO_ROPE_STRIDED_AXES) != 0;
  a.weight_f32 = weight_dtype == VICO_DTYPE_F32;
  a.eps = eps;
  return status_of(launch_qk_norm_rope(a, (hipStream_t)stream));
}

int vico_kv_append_q4(const void* k_chunk, const void* v_chunk, int32_t chunk_len, void* store_k, void* store_v,
                      void* scale_k, void* scale_v, int32_t store_slots, int64_t hist_len, int32_t num_kv_heads,
                      int32_t head_dim, void* stream) {
  if (chunk_len < 0 || store_slots < 0 || hist_len < 0 || !heads_ok(num_kv_heads, num_kv_heads))
    return VICO_ERR_INVALID_ARG;
  if (head_dim != 64 && head_dim != 128) return VICO_ERR_UNSUPPORTED;
  if (chunk_len > kMaxChunk || store_slots > kMaxKeys) return VICO_ERR_INVALID_ARG;
  if (chunk_len > store_slots) return VICO_ERR_CAPACITY;
  const int64_t cb = int64_t(chunk_len) * num_kv_heads * head_dim * 2;
  if (cb >= kMaxTensorBytes) return VICO_ERR_INVALID_ARG;
  if (chunk_len == 0) return VICO_OK;
  if (!k_chunk || !v_chunk || !store_k || !store_v || !scale_k || !scale_v) return VICO_ERR_INVALID_ARG;
  const void* ptrs[] = {k_chunk, v_chunk, store_k, store_v, scale_k, scale_v};
  for (const void* p : ptrs)
    if (!aligned16(p)) return VICO_ERR_MISALIGNED;
  const int64_t qb = code_bytes(store_slots, num_kv_heads, head_dim), sb = scale_bytes(store_slots, num_kv_heads, head_dim);
  const Region w[] = {{store_k, qb}, {store_v, qb}, {scale_k, sb}, {scale_v, sb}};
  const Region r[] = {{k_chunk, cb}, {v_chunk, cb}};
  if (collide(w, r)) return VICO_ERR_INVALID_ARG;
  AppendQ4Args a{(const uint16_t*)k_chunk, (const uint16_t*)v_chunk, (uint8_t*)store_k, (uint8_t*)store_v,
                 (uint8_t*)scale_k, (uint8_t*)scale_v, chunk_len, store_slots, (int)(hist_len % store_slots),
                 num_kv_heads * head_dim};
  return status_of(launch_append_q4(a, (hipStream_t)stream));
}

int vico_kv_load_q4(const void* store_k, const void* store_v, const void* scale_k, const void* scale_v,
                    int32_t store_slots, const int64_t* seg_start, const int32_t* seg_len, int32_t num_segments,
                    void* out_k, void* out_v, int32_t out_rows, int32_t* out_count, int32_t num_kv_heads,
                    int32_t head_dim, void* stream) {
  if (store_slots < 0 || num_segments < 0 || num_segments > kMaxSegments || out_rows < 0 ||
      !heads_ok(num_kv_heads, num_kv_heads))
    return VICO_ERR_INVALID_ARG;
  if (head_dim != 64 && head_dim != 128) return VICO_ERR_UNSUPPORTED;
  if (store_slots > kMaxKeys || int64_t(num_segments) * store_slots > kMaxKeys) return VICO_ERR_INVALID_ARG;
  const int64_t ob = int64_t(out_rows) * num_kv_heads * head_dim * 2;
  if (ob >= kMaxTensorBytes) return VICO_ERR_INVALID_ARG;
  if (out_rows == 0 && !out_count) return VICO_OK;
  if (out_rows > 0 && (!out_k || !out_v)) return VICO_ERR_INVALID_ARG;
  if (num_segments > 0 && (!seg_start || !seg_len)) return VICO_ERR_INVALID_ARG;
  if (num_segments > 0 && store_slots > 0 && (!store_k || !store_v || !scale_k || !scale_v)) return VICO_ERR_INVALID_ARG;
  const void* ptrs[] = {store_k, store_v, scale_k, scale_v, out_k, out_v};
  for (const void* p : ptrs)
    if (p && !aligned16(p)) return VICO_ERR_MISALIGNED;
  if (!aligned_to(seg_start, 8) || !aligned_to(seg_len, 4) || !aligned_to(out_count, 4)) return VICO_ERR_MISALIGNED;
  const int64_t qb = code_bytes(store_slots, num_kv_heads, head_dim), sb = scale_bytes(store_slots, num_kv_heads, head_dim);
  const Region w[] = {{out_k, ob}, {out_v, ob}, {out_count, 4}};
  const Region r[] = {{store_k, qb}, {store_v, qb}, {scale_k, sb}, {scale_v, sb},
                      {seg_start, int64_t(num_segments) * 8}, {seg_len, int64_t(num_segments) * 4}};
  if (collide(w, r)) return VICO_ERR_INVALID_ARG;
  LoadQ4Args a{(const uint8_t*)store_k, (const uint8_t*)store_v, (const uint8_t*)scale_k, (const uint8_t*)scale_v,
               seg_start, seg_len, (uint16_t*)out_k, (uint16_t*)out_v, out_count, store_slots, num_segments, out_rows,
               num_kv_heads * head_dim};
  return status_of(launch_load_q4(a, (hipStream_t)stream));
}

int vico_gather_plan_q4(int32_t q_len, int32_t tail_len, int32_t sink_len, int32_t store_slots, int32_t num_segments,
                        int64_t keys_hint, int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim,
                        int32_t num_splits, int32_t* num_splits_out, int64_t* workspace_bytes_out) {
  GatherQ4Shape sh;
  const int st = check_gather_q4_shape(q_len, tail_len, sink_len, store_slots, num_segments, keys_hint, num_q_heads,
                                       num_kv_heads, head_dim, num_splits, &sh);
  if (st != VICO_OK) return st;
  if (num_splits_out) *num_splits_out = sh.parts;
  if (workspace_bytes_out) *workspace_bytes_out = sh.ws_bytes;
  return VICO_OK;
}

int vico_gather_q4_route(int32_t q_len, int32_t tail_len, int32_t sink_len, int32_t store_slots, int32_t num_segments,
                         int64_t keys_hint, int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim,
                         int32_t num_splits, int32_t* route_out) {
  GatherQ4Shape sh;
  const int st = check_gather_q4_shape(q_len, tail_len, sink_len, store_slots, num_segments, keys_hint, num_q_heads,
                                       num_kv_heads, head_dim, num_splits, &sh);
  if (st != VICO_OK) return st;
  route_out[0] = sh.tile ? kRouteTile : kRouteRows;
  route_out[1] = sh.parts;
  route_out[2] = sh.Hkv * sh.n_rt * sh.parts;
  route_out[3] = sh.tile ? kBlockM : 16 * sh.row_blocks;
  return VICO_OK;
}

int vico_gather_attn_q4(const void* q, int32_t q_len, const void* tail_k, const void* tail_v, int32_t tail_len,
                        const void* sink_k, const void* sink_v, int32_t sink_len, const void* store_k,
                        const void* store_v, const void* scale_k, const void* scale_v, int32_t store_slots,
                        const int64_t* seg_start, const int32_t* seg_len, int32_t num_segments, int64_t keys_hint,
                        int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim, float softmax_scale, void* out,
                        int32_t out_dtype, float* lse_out, int32_t num_splits, void* workspace,
                        int64_t workspace_bytes, void* stream) {
  GatherQ4Shape sh;
  const int st = check_gather_q4_shape(q_len, tail_len, sink_len, store_slots, num_segments, keys_hint, num_q_heads,
                                       num_kv_heads, head_dim, num_splits, &sh);
  if (st != VICO_OK) return st;
  if (out_dtype != VICO_DTYPE_BF16 && out_dtype != VICO_DTYPE_F32) return VICO_ERR_UNSUPPORTED;
  if (isnan(softmax_scale) || isinf(softmax_scale) || workspace_bytes < 0) return VICO_ERR_INVALID_ARG;
  if (q_len == 0) return VICO_OK;
  if (!q || !tail_k || !tail_v || !out) return VICO_ERR_INVALID_ARG;
  if (sink_len > 0 && (!sink_k || !sink_v)) return VICO_ERR_INVALID_ARG;
  if (num_segments > 0 && (!seg_start || !seg_len)) return VICO_ERR_INVALID_ARG;
  if (num_segments > 0 && store_slots > 0 && (!store_k || !store_v || !scale_k || !scale_v)) return VICO_ERR_INVALID_ARG;
  const void* ptrs[] = {q, tail_k, tail_v, sink_k, sink_v, store_k, store_v, scale_k, scale_v, out, workspace};
  for (const void* p : ptrs)
    if (p && !aligned16(p)) return VICO_ERR_MISALIGNED;
  if (!aligned_to(seg_start, 8) || !aligned_to(seg_len, 4) || !aligned_to(lse_out, 4)) return VICO_ERR_MISALIGNED;
  if (sh.ws_bytes > 0 && (!workspace || workspace_bytes < sh.ws_bytes)) return VICO_ERR_WORKSPACE;
  const int64_t rows = int64_t(q_len) * num_q_heads, row = int64_t(num_kv_heads) * head_dim * 2;
  const int64_t qb = code_bytes(store_slots, num_kv_heads, head_dim), sb = scale_bytes(store_slots, num_kv_heads, head_dim);
  const Region w[] = {{out, rows * head_dim * (out_dtype == VICO_DTYPE_F32 ? 4 : 2)}, {lse_out, rows * 4},
                      {sh.ws_bytes > 0 ? workspace : nullptr, sh.ws_bytes}};
  const Region r[] = {{q, rows * head_dim * 2}, {tail_k, row * tail_len}, {tail_v, row * tail_len},
                      {sink_k, row * sink_len}, {sink_v, row * sink_len}, {store_k, qb}, {store_v, qb}, {scale_k, sb},
                      {scale_v, sb}, {seg_start, int64_t(num_segments) * 8}, {seg_len, int64_t(num_segments) * 4}};
  if (collide(w, r)) return VICO_ERR_INVALID_ARG;

  RowsQ4Args a{};
  a.q = (const uint16_t*)q;
  a.tail_k = (const uint16_t*)tail_k; a.tail_v = (const uint16_t*)tail_v;
  a.sink_k = (const uint16_t*)sink_k; a.sink_v = (const uint16_t*)sink_v;
  a.k4 = (const uint8_t*)store_k; a.v4 = (const uint8_t*)store_v;
  a.ks = (const uint8_t*)scale_k; a.vs = (const uint8_t*)scale_v;
  a.seg_start = seg_start; a.seg_len = seg_len;
  a.out = out;
  a.lse = lse_out;
  if (sh.parts > 1) {
    a.ws_o = (float*)workspace;
    a.ws_lse = (float*)((char*)workspace + align256(int64_t(4) * sh.parts * sh.Hq * sh.Lq * sh.D));
  }
  a.Lq = sh.Lq; a.T = sh.T; a.S = sh.S; a.cap = sh.cap; a.n_segs = sh.n_segs;
  a.Hq = sh.Hq; a.Hkv = sh.Hkv; a.D = sh.D;
  a.parts = sh.parts; a.n_rt = sh.n_rt; a.row_blocks = sh.row_blocks;
  a.by_g = FastDiv::by(a.Hq / a.Hkv);
  a.by_rt = FastDiv::by(a.n_rt);
  a.by_kv = FastDiv::by(a.Hkv);
  a.by_parts = FastDiv::by(a.parts);
  a.out_f32 = out_dtype == VICO_DTYPE_F32;
  const double scale = softmax_scale > 0.f ? double(softmax_scale) : 1.0 / sqrt(double(head_dim));
  a.scale_log2 = (float)(scale * 1.4426950408889634);
  hipError_t e = sh.tile ? launch_tile_q4(a, (hipStream_t)stream) : launch_rows_q4(a, (hipStream_t)stream);
  if (e == hipSuccess && a.parts > 1) {
    AttnArgs m{};
    m.out = a.out; m.lse = a.lse; m.ws_o = a.ws_o; m.ws_lse = a.ws_lse;
    m.C = a.Lq; m.Hq = a.Hq; m.Hkv = a.Hkv; m.D = a.D;
    m.splits = a.parts; m.out_f32 = a.out_f32; m.keep_nan = 1;
    e = launch_merge(m, (hipStream_t)stream);
  }
  return status_of(e);
}

}  // extern "C"
