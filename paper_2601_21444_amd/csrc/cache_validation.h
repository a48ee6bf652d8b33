// Host-side argument validation and planning of the cache's C ABI (include/apbv_cache.h); plain C++ as host_validation.h is.
#pragma once
#include "apbv_cache.h"
#include "host_validation.h"

namespace apbv {

constexpr int64_t kMaxSlots = ((int64_t)1 << 31) - 1;
constexpr int64_t kMaxCachedTokens = (int64_t)1 << 30;      // of one request
constexpr int kCacheBlock = 32;             // elements that share a scale
constexpr int64_t kMaxGroups = (1 << 24) - 1;               // of 256 threads: a launch counts its threads in 32 bits

// Workgroups of a store or load: each takes a head of 2048 / d tokens.
inline int64_t cache_row_groups(int64_t tokens, int hkv, int d) { return (tokens + 2048 / d - 1) / (2048 / d) * hkv; }

inline bool valid_page_size(int p) { return p == 16 || p == 32 || p == 64 || p == 128 || p == 256; }
inline int log2_page(int p) { return p == 16 ? 4 : p == 32 ? 5 : p == 64 ? 6 : p == 128 ? 7 : 8; }

inline apbv_status check_cache(const apbv_cache* c, int hkv, int d) {
  if (c == nullptr) return APBV_ERR_NULL;
  if (hkv < 1 || hkv > 65535) return APBV_ERR_SHAPE;
  if (d != 64 && d != 128) return APBV_ERR_UNSUPPORTED;
  if (!valid_page_size(c->page_size)) return APBV_ERR_UNSUPPORTED;
  if (c->n_pages < 1 || c->n_pages > kMaxSlots / c->page_size) return APBV_ERR_SHAPE;
  if (c->k_codes == nullptr || c->v_codes == nullptr || c->k_scales == nullptr || c->v_scales == nullptr) return APBV_ERR_NULL;
  for (const void* p : {c->k_codes, c->v_codes, c->k_scales, c->v_scales})
    if (!aligned(p, 16)) return APBV_ERR_SHAPE;
  const int64_t rows = (int64_t)hkv * c->page_size;
  if (c->page_stride_codes % 16 || c->page_stride_scales % 16) return APBV_ERR_SHAPE;
  if (c->n_pages > 1 && (c->page_stride_codes < rows * (d / 2) || c->page_stride_scales < rows * (d / kCacheBlock))) return APBV_ERR_SHAPE;
  // (a page's bytes are kept in 32 bits; pages lie within 2^62 bytes of the first)
  if (rows * (d / 2) > ((int64_t)1 << 30) || c->page_stride_codes >= (int64_t)1 << 31 || c->page_stride_scales >= (int64_t)1 << 31) return APBV_ERR_UNSUPPORTED;
  return APBV_OK;
}

// A table of max_blocks entries a request.
inline apbv_status check_table(int n_requests, int page_size, const void* table, int64_t stride, int64_t max_blocks) {
  if (n_requests < 1) return APBV_ERR_SHAPE;
  if (n_requests > APBV_CACHE_MAX_REQUESTS) return APBV_ERR_UNSUPPORTED;
  if (max_blocks < 1 || max_blocks > kMaxCachedTokens / page_size) return APBV_ERR_SHAPE;
  if (table == nullptr) return APBV_ERR_NULL;
  if (!aligned(table, 4)) return APBV_ERR_SHAPE;
  if (n_requests > 1 && stride < max_blocks) return APBV_ERR_SHAPE;
  return APBV_OK;
}

inline apbv_status validate_cache_map(int n_requests, int page_size, int64_t max_blocks, const int32_t* old_lengths,
                                      const int32_t* new_lengths, const int32_t* table, int64_t table_stride, const int32_t* free_pages,
                                      int64_t free_capacity, const int32_t* free_count, int64_t max_new_tokens, const int32_t* lengths_out,
                                      const int32_t* starts_out, const int32_t* slots_out, const int32_t* free_count_out) {
  if (!valid_page_size(page_size)) return APBV_ERR_UNSUPPORTED;
  const apbv_status st = check_table(n_requests, page_size, table, table_stride, max_blocks);
  if (st != APBV_OK) return st;
  if (free_capacity < 0 || free_capacity > kMaxSlots / page_size || max_new_tokens < 0 || max_new_tokens > kMaxTokens) return APBV_ERR_SHAPE;
  if (old_lengths == nullptr || new_lengths == nullptr || free_count == nullptr || lengths_out == nullptr || starts_out == nullptr ||
      free_count_out == nullptr || (free_pages == nullptr && free_capacity > 0) || (slots_out == nullptr && max_new_tokens > 0))
    return APBV_ERR_NULL;
  for (const void* p : {old_lengths, new_lengths, free_pages, free_count, lengths_out, starts_out, slots_out, free_count_out})
    if (!aligned(p, 4)) return APBV_ERR_SHAPE;
  if (lengths_out == new_lengths) return APBV_ERR_SHAPE;
  return APBV_OK;
}

inline apbv_status validate_cache_store(const apbv_cache* cache, int hkv, int d, const apbv_tensor& k, const apbv_tensor& v, const int32_t* slots) {
  apbv_status st = check_cache(cache, hkv, d);
  if (st != APBV_OK) return st;
  if ((st = check_view(k, hkv, d, 1, true)) != APBV_OK) return st;
  if ((st = check_view(v, hkv, d, 1, true)) != APBV_OK) return st;
  if (k.tokens != v.tokens) return APBV_ERR_SHAPE;
  if (k.tokens > 0 && slots == nullptr) return APBV_ERR_NULL;
  if (!aligned(slots, 4)) return APBV_ERR_SHAPE;
  return cache_row_groups(k.tokens, hkv, d) <= kMaxGroups ? APBV_OK : APBV_ERR_UNSUPPORTED;
}

inline apbv_status validate_cache_load(const apbv_cache* cache, int hkv, int d, int64_t tokens, const int32_t* slots, const void* k_out,
                                       const void* v_out) {
  const apbv_status st = check_cache(cache, hkv, d);
  if (st != APBV_OK) return st;
  if (tokens < 0 || tokens > kMaxTokens) return APBV_ERR_SHAPE;
  if (tokens > 0 && (slots == nullptr || k_out == nullptr || v_out == nullptr)) return APBV_ERR_NULL;
  if (!aligned(slots, 4) || !aligned(k_out, 16) || !aligned(v_out, 16)) return APBV_ERR_SHAPE;
  return cache_row_groups(tokens, hkv, d) <= kMaxGroups ? APBV_OK : APBV_ERR_UNSUPPORTED;
}

// The tiles of all (request, KV head, row tile) are numbered in 32 bits; the host knows the most there can be.
constexpr int kCacheKeyTile = 64;
inline bool cache_axis_fits(int64_t n_requests, int64_t n_rows, int hq, int hkv, int64_t max_len) {
  const int64_t row_tiles = (n_rows * (hq / hkv) / 16 + n_requests) * hkv;               // below 2^37 (2^24 tokens of 65535 query heads)
  return row_tiles <= (int64_t)0x7fff0000 / ((max_len + kCacheKeyTile - 1) / kCacheKeyTile);
}

inline apbv_status validate_cache_attention(const apbv_cache* cache, int n_requests, int hq, int hkv, int d, const apbv_tensor& q,
                                            const int32_t* table, int64_t table_stride, int64_t max_blocks, const int32_t* lengths,
                                            const int32_t* q_starts, int64_t max_q, float softmax_scale, const void* out,
                                            const float* lse_out) {
  apbv_status st = check_heads(1, hq, hkv, d);
  if (st != APBV_OK) return st;
  if ((st = check_cache(cache, hkv, d)) != APBV_OK) return st;
  if ((st = check_table(n_requests, cache->page_size, table, table_stride, max_blocks)) != APBV_OK) return st;
  if ((st = check_view(q, hq, d, 1, true)) != APBV_OK) return st;
  if (!cache_axis_fits(n_requests, q.tokens, hq, hkv, max_blocks * cache->page_size)) return APBV_ERR_UNSUPPORTED;
  if (lengths == nullptr) return APBV_ERR_NULL;
  if (!aligned(lengths, 4) || !aligned(q_starts, 4)) return APBV_ERR_SHAPE;
  if (q_starts == nullptr && q.tokens % n_requests) return APBV_ERR_SHAPE;
  if (q.tokens * (hq / hkv) > (int64_t)1 << 30) return APBV_ERR_UNSUPPORTED;      // rows of a KV head: kept in 32 bits
  // workgroups of the launches: one for every (request, KV head), or for four (row, head) of the output
  if ((int64_t)n_requests * hkv > kMaxGroups || q.tokens * hq > 4 * kMaxGroups) return APBV_ERR_UNSUPPORTED;
  if (max_q < 0 || max_q > kMaxTokens) return APBV_ERR_SHAPE;
  if (!(softmax_scale > 0.0f) || !std::isfinite(softmax_scale)) return APBV_ERR_SHAPE;
  if (q.tokens > 0 && out == nullptr) return APBV_ERR_NULL;
  if (!aligned(out, 16) || !aligned(lse_out, 4)) return APBV_ERR_SHAPE;
  return APBV_OK;
}

// ---- how an attention call is cut.  The keys of all requests, KV heads and row tiles are one axis of 64-key tiles (the
// device knows its length, the host does not), dealt to `workgroups` equal shares; a share that begins or ends inside a
// (request, head, row tile) leaves a part of it in the workspace: at most two a workgroup.
constexpr int kCacheBlockRows = 128;        // rows of a row tile of query blocks and chunks
constexpr int kCacheWaves = 4;              // waves of a workgroup
struct CachePlan {
  int rows;          // query rows (query x head of the KV group) of a row tile
  int workgroups;
  int short_tiles;   // where shares would be shorter than this, half as many workgroups share the axis
  int least_tiles;   // a share is not shorter than this
  int share_step;    // a share of more than three times this is a multiple of it
  int row_tiles;     // of a request
  bool whole;        // a workgroup for every (request, KV head, row tile)
  int join_waves;    // waves that join the parts of a row: 1 or 4
};
// Two workgroups fit a compute unit.  Where each would get but a few tiles, one is given the double: every share costs its start
// and end and two parts to join (us, 512 / 256 workgroups: one query over 133120 keys, 16 / 2 heads of 128, 8.1 tiles each of
// 512, 19.9 / 17.6; 256 requests of 65 to 4096 keys, 8 / 2 heads of 64, 16 tiles, 21.9 / 23.7; 64 queries over 16512 keys, 4 tiles,
// 35.7 / 32.8; 64 requests of 512 to 32768 keys, 28 / 4 heads of 128, 56 tiles, 49.4 / 50.1).  Shares of one tile rather than two
// cost the join more than they save (64 queries over 2000 keys 21.9 / 18.3).
//
// Few row tiles of 16 rows have hardly an end inside a workgroup, which a second one would fill with work: one is enough at
// head_dim 128, however long (one query, 16 / 2 heads, 512 / 256 workgroups: 262144 keys 25.0 / 22.1, 524288 34.5 / 31.8; with pages
// of 16 tokens 500000 keys 35.0 / 33.5; 64 / 8 heads, 400000 keys 88.7 / 90.4), and below 12 tiles each at 64 (8 / 2 heads: 133120
// keys, 8 tiles each of 512, 14.4 / 12.9; 500000, 31 tiles, 22.5 / 24.4).  Their waves take equally many tiles where that makes a
// share not much longer: the longest part is as long as before, and there are fewer to join (133120 keys, 17 or 20 tiles a share:
// 18.3 / 17.8; of 5 or 8, 40000 keys: 12.5 / 13.4; 64 requests, 57 or 60: 51.7 / 52.5).
//
// Where the table holds but a few tiles a request, a workgroup takes a whole (request, KV head, row tile): no axis to plan, no
// parts, no second launch.  It is alone with its keys, so a table of longer requests is cut as above unless there are many to
// even them out (us, cut / whole, one query each): 1 request of 700 keys, 16 / 2 heads of 128 9.6 / 7.8, 1280 9.4 / 10.3; 64 of 65 to
// 2048 13.0 / 13.7, 128 17.0 / 14.2; 64 of 8 / 2 heads of 64 11.7 / 10.6, 256 17.6 / 13.1; 512 of up to 4096, 16 / 2 heads of 128 42.5 /
// 45.9; 4096 of 8 / 2 heads of 64 198 / 154; 2048 of up to 8192 146 / 136, 4096 of up to 16384 414 / 452; 256 of 300 to 2048 keys, 5 to
// 8 queries 35.7 / 17.4.
//
// The second launch takes a wave per row of the output, or four where the rows are few and have many parts (us for the call, one
// wave / four: one query over 133120 keys, 16 / 2 heads of 128 22.3 / 17.9, 17 queries over 10000, 28 / 4 heads 24.4 / 23.0, 64
// queries over 16512, 16 / 2 heads 32.8 / 32.4; 4 x 64 queries, 8 / 2 heads of 64 19.6 / 23.0, 64 requests of one query, 28 / 4
// heads 49.6 / 52.2).
inline CachePlan choose_cache_plan(int n_requests, int hq, int hkv, int d, int64_t n_rows, int64_t max_q, int64_t max_len) {
  const int64_t rows = (max_q < n_rows ? max_q : n_rows) * (hq / hkv);      // at most 2^30
  CachePlan p;
  p.rows = rows <= 16 ? 16 : rows <= 32 ? 32 : kCacheBlockRows;
  p.workgroups = 512;
  p.row_tiles = rows <= p.rows ? 1 : (int)((rows + p.rows - 1) / p.rows);
  const bool few = p.rows == 16 && (int64_t)n_requests * hkv <= 8;
  p.short_tiles = few && d == 128 ? 1 << 30 : few || d == 128 ? 12 : 6;
  p.least_tiles = 2;
  p.share_step = few ? kCacheWaves : 1;
  const int64_t longest = (max_len + kCacheKeyTile - 1) / kCacheKeyTile;
  p.whole = p.rows != kCacheBlockRows && (longest <= 16 || (int64_t)n_requests * hkv * p.row_tiles >= (longest <= 32 ? 4 : 64) * longest);
  const int64_t parts = p.workgroups / ((int64_t)n_requests * hkv * p.row_tiles) + 1;      // of a row, if the requests are alike
  p.join_waves = parts > 8 && n_rows * hq <= 1024 ? 4 : 1;
  return p;
}
// Tiles of a workgroup's share of an axis of `total` tiles.
constexpr uint32_t cache_share(uint32_t total, uint32_t workgroups, uint32_t short_tiles, uint32_t least_tiles, uint32_t share_step) {
  uint32_t q = (total + workgroups - 1) / workgroups;
  if (q < short_tiles) q = (total + workgroups / 2 - 1) / (workgroups / 2);
  q = q > least_tiles ? q : least_tiles;
  if (q > 3 * share_step) q = (q + share_step - 1) / share_step * share_step;
  return q;
}
// An axis that is cut among workgroups which have other work, too (shared_validation.h).  Every die has an equal stretch of `stretch`
// tiles, which its workgroups take in shares of `share`, the first `full` of them, and of `rest`, the others; `used` of them are
// needed.  Shares are numbered die after die.
struct AxisCut {
  uint32_t stretch, share, rest, full, used;
};
constexpr uint32_t kCutDies = 8;
constexpr int kCutWords = 12;                 // a CutWord: left in front of where the requests begin
constexpr uint32_t cut_begin(const AxisCut& c, uint32_t die, uint32_t x) {
  return die * c.stretch + (x <= c.full ? x * c.share : c.full * c.share + (x - c.full) * c.rest);
}
constexpr uint32_t cut_end(const AxisCut& c, uint32_t die, uint32_t x) {
  const uint32_t e = cut_begin(c, die, x) + (x < c.full ? c.share : c.rest), top = (die + 1) * c.stretch;
  return e < top ? e : top;
}
// The number of the share that holds tile `pos`, by reciprocals: (a + 1/2) / b is no nearer to a whole number than 1 / (2 b), and a double's
// error is smaller (as query_of has it).
struct CutWord {
  AxisCut cut;
  uint32_t pad;
  double per_stretch, per_share, per_rest;
};
constexpr uint32_t cut_divide(uint32_t a, double per_b) { return (uint32_t)(((double)a + 0.5) * per_b); }
constexpr CutWord cut_word(const AxisCut& c) { return CutWord{c, 0, 1.0 / c.stretch, 1.0 / c.share, 1.0 / c.rest}; }
constexpr uint32_t cut_share_of(const CutWord& w, uint32_t pos) {
  const AxisCut& c = w.cut;
  const uint32_t die = cut_divide(pos, w.per_stretch), at = pos - die * c.stretch, in_full = c.full * c.share;
  return die * c.used + (at < in_full ? cut_divide(at, w.per_share) : c.full + cut_divide(at - in_full, w.per_rest));
}
inline size_t cache_part_bytes(int rows, int d) { return (size_t)rows * (size_t)(d + 3) * sizeof(float); }
inline size_t cache_parts_bytes(const CachePlan& p, int d) {
  const size_t heads = p.rows != 32 ? 0 : (size_t)kCacheWaves * p.rows * d * sizeof(float);      // pieces that have no room in LDS
  return align256((size_t)p.workgroups * (2 * cache_part_bytes(p.rows, d) + heads));
}
inline size_t cache_attention_workspace_bytes(int n_requests, int64_t n_rows, int hq, int hkv, int d, int64_t max_q) {
  if (check_heads(1, hq, hkv, d) != APBV_OK || n_requests < 1 || n_requests > APBV_CACHE_MAX_REQUESTS || n_rows < 0 || n_rows > kMaxTokens ||
      n_rows * (hq / hkv) > (int64_t)1 << 30 || max_q < 0 || max_q > kMaxTokens)
    return 0;
  const CachePlan p = choose_cache_plan(n_requests, hq, hkv, d, n_rows, max_q, 0);
  return cache_parts_bytes(p, d) + align256(((size_t)n_requests + 1) * sizeof(uint32_t));
}

}  // namespace apbv
