// Host-side argument validation and planning of include/apbv_shared.h; plain C++ as host_validation.h is.
#pragma once
#include "apbv_shared.h"
#include "cache_validation.h"

namespace apbv {

inline apbv_status validate_shared_attention(const apbv_cache* cache, int n_groups, int n_requests, int hq, int hkv, int d, const apbv_tensor& q,
                                             const int32_t* prefix_table, int64_t prefix_stride, int64_t max_prefix_blocks,
                                             const int32_t* prefix_lengths, const int32_t* group_starts, const int32_t* table,
                                             int64_t table_stride, int64_t max_blocks, const int32_t* lengths, const int32_t* q_starts,
                                             int64_t max_q, float softmax_scale, const void* out, const float* lse_out) {
  apbv_status st = validate_cache_attention(cache, n_requests, hq, hkv, d, q, table, table_stride, max_blocks, lengths, q_starts, max_q,
                                            softmax_scale, out, lse_out);
  if (st != APBV_OK) return st;
  if (n_groups < 1 || n_groups > n_requests) return APBV_ERR_SHAPE;
  if ((st = check_table(n_groups, cache->page_size, prefix_table, prefix_stride, max_prefix_blocks)) != APBV_OK) return st;
  if (!cache_axis_fits(n_groups, q.tokens, hq, hkv, max_prefix_blocks * cache->page_size)) return APBV_ERR_UNSUPPORTED;
  if (prefix_lengths == nullptr) return APBV_ERR_NULL;
  if (!aligned(prefix_lengths, 4) || !aligned(group_starts, 4)) return APBV_ERR_SHAPE;
  if (group_starts == nullptr && n_requests % n_groups) return APBV_ERR_SHAPE;
  return APBV_OK;
}

// How a call is cut: two axes of tiles as in cache_validation.h, one of the groups over their prefixes and one of the requests over
// their own keys, of both of which every workgroup takes a share.
constexpr int kSharedWorkgroups = 512;
struct SharedPlan {
  CachePlan prefix, own;
  int join_waves;            // waves that join the parts of a row: 1 or 4
  bool whole;                // a workgroup for every (group, KV head, 16 rows), with all their keys: prefix.row_tiles of a group
};
//
// Where the tables hold but a few tiles, a workgroup takes 16 rows and all the keys that they see, without a second launch: a
// microsecond for every four tiles, where a cut call has its second launch, and whole row tiles of 128 rows for few keys.  How many tiles
// are few depends on how many such workgroups there are to even them out (us, cut / whole; tiles of the prefix and of the own keys that
// a row tile sees: 2 requests, 2 / 1 heads of 64, 13 11.2 / 7.5, 24 11.9 / 9.3, 34 11.5 / 11.0, 48 11.9 / 13.0; 8 of 8 / 8 of 128, 12 12.0 /
// 9.3, 19 12.4 / 11.7, 24 12.1 / 14.0.  128-row tiles: 32 of 16 / 2 heads of 128, 32 workgroups, 19 17.1 / 10.3, 35 18.1 / 15.1, 56 18.4 /
// 22.3; 128 of 8 / 8, 64 workgroups, 28 22.8 / 17.1, 33 18.9 / 19.3, 49 20.2 / 25.6; 128 of 16 / 2, 128 workgroups, 28 26.3 / 14.5, 56 31.6 / 23.1, 70
// 31.8 / 26.7; 128 of 28 / 4, 224 workgroups, 56 29.9 / 30.1, 70 35.7 / 29.3).  max_prefix and max_len: keys that a row of the tables holds.
inline SharedPlan choose_shared_plan(int n_groups, int n_requests, int hq, int hkv, int d, int64_t n_rows, int64_t max_q, int64_t max_prefix,
                                     int64_t max_len) {
  SharedPlan p;
  p.prefix = choose_cache_plan(n_groups, hq, hkv, d, n_rows, (n_rows + n_groups - 1) / n_groups, 0);
  p.own = choose_cache_plan(n_requests, hq, hkv, d, n_rows, max_q, 0);
  // (row tiles of 32 own rows are taken in two of 16, and no row tile of own rows is higher than those of the prefix)
  if (p.own.rows == 32 || p.prefix.rows != kCacheBlockRows) {
    const int64_t rows = (max_q < n_rows ? max_q : n_rows) * (hq / hkv);
    p.own.rows = 16;
    p.own.row_tiles = (int)((rows + 15) / 16);
  }
  p.prefix.workgroups = p.own.workgroups = kSharedWorkgroups;
  // a row has as many parts over its prefix as workgroups share it, if the groups are alike
  const int64_t parts = kSharedWorkgroups / ((int64_t)n_groups * hkv * p.prefix.row_tiles) + 1;
  p.join_waves = parts > 8 && n_rows * hq <= 2048 ? 4 : 1;
  const int group = hq / hkv;
  const int64_t rows = (n_rows + n_groups - 1) / n_groups * group, row_tiles = (rows + 15) / 16;
  const int64_t per_tile = (int64_t)n_requests * 16 / (n_rows * group) + 1, of_group = (n_requests + n_groups - 1) / n_groups;      // requests
  const int64_t tiles = (max_prefix + kCacheKeyTile - 1) / kCacheKeyTile + (per_tile < of_group ? per_tile : of_group) * ((max_len + kCacheKeyTile - 1) / kCacheKeyTile);
  const int64_t groups16 = n_groups * (int64_t)hkv * row_tiles;
  const int64_t few = p.prefix.rows != kCacheBlockRows ? 22 : (groups16 < 160 ? 24 + groups16 / 4 : 64);
  p.whole = tiles <= few && groups16 + 2 * (int64_t)hkv * row_tiles <= (int64_t)1 << 22;
  if (p.whole) p.prefix.row_tiles = (int)row_tiles;
  return p;
}
// The cut of an axis of `total` tiles.  `busy` workgroups of each die, the last ones, have work of the other axis that costs as much as
// `cost` tiles of this one, and take so many fewer.  Where shares would be shorter than short_tiles, half of the workgroups take part.
constexpr AxisCut shared_cut(uint32_t total, uint32_t workgroups, uint32_t short_tiles, uint32_t least_tiles, uint32_t busy, uint32_t cost) {
  const uint32_t w = workgroups / kCutDies;
  AxisCut c = {0, 0, 0, 0, 0};
  c.stretch = (total + kCutDies - 1) / kCutDies;
  c.stretch = c.stretch > least_tiles ? c.stretch : least_tiles;
  busy = busy < w ? busy : w;
  const uint32_t even = (c.stretch + w - 1) / w;
  if (even < short_tiles || busy == 0 || busy == w || cost == 0) {      // (all alike)
    const uint32_t of = even < short_tiles ? w / 2 : w;
    c.share = (c.stretch + of - 1) / of;
    c.share = c.share > least_tiles ? c.share : least_tiles;
    c.rest = c.share;
    c.full = w;
  } else {
    c.full = w - busy;
    c.share = (uint32_t)((c.stretch + (uint64_t)busy * cost + w - 1) / w);
    if (c.share < cost + least_tiles) {                    // nothing is left for those
      c.share = (c.stretch + c.full - 1) / c.full;
      c.rest = c.share;
    } else {
      c.rest = c.share - cost;
    }
  }
  const uint32_t in_full = c.full * c.share;
  c.used = c.stretch <= in_full ? (c.stretch + c.share - 1) / c.share : c.full + (c.stretch - in_full + c.rest - 1) / c.rest;
  return c;
}

// Workspace: parts of the prefixes' axis, parts of the other, rows kept whole of either, and where both begin.
struct SharedSpace {
  size_t own_parts, prefix_kept, own_kept, prefix_begins, own_begins, bytes;
};
inline SharedSpace shared_space(const SharedPlan& p, int n_groups, int n_requests, int64_t n_rows, int hq, int d) {
  SharedSpace s;
  const size_t kept = align256((size_t)n_rows * (size_t)hq * (size_t)(d + 3) * sizeof(float));
  s.own_parts = cache_parts_bytes(p.prefix, d);
  s.prefix_kept = s.own_parts + cache_parts_bytes(p.own, d);
  s.own_kept = s.prefix_kept + kept;
  s.prefix_begins = s.own_kept + kept;
  s.own_begins = s.prefix_begins + align256(((size_t)n_groups + kCutWords) * sizeof(uint32_t));
  s.bytes = s.own_begins + align256(((size_t)n_requests + kCutWords) * sizeof(uint32_t));
  return s;
}
inline size_t shared_attention_workspace_bytes(int n_groups, int n_requests, int64_t n_rows, int hq, int hkv, int d, int64_t max_q) {
  if (n_groups < 1 || n_groups > n_requests || n_rows * (int64_t)hq > 4 * kMaxGroups ||
      cache_attention_workspace_bytes(n_requests, n_rows, hq, hkv, d, max_q) == 0)
    return 0;
  return shared_space(choose_shared_plan(n_groups, n_requests, hq, hkv, d, n_rows > 0 ? n_rows : 1, max_q, 0, 0), n_groups, n_requests, n_rows, hq, d).bytes;
}

}  // namespace apbv
