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
  size_t prefix_parts, own_parts;      // bytes of the workspace, whatever the tables hold
  int join_waves;            // waves that join the parts of a row: 1 or 4
  bool whole;                // a workgroup for every (group, KV head, 16 rows), with all their keys: prefix.row_tiles of a group where all are alike
  int short_waves;           // waves of such a workgroup
  int64_t slots;             // such workgroups for every KV head
};

// Where the host does not know how many rows each group has, its row tiles of 16 are found by slots: those of the e-th of all that may have
// rows (the groups, and where they are listed the requests in front of them and behind) begin at this one, `query` being its first query.  It
// has at most one slot more than row tiles, as r rows behind a have ceil(r / 16) <= (a + r) / 16 - a / 16 + 1; one without rows need not have any.
constexpr int first_slot(int query, int group, int e) { return (int)((int64_t)query * group / 16) + (e < query ? e : query); }

// Row tiles of 16 rows over the prefixes, though the rows would fill some of 32 or 128: a wave works on one by itself, from its start to
// its part in 2 us and a little more for every tile; a row tile of 128 takes a workgroup 5 us longer to start and to end, but a fourth
// of the time per row where it is full.  tiles_16, tiles: key tiles of the prefixes that the tables have room for, times row tiles.
//
// us, row tiles of 128 / of 16 (tiles_16, tiles): 21 requests of 16 / 2 heads of 128 behind 2440 keys 20.6 / 15.4 (858, 156), 8 behind
// 14128 22.3 / 16.8 (1768, 442), 80 behind 4 prefixes of 2743 29.3 / 21.1 (3440, 688), 37 behind 5 of 14265 39.7 / 32.5 (8920, 2230), 16
// behind 34286 28.7 / 30.3 (8576, 1072), 11 behind 67889 28.6 / 31.6 (12732, 2122), 27 behind 92268 46.6 / 55.9 (40376, 5768); 43 of 28 /
// 4 heads behind 8 of 21535, 37 rows, 56.8 / 44.4 (32352, 10784), 213 behind 18062 112 / 145 (106408, 13584).  Heads of 64: 91 of 2 / 1
// behind 3 of 5753 16.1 / 14.0 (1080, 270), 3 x 49 questions behind 16512 16.0 / 14.2 (2580, 516); 3 x 41 of 8 / 2 behind 10556 18.4 / 20.2
// (5280, 660), 215 behind 68601 65.7 / 86.6 (115776, 15008).
// Of 32 / of 16: 17 requests of 8 / 8 heads of 128 behind 3598 18.2 / 14.1 (tiles_16 912), 88 behind 4 of 4933 25.8 / 20.3 (4992), 74
// behind 3 of 20066 43.7 / 40.3 (15072), 4 of 28 / 4 behind 160000 39.0 / 41.5 (20000); 64: 6 of 8 / 2 behind 2293 12.8 / 11.9 (144), 96 of 2 / 1
// behind 8 of 19798 19.3 / 18.2 (4960), 48 of 8 / 2 behind 7 of 1500 to 16384 18.0 / 19.3 (7196).
// A line between these points, too; of those listed it takes the slower height for 16 requests behind 34286 keys (30.3 for 28.7) and 11 behind 67889
// (31.6 for 28.6).
inline bool low_row_tiles(int d, bool high, int64_t tiles_16, int64_t tiles) {
  if (!high) return tiles_16 <= (d == 128 ? 16000 : 5000);
  return tiles_16 <= (d == 128 ? 6000 + tiles * 7 / 2 : 1500 + tiles * 3);
}

// How many workgroups share a row over one axis, if all of its row tiles have as many key tiles as the tables have room for.  A row is
// joined by four waves where it has many parts and there are not many rows (us, one wave / four; parts, rows x query heads: 4 requests of 2 / 1
// heads of 64 behind 89171 keys 22.1 / 14.7 (256, 8), 2 of 28 / 4 of 128 behind 10897 17.5 / 14.1 (88, 56), 14 of 16 / 2 behind 78298 38.7 / 32.3
// (257, 224), 18 behind 13101 21.3 / 20.7 (16, 288), 75 behind 15930 38.2 / 37.6 (27, 1200); 70 of 8 / 2 of 64 behind 3527 14.5 / 15.4 (9, 560),
// 51 of 16 / 2 of 128 behind 4 of 1211 16.3 / 17.8 (8, 816), 70 of 28 / 4 behind 7 of 1632 22.9 / 27.4 (5, 1960), 235 of 8 / 2 of 64 behind 6037 26.2 /
// 30.0 (18, 1880)).
inline int64_t parts_of_a_row(const CachePlan& p, int64_t units, int64_t tiles) {
  const int64_t total = units * p.row_tiles * tiles;
  int64_t share = (total + kSharedWorkgroups - 1) / kSharedWorkgroups;
  if (share < p.short_tiles) share = (total + kSharedWorkgroups / 2 - 1) / (kSharedWorkgroups / 2);
  if (share < p.least_tiles) share = p.least_tiles;
  return tiles / share + 1;
}

// Where the tables hold but a few tiles, a workgroup takes 16 rows and all the keys that they see, without a second launch: 5 us and
// 0.25 for every tile, where a cut call takes 12 and more.  How many tiles are few depends on how many such workgroups there are to even them
// out (us, cut / whole; number of row tiles of 16, tiles of the prefix and of the own keys that one sees).  Heads of 64: 11 requests of 8 / 2, 6, 15
// 11.9 / 7.7; 4, 2, 22 11.7 / 9.5; 8, 4, 48 12.3 / 13.5; 10 x 22 questions, 110, 29 17.6 / 11.8; 114 requests of 2 / 1, 15, 53 14.6 / 15.6.  Heads of 128:
// 7 of 8 / 8, 8, 33 13.0 / 15.1; 60 behind 7 prefixes, 56, 41 16.3 / 17.7; 191, 96, 69 27.0 / 27.2; 154 of 16 / 2, 154, 54 25.1 / 19.0; 3 x 54
// questions, 162, 38 24.4 / 15.2; 256 requests of 28 / 4, 448, 19 35.9 / 15.9; 5 x 46 questions, 404, 34 42.0 / 24.4.
// It is a line between such points, and near it the slower form is taken: 83 requests of 8 / 2 heads of 64, 42, 33 cut, 14.5 / 11.1; 44, 22, 42 cut,
// 13.1 / 12.5; 65 of 28 / 4 of 128, 116, 70 whole, 25.2 / 26.2; 94, 168, 99 cut, 36.4 / 35.8; 10 x 27 questions of 8 / 8, 136, 82 cut, 32.7 / 28.5; 12 x 48
// of 28 / 4, 1008, 87 cut, 86.9 / 82.3.
// Eight waves share the tiles, four where there are more such workgroups than units anyway (us, eight / four waves: 11 requests of 8 / 2 heads
// of 64, 6, 15 7.7 / 9.1; 154 as above 19.5 / 22.6; 196 requests of 28 / 4, 344, 46 38.3 / 35.1; 248, 436, 19 23.1 / 19.2; 12 x 48 questions, 1008,
// 87 93.6 / 82.3).
// Groups whose sizes only the device knows are dealt by slots, so that the largest has as many workgroups as its rows need (us, cut / whole: 8
// requests of 8 / 8 heads of 128 behind 5 prefixes of 333 keys 12.4 / 8.9, 87 of 28 / 4 behind 2 of 300, 57 behind one, 16.7 / 8.3, 33 of 16 / 2
// behind 2 of 600 13.4 / 9.4, 60 of 8 / 8 behind 7 of 300 16.4 / 24.9, 92 behind 4 of 700 23.9 / 32.9; 4096 behind 1000 of 256, 3097 behind one,
// 246 / 149, spread evenly 247 / 142).  The same limit holds for them: over fifty such calls the form taken is as fast as the faster one, but for one
// (83 requests of 8 / 2 heads of 64, as above).
// max_prefix and max_len: keys that a row of the tables holds; even: groups are of equally many requests, and these of equally many rows.
inline SharedPlan choose_shared_plan(int n_groups, int n_requests, int hq, int hkv, int d, int64_t n_rows, int64_t max_q, int64_t max_prefix,
                                     int64_t max_len, bool even) {
  SharedPlan p;
  p.prefix = choose_cache_plan(n_groups, hq, hkv, d, n_rows, (n_rows + n_groups - 1) / n_groups, 0);
  p.own = choose_cache_plan(n_requests, hq, hkv, d, n_rows, max_q, 0);
  const int group = hq / hkv;
  const int64_t rows = (n_rows + n_groups - 1) / n_groups * group, row_tiles = (rows + 15) / 16;
  const bool high = p.prefix.rows == kCacheBlockRows;
  // (row tiles of 32 own rows are taken in two of 16, and no row tile of own rows is higher than those of the prefix)
  auto own_of_16 = [&]() {
    p.own.rows = 16;
    p.own.row_tiles = (int)(((max_q < n_rows ? max_q : n_rows) * group + 15) / 16);
  };
  if (p.own.rows == 32 || !high) own_of_16();
  p.prefix_parts = cache_parts_bytes(p.prefix, d);
  p.own_parts = cache_parts_bytes(p.own, d);
  const int64_t row_tiles_16 = n_groups * (int64_t)hkv * row_tiles, prefix_tiles = (max_prefix + kCacheKeyTile - 1) / kCacheKeyTile;
  if (p.prefix.rows > 16 && low_row_tiles(d, high, row_tiles_16 * prefix_tiles, n_groups * (int64_t)hkv * p.prefix.row_tiles * prefix_tiles)) {
    p.prefix.rows = 16;
    p.prefix.row_tiles = (int)row_tiles;
    own_of_16();
  }
  p.prefix.workgroups = p.own.workgroups = kSharedWorkgroups;
  const int64_t own_tiles = (max_len + kCacheKeyTile - 1) / kCacheKeyTile;
  const int64_t parts = parts_of_a_row(p.prefix, n_groups * (int64_t)hkv, prefix_tiles) + parts_of_a_row(p.own, n_requests * (int64_t)hkv, own_tiles);
  p.join_waves = parts > 15 && n_rows * hq <= 1200 ? 4 : 1;
  const int64_t per_tile = (int64_t)n_requests * 16 / (n_rows * group) + 1, of_group = (n_requests + n_groups - 1) / n_groups;      // requests
  const int64_t tiles = prefix_tiles + (per_tile < of_group ? per_tile : of_group) * own_tiles;
  const int64_t more = row_tiles_16 > 48 ? (row_tiles_16 - 48) * 7 / 10 : 0, some = (d == 128 ? 24 : 32) + more;
  const int64_t few = some < 80 ? some : 80;
  p.slots = even ? n_groups * row_tiles : n_rows * group / 16 + (n_groups + 2 < n_rows ? n_groups + 2 : n_rows);
  p.whole = tiles <= few && row_tiles_16 + 2 * (int64_t)hkv * row_tiles <= (int64_t)1 << 22 && p.slots * hkv <= (int64_t)1 << 22;
  p.short_waves = row_tiles_16 <= 320 ? 8 : 4;
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
  s.own_parts = p.prefix_parts;
  s.prefix_kept = s.own_parts + p.own_parts;
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
  return shared_space(choose_shared_plan(n_groups, n_requests, hq, hkv, d, n_rows > 0 ? n_rows : 1, max_q, 0, 0, true), n_groups, n_requests, n_rows, hq, d).bytes;
}

}  // namespace apbv
