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
struct SharedPlan {
  CachePlan prefix, own;
  int workgroups;
  int join_waves;            // waves that join the parts of a row: 1 or 4
};
inline SharedPlan choose_shared_plan(int n_groups, int n_requests, int hq, int hkv, int d, int64_t n_rows, int64_t max_q) {
  SharedPlan p;
  p.workgroups = 512;
  p.prefix = choose_cache_plan(n_groups, hq, hkv, d, n_rows, (n_rows + n_groups - 1) / n_groups, 0);
  p.own = choose_cache_plan(n_requests, hq, hkv, d, n_rows, max_q, 0);
  // (row tiles of 32 own rows are taken in two of 16, and no row tile of own rows is higher than those of the prefix)
  if (p.own.rows == 32 || p.prefix.rows != kCacheBlockRows) {
    const int64_t rows = (max_q < n_rows ? max_q : n_rows) * (hq / hkv);
    p.own.rows = 16;
    p.own.row_tiles = (int)((rows + 15) / 16);
  }
  p.prefix.workgroups = p.own.workgroups = p.workgroups;
  // a row has as many parts over its prefix as workgroups share it, if the groups are alike
  const int64_t parts = p.workgroups / ((int64_t)n_groups * hkv * p.prefix.row_tiles) + 1;
  p.join_waves = parts > 8 && n_rows * hq <= 2048 ? 4 : 1;
  return p;
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
  s.own_begins = s.prefix_begins + align256(((size_t)n_groups + 1) * sizeof(uint32_t));
  s.bytes = s.own_begins + align256(((size_t)n_requests + 1) * sizeof(uint32_t));
  return s;
}
inline size_t shared_attention_workspace_bytes(int n_groups, int n_requests, int64_t n_rows, int hq, int hkv, int d, int64_t max_q) {
  if (n_groups < 1 || n_groups > n_requests || n_rows * (int64_t)hq > 4 * kMaxGroups ||
      cache_attention_workspace_bytes(n_requests, n_rows, hq, hkv, d, max_q) == 0)
    return 0;
  return shared_space(choose_shared_plan(n_groups, n_requests, hq, hkv, d, n_rows, max_q), n_groups, n_requests, n_rows, hq, d).bytes;
}

}  // namespace apbv
