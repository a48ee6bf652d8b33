// Device/host declarations of the cache's kernels (internal; the public ABI is include/apbv_cache.h).
#pragma once
#include "apbv_common.h"
#include "cache_validation.h"

namespace apbv {

// One of the cache's four arrays is base + page * stride + (head * page_size + place in the page) * row bytes.
struct CacheView {
  uint8_t *k_codes, *v_codes, *k_scales, *v_scales;
  int64_t stride_codes, stride_scales;
  int n_pages, page_log2;
};
inline CacheView to_view(const apbv_cache& c) {
  CacheView v;
  v.k_codes = static_cast<uint8_t*>(c.k_codes);
  v.v_codes = static_cast<uint8_t*>(c.v_codes);
  v.k_scales = static_cast<uint8_t*>(c.k_scales);
  v.v_scales = static_cast<uint8_t*>(c.v_scales);
  v.stride_codes = c.page_stride_codes;
  v.stride_scales = c.page_stride_scales;
  v.n_pages = (int)c.n_pages;
  v.page_log2 = log2_page(c.page_size);
  return v;
}

struct CacheMapParams {
  const int32_t *old_lengths, *new_lengths, *free_count;
  int32_t *table, *free_pages, *lengths_out, *starts_out, *slots_out, *free_count_out;
  int64_t table_stride;
  int n_requests, page_log2, free_capacity, max_new;
  int cap;                 // the longest length a row of the table holds
};
apbv_status launch_cache_map(const CacheMapParams& p, hipStream_t stream);

struct CacheRowsParams {
  CacheView cache;
  View k, v;               // store: the rows
  bf16_t *k_out, *v_out;   // load: dense
  const int32_t* slots;
  int64_t tokens;
  int hkv;
};
apbv_status launch_cache_store(const CacheRowsParams& p, int head_dim, hipStream_t stream);
apbv_status launch_cache_load(const CacheRowsParams& p, int head_dim, hipStream_t stream);

struct CacheAttnParams {
  CacheView cache;
  View q;
  const int32_t *table, *lengths, *starts;
  int64_t table_stride;
  bf16_t* out;             // [n_rows, Hq, d]
  float* lse;              // [Hq, n_rows] or nullptr
  // [workgroups][2][rows][d]: O, not divided by the row sum; then [2][3][rows][workgroups]: maxima, sums of the weights as rounded
  // for the product with V, and, where the log-sum-exp is wanted, as they were before; then room for pieces (cache_attention.hip)
  float* parts;
  uint32_t* begins;        // [1 + n_requests], behind them: the length of a share, and where each request begins on the axis (more than 64); of kept
                           // row tiles a CutWord in place of the share, and always
  int n_requests, n_rows, each;     // each: rows of every request where starts is nullptr
  int max_len;             // the longest length a row of the table holds
  int hq, hkv, group, causal;
  int workgroups, short_tiles, least_tiles, share_step;
  int row_tiles;           // of a request, by max_q
  // of requests behind shared prefixes (shared_attention.hip): the axis of the prefixes has groups in place of requests, and row
  // tiles that one workgroup has to itself are kept, too: [n_rows, Hq, d], then [3][n_rows, Hq] as the parts' statistics
  const int32_t* members;  // [groups + 1]: the first request of each, or nullptr: every group has members_each
  float* kept;
  int n_members, members_each;      // requests of all groups, of each (more than 0; 0: no axis of groups)
  float scale_log2;        // softmax_scale * log2(e)
  double per_group;        // 1 / group
};
apbv_status launch_cache_block_attention(const CacheAttnParams& p, int head_dim, hipStream_t stream);      // the parts are left to join
apbv_status launch_cache_attention(const CacheAttnParams& p, const CachePlan& plan, int head_dim, hipStream_t stream);

}  // namespace apbv
