// C ABI of the attention behind shared prefixes (include/apbv_shared.h): argument validation on the host, then dispatch.
#include "shared.h"

using namespace apbv;

extern "C" {

size_t apbv_cache_shared_attention_workspace_bytes(int n_groups, int n_requests, int64_t n_rows, int n_q_heads, int n_kv_heads, int head_dim,
                                                   int64_t max_q) {
  return shared_attention_workspace_bytes(n_groups, n_requests, n_rows, n_q_heads, n_kv_heads, head_dim, max_q);
}

apbv_status apbv_cache_shared_attention(const apbv_cache* cache, int n_groups, int n_requests, int n_q_heads, int n_kv_heads, int head_dim,
                                        apbv_tensor q, const int32_t* prefix_table, int64_t prefix_table_stride, int64_t max_prefix_blocks,
                                        const int32_t* prefix_lengths, const int32_t* group_starts, const int32_t* block_table,
                                        int64_t table_stride, int64_t max_blocks, const int32_t* lengths, const int32_t* q_starts,
                                        int64_t max_q, int causal, float softmax_scale, void* out, float* lse_out, void* workspace,
                                        size_t workspace_bytes, void* hip_stream) {
  const apbv_status st = validate_shared_attention(cache, n_groups, n_requests, n_q_heads, n_kv_heads, head_dim, q, prefix_table,
                                                   prefix_table_stride, max_prefix_blocks, prefix_lengths, group_starts, block_table,
                                                   table_stride, max_blocks, lengths, q_starts, max_q, softmax_scale, out, lse_out);
  if (st != APBV_OK || q.tokens == 0) return st;
  const SharedPlan plan = choose_shared_plan(n_groups, n_requests, n_q_heads, n_kv_heads, head_dim, q.tokens, max_q,
                                             max_prefix_blocks * cache->page_size, max_blocks * cache->page_size,
                                             group_starts == nullptr && q_starts == nullptr);
  const SharedSpace space = shared_space(plan, n_groups, n_requests, q.tokens, n_q_heads, head_dim);
  if (workspace == nullptr || !aligned(workspace, 256) || workspace_bytes < space.bytes) return APBV_ERR_WORKSPACE;
  char* const ws = static_cast<char*>(workspace);
  CacheAttnParams p;
  p.cache = to_view(*cache);
  p.q = to_view(q);
  p.starts = q_starts;
  p.out = static_cast<bf16_t*>(out);
  p.lse = lse_out;
  p.n_rows = (int)q.tokens;
  p.each = (int)(q.tokens / n_requests);
  p.hq = n_q_heads;
  p.hkv = n_kv_heads;
  p.group = n_q_heads / n_kv_heads;
  p.members = group_starts;
  p.n_members = n_requests;
  p.members_each = n_requests / n_groups;
  p.scale_log2 = softmax_scale * 1.4426950408889634f;
  p.per_group = 1.0 / p.group;
  auto cut = [&](CacheAttnParams& x, const CachePlan& by) {
    x.workgroups = by.workgroups;
    x.short_tiles = by.short_tiles;
    x.least_tiles = by.least_tiles;
    x.share_step = by.share_step;
    x.row_tiles = by.row_tiles;
  };
  SharedParams s;
  s.prefix = s.own = p;
  cut(s.prefix, plan.prefix);
  s.prefix.table = prefix_table;
  s.prefix.table_stride = prefix_table_stride;
  s.prefix.lengths = prefix_lengths;
  s.prefix.max_len = (int)(max_prefix_blocks * cache->page_size);
  s.prefix.n_requests = n_groups;
  s.prefix.causal = 0;
  s.prefix.parts = reinterpret_cast<float*>(ws);
  s.prefix.kept = reinterpret_cast<float*>(ws + space.prefix_kept);
  s.prefix.begins = reinterpret_cast<uint32_t*>(ws + space.prefix_begins);
  cut(s.own, plan.own);
  s.own.table = block_table;
  s.own.table_stride = table_stride;
  s.own.lengths = lengths;
  s.own.max_len = (int)(max_blocks * cache->page_size);
  s.own.n_requests = n_requests;
  s.own.members = nullptr;
  s.own.members_each = 0;
  s.own.causal = causal != 0;
  s.own.parts = reinterpret_cast<float*>(ws + space.own_parts);
  s.own.kept = reinterpret_cast<float*>(ws + space.own_kept);
  s.own.begins = reinterpret_cast<uint32_t*>(ws + space.own_begins);
  return launch_shared_attention(s, plan, head_dim, static_cast<hipStream_t>(hip_stream));
}

}  // extern "C"
