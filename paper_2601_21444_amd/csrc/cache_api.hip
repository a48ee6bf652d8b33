// C ABI of the cache (include/apbv_cache.h): argument validation on the host, then dispatch to the kernel launchers.
#include "cache.h"

using namespace apbv;

extern "C" {

apbv_status apbv_cache_map(int n_requests, int page_size, int64_t max_blocks, const int32_t* old_lengths, const int32_t* new_lengths,
                           int32_t* block_table, int64_t table_stride, int32_t* free_pages, int64_t free_capacity,
                           const int32_t* free_count, int64_t max_new_tokens, int32_t* lengths_out, int32_t* starts_out,
                           int32_t* slots_out, int32_t* free_count_out, void* hip_stream) {
  const apbv_status st = validate_cache_map(n_requests, page_size, max_blocks, old_lengths, new_lengths, block_table, table_stride, free_pages,
                                            free_capacity, free_count, max_new_tokens, lengths_out, starts_out, slots_out, free_count_out);
  if (st != APBV_OK) return st;
  CacheMapParams p;
  p.old_lengths = old_lengths;
  p.new_lengths = new_lengths;
  p.free_count = free_count;
  p.table = block_table;
  p.free_pages = free_pages;
  p.lengths_out = lengths_out;
  p.starts_out = starts_out;
  p.slots_out = slots_out;
  p.free_count_out = free_count_out;
  p.table_stride = table_stride;
  p.n_requests = n_requests;
  p.page_log2 = log2_page(page_size);
  p.free_capacity = (int)free_capacity;
  p.max_new = (int)max_new_tokens;
  p.cap = (int)(max_blocks * page_size);
  return launch_cache_map(p, static_cast<hipStream_t>(hip_stream));
}

apbv_status apbv_cache_store(const apbv_cache* cache, int n_kv_heads, int head_dim, apbv_tensor k, apbv_tensor v, const int32_t* slots,
                             void* hip_stream) {
  const apbv_status st = validate_cache_store(cache, n_kv_heads, head_dim, k, v, slots);
  if (st != APBV_OK || k.tokens == 0) return st;
  CacheRowsParams p = {};
  p.cache = to_view(*cache);
  p.k = to_view(k);
  p.v = to_view(v);
  p.slots = slots;
  p.tokens = k.tokens;
  p.hkv = n_kv_heads;
  return launch_cache_store(p, head_dim, static_cast<hipStream_t>(hip_stream));
}

apbv_status apbv_cache_load(const apbv_cache* cache, int n_kv_heads, int head_dim, int64_t tokens, const int32_t* slots, void* k_out,
                            void* v_out, void* hip_stream) {
  const apbv_status st = validate_cache_load(cache, n_kv_heads, head_dim, tokens, slots, k_out, v_out);
  if (st != APBV_OK || tokens == 0) return st;
  CacheRowsParams p = {};
  p.cache = to_view(*cache);
  p.k_out = static_cast<bf16_t*>(k_out);
  p.v_out = static_cast<bf16_t*>(v_out);
  p.slots = slots;
  p.tokens = tokens;
  p.hkv = n_kv_heads;
  return launch_cache_load(p, head_dim, static_cast<hipStream_t>(hip_stream));
}

size_t apbv_cache_attention_workspace_bytes(int n_requests, int64_t n_rows, int n_q_heads, int n_kv_heads, int head_dim, int64_t max_q) {
  return cache_attention_workspace_bytes(n_requests, n_rows, n_q_heads, n_kv_heads, head_dim, max_q);
}

apbv_status apbv_cache_attention(const apbv_cache* cache, int n_requests, int n_q_heads, int n_kv_heads, int head_dim, apbv_tensor q,
                                 const int32_t* block_table, int64_t table_stride, int64_t max_blocks, const int32_t* lengths,
                                 const int32_t* q_starts, int64_t max_q, int causal, float softmax_scale, void* out, float* lse_out,
                                 void* workspace, size_t workspace_bytes, void* hip_stream) {
  const apbv_status st = validate_cache_attention(cache, n_requests, n_q_heads, n_kv_heads, head_dim, q, block_table, table_stride, max_blocks,
                                                  lengths, q_starts, max_q, softmax_scale, out, lse_out);
  if (st != APBV_OK || q.tokens == 0) return st;
  const CachePlan plan = choose_cache_plan(n_requests, n_q_heads, n_kv_heads, head_dim, q.tokens, max_q, max_blocks * cache->page_size);
  const size_t need = cache_attention_workspace_bytes(n_requests, q.tokens, n_q_heads, n_kv_heads, head_dim, max_q);
  if (workspace == nullptr || !aligned(workspace, 256) || workspace_bytes < need) return APBV_ERR_WORKSPACE;
  CacheAttnParams p;
  p.cache = to_view(*cache);
  p.q = to_view(q);
  p.table = block_table;
  p.lengths = lengths;
  p.starts = q_starts;
  p.table_stride = table_stride;
  p.out = static_cast<bf16_t*>(out);
  p.lse = lse_out;
  p.parts = static_cast<float*>(workspace);
  p.begins = reinterpret_cast<uint32_t*>(static_cast<char*>(workspace) + cache_parts_bytes(plan, head_dim));
  p.n_requests = n_requests;
  p.n_rows = (int)q.tokens;
  p.each = (int)(q.tokens / n_requests);
  p.max_len = (int)(max_blocks * cache->page_size);
  p.hq = n_q_heads;
  p.hkv = n_kv_heads;
  p.group = n_q_heads / n_kv_heads;
  p.causal = causal != 0;
  p.workgroups = plan.workgroups;
  p.short_tiles = plan.short_tiles;
  p.least_tiles = plan.least_tiles;
  p.share_step = plan.share_step;
  p.row_tiles = plan.row_tiles;
  p.scale_log2 = softmax_scale * 1.4426950408889634f;
  p.per_group = 1.0 / p.group;
  return launch_cache_attention(p, plan, head_dim, static_cast<hipStream_t>(hip_stream));
}

}  // extern "C"
