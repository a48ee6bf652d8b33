/*
 * apbv_shared.h -- attention of many requests that share cached prefixes (questions about one video, answers behind one system
 * prompt): the keys of a prefix are read once for all rows of its requests.  The cache is that of apbv_cache.h, whose conventions
 * hold here too.  These calls keep no state and need no set-up before a capture.
 */
#ifndef APBV_SHARED_H_
#define APBV_SHARED_H_

#include "apbv_cache.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Host, pure.  Bytes of workspace apbv_cache_shared_attention needs (0 on invalid arguments); 256-byte aligned.  Its contents need no
 * initialisation and are garbage afterwards.  n_rows = q.tokens, max_q as passed to the call. */
size_t apbv_cache_shared_attention_workspace_bytes(int n_groups, int n_requests, int64_t n_rows, int n_q_heads, int n_kv_heads,
                                                   int head_dim, int64_t max_q);

/*
 * apbv_cache_attention where the requests of a group have a prefix in common: the keys that a row sees are those of its group's prefix,
 * all of them, and behind them those of its request's own that apbv_cache_attention would let it see, under one softmax.
 *   - Group g is the requests group_starts[g] to group_starts[g + 1] - 1; its prefix is prefix_lengths[g] keys, key j at slot
 *     prefix_table[g, j / page_size] * page_size + j % page_size.
 *   - Request b has the rows q_starts[b] to q_starts[b + 1] - 1 and lengths[b] keys of its own, found through block_table.
 *     With n rows, its row i sees the own keys j <= lengths[b] - n + i (causal) or all of them (causal == 0).
 *
 *   prefix_table    [n_groups, max_prefix_blocks] int32, rows prefix_table_stride elements apart
 *   prefix_lengths  [n_groups] int32; outside [0, max_prefix_blocks * page_size] the nearest in it is taken.  0: no prefix
 *   group_starts    [n_groups + 1] int32, not descending, within [0, n_requests] (cut off there); or NULL: every group has
 *                   n_requests / n_groups requests.  A request of no group has its own keys alone
 *   the others      as in apbv_cache_attention; lengths[b] == 0: the prefix alone.  q_starts ascends over the groups, too: the rows
 *                   of a group follow one another
 * Rows of no request are left as they were.  A row that sees no key gets zeros and -inf.  Keys on a page outside [0, n_pages) are taken
 * as not there.  Arithmetic as in apbv_cache_attention; what lies in several parts (the prefix, the own keys) is kept and joined
 * in fp32, so that the result is that of one softmax.  Results of the same call are repeatable.
 * Supported: as apbv_cache_attention, for the groups over their prefixes and for the requests over their own keys; 1 <= n_groups <=
 * n_requests; the workspace holds 8 * (head_dim + 3) bytes for every row and query head.
 */
apbv_status apbv_cache_shared_attention(const apbv_cache* cache, int n_groups, int n_requests, int n_q_heads, int n_kv_heads, int head_dim,
                                        apbv_tensor q, const int32_t* prefix_table, int64_t prefix_table_stride, int64_t max_prefix_blocks,
                                        const int32_t* prefix_lengths, const int32_t* group_starts,
                                        const int32_t* block_table, int64_t table_stride, int64_t max_blocks, const int32_t* lengths,
                                        const int32_t* q_starts, int64_t max_q, int causal, float softmax_scale, void* out, float* lse_out,
                                        void* workspace, size_t workspace_bytes, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* APBV_SHARED_H_ */
