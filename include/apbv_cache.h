/*
 * apbv_cache.h -- a key/value cache held in 4 bits, its block tables, and the attention that reads it.
 *
 * The cache outlives the prefill: requests of different lengths share one pool of pages, decoding appends to it and
 * attends over it.  Per layer: apbv_cache_map once for all layers, then apbv_cache_store and apbv_cache_attention in every
 * layer; apbv_cache_load gives a cached prefix back to the entry points of apbv.h, whose conventions (device pointers, the
 * caller owns every buffer, asynchronous on `hip_stream`, errors found on the host before anything is launched, capture
 * into a HIP graph) hold here too.  These calls keep no state and need no set-up before a capture.  Integers that lie on the
 * device are not seen by the host: what the calls do with values that are out of range is said for each.
 *
 * Format (OCP Microscaling, MXFP4).  A row is head_dim elements of one token and KV head.  Elements are E2M1 (magnitudes 0,
 * 0.5, 1, 1.5, 2, 3, 4, 6 as codes 0 to 7, bit 3 the sign), element 2i in the low half of byte i; every 32 consecutive
 * elements share a scale byte e that stands for 2^(e - 127): 4.25 bits an element.  Written by apbv_cache_store:
 *   m = max |x| of the block;  s = floor(log2 m) - 2, one more if m > 7 * 2^s, kept within [-125, 125];  e = s + 127;
 *   code = x / 2^s rounded to the nearest magnitude, halves to the even code, 6 at most.
 * (A maximum up to 7 * 2^s is held as 6 * 2^s: its error is no larger than a doubled scale would leave it, and the others'
 * is half.)  Every value a stored row stands for is finite and exact in bf16.  An infinity is stored as the largest finite
 * bf16 of its sign would be, a NaN as zero.
 */
#ifndef APBV_CACHE_H_
#define APBV_CACHE_H_

#include "apbv.h"

#ifdef __cplusplus
extern "C" {
#endif

/* A pool of pages of page_size tokens (16, 32, 64, 128 or 256).  Inside a page codes are [n_kv_heads, page_size, head_dim / 2]
 * bytes and scales [n_kv_heads, page_size, head_dim / 32] bytes, both dense; pages are page_stride_* BYTES apart (multiples
 * of 16, below 2^31), so the pages of several layers, or K and V, may be interleaved in one allocation.  Pointers are 16-byte
 * aligned; a page holds at most 2^30 bytes of codes.
 * The slot of a token is page * page_size + its place in the page; n_pages * page_size < 2^31.  Contents need no
 * initialisation: slots that no visible key of a request names are never part of a result. */
typedef struct {
  void* k_codes;
  void* v_codes;
  void* k_scales;
  void* v_scales;
  int64_t n_pages;
  int64_t page_stride_codes;
  int64_t page_stride_scales;
  int32_t page_size;
} apbv_cache;

/*
 * Lengths, block tables and slots of a step: every request grows or shrinks from old_lengths[b] to new_lengths[b] tokens.
 *   - A request that shrinks gives back the pages it no longer needs (its table entries stay as they are): they are appended
 *     to free_pages, request after request, blocks ascending.  Length 0 gives everything back.
 *   - A request that grows takes pages from the end of the list (after those given back), request after request, blocks
 *     ascending; they are written into its row of block_table behind the blocks it has.
 *   - The new tokens of all requests, request after request, are numbered from 0: starts_out[b] is the first of request b, and
 *     slots_out[t] the slot of token t (-1 for t >= starts_out[n_requests]).
 * A request is refused -- lengths_out[b] = old_lengths[b], its slots -1, nothing taken -- if its new length is negative or
 * exceeds max_blocks * page_size; if it needs pages and those asked for up to and with it exceed what the list holds; or if
 * the new tokens up to and with it exceed max_new_tokens.  Its tokens keep their numbers (starts_out is not below
 * max_new_tokens only in that last case, where it is cut off there).
 *
 *   old_lengths, new_lengths  [n_requests] int32; an old length outside [0, max_blocks * page_size] counts as the nearest in it
 *   block_table               [n_requests, max_blocks] int32, rows table_stride elements apart; in and out
 *   free_pages, free_count    [free_capacity] and [1] int32: the first free_count entries are the free pages; in and out.  A
 *                             count outside [0, free_capacity] counts as the nearest in it; pages beyond the capacity are lost
 *   lengths_out               [n_requests] int32; may be old_lengths, not new_lengths
 *   starts_out                [n_requests + 1] int32;  slots_out [max_new_tokens] int32 (may be NULL if that is 0)
 *   free_count_out            [1] int32; may be free_count (in place: a second launch where max_new_tokens exceeds 8192)
 * 1 <= n_requests <= 4096; 0 <= max_new_tokens <= 2^24; 1 <= max_blocks, max_blocks * page_size <= 2^30;
 * 0 <= free_capacity, free_capacity * page_size < 2^31 (no pool has more pages).
 */
#define APBV_CACHE_MAX_REQUESTS 4096
apbv_status apbv_cache_map(int n_requests, int page_size, int64_t max_blocks,
                           const int32_t* old_lengths, const int32_t* new_lengths,
                           int32_t* block_table, int64_t table_stride,
                           int32_t* free_pages, int64_t free_capacity, const int32_t* free_count,
                           int64_t max_new_tokens,
                           int32_t* lengths_out, int32_t* starts_out, int32_t* slots_out, int32_t* free_count_out,
                           void* hip_stream);

/*
 * Writes the rows of k and v ([tokens, n_kv_heads, head_dim] bf16) into the cache, token t at slots[t].  A slot outside
 * [0, n_pages * page_size) (-1: padding) is skipped.  Slots must differ: what a slot named twice holds afterwards is
 * unspecified (other slots are not touched).  tokens == 0 does nothing.  0 <= tokens <= 2^24, and tokens * head_dim / 2048
 * (rounded up) * n_kv_heads below 2^24; apbv_cache_load alike.
 */
apbv_status apbv_cache_store(const apbv_cache* cache, int n_kv_heads, int head_dim,
                             apbv_tensor k, apbv_tensor v, const int32_t* slots, void* hip_stream);

/*
 * Reads rows back: k_out, v_out [tokens, n_kv_heads, head_dim] bf16, dense, take the values held at slots[t] (exactly); zero
 * for a slot outside [0, n_pages * page_size).  A slot may be named any number of times.
 */
apbv_status apbv_cache_load(const apbv_cache* cache, int n_kv_heads, int head_dim, int64_t tokens,
                            const int32_t* slots, void* k_out, void* v_out, void* hip_stream);

/* Host, pure.  Bytes of workspace apbv_cache_attention needs (0 on invalid arguments; a call may still be larger than what is
 * supported, which it says itself); 256-byte aligned.  n_rows = q.tokens, max_q as passed to the call. */
size_t apbv_cache_attention_workspace_bytes(int n_requests, int64_t n_rows, int n_q_heads, int n_kv_heads, int head_dim,
                                            int64_t max_q);

/*
 * Attention of the query rows of many requests over their cached keys:
 *   out[i, h, :] = sum_j softmax_j(softmax_scale * q[i, h, :] . K[j, h/G, :]) V[j, h/G, :],  G = n_q_heads / n_kv_heads
 * over the keys j of the row's request that the row sees.  Request b has the rows q_starts[b] to q_starts[b + 1] - 1 and
 * lengths[b] keys, of which key j lies at slot block_table[b, j / page_size] * page_size + j % page_size.  With n rows, its
 * row i sees the keys j <= lengths[b] - n + i (causal: the rows are the last n positions, already stored) or all of them
 * (causal == 0: a partial result, to be merged by apbv_merge_lse, whose layouts out and lse_out have).
 *
 *   q            [n_rows, n_q_heads, head_dim], any number of rows (0: nothing is done)
 *   block_table  [n_requests, max_blocks] int32, rows table_stride elements apart; entries beyond a request's keys are not read.  How
 *                wide it is decides how the work is cut, as the host knows no lengths: the columns that are needed, of a wider table,
 *                are faster for short requests (256 of up to 2048 keys 13 us, in a table of 131072 tokens 18)
 *   lengths      [n_requests] int32; outside [0, max_blocks * page_size] the nearest in it is taken
 *   q_starts     [n_requests + 1] int32, not descending, within [0, n_rows] (cut off there); or NULL: every request has
 *                n_rows / n_requests rows
 *   max_q        the largest number of rows of a request, or more: a question of speed and workspace only (above 32 rows per KV head
 *                every request is worked on in tiles of 128: 256 requests of one query 13 us with max_q = 1, 32 with 256)
 *   out          [n_rows, n_q_heads, head_dim] bf16, dense;  lse_out optional (may be NULL) [n_q_heads, n_rows] fp32
 * Rows of no request (before q_starts[0], behind q_starts[n_requests]) are left as they were.  A row that sees no key gets
 * zeros and -inf.  Keys on a page outside [0, n_pages) are taken as not there.
 *
 * Arithmetic: the cached values are exact in bf16; bf16 operands, fp32 accumulation and softmax, probabilities rounded to
 * bf16 before the product with V and divided by their rounded sum (the lse is of their exact one), the parts of a row that
 * several workgroups share are kept and joined in fp32, output rounded to bf16.  How the keys are cut depends on the shape of the
 * call and on all lengths; results of the same call are repeatable.
 * Supported: head_dim in {64, 128}; n_q_heads % n_kv_heads == 0; 1 <= n_requests <= 4096; max_blocks * page_size <= 2^30;
 * n_rows * G <= 2^30; (n_rows * G / 16 + n_requests) * n_kv_heads * (max_blocks * page_size / 64) below 2^31 (a table of
 * 4096 rows for 2^20 tokens, with 8 KV heads); n_rows * n_q_heads <= 2^26 - 4; n_requests * n_kv_heads below 2^24.
 */
apbv_status apbv_cache_attention(const apbv_cache* cache, int n_requests, int n_q_heads, int n_kv_heads, int head_dim,
                                 apbv_tensor q, const int32_t* block_table, int64_t table_stride, int64_t max_blocks,
                                 const int32_t* lengths, const int32_t* q_starts, int64_t max_q, int causal,
                                 float softmax_scale, void* out, float* lse_out,
                                 void* workspace, size_t workspace_bytes, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* APBV_CACHE_H_ */
