/*
 * apbv_positions.h -- positions of queries and keys: the norm of every head's row and its rotation, before the attention of apbv.h
 * (apbv_rotate) and on the way into the cache of apbv_cache.h (apbv_cache_append), whose conventions (device pointers, the caller
 * owns every buffer, asynchronous on `hip_stream`, errors found on the host before anything is launched, capture into a HIP graph)
 * hold here too.  These calls keep no state and need no set-up before a capture.
 */
#ifndef APBV_POSITIONS_H_
#define APBV_POSITIONS_H_

#include "apbv_cache.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * What is done with the rows x [head_dim] of a token's queries and keys:
 *   y = x, or with a weight w   y[e] = x[e] * w[e] / sqrt(sum_e x[e]^2 / head_dim + eps)
 *   of the first rot_dim elements pair i < rot_dim / 2, (a, b) = (y[i], y[i + rot_dim / 2]), or (y[2i], y[2i + 1]) if `adjacent`,
 *   becomes (a cos t - b sin t, b cos t + a sin t),  t = positions[axis[i]][token] * inv_freq[i];  the other elements stay.
 * Positions with one axis are those of text; with several, time, height and width of a frame's tokens, each pair going with one.
 * Angles are formed and reduced in float64 (the product exact below 2^29, angles beyond 2^52 unspecified), whatever the position: negated
 * positions turn back.
 */
typedef struct {
  const float* inv_freq;    /* [rot_dim / 2]                                                           */
  const void* q_weight;     /* [head_dim] bf16, 16-byte aligned; NULL: queries are not normed          */
  const void* k_weight;     /* ... keys                                                                */
  float eps;                /* finite, not negative                                                    */
  int32_t rot_dim;          /* a multiple of 16, 16 to head_dim                                        */
  int32_t n_axes;           /* 1 to 4                                                                  */
  int32_t adjacent;         /* 0 or 1                                                                  */
  uint8_t axis[64];         /* of pair i, below n_axes                                                 */
} apbv_rotation;

/*
 * Norms and turns the rows of queries and keys.
 *   q [tokens, n_q_heads, head_dim], k [tokens, n_kv_heads, head_dim] bf16, any strides of apbv_tensor (a projection's joint output);
 *              one of them may be left out (0 tokens)
 *   positions  [n_axes, tokens] int32, axes position_stride elements apart (0: all axes the same)
 *   q_out, k_out   bf16, dense; q_out may be q itself and k_out k itself where that is dense (else they overlap neither inputs nor each
 *              other: an output that begins where the other or the other's input does is refused).  Not read where q or k is left out
 * Arithmetic: float32 (the sum of squares and the angles in float64), rounded once, to bf16.  No tokens: nothing is done.
 * Supported: head_dim in {64, 128}; tokens <= 2^24; tokens * (n_q_heads + n_kv_heads) below 2^29.
 */
apbv_status apbv_rotate(int n_q_heads, int n_kv_heads, int head_dim, const apbv_rotation* rotation, apbv_tensor q, apbv_tensor k,
                        const int32_t* positions, int64_t position_stride, void* q_out, void* k_out, void* hip_stream);

/*
 * A step's queries, keys and values [tokens, heads, head_dim]: queries as apbv_rotate leaves them, in q_out; keys, normed and turned,
 * and values into the cache, token t at slots[t].  Slots are as in apbv_cache_store: one outside [0, n_pages * page_size) (-1: padding)
 * is skipped, its query is turned all the same; what a slot named twice holds is unspecified.
 *   q_out   bf16, dense; may be q itself where that is dense, not k or v (refused)
 * Keys are formed in float64 and rounded once, to the codes of the cache (a key that apbv_rotate has rounded to bf16 and
 * apbv_cache_store then stores may be held one code away); a NaN is stored as zero, what lies beyond the largest finite bf16 as that.
 * Queries may be left out (0 tokens: keys and values alone).
 * Supported: as apbv_rotate and apbv_cache_store; tokens * n_kv_heads up to 2^26.
 */
apbv_status apbv_cache_append(const apbv_cache* cache, int n_q_heads, int n_kv_heads, int head_dim, const apbv_rotation* rotation,
                              apbv_tensor q, apbv_tensor k, apbv_tensor v, const int32_t* positions, int64_t position_stride,
                              const int32_t* slots, void* q_out, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* APBV_POSITIONS_H_ */
