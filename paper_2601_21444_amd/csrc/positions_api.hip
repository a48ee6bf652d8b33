// C ABI of the positions (include/apbv_positions.h): argument validation on the host, then dispatch to the kernel launchers.
#include "positions.h"

using namespace apbv;

extern "C" {

apbv_status apbv_rotate(int n_q_heads, int n_kv_heads, int head_dim, const apbv_rotation* rotation, apbv_tensor q, apbv_tensor k,
                        const int32_t* positions, int64_t position_stride, void* q_out, void* k_out, void* hip_stream) {
  const apbv_status st = validate_rotate(n_q_heads, n_kv_heads, head_dim, rotation, q, k, positions, position_stride, q_out, k_out);
  if (st != APBV_OK || (q.tokens == 0 && k.tokens == 0)) return st;
  TurnParams p;
  p.rot = to_rotation(*rotation, positions, position_stride);
  p.q = to_view(q);
  p.k = to_view(k);
  p.q_out = static_cast<bf16_t*>(q_out);
  p.k_out = static_cast<bf16_t*>(k_out);
  p.tokens = q.tokens > 0 ? q.tokens : k.tokens;
  p.hq = q.tokens > 0 ? n_q_heads : 0;
  p.hkv = k.tokens > 0 ? n_kv_heads : 0;
  return launch_rotate(p, head_dim, static_cast<hipStream_t>(hip_stream));
}

apbv_status apbv_cache_append(const apbv_cache* cache, int n_q_heads, int n_kv_heads, int head_dim, const apbv_rotation* rotation,
                              apbv_tensor q, apbv_tensor k, apbv_tensor v, const int32_t* positions, int64_t position_stride,
                              const int32_t* slots, void* q_out, void* hip_stream) {
  const apbv_status st = validate_cache_append(cache, n_q_heads, n_kv_heads, head_dim, rotation, q, k, v, positions, position_stride, slots, q_out);
  if (st != APBV_OK || k.tokens == 0) return st;
  AppendParams p;
  p.turn.rot = to_rotation(*rotation, positions, position_stride);
  p.turn.q = to_view(q);
  p.turn.k = {};
  p.turn.q_out = static_cast<bf16_t*>(q_out);
  p.turn.k_out = nullptr;
  p.turn.tokens = k.tokens;
  p.turn.hq = q.tokens > 0 ? n_q_heads : 0;
  p.turn.hkv = 0;
  p.cache = to_view(*cache);
  p.k = to_view(k);
  p.v = to_view(v);
  p.slots = slots;
  p.hkv = n_kv_heads;
  return launch_cache_append(p, head_dim, static_cast<hipStream_t>(hip_stream));
}

}  // extern "C"
