// Device/host declarations of the position kernels (internal; the public ABI is include/apbv_positions.h).
#pragma once
#include "cache.h"
#include "positions_validation.h"

namespace apbv {

struct Rotation {
  const float* inv_freq;
  const bf16_t *q_weight, *k_weight;
  const int32_t* positions;
  int64_t position_stride;
  double eps;
  int rot, adjacent;
  uint64_t axis[2];        // two bits a pair, 32 pairs each
};
inline Rotation to_rotation(const apbv_rotation& r, const int32_t* positions, int64_t stride) {
  Rotation x;
  x.inv_freq = r.inv_freq;
  x.q_weight = static_cast<const bf16_t*>(r.q_weight);
  x.k_weight = static_cast<const bf16_t*>(r.k_weight);
  x.positions = positions;
  x.position_stride = stride;
  x.eps = r.eps;
  x.rot = r.rot_dim;
  x.adjacent = r.adjacent;
  x.axis[0] = x.axis[1] = 0;
  for (int i = 0; i < r.rot_dim / 2; ++i) x.axis[i / 32] |= (uint64_t)r.axis[i] << (2 * (i % 32));
  return x;
}

// Rows that are turned: heads of q, behind them those of k (of a token).
struct TurnParams {
  Rotation rot;
  View q, k;
  bf16_t *q_out, *k_out;
  int64_t tokens;
  int hq, hkv;             // 0: none
  int tile_tokens, tile_heads, head_tiles;      // TurnPlan
};
struct AppendParams {
  TurnParams turn;         // the queries
  CacheView cache;
  View k, v;
  const int32_t* slots;
  int hkv, row_groups;     // workgroups of keys and values, in front of those of the queries
  int tile_tokens, tile_heads, head_tiles;      // append_plan
};
apbv_status launch_rotate(TurnParams& p, int head_dim, hipStream_t stream);
apbv_status launch_cache_append(AppendParams& p, int head_dim, hipStream_t stream);

}  // namespace apbv
