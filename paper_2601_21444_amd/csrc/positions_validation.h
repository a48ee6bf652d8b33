// Host-side argument validation and planning of include/apbv_positions.h; plain C++ as host_validation.h is.
#pragma once
#include "apbv_positions.h"
#include "cache_validation.h"

namespace apbv {

constexpr int kMaxAxes = 4;
constexpr int kMaxPairs = 64;

inline apbv_status check_rotation(const apbv_rotation* r, int d) {
  if (r == nullptr) return APBV_ERR_NULL;
  if (r->rot_dim < 16 || r->rot_dim > d || r->rot_dim % 16) return APBV_ERR_SHAPE;
  if (r->n_axes < 1 || r->n_axes > kMaxAxes || r->adjacent < 0 || r->adjacent > 1) return APBV_ERR_SHAPE;
  if (!(r->eps >= 0.0f) || !std::isfinite(r->eps)) return APBV_ERR_SHAPE;
  for (int i = 0; i < r->rot_dim / 2; ++i)
    if (r->axis[i] >= r->n_axes) return APBV_ERR_SHAPE;
  if (r->inv_freq == nullptr) return APBV_ERR_NULL;
  if (!aligned(r->inv_freq, 4) || !aligned(r->q_weight, 16) || !aligned(r->k_weight, 16)) return APBV_ERR_SHAPE;
  return APBV_OK;
}

// Rows that a call turns, dense where they are written: `out` may be the rows themselves only if they are dense, too.
inline apbv_status check_turned(const apbv_tensor& t, int heads, int d, const void* out) {
  if (t.tokens != 0 && (heads < 1 || heads > 65535)) return APBV_ERR_SHAPE;
  const apbv_status st = check_view(t, heads, d, 1, true);
  if (st != APBV_OK || t.tokens == 0) return st;
  if (out == nullptr) return APBV_ERR_NULL;
  if (!aligned(out, 16)) return APBV_ERR_SHAPE;
  if (out == t.ptr && ((t.tokens > 1 && t.stride_token != (int64_t)heads * d) || (heads > 1 && t.stride_head != d))) return APBV_ERR_SHAPE;
  return APBV_OK;
}

inline apbv_status check_positions(const int32_t* positions, int64_t stride) {
  if (positions == nullptr) return APBV_ERR_NULL;
  return aligned(positions, 4) && stride >= 0 ? APBV_OK : APBV_ERR_SHAPE;
}

// How rows are dealt: a workgroup takes `tokens` tokens of `heads` heads each, at most `most` rows.
struct TurnPlan {
  int tokens, heads;
  int64_t token_tiles, head_tiles;
  int64_t workgroups() const { return token_tiles * head_tiles; }
};
constexpr int kMaxTurnTokens = 64;          // whose angles fit a workgroup's LDS
// Rows of a workgroup: one for every d / 16 of its threads, or four where there are enough to fill the chip all the same.
constexpr int64_t kFewTurnRows = 32768;
inline int turn_rows(int64_t rows, int d) { return (rows > kFewTurnRows ? 4 : 1) * (256 * 16 / d); }
inline TurnPlan turn_plan(int64_t tokens, int heads, int most) {
  TurnPlan p;
  p.heads = heads < most ? heads : most;
  p.tokens = most / p.heads < kMaxTurnTokens ? most / p.heads : kMaxTurnTokens;
  p.token_tiles = (tokens + p.tokens - 1) / p.tokens;
  p.head_tiles = (heads + p.heads - 1) / p.heads;
  return p;
}

// Keys and values: 2048 / d rows a workgroup, of up to 8 heads, whose tokens' angles it forms once for them.
inline TurnPlan append_plan(int64_t tokens, int hkv, int d) {
  const int rows = 2048 / d;
  TurnPlan p;
  p.heads = hkv < 8 ? hkv : 8;
  p.tokens = rows / p.heads;
  p.token_tiles = (tokens + p.tokens - 1) / p.tokens;
  p.head_tiles = (hkv + p.heads - 1) / p.heads;
  return p;
}

inline apbv_status validate_rotate(int hq, int hkv, int d, const apbv_rotation* r, const apbv_tensor& q, const apbv_tensor& k,
                                   const int32_t* positions, int64_t stride, const void* q_out, const void* k_out) {
  if (d != 64 && d != 128) return APBV_ERR_UNSUPPORTED;
  apbv_status st = check_rotation(r, d);
  if (st != APBV_OK) return st;
  if ((st = check_turned(q, hq, d, q_out)) != APBV_OK) return st;
  if ((st = check_turned(k, hkv, d, k_out)) != APBV_OK) return st;
  if (q.tokens != 0 && k.tokens != 0 && q.tokens != k.tokens) return APBV_ERR_SHAPE;
  if (q.tokens == 0 && k.tokens == 0) return APBV_OK;
  // (each output may be its own input, which a thread reads before it writes; the other's would be written before it is read)
  if (q.tokens != 0 && k.tokens != 0 && (q_out == k_out || q_out == k.ptr || k_out == q.ptr)) return APBV_ERR_SHAPE;
  if (q.tokens * hq + k.tokens * hkv >= (int64_t)1 << 29) return APBV_ERR_UNSUPPORTED;
  return check_positions(positions, stride);
}

inline apbv_status validate_cache_append(const apbv_cache* cache, int hq, int hkv, int d, const apbv_rotation* r, const apbv_tensor& q,
                                         const apbv_tensor& k, const apbv_tensor& v, const int32_t* positions, int64_t stride,
                                         const int32_t* slots, const void* q_out) {
  apbv_status st = validate_cache_store(cache, hkv, d, k, v, slots);
  if (st != APBV_OK) return st;
  if ((st = check_rotation(r, d)) != APBV_OK) return st;
  if ((st = check_turned(q, hq, d, q_out)) != APBV_OK) return st;
  if (q.tokens != 0 && q.tokens != k.tokens) return APBV_ERR_SHAPE;
  if (k.tokens == 0) return APBV_OK;
  if (q.tokens != 0 && (q_out == k.ptr || q_out == v.ptr)) return APBV_ERR_SHAPE;
  if (q.tokens * hq + k.tokens * hkv >= (int64_t)1 << 29) return APBV_ERR_UNSUPPORTED;
  if (k.tokens * hkv > (int64_t)1 << 26) return APBV_ERR_UNSUPPORTED;      // (below 2^24 workgroups, then: tests/host/positions_check.cpp)
  return check_positions(positions, stride);
}

}  // namespace apbv
