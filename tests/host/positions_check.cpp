// Host checks of the positions' validation and of how their rows are dealt (built with sanitizers by tests/test_positions_host.py).
#include <stdio.h>
#include <stdlib.h>
#include "positions_validation.h"

using namespace apbv;

#define CHECK(x)                                                \
  do {                                                          \
    if (!(x)) {                                                 \
      printf("line %d: %s\n", __LINE__, #x);                    \
      exit(1);                                                  \
    }                                                           \
  } while (0)

int main() {
  // every row is some thread's exactly once, and no workgroup holds more tokens than its angles have room for
  for (int d : {64, 128})
    for (int heads : {1, 2, 3, 9, 31, 32, 33, 36, 63, 64, 65, 127, 128, 129, 255, 256, 257, 300, 5000, 65535})
      for (int64_t tokens : {1, 2, 7, 63, 64, 65, 1000, 32768, 100003}) {
        if (tokens * heads >= (int64_t)1 << 29) continue;
        const int most = turn_rows(tokens * heads, d), at_once = 4096 / d;
        CHECK(most == at_once || most == 4 * at_once);
        const TurnPlan p = turn_plan(tokens, heads, most);
        CHECK(p.tokens >= 1 && p.tokens <= kMaxTurnTokens && p.heads >= 1 && p.heads <= heads && p.tokens * p.heads <= most);
        CHECK(p.token_tiles * p.tokens >= tokens && (p.token_tiles - 1) * p.tokens < tokens);
        CHECK(p.head_tiles * p.heads >= heads && (p.head_tiles - 1) * p.heads < heads);
        CHECK(p.workgroups() <= kMaxGroups);
        CHECK((size_t)p.tokens * d * 4 <= 65536);
        // the threads' walk over a workgroup's rows, as the kernel steps through them
        if (tokens * heads < 5000) {
          int seen = 0;
          for (int row = 0; row < at_once; ++row) {
            int t = row / p.heads, h = row - t * p.heads;
            const int step_t = at_once / p.heads, step_h = at_once - step_t * p.heads;
            for (int u = 0; u < most / at_once; ++u) {
              CHECK(t * p.heads + h == row + u * at_once && h >= 0 && h < p.heads);
              seen += t < p.tokens;
              t += step_t;
              h += step_h;
              if (h >= p.heads) h -= p.heads, ++t;
            }
          }
          CHECK(seen == p.tokens * p.heads);
        }
      }
  for (int d : {64, 128})
    for (int hkv : {1, 2, 3, 5, 7, 8, 9, 16, 17, 100, 65535})
      for (int64_t tokens : {1, 2, 15, 16, 17, 1000, 100003}) {
        const TurnPlan p = append_plan(tokens, hkv, d);
        CHECK(p.tokens >= 2 && p.heads >= 1 && p.tokens * p.heads <= 2048 / d && p.tokens * p.heads > 2048 / d - p.heads);
        CHECK(p.token_tiles * p.tokens >= tokens && (p.token_tiles - 1) * p.tokens < tokens && p.head_tiles * p.heads >= hkv && (p.head_tiles - 1) * p.heads < hkv);
        CHECK((size_t)p.tokens * (d / 2) * 16 <= 65536);
      }
  CHECK(turn_plan((int64_t)1 << 24, 31, turn_rows((int64_t)31 << 24, 128)).workgroups() <= kMaxGroups);
  CHECK(turn_plan(((int64_t)1 << 29) / 65 - 1, 65, turn_rows(((int64_t)1 << 29) - 65, 128)).workgroups() <= kMaxGroups);
  // the most workgroups that an append may take: as many keys as are supported, and queries up to the limit of both
  for (int d : {64, 128})
    for (int hkv : {1, 2, 3, 5, 7, 8, 9, 15, 16, 17, 63, 64, 65, 1000, 65535})
      for (int64_t tokens : {((int64_t)1 << 26) / hkv, ((int64_t)1 << 26) / hkv / 3, ((int64_t)1 << 24)}) {
        if (tokens > kMaxTokens || tokens * hkv > (int64_t)1 << 26) continue;
        for (int hq : {1, 2, 31, 33, 64, 65, 127, 128, 129, 65535}) {
          if (tokens * (hq + hkv) >= (int64_t)1 << 29) continue;
          CHECK(append_plan(tokens, hkv, d).workgroups() + turn_plan(tokens, hq, turn_rows(tokens * hq, d)).workgroups() <= kMaxGroups);
        }
      }
  apbv_rotation r = {};
  CHECK(check_rotation(nullptr, 128) == APBV_ERR_NULL);
  r.rot_dim = 128;
  r.n_axes = 1;
  CHECK(check_rotation(&r, 128) == APBV_ERR_NULL && check_rotation(&r, 64) == APBV_ERR_SHAPE);
  float f[64];
  r.inv_freq = f;
  CHECK(check_rotation(&r, 128) == APBV_OK);
  r.axis[63] = 1;
  CHECK(check_rotation(&r, 128) == APBV_ERR_SHAPE);
  r.rot_dim = 64;
  CHECK(check_rotation(&r, 128) == APBV_OK);
  printf("positions checks OK\n");
  return 0;
}
