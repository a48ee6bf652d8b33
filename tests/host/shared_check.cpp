// Host checks of how a call behind shared prefixes is cut (built with sanitizers by tests/test_shared_host.py).
#include <stdio.h>
#include <stdlib.h>
#include "shared_validation.h"

using namespace apbv;

#define CHECK(x)                                                \
  do {                                                          \
    if (!(x)) {                                                 \
      printf("line %d: %s\n", __LINE__, #x);                    \
      exit(1);                                                  \
    }                                                           \
  } while (0)

int main() {
  // every tile is in one share, shares are numbered as the dies' workgroups take them, and there are no more than workgroups
  for (uint32_t w : {16u, 512u})
    for (uint32_t total : {0u, 1u, 5u, 16u, 17u, 100u, 999u, 4096u, 16640u, 100001u, 0x7fff0000u})
      for (uint32_t short_tiles : {0u, 6u, 12u, 1u << 30})
        for (uint32_t busy : {0u, 1u, 5u, 22u, 63u, 64u, 100u})
          for (uint32_t cost : {0u, 1u, 3u, 30u}) {
            const AxisCut c = shared_cut(total, w, short_tiles, 2, busy, cost);
            CHECK(c.share >= 1 && c.rest >= 1 && c.used >= 1 && c.used <= w / 8 && c.stretch * 8 >= total && c.full <= w / 8);
            uint32_t at = 0;
            for (uint32_t die = 0; die < 8; ++die) {
              CHECK(cut_begin(c, die, 0) == die * c.stretch);
              for (uint32_t x = 0; x < c.used; ++x) {
                const uint32_t b = cut_begin(c, die, x), e = cut_end(c, die, x);
                CHECK(b == at && e > b && e <= (die + 1) * c.stretch);
                for (uint32_t t : {b, e - 1}) CHECK(cut_share_of(cut_word(c), t) == die * c.used + x);
                at = e;
              }
              CHECK(at == (die + 1) * c.stretch);
            }
            CHECK(at >= total);
          }
  static_assert(sizeof(CutWord) == kCutWords * 4, "");
  CHECK(shared_cut(16640, 512, 12, 2, 22, 2).share == 34 && shared_cut(16640, 512, 12, 2, 22, 2).rest == 32);
  // the launches there are: tiles of 16 or 32 rows of the prefix with 16 of the own keys, or of 128 with 16 or 128
  for (int d : {64, 128})
    for (int groups : {1, 2, 7, 64, 4096})
      for (int n : {1, 2, 64, 333, 4096})
        for (int hkv : {1, 2, 8})
          for (int g : {1, 2, 7, 8, 33})
            for (int64_t each : {1, 2, 3, 40, 700}) {
              if (groups > n) continue;
              const int64_t rows = n * each;
              for (int64_t max_q : {(int64_t)0, each, rows, rows + 5}) {
                const SharedPlan p = choose_shared_plan(groups, n, hkv * g, hkv, d, rows, max_q, 1 << 30, 1 << 20, true);
                CHECK(p.prefix.rows == 16 || p.prefix.rows == 32 || p.prefix.rows == kCacheBlockRows);
                CHECK(p.own.rows == 16 || (p.own.rows == kCacheBlockRows && p.prefix.rows == kCacheBlockRows));
                CHECK(p.own.row_tiles >= 0 && kSharedWorkgroups % 8 == 0);
                CHECK(!p.whole);
                const SharedPlan few = choose_shared_plan(groups, n, hkv * g, hkv, d, rows, max_q, 64, 64, true);
                if (few.whole) CHECK(few.prefix.row_tiles >= 1 && (groups + 2) * (int64_t)hkv * few.prefix.row_tiles <= 1 << 22 && few.prefix.row_tiles * (int64_t)16 * groups >= rows * g);
                // whatever the tables hold, the workspace is the same, and tiles of 16 rows fit what it has for higher ones
                for (int64_t max_prefix : {(int64_t)0, (int64_t)1000, (int64_t)30000, (int64_t)1 << 30})
                  for (bool even : {false, true}) {
                    const SharedPlan x = choose_shared_plan(groups, n, hkv * g, hkv, d, rows, max_q, max_prefix, 1 << 20, even);
                    CHECK(x.prefix.rows <= p.prefix.rows && x.own.rows <= p.own.rows && x.prefix.row_tiles >= 1);
                    CHECK(x.prefix.rows == p.prefix.rows || (x.prefix.rows == 16 && x.own.rows == 16));
                    CHECK(shared_space(x, groups, n, rows, hkv * g, d).bytes == shared_space(p, groups, n, rows, hkv * g, d).bytes);
                    CHECK(x.prefix_parts >= cache_parts_bytes(x.prefix, d) && x.own_parts >= cache_parts_bytes(x.own, d));
                  }
                const SharedSpace s = shared_space(p, groups, n, rows, hkv * g, d);
                // regions follow one another, hold what is written into them, and start where float4s may
                CHECK(s.own_parts >= (size_t)kSharedWorkgroups * 2 * p.prefix.rows * (d + 3) * 4);
                CHECK(s.prefix_kept - s.own_parts >= (size_t)kSharedWorkgroups * 2 * p.own.rows * (d + 3) * 4);
                CHECK(s.own_kept - s.prefix_kept >= (size_t)rows * hkv * g * (d + 3) * 4 && s.prefix_begins - s.own_kept == s.own_kept - s.prefix_kept);
                CHECK(s.own_begins - s.prefix_begins >= (size_t)(groups + kCutWords) * 4 && s.bytes - s.own_begins >= (size_t)(n + kCutWords) * 4);
                CHECK(s.own_parts % 256 == 0 && s.prefix_kept % 256 == 0 && s.own_kept % 256 == 0 && s.prefix_begins % 256 == 0 && s.own_begins % 256 == 0);
                if (rows * hkv * g <= 4 * kMaxGroups) CHECK(shared_attention_workspace_bytes(groups, n, rows, hkv * g, hkv, d, max_q) == s.bytes);
              }
            }
  printf("shared checks OK\n");
  return 0;
}
