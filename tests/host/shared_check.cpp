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
                const SharedPlan p = choose_shared_plan(groups, n, hkv * g, hkv, d, rows, max_q, 1 << 20, 1 << 20);
                CHECK(p.prefix.rows == 16 || p.prefix.rows == 32 || p.prefix.rows == kCacheBlockRows);
                CHECK(p.own.rows == 16 || (p.own.rows == kCacheBlockRows && p.prefix.rows == kCacheBlockRows));
                CHECK(p.own.row_tiles >= 0 && p.workgroups % 8 == 0);
                CHECK(!p.whole);
                const SharedPlan few = choose_shared_plan(groups, n, hkv * g, hkv, d, rows, max_q, 64, 64);
                if (few.whole) CHECK(few.prefix.row_tiles >= 1 && (groups + 2) * (int64_t)hkv * few.prefix.row_tiles <= 1 << 22 && few.prefix.row_tiles * (int64_t)16 * groups >= rows * g);
                const SharedSpace s = shared_space(p, groups, n, rows, hkv * g, d);
                // regions follow one another, hold what is written into them, and start where float4s may
                CHECK(s.own_parts >= (size_t)p.workgroups * 2 * p.prefix.rows * (d + 3) * 4);
                CHECK(s.prefix_kept - s.own_parts >= (size_t)p.workgroups * 2 * p.own.rows * (d + 3) * 4);
                CHECK(s.own_kept - s.prefix_kept >= (size_t)rows * hkv * g * (d + 3) * 4 && s.prefix_begins - s.own_kept == s.own_kept - s.prefix_kept);
                CHECK(s.own_begins - s.prefix_begins >= (size_t)(groups + 1) * 4 && s.bytes - s.own_begins >= (size_t)(n + 1) * 4);
                CHECK(s.own_parts % 256 == 0 && s.prefix_kept % 256 == 0 && s.own_kept % 256 == 0 && s.prefix_begins % 256 == 0 && s.own_begins % 256 == 0);
                if (rows * hkv * g <= 4 * kMaxGroups) CHECK(shared_attention_workspace_bytes(groups, n, rows, hkv * g, hkv, d, max_q) == s.bytes);
              }
            }
  printf("shared checks OK\n");
  return 0;
}
