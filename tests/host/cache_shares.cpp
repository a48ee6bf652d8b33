// How an attention call over the cache is cut: reads "query heads, KV heads, head_dim, longest length of the table, requests, then
// the queries and keys of each" from stdin, a call a line, and prints rows of a row tile, whether a workgroup takes it whole, waves
// of the join, tiles of a share, and the most parts that a row tile has (taken whole: its most tiles, and its waves).
#include <cstdio>
#include <vector>
#include "cache_validation.h"

using namespace apbv;

int main() {
  int hq, hkv, d, n;
  long long max_len;
  while (std::scanf("%d %d %d %lld %d", &hq, &hkv, &d, &max_len, &n) == 5) {
    std::vector<long long> q(n), k(n);
    long long rows = 0, most = 0;
    for (int b = 0; b < n; ++b) {
      if (std::scanf("%lld %lld", &q[b], &k[b]) != 2) return 1;
      rows += q[b];
      most = q[b] > most ? q[b] : most;
    }
    const CachePlan p = choose_cache_plan(n, hq, hkv, d, rows, most, max_len);
    long long total = 0;
    for (int b = 0; b < n; ++b) total += (q[b] * (hq / hkv) + p.rows - 1) / p.rows * hkv * (q[b] > 0 ? (k[b] + kCacheKeyTile - 1) / kCacheKeyTile : 0);
    const uint32_t share = cache_share((uint32_t)total, p.workgroups, p.short_tiles, p.least_tiles, p.share_step);
    long long parts = 0, at = 0;
    for (int b = 0; b < n; ++b) {
      const long long tiles = (k[b] + kCacheKeyTile - 1) / kCacheKeyTile, items = (q[b] * (hq / hkv) + p.rows - 1) / p.rows * hkv;
      for (long long i = 0; i < items && tiles > 0; ++i, at += tiles) {
        const long long here = (at + tiles - 1) / share - at / share + 1;
        parts = here > parts ? here : parts;
      }
    }
    if (p.whole) {
      std::printf("%d 1 0 %lld %d\n", p.rows, (max_len + kCacheKeyTile - 1) / kCacheKeyTile, kCacheWaves);
      continue;
    }
    std::printf("%d 0 %d %u %lld\n", p.rows, p.join_waves, share, parts);
  }
  return 0;
}
