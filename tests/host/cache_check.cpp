// Host checks of the cache's validation and plans (csrc/cache_validation.h), built with the host compiler's sanitizers.
#include <cstdio>
#include <cstdlib>
#include "cache_validation.h"

using namespace apbv;

#define CHECK(x) do { if (!(x)) { std::printf("line %d: %s\n", __LINE__, #x); std::exit(1); } } while (0)

int main() {
  CHECK(log2_page(16) == 4 && log2_page(32) == 5 && log2_page(64) == 6 && log2_page(128) == 7 && log2_page(256) == 8);
  for (int p = -1; p < 300; ++p) CHECK(!valid_page_size(p) || (1 << log2_page(p)) == p);
  void* at = reinterpret_cast<void*>(0x10000);
  apbv_cache c = {at, at, at, at, 5, 2 * 64 * 64, 2 * 64 * 4, 64};
  CHECK(check_cache(&c, 2, 128) == APBV_OK && check_cache(&c, 4, 64) == APBV_OK && check_cache(nullptr, 2, 128) == APBV_ERR_NULL);
  CHECK(check_cache(&c, 3, 128) == APBV_ERR_SHAPE);             // pages overlap
  c.n_pages = 1;
  CHECK(check_cache(&c, 3, 128) == APBV_OK);                    // one page: no distance between pages
  c.n_pages = kMaxSlots / 64;
  CHECK(check_cache(&c, 2, 128) == APBV_OK);
  c.n_pages += 1;
  CHECK(check_cache(&c, 2, 128) == APBV_ERR_SHAPE);
  c.n_pages = -5;
  CHECK(check_cache(&c, 2, 128) == APBV_ERR_SHAPE);
  // the longest table: its last key's tile ends within 32 bits
  CHECK(check_table(1, 16, at, 0, kMaxCachedTokens / 16) == APBV_OK && check_table(1, 16, at, 0, kMaxCachedTokens / 16 + 1) == APBV_ERR_SHAPE);
  CHECK(kMaxCachedTokens + kCacheKeyTile < kMaxSlots);
  // plans: the workspace holds two parts of a row tile for every workgroup
  const int heads[][2] = {{1, 1}, {2, 1}, {16, 2}, {28, 4}, {8, 8}, {64, 1}, {128, 1}};
  for (auto& h : heads)
    for (int64_t q : {0, 1, 2, 3, 5, 16, 64, 333, 4096})
      for (int n : {1, 7, 64, 4096})
        for (int d : {64, 128}) {
          const int64_t rows = q * n < 1 << 20 ? q * n : 1 << 20;
          const CachePlan p = choose_cache_plan(n, h[0], h[1], d, rows, q, 1000);
          CHECK(p.rows >= 16 && p.rows % 16 == 0 && p.workgroups % 16 == 0 && p.least_tiles >= 1);
          CHECK(cache_attention_workspace_bytes(n, rows, h[0], h[1], d, q) >= (size_t)p.workgroups * 2 * p.rows * (d + 3) * 4);
        }
  // a workgroup for every (request, head, row tile): short tables, or rather short ones of many
  CHECK(choose_cache_plan(1, 2, 1, 64, 1, 1, 1024).whole && !choose_cache_plan(1, 2, 1, 64, 1, 1, 1025).whole);
  CHECK(choose_cache_plan(64, 16, 2, 128, 64, 1, 2048).whole && !choose_cache_plan(63, 16, 2, 128, 63, 1, 2048).whole);
  CHECK(choose_cache_plan(4096, 8, 2, 64, 4096, 1, 8192).whole && !choose_cache_plan(4096, 8, 2, 64, 4096, 1, 8193).whole);
  CHECK(!choose_cache_plan(1, 16, 2, 128, 5, 5, 64).whole && choose_cache_plan(1, 16, 2, 128, 4, 4, 64).whole);      // more than 32 rows: shared keys
  // the axis: as many tiles as 32 bits number, and no more
  CHECK(cache_axis_fits(1, 1, 1, 1, kMaxCachedTokens) && cache_axis_fits(4096, 4096, 28, 4, 1 << 20) && !cache_axis_fits(4096, 4096, 8, 8, kMaxCachedTokens));
  CHECK(!cache_axis_fits(1, (int64_t)1 << 24, 16, 16, 1 << 20) && cache_axis_fits(64, 8192, 64, 8, 1 << 18));
  CHECK(cache_attention_workspace_bytes(1, (int64_t)1 << 24, 65535, 1, 128, 1) == 0);
  std::printf("cache checks OK\n");
  return 0;
}
