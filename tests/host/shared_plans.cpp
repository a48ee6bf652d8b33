// Which kernels a call behind shared prefixes takes: reads "groups, requests, query heads, KV heads, head_dim, rows, max_q, keys that a row of the
// prefix table holds, of the requests' table, whether groups and requests are equal" from stdin, a call a line, and prints "whole <waves>" or
// "cut <rows of the prefixes' tiles> <of the own keys'> <waves of the join>".
#include <cstdio>
#include "shared_validation.h"

using namespace apbv;

int main() {
  int groups, n, hq, hkv, d, even;
  long long rows, max_q, max_prefix, max_len;
  while (std::scanf("%d %d %d %d %d %lld %lld %lld %lld %d", &groups, &n, &hq, &hkv, &d, &rows, &max_q, &max_prefix, &max_len, &even) == 10) {
    const SharedPlan p = choose_shared_plan(groups, n, hq, hkv, d, rows, max_q, max_prefix, max_len, even != 0);
    if (p.whole)
      std::printf("whole %d\n", p.short_waves);
    else
      std::printf("cut %d %d %d\n", p.prefix.rows, p.own.rows, p.join_waves);
  }
  return 0;
}
