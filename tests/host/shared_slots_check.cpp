// Host replay of how a workgroup of the one-launch form finds its group and row tile (built with sanitizers by tests/test_shared_slots.py).
#include <stdio.h>
#include <stdlib.h>
#include <algorithm>
#include <random>
#include <vector>
#include "shared_validation.h"

using namespace apbv;

#define CHECK(x)                                                \
  do {                                                          \
    if (!(x)) {                                                 \
      printf("line %d: %s\n", __LINE__, #x);                    \
      exit(1);                                                  \
    }                                                           \
  } while (0)

static int clip(int x, int hi) { return x < 0 ? 0 : (x > hi ? hi : x); }

struct Call {
  int n_groups, n_requests, group, n_rows, members_each, each;
  const std::vector<int32_t>*members, *starts;       // null: equal groups, equally many rows
  int row_of(int b) const { return clip(starts ? starts->at(b) : b * each, n_rows); }
};
struct Found {
  int g, rt, from, to, first, past;
};

// shared_short.hip, lane after lane; `at` checks every index.
static bool find(const Call& c, int slot, Found& f) {
  const int n = c.n_groups + (c.members ? 2 : 0);
  int e = 0, top = n, step = (n + 64) / 64, rounds = 0;
  for (;;) {
    CHECK(++rounds <= 3);
    int last = -1, b[64], q[64], begin[64];
    for (int lane = 0; lane < 64; ++lane) {
      const int x = e + lane * step < top ? e + lane * step : top;
      b[lane] = !c.members ? x * c.members_each : x == 0 ? 0 : x == n ? c.n_requests : clip(c.members->at(x - 1), c.n_requests);
      q[lane] = c.row_of(b[lane]);
      begin[lane] = first_slot(q[lane], c.group, x);
      if (e + lane * step < top && begin[lane] <= slot) last = lane;
    }
    if (last < 0) return false;
    e += last * step;
    if (step == 1) {
      CHECK(last < 63);
      f = Found{c.members ? e - 1 : e, slot - begin[last], b[last], b[last + 1], q[last], q[last + 1]};
      return true;
    }
    top = e + step < n ? e + step : n;
    step = (step + 64) / 64;
  }
}

static std::mt19937 rng(5);
static int below(int n) { return (int)(rng() % (unsigned)n); }

static void replay(int n_groups, int n_requests, int group, bool listed, bool ragged, int shape) {
  std::vector<int32_t> starts(n_requests + 1), members(n_groups + 1);
  const int lead = ragged ? below(20) : 0, each = 1 + below(3);
  starts[0] = lead;
  for (int b = 0; b < n_requests; ++b) starts[b + 1] = starts[b] + (shape == 1 ? below(2) : shape == 4 ? (below(40) ? 0 : below(3)) : shape == 2 ? (b == n_requests / 2 ? 500 : 1) : below(4));
  for (int& m : members) m = below(n_requests + 1);
  std::sort(members.begin(), members.end());
  if (shape == 3)                                      // one group has nearly all
    for (int g = 0; g <= n_groups; ++g) members[g] = g <= n_groups / 2 ? g % 2 : n_requests - (n_groups - g) % 2;
  std::sort(members.begin(), members.end());
  Call c;
  c.n_groups = n_groups;
  c.n_requests = n_requests;
  c.group = group;
  c.n_rows = ragged ? starts[n_requests] + below(9) : n_requests * each;
  c.each = c.n_rows / n_requests;
  c.members_each = n_requests / n_groups;
  c.members = listed ? &members : nullptr;
  c.starts = ragged ? &starts : nullptr;
  if (c.n_rows == 0) return;
  const SharedPlan p = choose_shared_plan(n_groups, n_requests, 2 * group, 2, 64, c.n_rows, 4, 64, 64, false);
  CHECK(p.slots <= (int64_t)c.n_rows * group / 16 + std::min(n_groups + 2, c.n_rows));
  // rows of every group, and of those in front and behind, each to be taken once
  std::vector<int> taken(c.n_rows * group, 0);
  int idle = 0;
  for (int slot = 0; slot < p.slots; ++slot) {
    Found f;
    if (!find(c, slot, f)) {
      ++idle;
      continue;
    }
    CHECK(f.g >= -1 && f.g <= n_groups && f.rt >= 0);
    const int rows = (f.past > f.first ? f.past - f.first : 0) * group, r0 = f.rt * 16;
    if (f.from >= f.to || r0 >= rows) {
      ++idle;
      continue;
    }
    const bool grouped = f.g >= 0 && f.g < n_groups;
    CHECK(f.from == (!listed ? f.g * c.members_each : f.g < 0 ? 0 : members[f.g]));
    CHECK(f.to == (!listed ? f.from + c.members_each : f.g == n_groups ? n_requests : members[f.g + 1]));
    CHECK(grouped || listed);
    for (int r = r0; r < rows && r < r0 + 16; ++r) ++taken[f.first * group + r];
  }
  for (int r = 0; r < c.n_rows * group; ++r) {
    const bool somebody = r >= c.row_of(0) * group && r < c.row_of(n_requests) * group;
    CHECK(taken[r] == (somebody ? 1 : 0));
  }
  CHECK(idle <= n_groups + 3 + lead * group / 16 + 9 * group / 16 + 1);
}

int main() {
  for (int n_groups : {1, 2, 3, 61, 62, 63, 64, 65, 130, 1000, 4094, 4095, 4096})
    for (int times : {1, 2, 5})
      for (int group : {1, 2, 7, 8, 33})
        for (int shape = 0; shape < 5; ++shape) {
          const int n_requests = n_groups * times;
          if (n_requests > 4096 || (n_groups >= 1000 && group > 2)) continue;
          replay(n_groups, n_requests, group, true, true, shape);
          replay(n_groups, n_requests, group, true, false, shape);
          replay(n_groups, n_requests, group, false, true, shape);
        }
  // starts that descend and members that are anything: whatever is found, no index leaves its array
  for (int k = 0; k < 300; ++k) {
    const int n_groups = 1 + below(200), n_requests = n_groups + below(300);
    std::vector<int32_t> starts(n_requests + 1), members(n_groups + 1);
    for (int& x : starts) x = (int32_t)rng();
    for (int& x : members) x = (int32_t)rng();
    const Call c = {n_groups, n_requests, 3, 1000, 1, 1, &members, &starts};
    Found f;
    for (int slot = 0; slot < 1000 * 3 / 16 + n_groups + 2; ++slot)      // (more than there are)
      if (find(c, slot, f)) CHECK(f.rt >= 0 && f.from >= 0 && f.from <= n_requests && f.first >= 0 && f.first <= 1000 && f.past <= 1000);
  }
  // the launch: never more workgroups than 2^22, and of groups of unknown sizes no fewer than their row tiles may be
  for (int n_groups : {1, 2, 7, 100, 1000, 4096})
    for (int n_requests : {1, 8, 100, 4096})
      for (int hkv : {1, 8, 100})
        for (int group : {1, 7, 33})
          for (int64_t rows : {(int64_t)n_requests, (int64_t)n_requests * 40, (int64_t)1 << 20}) {
            if (n_groups > n_requests || rows * hkv * group > 4 * kMaxGroups) continue;
            for (bool even : {false, true}) {
              const SharedPlan p = choose_shared_plan(n_groups, n_requests, hkv * group, hkv, 128, rows, 1, 64, 64, even);
              if (!p.whole) continue;
              CHECK(p.slots >= 1 && p.slots * hkv <= 1 << 22);
              CHECK(even ? p.slots == (int64_t)n_groups * p.prefix.row_tiles : p.slots * 16 > rows * group && p.slots <= rows * group / 16 + rows);
            }
          }
  printf("slot checks OK\n");
  return 0;
}
