// Host replay of a call behind shared prefixes that is cut (built with sanitizers by tests/test_shared_slots.py): both axes laid out, every
// share walked as attend_few_rows and attend_block_rows walk it, wave after wave, and every row's list of parts made as parts_of makes it.
// Every tile of every row tile is in exactly one part that is joined, a part is written once and joined by the rows of its row tile alone,
// and nothing lies outside the workspace.
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

static std::mt19937 rng(11);
static int below(int n) { return (int)(rng() % (unsigned)n); }

struct Unit {                      // a request, or a group
  int first, queries, tiles;
};
struct Item {                      // a row tile of a unit and KV head
  int b, head, rt, tiles;
  uint32_t begin;
};
struct Piece {
  int item, t0, t1;
};
struct Axis {
  int R, hkv, group;
  std::vector<Unit> units;
  std::vector<Item> items;
  std::vector<uint32_t> unit_begin;      // on the axis
  uint32_t total = 0;
  AxisCut cut;
  // what the first launch leaves behind
  std::vector<Piece> part[2];            // [slot][share]
  std::vector<int> kept;                 // of an item: how often it was written whole
  std::vector<int64_t> begins;           // where a unit begins, if it was left word of
  bool word = false;

  void lay_out() {
    for (int b = 0; b < (int)units.size(); ++b) {
      const Unit& u = units[b];
      unit_begin.push_back(total);
      if (u.queries == 0 || u.tiles == 0) continue;
      const int row_tiles = (u.queries * group + R - 1) / R;
      for (int h = 0; h < hkv; ++h)
        for (int rt = 0; rt < row_tiles; ++rt) {
          items.push_back({b, h, rt, u.tiles, total});
          total += u.tiles;
        }
    }
    part[0].assign(kSharedWorkgroups, {-1, 0, 0});
    part[1] = part[0];
    kept.assign(items.size(), 0);
    begins.assign(units.size(), -1);
  }
  int item_at(uint32_t pos) const {
    int lo = 0, hi = (int)items.size() - 1;
    while (lo < hi) {
      const int m = (lo + hi + 1) / 2;
      if (items[m].begin <= pos)
        lo = m;
      else
        hi = m - 1;
    }
    return lo;
  }
  void leave(int wg, int slot, const Piece& p) {
    CHECK(wg >= 0 && wg < kSharedWorkgroups && part[slot][wg].item < 0);
    part[slot][wg] = p;
  }
  // pieces of [pos, end), as a wave (few rows) or a workgroup (128 rows) takes them
  std::vector<Piece> walk(uint32_t pos, uint32_t end) {
    std::vector<Piece> out;
    while (pos < end) {
      const int i = item_at(pos);
      const int t0 = (int)(pos - items[i].begin), t1 = end - pos < (uint32_t)(items[i].tiles - t0) ? t0 + (int)(end - pos) : items[i].tiles;
      if (pos == unit_begin[items[i].b]) {                 // the unit's first tile: word is left of where it begins
        CHECK(begins[items[i].b] < 0);
        begins[items[i].b] = pos;
        if (pos == 0) word = true;
      }
      out.push_back({i, t0, t1});
      pos += t1 - t0;
    }
    return out;
  }
  void first_launch() {
    for (uint32_t block = 0; block < (uint32_t)kSharedWorkgroups; ++block) {
      const uint32_t die = block % kCutDies, x = block / kCutDies;
      if (x >= cut.used) continue;
      const uint32_t begin = cut_begin(cut, die, x), past = cut_end(cut, die, x), end = past < total ? past : total;
      if (begin >= end) continue;
      const int wg = (int)(die * cut.used + x);
      if (R == kCacheBlockRows) {
        for (const Piece& p : walk(begin, end)) {
          if (p.t0 == 0 && p.t1 == items[p.item].tiles)
            ++kept[p.item];
          else
            leave(wg, p.t0 == 0 ? 1 : 0, p);
        }
        continue;
      }
      constexpr int W = kCacheWaves;
      enum { kHead = 1, kTail = 2, kSpan = 4 };
      const uint32_t wave_share = (end - begin + W - 1) / W;
      int keeps[W] = {};
      Piece head[W], tail[W];
      for (int w = 0; w < W; ++w) {
        const uint32_t pos = begin + w * wave_share, to = pos + wave_share < end ? pos + wave_share : end;
        if (pos >= to) continue;
        for (const Piece& p : walk(pos, to)) {
          const int tiles = items[p.item].tiles;
          if (p.t0 == 0 && p.t1 == tiles) {
            ++kept[p.item];
          } else if (p.t1 == tiles) {
            CHECK((keeps[w] & kHead) == 0);
            keeps[w] |= kHead;
            head[w] = p;
          } else {
            CHECK((keeps[w] & (kTail | kSpan)) == 0);
            keeps[w] |= p.t0 == 0 ? kTail : kSpan;
            tail[w] = p;
          }
        }
      }
      int used_head[W] = {}, used_tail[W] = {};
      for (int chain = 0; chain <= W; ++chain) {
        const int from = chain == 0 ? 0 : chain - 1;
        if (!(chain == 0 ? keeps[from] & (kHead | kSpan) : keeps[from] & kTail)) continue;
        int to = from;
        bool ends = chain == 0 && (keeps[0] & kHead);
        while (!ends && to + 1 < W) {
          if (keeps[to + 1] & kHead)
            ends = true;
          else if (!(keeps[to + 1] & kSpan))
            break;
          ++to;
        }
        Piece all = {-1, 0, 0};
        for (int w = from; w <= to; ++w) {
          const bool is_head = w == to && ends;
          const Piece& p = is_head ? head[w] : tail[w];
          CHECK(!(is_head ? used_head : used_tail)[w]);
          (is_head ? used_head : used_tail)[w] = 1;
          CHECK(w == from || (p.item == all.item && p.t0 == all.t1));
          all = w == from ? p : Piece{p.item, all.t0, p.t1};
        }
        if (chain > 0 && ends) {
          CHECK(all.t0 == 0 && all.t1 == items[all.item].tiles);
          ++kept[all.item];
        } else {
          leave(wg, chain > 0 ? 1 : 0, all);
        }
      }
      for (int w = 0; w < W; ++w) CHECK(used_head[w] == (keeps[w] & kHead ? 1 : 0) && used_tail[w] == (keeps[w] & (kTail | kSpan) ? 1 : 0));
    }
  }
  // parts_of: what is joined for row `row` of query head h; the tiles that are found, -1: a row that is of none
  int join(int row, int h, std::vector<int> (&joined)[2], std::vector<int>& read) const {
    const int n = (int)units.size();
    int base = 0;
    if (n > 64) {
      const int per = (n + 63) / 64;
      int last = -1;
      for (int lane = 0; lane < 64; ++lane)
        if (lane * per < n && units[lane * per].first <= row) last = lane;
      base = last < 0 ? 0 : last * per;
    }
    int at = -1;
    for (int lane = 0; lane < 64; ++lane)
      if (base + lane < n && units[base + lane].first <= row) at = lane;
    const int b = base + (at < 0 ? 0 : at);
    const Unit& u = units[b];
    const int i = row - u.first;
    if (!(i >= 0 && i < u.queries)) return -1;
    if (u.tiles == 0) return 0;
    const int r = i * group + h % group, rt = r / R, row_tiles = (u.queries * group + R - 1) / R;
    CHECK(word && begins[b] >= 0);                         // (of units without tiles nothing is read)
    const uint32_t from = (uint32_t)begins[b] + (uint32_t)(h / group * row_tiles + rt) * (uint32_t)u.tiles;
    const CutWord w = cut_word(cut);
    const uint32_t first = cut_share_of(w, from), last = cut_share_of(w, from + u.tiles - 1);
    CHECK(last >= first && last < (uint32_t)kSharedWorkgroups);
    const int item = item_at(from);
    CHECK(items[item].begin == from && items[item].b == b && items[item].head == h / group && items[item].rt == rt);
    if (first == last) {
      CHECK(kept[item] == 1);
      read[item] = 1;
      return u.tiles;
    }
    CHECK(kept[item] == 0);
    int tiles = 0;
    for (uint32_t s = first; s <= last; ++s) {
      const int slot = s == first ? 1 : 0;
      const Piece& p = part[slot][s];
      CHECK(p.item == item && p.t0 == tiles);
      joined[slot][s] = 1;
      tiles = p.t1;
    }
    return tiles;
  }
};

static void replay(int n_groups, int n, int hq, int hkv, int d, int longest_prefix, int longest, int queries, int RP, int RO, int busy_cost) {
  const int group = hq / hkv;
  std::vector<int> starts(n + 1), members(n_groups + 1);
  starts[0] = below(3);
  for (int b = 0; b < n; ++b) starts[b + 1] = starts[b] + (queries == 1 ? (below(8) ? 1 : 0) : below(queries + 1));
  for (int& m : members) m = below(n + 1);
  std::sort(members.begin(), members.end());
  const int n_rows = starts[n] + below(4);
  if (n_rows == 0) return;
  SharedPlan plan = choose_shared_plan(n_groups, n, hq, hkv, d, n_rows, queries, 1 << 24, 1 << 20, false);
  plan.prefix.rows = RP;
  plan.own.rows = RO;
  const size_t prefix_room = cache_parts_bytes(plan.prefix, d), own_room = cache_parts_bytes(plan.own, d);
  Axis a, o;
  a.R = RP, o.R = RO;
  a.hkv = o.hkv = hkv;
  a.group = o.group = group;
  for (int g = 0; g < n_groups; ++g) a.units.push_back({starts[members[g]], starts[members[g + 1]] - starts[members[g]], below(5) ? below(longest_prefix + 1) : 0});
  for (int b = 0; b < n; ++b) o.units.push_back({starts[b], starts[b + 1] - starts[b], below(5) ? below(longest + 1) : 0});
  a.lay_out();
  o.lay_out();
  o.cut = shared_cut(o.total, kSharedWorkgroups, plan.own.short_tiles, plan.own.least_tiles, 0, 0);
  a.cut = shared_cut(a.total, kSharedWorkgroups, plan.prefix.short_tiles, plan.prefix.least_tiles, o.total > 0 ? o.cut.used : 0, busy_cost);
  a.first_launch();
  o.first_launch();
  std::vector<int> joined_a[2], joined_o[2], read_a(a.items.size()), read_o(o.items.size());
  for (auto* j : {joined_a, joined_o}) j[0].assign(kSharedWorkgroups, 0), j[1] = j[0];
  for (int row = 0; row < n_rows; ++row)
    for (int h = 0; h < hq; ++h) {
      const int of_own = o.join(row, h, joined_o, read_o), of_prefix = a.join(row, h, joined_a, read_a);
      // who the row's request and group are
      int b = -1, g = -1;
      for (int x = 0; x < n; ++x)
        if (row >= starts[x] && row < starts[x + 1]) b = x;
      for (int x = 0; x < n_groups; ++x)
        if (b >= members[x] && b < members[x + 1]) g = x;
      CHECK(of_own == (b < 0 ? -1 : o.units[b].tiles));
      if (b >= 0) CHECK(of_prefix == (g < 0 ? -1 : a.units[g].tiles));
    }
  // every part that was left is joined by somebody, every item is written, kept or in parts
  for (int slot = 0; slot < 2; ++slot)
    for (int wg = 0; wg < kSharedWorkgroups; ++wg)
      CHECK(joined_a[slot][wg] == (a.part[slot][wg].item >= 0) && joined_o[slot][wg] == (o.part[slot][wg].item >= 0));
  for (size_t i = 0; i < a.items.size(); ++i) CHECK(a.kept[i] <= 1 && a.kept[i] == read_a[i]);
  for (size_t i = 0; i < o.items.size(); ++i) CHECK(o.kept[i] <= 1 && o.kept[i] == read_o[i]);
  // the last word of the last part, and of its statistics
  for (const auto& x : {std::make_pair(RP, prefix_room), std::make_pair(RO, own_room)}) {
    const size_t R = x.first, wgs = kSharedWorkgroups, last = wgs - 1;
    CHECK(((last * 2 + 1) * (R * d) + (R - 1) * d + d) * 4 <= x.second);
    CHECK((wgs * 2 * (R * d) + 1 * (3 * R) * wgs + (2 * R + R - 1) * wgs + last + 1) * 4 <= x.second);
  }
}

int main() {
  for (int k = 0; k < 12; ++k)
    for (int n_groups : {1, 2, 5, 64, 65, 150})
      for (int times : {1, 3})
        for (auto heads : {std::make_pair(2, 1), std::make_pair(8, 2), std::make_pair(21, 3), std::make_pair(4, 4)})
          for (auto rows : {std::make_pair(16, 16), std::make_pair(32, 16), std::make_pair(128, 16), std::make_pair(128, 128)}) {
            if ((k + n_groups + times + heads.first + rows.first + rows.second) % 3) continue;
            replay(n_groups, n_groups * times + below(5), heads.first, heads.second, k % 2 ? 128 : 64, k % 4 == 0 ? 3 : k % 4 == 1 ? 40 : k % 4 == 2 ? 700 : 20000,
                   k % 3 == 0 ? 2 : k % 3 == 1 ? 30 : 900, k % 5 == 0 ? 1 : k % 5 == 1 ? 9 : 3, rows.first, rows.second, below(40));
          }
  printf("replay checks OK\n");
  return 0;
}
