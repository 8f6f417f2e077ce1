// Plans of the attention over a 4-bit cache against a walk over what their workgroups do: every key that a tile of rows sees belongs to
// one part of it, partial results have places of their own, and what the join is told leads to all of a tile's parts.
#include <cstdio>
#include <cstdlib>
#include <map>
#include <random>
#include <set>
#include <tuple>
#include <vector>

#include "mx4_plan.h"

using namespace efim;

#define CHECK(x)                                                  \
  do {                                                            \
    if (!(x)) {                                                   \
      std::printf("%s:%d: %s (seed %d)\n", __FILE__, __LINE__, #x, g_seed); \
      std::exit(1);                                               \
    }                                                             \
  } while (0)
static int g_seed;

using Tile = std::tuple<int, int, int>;  // block table row, head, tile
using Keys = std::map<Tile, int64_t>;    // keys that are done, from the first one on

template <int MAXREQ>
static void walk_few(const efim_batch_t& b, const Mx4FewPlan& plan, std::map<int, int>* launched) {
  Mx4Cursor at;
  Mx4FewTable<MAXREQ> t;
  while (mx4_next(&b, plan, &at, &t)) {
    CHECK(t.nreq > 0 && t.nreq <= MAXREQ && t.slots <= plan.slots && t.groups <= kMx4MostGroups);
    int group = 0, splits = 0, slots = 0;
    for (int k = 0; k < t.nreq; ++k) {
      const int r = t.req[k];
      CHECK(!(*launched)[r]++ && t.cached[k] == b.cached_len[r] && t.new_len[k] == b.new_len[r]);
      int64_t rows = 0;
      for (int i = 0; i < r; ++i) rows += b.new_len[i];
      CHECK(t.row_start[k] == rows && t.new_len[k] * t.group_heads <= plan.row_tile);
      CHECK(t.group_start[k] == group && t.split_start[k] == splits && t.slot_start[k] == slots);
      const int keys = t.cached[k] + t.new_len[k], units = (keys + kMx4FewKeys - 1) / kMx4FewKeys, parts = t.parts[k];
      CHECK(parts >= 1 && parts <= units);
      CHECK(mx4_first_of(units, parts, 0) == 0 && mx4_first_of(units, parts, parts) == units);
      for (int j = 0; j < parts; ++j) {
        const int of_part = mx4_first_of(units, parts, j + 1) - mx4_first_of(units, parts, j);
        CHECK(of_part >= 1 && of_part <= plan.part_units);
      }
      group += parts * t.kv_heads;
      if (parts > 1) {
        splits += t.kv_heads;
        slots += parts * t.kv_heads;
      }
    }
    CHECK(t.groups == group && t.splits == splits && t.slots == slots);
  }
}

// The tile at a place of the order by length, as a wave looks for it.
static Tile nth_tile(const Mx4Table& t, int n, int* units) {
  auto of_all = [&](int c) {
    int all = 0;
    for (int k = 0; k < t.nreq; ++k) all += t.kv_heads * mx4_tiles_from(t.req[k], t.group_heads, kMx4ManyRows, t.unit_shift, c);
    return all;
  };
  int low = 1, high = t.most_units + 1;
  while (high - low > 1) {
    const int middle = low + (high - low) / 2;
    (of_all(middle) > n ? low : high) = middle;
  }
  int in = n - of_all(high);
  *units = low;
  for (int k = 0; k < t.nreq; ++k) {
    const Mx4Req& q = t.req[k];
    const int from = mx4_tiles_from(q, t.group_heads, kMx4ManyRows, t.unit_shift, low);
    const int mine = t.kv_heads * (from - mx4_tiles_from(q, t.group_heads, kMx4ManyRows, t.unit_shift, high));
    if (in < mine) return {k, in % t.kv_heads, mx4_tiles(q, t.group_heads, kMx4ManyRows) - from + in / t.kv_heads};
    in -= mine;
  }
  CHECK(!"a tile for each place");
  return {};
}

static int g_ways[3];  // launches of whole tiles, of one unit and of several to a workgroup

static void walk_many(const efim_batch_t& b, const Mx4ManyPlan& plan, std::map<int, int>* launched) {
  Mx4Cursor at;
  Mx4Table t;
  while (mx4_next(&b, plan, &at, &t)) {
    const int g = t.group_heads;
    std::vector<Tile> order;  // as the units lie
    std::vector<int64_t> starts;
    int64_t units = 0;
    for (int k = 0; k < t.nreq; ++k) {
      const Mx4Req& q = t.req[k];
      CHECK(!(*launched)[q.req]++ && q.cached == b.cached_len[q.req] && q.new_len == b.new_len[q.req]);
      CHECK(t.by_tile || q.unit_start == units);
      for (int h = 0; h < t.kv_heads; ++h) {
        const int64_t before = units;
        for (int tile = 0; tile < mx4_tiles(q, g, kMx4ManyRows); ++tile) {
          order.push_back({k, h, tile});
          starts.push_back(units);
          units += mx4_units_of(q, g, kMx4ManyRows, t.unit_shift, tile);
        }
        CHECK(q.units_per_head == units - before);
      }
    }
    if (t.by_tile) {
      ++g_ways[0];
      CHECK(t.groups == (int)order.size());
      std::set<Tile> seen;
      int last = t.most_units;
      for (int n = 0; n < t.groups; ++n) {
        int length = 0;
        const Tile tile = nth_tile(t, n, &length);
        const Mx4Req& q = t.req[std::get<0>(tile)];
        CHECK(std::get<2>(tile) >= 0 && std::get<2>(tile) < mx4_tiles(q, g, kMx4ManyRows));
        CHECK(length == mx4_units_of(q, g, kMx4ManyRows, t.unit_shift, std::get<2>(tile)) && length <= last);
        CHECK(seen.insert(tile).second);
        last = length;
      }
      continue;
    }
    ++g_ways[t.share == 1 && t.longer == 0 && t.unit_shift > kMx4ManyShift ? 1 : 2];
    CHECK(t.groups >= 1 && t.groups <= plan.places && t.first_unit(0) == 0 && t.first_unit(t.groups) == units);
    std::set<int64_t> slots;
    std::map<size_t, std::vector<int64_t>> parts;  // slots of split tiles
    std::map<size_t, std::pair<int, int>> told;    // the first and the last workgroup
    Keys done;
    size_t i = 0;
    for (int group = 0; group < t.groups; ++group) {
      const int64_t end = t.first_unit(group + 1);
      int64_t begin = t.first_unit(group);
      CHECK(begin < end);
      while (begin < end) {
        while (i + 1 < order.size() && starts[i + 1] <= begin) ++i;
        const Mx4Req& q = t.req[std::get<0>(order[i])];
        const int tile = std::get<2>(order[i]), length = mx4_units_of(q, g, kMx4ManyRows, t.unit_shift, tile);
        const int64_t u0 = begin - starts[i], u1 = std::min<int64_t>(length, end - starts[i]);
        CHECK(u0 >= 0 && u1 > u0 && done[order[i]] == u0 << t.unit_shift);
        done[order[i]] = std::min<int64_t>(u1 << t.unit_shift, mx4_keys_of(q, g, kMx4ManyRows, tile));
        if (u0 > 0 || u1 < length) {
          const int64_t slot = mx4_slot(group, u0 > 0);
          CHECK(slot < (int64_t)plan.slots && slots.insert(slot).second);
          parts[i].push_back(slot);
          if (u0 == 0) {
            CHECK(starts[i] + length >= end);
            int last = group;
            while (last + 1 < t.groups && t.first_unit(last + 1) < starts[i] + length) ++last;
            told[i] = {group, last};
          }
        }
        begin = starts[i] + length;
      }
    }
    for (const Tile& tile : order) CHECK(done[tile] == mx4_keys_of(t.req[std::get<0>(tile)], g, kMx4ManyRows, std::get<2>(tile)));
    CHECK(parts.size() == told.size());
    std::set<int> firsts;
    for (auto& [k, of] : parts) {
      CHECK(firsts.insert(told[k].first).second && told[k].first < t.groups - 1);
      std::vector<int64_t> joined;
      for (int group = told[k].first; group <= told[k].second; ++group) joined.push_back(mx4_slot(group, group > told[k].first));
      CHECK(joined == of);
    }
  }
}

int main() {
  for (g_seed = 0; g_seed < 1500; ++g_seed) {
    std::mt19937 rng(g_seed);
    auto upto = [&](int n) { return (int)(rng() % (unsigned)(n + 1)); };
    const int heads[][2] = {{4, 4}, {28, 4}, {32, 8}, {8, 1}, {64, 1}, {3, 3}, {33, 1}, {1, 1}};
    const auto& h = heads[upto(7)];
    const int batch = upto(8) == 0 ? upto(260) : upto(40), long_new = upto(2) == 0 ? 700 : 60, long_past = upto(1) ? 300 : 20000;
    std::vector<int32_t> cached(batch), fresh(batch);
    for (int r = 0; r < batch; ++r) {
      cached[r] = upto(3) == 0 ? 0 : upto(long_past);
      fresh[r] = upto(5) == 0 ? 0 : 1 + upto(upto(1) ? 5 : long_new);
    }
    efim_batch_t b{};
    b.batch = batch;
    b.cached_len = cached.data();
    b.new_len = fresh.data();
    b.num_q_heads = h[0];
    b.num_kv_heads = h[1];
    b.head_dim = 128;
    b.page_size = 16;
    b.max_pages_per_req = 2000;
    const int units[] = {1, 8, 256, 304};
    const int cus = units[upto(3)];
    std::map<int, int> launched;
    const Mx4FewPlan few = plan_mx4_few(&b, cus);
    if (few.any) upto(1) ? walk_few<64>(b, few, &launched) : walk_few<kMx4FewReqs>(b, few, &launched);
    const Mx4ManyPlan many = plan_mx4_many(&b, cus);
    if (many.any) walk_many(b, many, &launched);
    for (int r = 0; r < batch; ++r) CHECK(launched.count(r) == (fresh[r] > 0));
  }
  CHECK(g_ways[0] > 50 && g_ways[1] > 50 && g_ways[2] > 50);
  std::printf("4-bit plan ok\n");
  return 0;
}
