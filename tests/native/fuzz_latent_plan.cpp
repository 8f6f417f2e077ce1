// Plans of the latent attention on random batches: the shares of the workgroups are the units of all tiles once each, every
// query row of every request lies in one tile and the tile's units hold the keys that it sees, no workgroup has more than
// two parts of tiles that it does not have whole, and their places are its own and within the workspace.  Of the expanded
// form: every request has its key tiles and row tiles.
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

#include "efim_internal.h"
#include "latent_plan.h"

using namespace efim;

#define CHECK(x) do { if (!(x)) { printf("line %d: %s\n", __LINE__, #x); return 1; } } while (0)

int main() {
  std::mt19937_64 rng(11);
  long parts = 0, launches = 0, by_tile = 0, one_team = 0, two_teams = 0;
  for (int iter = 0; iter < 4000; ++iter) {
    const int B = (int)(rng() % 8 == 0 ? rng() % 400 : rng() % 24);
    std::vector<int32_t> cached(B), fresh(B);
    const int long_keys = 1 + (int)(rng() % 20000), most_new = 1 + (int)(rng() % (rng() % 3 ? 4 : 300));
    for (int r = 0; r < B; ++r) {
      cached[r] = (int)(rng() % long_keys);
      fresh[r] = (int)(rng() % (most_new + 1));
    }
    efim_batch_t b{};
    b.batch = B;
    const int heads[] = {1, 3, 16, 28, 32, 128, 256};
    b.num_q_heads = heads[rng() % 7];
    b.num_kv_heads = 1;
    b.head_dim = kLatentRow;
    b.page_size = 8 << (rng() % 6);
    b.max_pages_per_req = 40000;
    b.num_pages = 40000;
    b.cached_len = cached.data();
    b.new_len = fresh.data();
    b.block_table = reinterpret_cast<const int32_t*>(0x1000);
    int64_t total = 0;
    CHECK(validate_latent_batch(&b, &total) == EFIM_OK);
    const LatentPlan plan = plan_latent(&b, rng() % 2 ? 256 : 1 + (int)(rng() % 300));
    const LatentBytes bytes = latent_bytes(plan);
    LatentCursor at;
    LatentTable t;
    int expect = 0;
    int64_t row = 0;
    while (latent_next(&b, plan, &at, &t)) {
      ++launches;
      CHECK(t.nreq > 0 && t.nreq <= kLatentTableReqs && t.groups > 0 && t.groups <= plan.units);
      CHECK(t.by_tile || (t.first_unit(0) == 0 && t.first_unit(t.groups) == t.units));
      by_tile += t.by_tile;
      int group = 0, of_group = 0;       // the workgroup at hand, and how many parts of it are done
      std::vector<int> used(plan.slots, 0);
      int64_t unit = 0, longest = t.by_tile ? 0 : t.share + (t.longer > 0);
      for (int k = 0; k < t.nreq; ++k) {
        const LatentReq& q = t.req[k];
        while (fresh[expect] == 0) ++expect;
        CHECK(q.req == expect && q.cached == cached[expect] && q.new_len == fresh[expect] && q.row_start == row && (t.by_tile || q.unit_start == unit));
        const int n = t.by_tile ? (int)(q.unit_start >> 32) : 0;
        CHECK(!t.by_tile || (n > 0 && (int)(uint32_t)q.unit_start == group));
        int rows = 0;
        const int tiles = latent_tiles(q, t.heads, plan.row_tile);
        for (int tile = 0; tile < tiles; ++tile) {
          const int mine = latent_rows_of(q, t.heads, plan.row_tile, tile), units = latent_units_of(q, t.heads, plan.row_tile, tile);
          CHECK(mine > 0 && mine <= plan.row_tile);
          rows += mine;
          const int seen = q.cached + (rows - 1) / t.heads + 1;  // of the last row
          CHECK(latent_keys_of(q, t.heads, plan.row_tile, tile) == seen && units * kLatentTileKeys >= seen && (units - 1) * kLatentTileKeys < seen);
          for (int j = 0; j < n; ++j, ++group) {
            const int from = LatentTable::first_of(units, n, j), to = LatentTable::first_of(units, n, j + 1);
            CHECK(from < to && (j > 0 || from == 0) && (j < n - 1 || to == units));
            if (to - from > longest) longest = to - from;
            if (n > 1) {
              ++parts;
              const int slot = latent_slot(group, true);
              CHECK(slot < plan.slots && !used[slot]++);
            }
          }
          for (int64_t u = unit; !t.by_tile && u < unit + units;) {
            while (t.first_unit(group + 1) <= u) {
              ++group;
              of_group = 0;
            }
            CHECK(group < t.groups && t.first_unit(group) <= u);
            const int64_t end = t.first_unit(group + 1) < unit + units ? t.first_unit(group + 1) : unit + units;
            if (u > unit || end < unit + units) {
              ++parts;
              const int slot = latent_slot(group, of_group == 0);
              CHECK(slot < plan.slots && !used[slot]++);
              CHECK(((size_t)slot + 1) * plan.row_tile * kLatentRank * 2 <= bytes.off_ml && bytes.off_ml + ((size_t)slot + 1) * plan.row_tile * 16 <= bytes.total);
            }
            ++of_group;
            u = end;
          }
          unit += units;
        }
        CHECK(rows == q.new_len * t.heads);
        row += q.new_len;
        ++expect;
      }
      CHECK(unit == t.units && longest == t.longest && group == (t.by_tile ? t.groups : t.groups - 1));
    }
    CHECK(row == total);

    const ExpandedPlan ep = plan_expanded(&b, 256);
    CHECK(ep.ok);
    (ep.teams == 2 ? two_teams : one_team) += 1;
    LatentCursor ea;
    ExpandedTable e;
    expect = 0;
    row = 0;
    while (expanded_next(&b, ep, &ea, &e)) {
      CHECK(e.slices >= 1 && e.slices <= e.key_tiles * kExpandedTileKeys / 32 && e.slices * (int64_t)e.heads <= 4 * 256 + e.heads);
      CHECK(e.key_tiles % 2 == 0 && (size_t)e.key_tiles * b.num_q_heads * kExpandedTileBytes <= ep.bytes);
      for (int k = 0; k < e.nreq; ++k) {
        const LatentReq& q = e.req[k];
        while (fresh[expect] == 0) ++expect;
        CHECK(q.req == expect && q.row_start == row);
        const int64_t key_tiles = (k + 1 < e.nreq ? e.req[k + 1].unit_start : e.key_tiles) - q.unit_start;
        const int row_tiles = (k + 1 < e.nreq ? e.row_tile_start[k + 1] : e.row_tiles) - e.row_tile_start[k];
        CHECK(key_tiles % 2 == 0 && key_tiles * kExpandedTileKeys >= q.cached + q.new_len && (key_tiles - 2) * kExpandedTileKeys < q.cached + q.new_len);
        CHECK(row_tiles == (q.new_len + kExpandedRowTile - 1) / kExpandedRowTile);
        row += q.new_len;
        ++expect;
      }
    }
    CHECK(row == total);
  }
  CHECK(parts > 0 && by_tile > 0 && by_tile < launches && one_team > 0 && two_teams > 0);
  printf("latent plan ok, %ld launches, %ld parts\n", launches, parts);
  return 0;
}
