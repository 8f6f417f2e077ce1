// Plans of the latent attention on random batches: every query row of every request lies in one tile, the ranges of a tile
// cover the keys that it sees once each, partial results have places of their own within the workspace, and no launch is
// beyond what a grid takes.  Of the expanded form: every request has its key tiles and row tiles.
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
  long split = 0, launches = 0, tiles128 = 0, tiles256 = 0;
  for (int iter = 0; iter < 6000; ++iter) {
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
    const LatentPlan plan = plan_latent(&b, 256);
    const LatentBytes bytes = latent_bytes(plan);
    CHECK(plan.range > 0 && plan.range % kLatentRangeStep == 0);
    LatentCursor at;
    LatentTable t;
    int expect = 0;
    int64_t row = 0;
    while (latent_next(&b, plan, &at, &t)) {
      ++launches;
      CHECK(t.nreq <= kLatentTableReqs && t.items > 0 && (int64_t)t.items * 256 <= INT32_MAX);
      std::vector<char> used(plan.slots, 0);
      int item = 0;
      for (int k = 0; k < t.nreq; ++k) {
        const LatentReq& q = t.req[k];
        while (fresh[expect] == 0) ++expect;
        CHECK(q.req == expect && q.cached == cached[expect] && q.new_len == fresh[expect] && q.row_start == row && q.item_start == item);
        const int end = k + 1 < t.nreq ? t.req[k + 1].item_start : t.items;
        int rows = 0, keys = 0, whole = 0;  // of the tile at hand
        for (; item < end; ++item) {
          const LatentItem it = latent_item(t, q, item, plan.row_tile);
          if (it.row0 != rows - whole) {  // the next tile
            CHECK(it.row0 == rows);
          }
          if (it.k0 == 0) {
            CHECK(it.row0 == rows);
            whole = it.rows;
            rows += it.rows;
            keys = 0;
          }
          CHECK(it.rows > 0 && it.rows <= plan.row_tile && it.row0 + it.rows == rows);
          const int key_end = q.cached + (rows - 1) / b.num_q_heads + 1;
          if (it.k0 < it.k1) {
            CHECK(it.k0 == keys && it.k1 <= key_end);
            keys = it.k1;
          } else {
            CHECK(keys == key_end);
          }
          if (it.slot >= 0) {
            ++split;
            CHECK(it.slot < plan.slots && !used[it.slot]);
            used[it.slot] = 1;
            CHECK(((size_t)it.slot + 1) * plan.row_tile * kLatentRank * 4 <= bytes.off_ml);
            CHECK(bytes.off_ml + ((size_t)it.slot + 1) * plan.row_tile * 8 <= bytes.total);
            CHECK(t.split_rows >= q.new_len * b.num_q_heads);
          }
          const LatentItem next = item + 1 < end ? latent_item(t, q, item + 1, plan.row_tile) : LatentItem{-1, 0, 0, 0, 0};
          if (next.row0 != it.row0) CHECK(keys == key_end);
        }
        CHECK(rows == q.new_len * b.num_q_heads);
        row += q.new_len;
        ++expect;
      }
      CHECK(item == t.items);
    }
    CHECK(row == total);

    const ExpandedPlan ep = plan_expanded(&b, 256);
    CHECK(ep.ok);
    (ep.row_tile == 256 ? tiles256 : tiles128) += 1;
    LatentCursor ea;
    int row_items = 0;
    expect = 0;
    row = 0;
    while (expanded_next(&b, ep, &ea, &t, &row_items)) {
      CHECK(t.items % 2 == 0 && (size_t)t.items * b.num_q_heads * kExpandedTileBytes <= ep.bytes);
      for (int k = 0; k < t.nreq; ++k) {
        const LatentReq& q = t.req[k];
        while (fresh[expect] == 0) ++expect;
        CHECK(q.req == expect && q.row_start == row);
        const int key_tiles = (k + 1 < t.nreq ? t.req[k + 1].slot_start : t.items) - q.slot_start;
        const int row_tiles = (k + 1 < t.nreq ? t.req[k + 1].item_start : row_items) - q.item_start;
        CHECK(key_tiles % 2 == 0 && key_tiles * kExpandedTileKeys >= q.cached + q.new_len && (key_tiles - 2) * kExpandedTileKeys < q.cached + q.new_len);
        CHECK(row_tiles == (q.new_len + ep.row_tile - 1) / ep.row_tile);
        row += q.new_len;
        ++expect;
      }
    }
    CHECK(row == total);
  }
  CHECK(split > 0 && tiles128 > 0 && tiles256 > 0);
  printf("latent plan ok, %ld launches, %ld parts\n", launches, split);
  return 0;
}
