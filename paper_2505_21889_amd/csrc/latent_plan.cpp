// Work items of the absorbed latent attention (host code).
#include "latent_plan.h"

#include "efim_internal.h"

namespace efim {

namespace {

struct Count {
  int64_t items = 0, slots = 0;
};

// Items of the whole batch with key ranges of `range`.
Count count_items(const efim_batch_t* b, int row_tile, int range) {
  Count n;
  for (int r = 0; r < b->batch; ++r) {
    if (b->new_len[r] == 0) continue;
    const int64_t tiles = ((int64_t)b->new_len[r] * b->num_q_heads + row_tile - 1) / row_tile;
    const int splits = latent_splits(b->cached_len[r] + b->new_len[r], range);
    n.items += tiles * splits;
    if (splits > 1) n.slots += tiles * splits;
  }
  return n;
}

}  // namespace

LatentPlan plan_latent(const efim_batch_t* b, int units) {
  LatentPlan plan;
  int64_t most_rows = 0, most_keys = 0;
  for (int r = 0; r < b->batch; ++r) {
    if (b->new_len[r] == 0) continue;
    const int64_t rows = (int64_t)b->new_len[r] * b->num_q_heads, keys = (int64_t)b->cached_len[r] + b->new_len[r];
    most_rows = rows > most_rows ? rows : most_rows;
    most_keys = keys > most_keys ? keys : most_keys;
  }
  plan.row_tile = most_rows <= 16 ? 16 : most_rows <= 32 ? 32 : 128;
  const int64_t whole = (most_keys + kLatentRangeStep - 1) / kLatentRangeStep;  // steps of the longest request
  if (whole == 0) {
    plan.range = kLatentRangeStep;
    return plan;
  }
  // A unit runs one item at a time.  For one, two, three ... items a unit the shortest range that leaves no more items
  // than that; the best is where they, with what an item costs beside its keys, end first.
  constexpr int64_t kItemSteps = 2;
  int64_t best_cost = -1;
  for (int64_t rounds = 1; rounds <= 4; ++rounds) {
    int64_t lo = 1, hi = whole;
    while (lo < hi) {
      const int64_t mid = (lo + hi) / 2;
      if (count_items(b, plan.row_tile, (int)(mid * kLatentRangeStep)).items <= rounds * units) hi = mid;
      else lo = mid + 1;
    }
    const int64_t items = count_items(b, plan.row_tile, (int)(lo * kLatentRangeStep)).items;
    const int64_t cost = (items + units - 1) / units * (lo + kItemSteps);
    if (best_cost < 0 || cost < best_cost) {
      best_cost = cost;
      plan.range = (int)(lo * kLatentRangeStep);
    }
  }
  plan.slots = count_items(b, plan.row_tile, plan.range).slots;
  return plan;
}

LatentBytes latent_bytes(const LatentPlan& plan) {
  LatentBytes at;
  at.off_ml = (size_t)plan.slots * plan.row_tile * kLatentRank * sizeof(float);
  at.total = at.off_ml + (size_t)plan.slots * plan.row_tile * 2 * sizeof(float);
  return at;
}

bool latent_next(const efim_batch_t* b, const LatentPlan& plan, LatentCursor* at, LatentTable* t) {
  t->nreq = 0;
  t->heads = b->num_q_heads;
  t->range = plan.range;
  t->max_pages = b->max_pages_per_req;
  t->page_shift = 0;
  while ((1 << t->page_shift) < b->page_size) ++t->page_shift;
  t->split_rows = 0;
  int64_t items = 0, slots = 0;
  for (; at->req < b->batch && t->nreq < kLatentTableReqs; ++at->req) {
    const int n = b->new_len[at->req];
    if (n == 0) continue;
    const int64_t rows = (int64_t)n * b->num_q_heads, tiles = (rows + plan.row_tile - 1) / plan.row_tile;
    const int splits = latent_splits(b->cached_len[at->req] + n, plan.range);
    if (items + tiles * splits > INT32_MAX / (64 * 4)) break;  // threads of a launch
    t->req[t->nreq++] = LatentReq{at->req, b->cached_len[at->req], n, (int32_t)at->row, (int32_t)items, (int32_t)slots};
    items += tiles * splits;
    if (splits > 1) {
      slots += tiles * splits;
      if (rows > t->split_rows) t->split_rows = (int32_t)rows;
    }
    at->row += n;
  }
  t->items = (int32_t)items;
  return t->nreq > 0;
}

ExpandedPlan plan_expanded(const efim_batch_t* b, int units) {
  ExpandedPlan plan;
  // 256 rows share a gathered tile once more than 128 do, 128 leave more workgroups and less of a short last tile empty:
  // the larger one where it still leaves every unit two of them.
  int64_t large = 0;
  for (int r = 0; r < b->batch; ++r) large += ((int64_t)b->new_len[r] + 255) / 256 * b->num_q_heads;
  plan.row_tile = large >= 2 * (int64_t)units ? 256 : 128;
  plan.ok = true;
  LatentTable table;
  LatentCursor at;
  int row_items = 0;
  while (expanded_next(b, plan, &at, &table, &row_items)) {
    const int64_t heads = b->num_q_heads;
    // (a request alone can pass the limit of threads of a launch)
    if ((int64_t)table.items / 2 * heads > INT32_MAX / 512 || row_items * heads > INT32_MAX / 512) plan.ok = false;
    const size_t bytes = (size_t)table.items * (size_t)heads * kExpandedTileBytes;
    if (bytes > plan.bytes) plan.bytes = bytes;
  }
  return plan;
}

bool expanded_next(const efim_batch_t* b, const ExpandedPlan& plan, LatentCursor* at, LatentTable* t, int* row_items) {
  t->nreq = 0;
  t->heads = b->num_q_heads;
  t->range = 0;
  t->split_rows = 0;
  t->max_pages = b->max_pages_per_req;
  t->page_shift = 0;
  while ((1 << t->page_shift) < b->page_size) ++t->page_shift;
  int64_t key_tiles = 0, row_tiles = 0;
  for (; at->req < b->batch && t->nreq < kLatentTableReqs; ++at->req) {
    const int n = b->new_len[at->req];
    if (n == 0) continue;
    const int64_t more_keys = ((int64_t)b->cached_len[at->req] + n + 2 * kExpandedTileKeys - 1) / (2 * kExpandedTileKeys) * 2;
    const int64_t more_rows = ((int64_t)n + plan.row_tile - 1) / plan.row_tile;
    if (t->nreq > 0 && ((key_tiles + more_keys) * b->num_q_heads > INT32_MAX / 512 ||
                        (row_tiles + more_rows) * b->num_q_heads > INT32_MAX / 512))
      break;
    t->req[t->nreq++] = LatentReq{at->req, b->cached_len[at->req], n, (int32_t)at->row, (int32_t)row_tiles, (int32_t)key_tiles};
    key_tiles += more_keys;
    row_tiles += more_rows;
    at->row += n;
  }
  t->items = (int32_t)key_tiles;
  *row_items = (int)row_tiles;
  return t->nreq > 0;
}

}  // namespace efim
