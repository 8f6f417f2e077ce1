// Work of the latent attention (host code).
#include "latent_plan.h"

#include "efim_internal.h"

namespace efim {

namespace {

int page_shift_of(const efim_batch_t* b) {
  int shift = 0;
  while ((1 << shift) < b->page_size) ++shift;
  return shift;
}

// Units of all tiles of a request.
int64_t units_of(const LatentReq& q, int heads, int row_tile) {
  int64_t n = 0;
  for (int tile = latent_tiles(q, heads, row_tile) - 1; tile >= 0; --tile) n += latent_units_of(q, heads, row_tile, tile);
  return n;
}

// Deals by tile where that shortens the longest workgroup.  Dealt evenly most have two parts, and a part costs its rows' queries
// and outputs besides its units: about as much as kPartUnits.  us evenly and by tile, 32 requests and 256 workgroups: 16 heads
// and 1k to 8k keys 49 / 43, 128 heads and 0.5k to 4k keys 64 / 53.
void deal_by_tile(LatentTable* t, int row_tile) {
  const int64_t kPartUnits = row_tile == 128 ? 6 : 3;
  int tiles[kLatentTableReqs], least[kLatentTableReqs], most[kLatentTableReqs];  // units of a request's first and last tile
  int64_t all = 0;
  int longest = 0;
  for (int r = 0; r < t->nreq; ++r) {
    tiles[r] = latent_tiles(t->req[r], t->heads, row_tile);
    least[r] = latent_units_of(t->req[r], t->heads, row_tile, 0);
    most[r] = latent_units_of(t->req[r], t->heads, row_tile, tiles[r] - 1);
    longest = most[r] > longest ? most[r] : longest;
    all += tiles[r];
  }
  t->by_tile = 0;
  if (all > t->groups) return;
  // the least number of units, at least four, by which the parts are no more than the workgroups
  auto parts_of = [&](int r, int units) {
    const int n = (most[r] + units - 1) / units;
    return n < least[r] ? n : least[r];
  };
  int low = 4, high = longest < 4 ? 4 : longest;
  while (low < high) {
    const int middle = (low + high) / 2;
    int64_t groups = 0;
    for (int r = 0; r < t->nreq; ++r) groups += (int64_t)tiles[r] * parts_of(r, middle);
    if (groups <= t->groups) high = middle;
    else low = middle + 1;
  }
  int worst = 0;
  int64_t groups = 0;
  for (int r = 0; r < t->nreq; ++r) {
    const int n = parts_of(r, low), units = (most[r] + n - 1) / n;
    worst = units > worst ? units : worst;
    groups += (int64_t)tiles[r] * n;
  }
  if (groups > t->groups || worst >= t->share + (t->longer > 0) + kPartUnits) return;
  t->by_tile = 1;
  t->longest = worst;
  groups = 0;
  for (int r = 0; r < t->nreq; ++r) {
    const int64_t n = parts_of(r, low);
    t->req[r].unit_start = groups | n << 32;
    groups += tiles[r] * n;
  }
  t->groups = (int32_t)groups;
}

}  // namespace

LatentPlan plan_latent(const efim_batch_t* b, int units) {
  LatentPlan plan;
  int64_t most_rows = 0;
  for (int r = 0; r < b->batch; ++r) {
    const int64_t rows = (int64_t)b->new_len[r] * b->num_q_heads;
    most_rows = rows > most_rows ? rows : most_rows;
  }
  // The least tile that holds the longest request: empty rows are multiplied too.  us with 16 / 32 / 128 rows, 32 requests of 1k to
  // 8k keys: 16 rows 39 / 47 / 61, 32 rows - / 49 / 59; one request of 2344 keys: 16 rows 17 / 22 / 23, 28 rows - / 24 / 24.
  plan.row_tile = most_rows <= 16 ? 16 : most_rows <= 32 ? 32 : 128;
  plan.units = units;
  plan.slots = 2 * units;
  return plan;
}

LatentBytes latent_bytes(const LatentPlan& plan) {
  LatentBytes at;
  at.off_ml = (size_t)plan.slots * plan.row_tile * kLatentRank * sizeof(uint16_t);
  at.total = at.off_ml + (size_t)plan.slots * plan.row_tile * 4 * sizeof(float);
  return at;
}

bool latent_next(const efim_batch_t* b, const LatentPlan& plan, LatentCursor* at, LatentTable* t) {
  t->nreq = 0;
  t->heads = b->num_q_heads;
  t->max_pages = b->max_pages_per_req;
  t->page_shift = page_shift_of(b);
  t->units = 0;
  for (; at->req < b->batch && t->nreq < kLatentTableReqs; ++at->req) {
    const int n = b->new_len[at->req];
    if (n == 0) continue;
    LatentReq& q = t->req[t->nreq++];
    q = LatentReq{t->units, at->req, b->cached_len[at->req], n, (int32_t)at->row};
    t->units += units_of(q, t->heads, plan.row_tile);
    at->row += n;
  }
  // Four units to a workgroup at least, one for each wave: fewer cost more in starting and joining than they shorten.  us with 2, 4, 6
  // and 8 of 128 rows: one request of 8000 keys 41 / 33 / 32 / 33, two of 2000 24 / 24 / 27 / 27, 11 of 660 23 / 24 / 27 / 32, 8 of 64 rows
  // and 2000 keys 31 / 28 / 29 / 31.
  const int64_t most = (t->units + 3) / 4;
  t->groups = (int32_t)(most < plan.units ? most : plan.units);
  if (t->nreq == 0) return false;
  t->share = t->units / t->groups;
  t->longer = (int32_t)(t->units - t->share * t->groups);
  t->longest = t->share + (t->longer > 0);
  deal_by_tile(t, plan.row_tile);
  return true;
}

// Slices of a head's `keys` units of 32 keys, a workgroup each: the number by which the device's rounds of workgroups take
// least, where a workgroup spends about as long on its weight as on kWeightUnits units.
static int expanded_slices(int64_t keys, int64_t heads, int units) {
  constexpr int64_t kWeightUnits = 4;
  int64_t best = 1, best_cost = INT64_MAX;
  const int64_t most = 4 * (int64_t)units / heads + 1;
  for (int64_t s = 1; s <= most && s <= keys; ++s) {
    const int64_t cost = (heads * s + units - 1) / units * ((keys + s - 1) / s + kWeightUnits);
    if (cost < best_cost) best = s, best_cost = cost;
  }
  return (int)best;
}

ExpandedPlan plan_expanded(const efim_batch_t* b, int units) {
  ExpandedPlan plan;
  plan.units = units;
  // Two teams to a workgroup, which halve its keys, while there are no more than two workgroups for each unit: then the longest
  // workgroup or the second round of them sets the time.  Beyond, one team, two workgroups to a unit.  us with two and one
  // (256 units): 64 workgroups of 3400 keys 87 / 104, 304 of up to 2355 70 / 80, 512 122 / 138, 608 168 / 167, 928 201 / 174.
  int64_t groups = 0;
  for (int r = 0; r < b->batch; ++r) groups += ((int64_t)b->new_len[r] + kExpandedRowTile - 1) / kExpandedRowTile * b->num_q_heads;
  plan.teams = groups > 2 * (int64_t)units ? 1 : 2;
  plan.ok = true;
  ExpandedTable table;
  LatentCursor at;
  while (expanded_next(b, plan, &at, &table)) {
    const int64_t heads = b->num_q_heads;
    // (a request alone can pass the limit of threads of a launch)
    if ((int64_t)table.key_tiles / 2 * heads > INT32_MAX / 512 || table.row_tiles * heads > INT32_MAX / 512) plan.ok = false;
    const size_t bytes = (size_t)table.key_tiles * (size_t)heads * kExpandedTileBytes;
    if (bytes > plan.bytes) plan.bytes = bytes;
  }
  return plan;
}

bool expanded_next(const efim_batch_t* b, const ExpandedPlan& plan, LatentCursor* at, ExpandedTable* t) {
  t->nreq = 0;
  t->heads = b->num_q_heads;
  t->max_pages = b->max_pages_per_req;
  t->page_shift = page_shift_of(b);
  int64_t key_tiles = 0, row_tiles = 0;
  for (; at->req < b->batch && t->nreq < kLatentTableReqs; ++at->req) {
    const int n = b->new_len[at->req];
    if (n == 0) continue;
    const int64_t more_keys = ((int64_t)b->cached_len[at->req] + n + 2 * kExpandedTileKeys - 1) / (2 * kExpandedTileKeys) * 2;
    const int64_t more_rows = ((int64_t)n + kExpandedRowTile - 1) / kExpandedRowTile;
    if (t->nreq > 0 && ((key_tiles + more_keys) * b->num_q_heads > INT32_MAX / 512 ||
                        (row_tiles + more_rows) * b->num_q_heads > INT32_MAX / 512))
      break;
    t->row_tile_start[t->nreq] = (int32_t)row_tiles;
    t->req[t->nreq++] = LatentReq{key_tiles, at->req, b->cached_len[at->req], n, (int32_t)at->row};
    key_tiles += more_keys;
    row_tiles += more_rows;
    at->row += n;
  }
  t->key_tiles = (int32_t)key_tiles;
  t->slices = t->nreq > 0 ? expanded_slices(key_tiles * 2, b->num_q_heads, plan.units) : 0;
  t->row_tiles = (int32_t)row_tiles;
  return t->nreq > 0;
}

}  // namespace efim
