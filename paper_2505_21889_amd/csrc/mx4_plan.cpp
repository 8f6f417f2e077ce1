// Work of the attention over a 4-bit cache (host code).
#include "mx4_plan.h"

#include "efim_internal.h"

namespace efim {

namespace {

int group_of(const efim_batch_t* b) { return b->num_q_heads / b->num_kv_heads; }
bool is_few(const efim_batch_t* b, int r) { return b->new_len[r] > 0 && (int64_t)b->new_len[r] * group_of(b) <= kMx4FewRows; }
bool is_many(const efim_batch_t* b, int r) { return (int64_t)b->new_len[r] * group_of(b) > kMx4FewRows; }
int page_shift_of(const efim_batch_t* b) {
  int shift = 0;
  while ((1 << shift) < b->page_size) ++shift;
  return shift;
}

// Units of a request of few rows, and its parts of at most `most` of them.
int few_units(const efim_batch_t* b, int r) {
  return (int)(((int64_t)b->cached_len[r] + b->new_len[r] + kMx4FewKeys - 1) / kMx4FewKeys);
}
int few_parts(const efim_batch_t* b, int r, int most) { return (few_units(b, r) + most - 1) / most; }

}  // namespace

Mx4FewPlan plan_mx4_few(const efim_batch_t* b, int compute_units) {
  Mx4FewPlan plan;
  int64_t most = 0, units = 0, tiles = 0;
  int longest = 1;
  for (int r = 0; r < b->batch; ++r) {
    if (!is_few(b, r)) continue;
    plan.any = true;
    const int64_t rows = (int64_t)b->new_len[r] * group_of(b);
    most = rows > most ? rows : most;
    const int mine = few_units(b, r);
    longest = mine > longest ? mine : longest;
    units += (int64_t)mine * b->num_kv_heads;
    tiles += b->num_kv_heads;
  }
  if (!plan.any) return plan;
  plan.row_tile = most <= 16 ? 16 : 32;
  // Two workgroups to a compute unit, none longer than it has to be; where the tiles alone are more than those, the ones of more than
  // the mean work of a place are cut.  us with one, two, three and six: 32 requests of 2048..8192 keys and a token, 28/4 heads 28.5 / 24.5
  // / 25.1 / 28.0, 16 of 1024..4096 and 24 rows 23.6 / 21.2 / 24.3 / 30.7.  Parts of two units at least: with one even a step of short
  // requests has a join (5.7 -> 9.2); one request of 2344 keys takes the same with one, two and three.
  constexpr int kLeastUnits = 2;
  const int64_t places = 2 * (int64_t)compute_units;
  int low = kLeastUnits, high = longest > low ? longest : low;
  if (tiles >= places) {
    low = high = (int)((units + places - 1) / places);
  }
  while (low < high) {
    const int middle = (low + high) / 2;
    int64_t groups = 0;
    for (int r = 0; r < b->batch; ++r)
      if (is_few(b, r)) groups += (int64_t)few_parts(b, r, middle) * b->num_kv_heads;
    if (groups <= places) high = middle;
    else low = middle + 1;
  }
  plan.part_units = low;
  Mx4Cursor at;
  Mx4FewTable<kMx4FewReqs> t;
  while (mx4_next(b, plan, &at, &t)) plan.slots = t.slots > plan.slots ? t.slots : plan.slots;
  return plan;
}

Mx4ManyPlan plan_mx4_many(const efim_batch_t* b, int compute_units) {
  Mx4ManyPlan plan;
  for (int r = 0; r < b->batch; ++r) plan.any = plan.any || is_many(b, r);
  if (!plan.any) return plan;
  plan.places = 2 * compute_units;
  Mx4Cursor at;
  Mx4Table t;
  while (mx4_next(b, plan, &at, &t))
    if (!t.by_tile && 2 * (size_t)t.groups > plan.slots) plan.slots = 2 * (size_t)t.groups;
  return plan;
}

Mx4Bytes mx4_bytes(size_t slots, int row_tile, int head_dim) {
  Mx4Bytes at;
  const size_t rows = slots * row_tile;
  at.off_ml = rows * head_dim * sizeof(float);
  at.total = (at.off_ml + rows * 2 * sizeof(float) + 255) / 256 * 256;
  return at;
}

template <int MAXREQ>
bool mx4_next(const efim_batch_t* b, const Mx4FewPlan& plan, Mx4Cursor* at, Mx4FewTable<MAXREQ>* t) {
  t->nreq = t->groups = t->splits = t->slots = 0;
  t->kv_heads = b->num_kv_heads;
  t->group_heads = group_of(b);
  t->max_pages = b->max_pages_per_req;
  t->page_shift = page_shift_of(b);
  for (; at->req < b->batch && t->nreq < MAXREQ; ++at->req) {
    const int r = at->req;
    if (is_few(b, r)) {
      const int n = few_parts(b, r, plan.part_units);
      const int64_t groups = (int64_t)n * t->kv_heads;
      if (t->nreq > 0 && t->groups + groups > kMx4MostGroups) break;  // (a request alone has fewer than 2^30)
      const int k = t->nreq++;
      t->group_start[k] = t->groups;
      t->parts[k] = n;
      t->split_start[k] = t->splits;
      t->slot_start[k] = t->slots;
      t->req[k] = r;
      t->cached[k] = b->cached_len[r];
      t->new_len[k] = b->new_len[r];
      t->row_start[k] = (int32_t)at->row;
      t->groups += (int32_t)groups;
      if (n > 1) {
        t->splits += t->kv_heads;
        t->slots += (int32_t)groups;
      }
    }
    at->row += b->new_len[r];
  }
  return t->nreq > 0;
}
template bool mx4_next<64>(const efim_batch_t*, const Mx4FewPlan&, Mx4Cursor*, Mx4FewTable<64>*);
template bool mx4_next<kMx4FewReqs>(const efim_batch_t*, const Mx4FewPlan&, Mx4Cursor*, Mx4FewTable<kMx4FewReqs>*);

bool mx4_next(const efim_batch_t* b, const Mx4ManyPlan& plan, Mx4Cursor* at, Mx4Table* t) {
  t->nreq = t->most_units = 0;
  t->kv_heads = b->num_kv_heads;
  t->group_heads = group_of(b);
  t->max_pages = b->max_pages_per_req;
  t->page_shift = page_shift_of(b);
  t->unit_shift = kMx4ManyShift;
  const int g = t->group_heads;
  int64_t units = 0, tiles = 0;
  int least = INT32_MAX;
  for (; at->req < b->batch && t->nreq < kMx4TableReqs; ++at->req) {
    const int n = b->new_len[at->req];
    if (is_many(b, at->req)) {
      Mx4Req& q = t->req[t->nreq++];
      q = Mx4Req{units, 0, at->req, b->cached_len[at->req], n, (int32_t)at->row};
      const int mine = mx4_tiles(q, g, kMx4ManyRows);
      for (int tile = 0; tile < mine; ++tile) q.units_per_head += mx4_units_of(q, g, kMx4ManyRows, kMx4ManyShift, tile);
      const int last = mx4_units_of(q, g, kMx4ManyRows, kMx4ManyShift, mine - 1);
      const int first = mx4_units_of(q, g, kMx4ManyRows, kMx4ManyShift, 0);
      t->most_units = last > t->most_units ? last : t->most_units;
      least = first < least ? first : least;
      units += q.units_per_head * t->kv_heads;
      tiles += (int64_t)mine * t->kv_heads;
    }
    at->row += n;
  }
  if (t->nreq == 0) return false;
  // What the ways take, in units of 64 keys (us even shares / whole tiles: 32 requests of 2048..8192 keys and 8..64 tokens, 28/4 heads
  // 117 / 165; one of 3712 keys, 32 tiles 32 / 74; prompts of 1024..4096 tokens, 32/8 heads 686 / 570; two of 600 tokens 44 / 20).  A tile's
  // start and end are as long as six units.  Whole tiles, the longest first, end by the shortest one apart at most.  Even
  // shares have up to two parts more than tiles, which are joined.
  constexpr int kTileCost = 6, kJoinCost = 14;
  const int64_t even = (units + kTileCost * tiles) / plan.places;
  const int64_t whole = tiles <= plan.places || even + least < t->most_units ? t->most_units : even + least;
  t->by_tile = whole <= even + kJoinCost;
  t->groups = (int32_t)(t->by_tile ? tiles : units < plan.places ? units : plan.places);
  // Where the device has a place for each of the units of eight (or sixteen, ..) times as many keys, and they are not much longer than
  // an even share with its second part: those.  (The one request above 27 us, in shares that are not cut at tiles' ends 33.)
  constexpr int kLeast = 8;
  // (Up to 2^30 keys, which is all that a request may have: with tiles by the ten thousand an even share is longer than that.)
  constexpr int kLongest = 30;
  const int64_t longest_unit = (even < kLeast ? kLeast : even) + kTileCost;
  for (int shift = kMx4ManyShift + 3; !t->by_tile && shift <= kLongest && (int64_t)1 << (shift - kMx4ManyShift) <= longest_unit; ++shift) {
    int64_t starts[kMx4TableReqs], heads[kMx4TableReqs], all = 0;
    for (int k = 0; k < t->nreq; ++k) {
      starts[k] = all;
      heads[k] = 0;
      for (int tile = mx4_tiles(t->req[k], g, kMx4ManyRows) - 1; tile >= 0; --tile) heads[k] += mx4_units_of(t->req[k], g, kMx4ManyRows, shift, tile);
      all += heads[k] * t->kv_heads;
    }
    if (all > plan.places) continue;
    for (int k = 0; k < t->nreq; ++k) {
      t->req[k].unit_start = starts[k];
      t->req[k].units_per_head = heads[k];
    }
    t->unit_shift = shift;
    t->groups = (int32_t)(units = all);
    break;
  }
  t->share = units / t->groups;
  t->longer = (int32_t)(units - t->share * t->groups);
  return true;
}

}  // namespace efim
