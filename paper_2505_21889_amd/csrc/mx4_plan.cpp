// Work of the attention over a 4-bit cache (host code).
#include "mx4_plan.h"

#include "efim_internal.h"

namespace efim {

namespace {

bool is_few(const efim_batch_t* b, int r) {
  return (int64_t)b->new_len[r] * (b->num_q_heads / b->num_kv_heads) <= kMx4FewRows;
}

}  // namespace

Mx4Plan plan_mx4(const efim_batch_t* b, bool few, int compute_units) {
  Mx4Plan plan;
  plan.few = few;
  int64_t most = 0;
  for (int r = 0; r < b->batch; ++r) {
    if (b->new_len[r] == 0 || is_few(b, r) != few) continue;
    plan.any = true;
    const int64_t rows = (int64_t)b->new_len[r] * (b->num_q_heads / b->num_kv_heads);
    most = rows > most ? rows : most;
  }
  plan.row_tile = few ? (most <= 16 ? 16 : 32) : kMx4ManyRows;
  plan.unit_keys = few ? kMx4FewKeys : kMx4ManyKeys;
  plan.max_groups = compute_units * (few ? (plan.row_tile == 16 ? 4 : 2) : 2);
  return plan;
}

Mx4Bytes mx4_bytes(const Mx4Plan& plan, int head_dim) {
  Mx4Bytes at;
  if (!plan.any) return at;
  const size_t rows = (size_t)2 * plan.max_groups * plan.row_tile;
  at.off_ml = rows * head_dim * sizeof(float);
  at.total = (at.off_ml + rows * 2 * sizeof(float) + 255) / 256 * 256;
  return at;
}

bool mx4_next(const efim_batch_t* b, const Mx4Plan& plan, Mx4Cursor* at, Mx4Table* t) {
  t->nreq = 0;
  t->kv_heads = b->num_kv_heads;
  t->group_heads = b->num_q_heads / b->num_kv_heads;
  t->max_pages = b->max_pages_per_req;
  t->page_shift = 0;
  while ((1 << t->page_shift) < b->page_size) ++t->page_shift;
  int64_t units = 0;
  for (; at->req < b->batch && t->nreq < kMx4TableReqs; ++at->req) {
    const int n = b->new_len[at->req];
    if (n > 0 && is_few(b, at->req) == plan.few) {
      Mx4Req& q = t->req[t->nreq++];
      q = Mx4Req{units, 0, at->req, b->cached_len[at->req], n, (int32_t)at->row};
      for (int tile = mx4_tiles(q, t->group_heads, plan.row_tile) - 1; tile >= 0; --tile)
        q.units_per_head += mx4_units_of(q, t->group_heads, plan.row_tile, plan.unit_keys, tile);
      units += q.units_per_head * t->kv_heads;
    }
    at->row += n;
  }
  if (t->nreq == 0) return false;
  t->groups = (int32_t)(units < plan.max_groups ? units : plan.max_groups);
  t->share = units / t->groups;
  t->longer = (int32_t)(units - t->share * t->groups);
  return true;
}

}  // namespace efim
