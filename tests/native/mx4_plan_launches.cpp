// The launches that a batch over a 4-bit cache is cut into, one line each.  Reads: query heads, heads of keys, compute units, requests, then
// the requests' cached and new lengths.
#include <cstdio>
#include <vector>

#include "mx4_plan.h"

using namespace efim;

int main() {
  efim_batch_t b{};
  int compute_units = 0;
  if (std::scanf("%d %d %d %d", &b.num_q_heads, &b.num_kv_heads, &compute_units, &b.batch) != 4) return 1;
  std::vector<int32_t> cached(b.batch), fresh(b.batch);
  for (int r = 0; r < b.batch; ++r)
    if (std::scanf("%d %d", &cached[r], &fresh[r]) != 2) return 1;
  b.cached_len = cached.data();
  b.new_len = fresh.data();
  b.head_dim = 64;
  b.page_size = 256;
  b.max_pages_per_req = 1 << 22;
  const Mx4FewPlan few = plan_mx4_few(&b, compute_units);
  Mx4Cursor at;
  Mx4FewTable<kMx4FewReqs> f;
  while (few.any && mx4_next(&b, few, &at, &f)) std::printf("few %d %d %d %d %d\n", few.row_tile, f.nreq, f.groups, f.splits, f.slots);
  const Mx4ManyPlan many = plan_mx4_many(&b, compute_units);
  Mx4Table m;
  at = Mx4Cursor();
  while (many.any && mx4_next(&b, many, &at, &m)) {
    // the units that the shares are made of, counted again
    int64_t units = 0, tiles = 0;
    for (int k = 0; k < m.nreq; ++k)
      for (int tile = 0; tile < mx4_tiles(m.req[k], m.group_heads, kMx4ManyRows); ++tile) {
        units += (int64_t)m.kv_heads * mx4_units_of(m.req[k], m.group_heads, kMx4ManyRows, m.unit_shift, tile);
        tiles += m.kv_heads;
      }
    const bool dealt = m.by_tile ? m.groups == tiles : m.first_unit(0) == 0 && m.first_unit(m.groups) == units;
    std::printf("many %d %d %d %d %d\n", m.nreq, m.by_tile, m.unit_shift, m.groups, dealt);
  }
  std::printf("end\n");
  return 0;
}
