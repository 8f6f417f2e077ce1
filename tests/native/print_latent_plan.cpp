// Prints the absorbed attention's plan of batches from standard input: lines of compute units, heads, number of requests
// and, for each, cached and new length; one line of row tile, and for the first launch by_tile, longest, groups, tiles.
#include <cstdio>
#include <vector>

#include "efim_internal.h"
#include "latent_plan.h"

using namespace efim;

int main() {
  int units, heads, n;
  while (scanf("%d %d %d", &units, &heads, &n) == 3) {
    std::vector<int32_t> cached(n), fresh(n);
    for (int r = 0; r < n; ++r)
      if (scanf("%d %d", &cached[r], &fresh[r]) != 2) return 1;
    efim_batch_t b{};
    b.batch = n;
    b.num_q_heads = heads;
    b.num_kv_heads = 1;
    b.head_dim = kLatentRow;
    b.page_size = 64;
    b.max_pages_per_req = b.num_pages = 1 << 20;
    b.cached_len = cached.data();
    b.new_len = fresh.data();
    b.block_table = reinterpret_cast<const int32_t*>(0x1000);
    if (validate_latent_batch(&b, nullptr) != EFIM_OK) return 1;
    const LatentPlan plan = plan_latent(&b, units);
    LatentCursor at;
    LatentTable t;
    if (!latent_next(&b, plan, &at, &t)) return 1;
    long tiles = 0;
    for (int k = 0; k < t.nreq; ++k) tiles += latent_tiles(t.req[k], t.heads, plan.row_tile);
    printf("%d %d %lld %d %ld\n", plan.row_tile, t.by_tile, (long long)t.longest, t.groups, tiles);
  }
  return 0;
}
