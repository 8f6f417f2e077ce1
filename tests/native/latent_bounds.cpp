// The longest request that the latent attention takes: what its plan and its kernels count fits the types that hold it.
#include <cstdio>
#include <limits>

#include "efim_internal.h"
#include "latent_plan.h"

using namespace efim;

#define CHECK(x) do { if (!(x)) { printf("line %d: %s\n", __LINE__, #x); return 1; } } while (0)

int main() {
  const int32_t new_len = 32, cached = (1 << 30) - new_len;
  efim_batch_t b{};
  b.batch = 1;
  b.num_q_heads = kMaxLatentHeads;
  b.num_kv_heads = 1;
  b.head_dim = kLatentRow;
  b.page_size = 256;
  b.max_pages_per_req = b.num_pages = 1 << 22;
  b.cached_len = &cached;
  b.new_len = &new_len;
  b.block_table = reinterpret_cast<const int32_t*>(0x1000);
  CHECK(validate_latent_batch(&b, nullptr) == EFIM_OK);
  const int32_t longer = cached + 1;
  b.cached_len = &longer;
  CHECK(validate_latent_batch(&b, nullptr) == EFIM_ERR_UNSUPPORTED);
  b.cached_len = &cached;
  const LatentPlan plan = plan_latent(&b, 256);
  LatentCursor at;
  LatentTable t;
  CHECK(latent_next(&b, plan, &at, &t));
  const int tiles = latent_tiles(t.req[0], t.heads, plan.row_tile);
  CHECK(tiles >= kLatentWaveTiles);
  int64_t all = 0, of_wave = 0;
  for (int tile = 0; tile < tiles; ++tile) {
    const int units = latent_units_of(t.req[0], t.heads, plan.row_tile, tile);
    CHECK(units > 0 && (int64_t)units * kLatentTileKeys <= std::numeric_limits<int32_t>::max());
    all += units;
    of_wave = tile % kLatentWaveTiles ? of_wave + units : units;
    CHECK(of_wave <= (int64_t)std::numeric_limits<LatentWaveUnits>::max());
  }
  CHECK(all == t.units && t.share <= t.longest && t.longest <= std::numeric_limits<int32_t>::max());
  printf("latent bounds ok\n");
  return 0;
}
