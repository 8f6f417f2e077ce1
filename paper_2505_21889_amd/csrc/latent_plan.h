// How the latent attention cuts a batch into work.  Host code without state: a call derives everything from the lengths and
// hands the kernels a table of the requests, from which each workgroup works its part out.
#pragma once
#include <cstddef>
#include <cstdint>

#include "efim.h"

#if defined(__HIPCC__) || defined(__HIP__)
#define EFIM_HOST_DEVICE __host__ __device__
#else
#define EFIM_HOST_DEVICE
#endif

namespace efim {

constexpr int kXcds = 8;                // of the device: workgroup i runs on XCD i % 8
constexpr int kLatentTableReqs = 128;   // requests of a launch (kernel arguments end at 4 KB)

// --- absorbed form ---------------------------------------------------------------------------------------------------------
// A tile is `row_tile` query rows (token x head) of a request.  Its work is a unit for each 32 keys in front of and at the
// last one that its rows see.  They are dealt out to as many workgroups as the device has compute units.
//   * Evenly: the units of all tiles one behind the other, whatever the requests' lengths.  A workgroup's share is a run of them,
//     which may begin and end inside a tile.
//   * By tile, where there are few: each tile of a request has the same number of workgroups, which have a part of it each.
// The parts of a tile that several workgroups share are joined by a second kernel.
constexpr int kLatentTileKeys = 32;

struct LatentReq {
  int64_t unit_start;  // units in front of the request in the launch (expanded form: key tiles, of one head; dealt by tile:
                       // workgroups in front, and from bit 32 on the workgroups of each of its tiles)
  int32_t req;         // block table row
  int32_t cached;      // C_r
  int32_t new_len;     // N_r > 0
  int32_t row_start;   // first packed new-token row
};

struct LatentTable {
  LatentReq req[kLatentTableReqs];
  int64_t units;
  int64_t share;       // units of a workgroup; the first `longer` have one more
  int32_t longer;
  int32_t groups;      // workgroups with a share
  int32_t by_tile;     // how they are dealt
  int64_t longest;     // units of the longest share
  int32_t nreq;
  int32_t heads;
  int32_t max_pages;
  int32_t page_shift;

  EFIM_HOST_DEVICE int64_t first_unit(int group) const { return group * share + (group < longer ? group : longer); }
  // by tile: the first of a tile's units that part j of n has
  EFIM_HOST_DEVICE static int first_of(int units, int n, int j) { return units / n * j + (j < units % n ? j : units % n); }
};

// Tiles of a request, the rows of one and its units.
EFIM_HOST_DEVICE inline int latent_tiles(const LatentReq& q, int heads, int row_tile) {
  return (q.new_len * heads + row_tile - 1) / row_tile;
}
EFIM_HOST_DEVICE inline int latent_rows_of(const LatentReq& q, int heads, int row_tile, int tile) {
  const int left = q.new_len * heads - tile * row_tile;
  return left < row_tile ? left : row_tile;
}
EFIM_HOST_DEVICE inline int latent_keys_of(const LatentReq& q, int heads, int row_tile, int tile) {
  return q.cached + (tile * row_tile + latent_rows_of(q, heads, row_tile, tile) - 1) / heads + 1;
}
EFIM_HOST_DEVICE inline int latent_units_of(const LatentReq& q, int heads, int row_tile, int tile) {
  return (latent_keys_of(q, heads, row_tile, tile) + kLatentTileKeys - 1) / kLatentTileKeys;
}

// Units of 64 tiles, which a wave looks through at a time: a request has up to 2^30 keys, and they then 2^31 units.
constexpr int kLatentWaveTiles = 64;
using LatentWaveUnits = uint32_t;

// A workgroup has at most two parts of tiles that it does not have whole: its first and its last.
EFIM_HOST_DEVICE inline int latent_slot(int group, bool first) { return 2 * group + (first ? 0 : 1); }

struct LatentPlan {
  int row_tile = 0;    // 16 or 32 (a workgroup's waves share the rows), 128 (a wave has 32 of them)
  int units = 0;       // compute units to deal to
  int slots = 0;       // partial results
};
LatentPlan plan_latent(const efim_batch_t* b, int units);

// Workspace: partial outputs [slots][row_tile][512] in binary16 and, for each row of them, four floats.
struct LatentBytes {
  size_t off_ml = 0, total = 0;
};
LatentBytes latent_bytes(const LatentPlan& plan);

// Where the next launch of a batch begins.
struct LatentCursor {
  int req = 0;
  int64_t row = 0;
};
// Fills the table of the next launch; false where no request with new tokens is left.
bool latent_next(const efim_batch_t* b, const LatentPlan& plan, LatentCursor* at, LatentTable* table);

// --- expanded form ---------------------------------------------------------------------------------------------------------
// Key tiles (unit_start) are made in pairs, so a request has an even number of them.
constexpr int kExpandedTileKeys = 64;
constexpr int kExpandedTileBytes = 64 * (192 + 128) * 2;
constexpr int kExpandedRowTile = 128;

struct ExpandedTable {
  LatentReq req[kLatentTableReqs];
  int32_t row_tile_start[kLatentTableReqs];  // tiles of query rows, of one head, in front of the request
  int32_t nreq;
  int32_t heads;
  int32_t max_pages;
  int32_t page_shift;
  int32_t key_tiles;                         // of one head
  int32_t slices;                            // of its keys, each expanded by a workgroup
  int32_t row_tiles;
};

struct ExpandedPlan {
  bool ok = false;       // every launch's numbers of workgroups are within a launch's reach
  int teams = 0;         // of a workgroup of the attention: 1 or 2
  int units = 0;         // compute units
  size_t bytes = 0;      // workspace: the expanded tiles of the largest launch
};
ExpandedPlan plan_expanded(const efim_batch_t* b, int units);
bool expanded_next(const efim_batch_t* b, const ExpandedPlan& plan, LatentCursor* at, ExpandedTable* table);

}  // namespace efim
