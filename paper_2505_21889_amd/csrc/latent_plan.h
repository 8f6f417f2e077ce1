// How the absorbed latent attention cuts a batch into work items.  Host code without state: a call derives everything from
// the lengths and hands the kernel a table of the requests, from which each workgroup works its item out.
#pragma once
#include <cstddef>
#include <cstdint>

#include "efim.h"

namespace efim {

constexpr int kLatentTileKeys = 32;     // keys of a tile
constexpr int kLatentTableReqs = 128;   // requests of a launch (kernel arguments end at 4 KB)
constexpr int kLatentRangeStep = 128;   // key ranges are multiples of this: a tile for each of four waves

struct LatentReq {
  int32_t req;         // block table row
  int32_t cached;      // C_r
  int32_t new_len;     // N_r > 0
  int32_t row_start;   // first packed new-token row
  int32_t item_start;  // first work item in the launch
  int32_t slot_start;  // first partial result in the launch, where the key range is cut
};

struct LatentTable {
  LatentReq req[kLatentTableReqs];
  int32_t nreq;
  int32_t items;       // of the launch
  int32_t heads;
  int32_t range;       // keys of a range
  int32_t max_pages;
  int32_t page_shift;
  int32_t split_rows;  // most rows of a request whose range is cut, 0: none is
};

#if defined(__HIPCC__) || defined(__HIP__)
#define EFIM_HOST_DEVICE __host__ __device__
#else
#define EFIM_HOST_DEVICE
#endif

// Ranges of a request of `keys` keys.
EFIM_HOST_DEVICE inline int latent_splits(int keys, int range) { return (int)(((int64_t)keys + range - 1) / range); }

// A work item: a tile of a request's query rows (token x head) against a range of its keys.
struct LatentItem {
  int row0, rows;      // of the request
  int k0, k1;          // empty (k0 >= k1) where the range lies behind the last key that the tile sees
  int slot;            // partial result, -1: the range is whole
};
EFIM_HOST_DEVICE inline LatentItem latent_item(const LatentTable& t, const LatentReq& q, int item, int row_tile) {
  const int splits = latent_splits(q.cached + q.new_len, t.range);
  const int within = item - q.item_start;
  const int tile = within / splits, split = within - tile * splits;
  const int left = q.new_len * t.heads - tile * row_tile;
  LatentItem it;
  it.row0 = tile * row_tile;
  it.rows = left < row_tile ? left : row_tile;
  const int key_end = q.cached + (it.row0 + it.rows - 1) / t.heads + 1;
  it.k0 = split * t.range;
  it.k1 = key_end - it.k0 < t.range ? key_end : it.k0 + t.range;
  it.slot = splits > 1 ? q.slot_start + within : -1;
  return it;
}

struct LatentPlan {
  int row_tile = 0;      // query rows of an item: 16 or 32 (waves share the rows), 128 (a wave has 32 of them)
  int range = 0;         // keys of a range
  int64_t slots = 0;     // partial results of the largest launch
};
LatentPlan plan_latent(const efim_batch_t* b, int units);

// Workspace: partial outputs [slots][row_tile][512] and their (reference, sum).
struct LatentBytes {
  size_t off_o = 0, off_ml = 0, total = 0;
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
// The table's item_start counts tiles of query rows and slot_start tiles of keys, of one head each; `items` is the key
// tiles of a head.  A request has an even number of key tiles: the expansion makes them in pairs.
constexpr int kExpandedTileKeys = 64;
constexpr int kExpandedTileBytes = 64 * (192 + 128) * 2;

struct ExpandedPlan {
  bool ok = false;       // every launch's numbers of workgroups are within a launch's reach
  int row_tile = 0;      // query rows of a workgroup: 128 or 256
  size_t bytes = 0;      // workspace: the expanded tiles of the largest launch
};
ExpandedPlan plan_expanded(const efim_batch_t* b, int units);
bool expanded_next(const efim_batch_t* b, const ExpandedPlan& plan, LatentCursor* at, LatentTable* table, int* row_items);

}  // namespace efim
