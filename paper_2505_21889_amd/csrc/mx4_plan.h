// How the attention over a 4-bit cache cuts a batch into work.  Host code without state: a call derives everything from the
// lengths and hands the kernels a table of the requests, from which each workgroup works its share out.
//
// A tile is `row_tile` query rows (token x head of the group) of a request and kv head.  Requests of few rows and of many are
// different launches: a mixed step's single tokens would be multiplied as tiles of mostly empty rows otherwise.
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

constexpr int kMx4FewRows = 32;    // query rows of a request and kv head that the kernel for few rows takes
constexpr int kMx4FewKeys = 128;   // keys of its units: 32 for each of its four waves
constexpr int kMx4ManyRows = 128;  // row tile of the kernel for many rows
constexpr int kMx4ManyShift = 6;   // log2 of the keys of its units

// --- few rows ---------------------------------------------------------------------------------------------------------------
// A request is one tile a kv head.  Its keys are cut into parts of as many units, a workgroup each; the parts of a tile that has
// several are joined by a second kernel.
template <int MAXREQ>
struct Mx4FewTable {
  int32_t group_start[MAXREQ];  // workgroups in front of the request in the launch
  int32_t parts[MAXREQ];        // of each of its tiles
  int32_t split_start[MAXREQ];  // split tiles in front of it
  int32_t slot_start[MAXREQ];   // partial results in front of it
  int32_t req[MAXREQ];          // block table row
  int32_t cached[MAXREQ];       // C_r
  int32_t new_len[MAXREQ];      // N_r > 0
  int32_t row_start[MAXREQ];    // first packed new-token row
  int32_t nreq;
  int32_t groups;               // workgroups of the launch
  int32_t splits;               // split tiles
  int32_t slots;                // partial results
  int32_t kv_heads;
  int32_t group_heads;          // query heads of a kv head
  int32_t max_pages;
  int32_t page_shift;
};
constexpr int64_t kMx4MostGroups = 1 << 22;  // of a launch (its threads are counted in 32 bits)
constexpr int kMx4FewReqs = 120;  // of a launch (kernel arguments end at 4 KB); batches of up to 64 take a smaller table

// The first of a tile's units that part j of n has.
EFIM_HOST_DEVICE inline int mx4_first_of(int units, int n, int j) { return units / n * j + (j < units % n ? j : units % n); }

struct Mx4FewPlan {
  bool any = false;    // the batch has such requests
  int row_tile = 0;    // 16 or 32
  int part_units = 0;  // the most units of a part
  int slots = 0;       // partial results of the largest launch
};

// --- many rows --------------------------------------------------------------------------------------------------------------
// A tile's work is a unit for each 64 keys in front of and at the last one that its rows see.  Either a workgroup has a tile, the
// longest first; or a unit of so many more keys that there is one for each workgroup; or the units of all tiles, one behind the other,
// are dealt evenly to the workgroups: a share is a run of them, which may begin and end inside a tile.  The parts of a tile that
// several workgroups share are joined by a second kernel.
constexpr int kMx4TableReqs = 96;  // requests of a launch

struct Mx4Req {
  int64_t unit_start;      // units in front of the request in the launch
  int64_t units_per_head;  // of all its tiles of one kv head
  int32_t req;             // block table row
  int32_t cached;          // C_r
  int32_t new_len;         // N_r > 0
  int32_t row_start;       // first packed new-token row
};

struct Mx4Table {
  Mx4Req req[kMx4TableReqs];
  int64_t share;       // units of a workgroup; the first `longer` have one more
  int32_t longer;
  int32_t groups;      // workgroups with a share, or tiles
  int32_t by_tile;
  int32_t most_units;  // of a tile
  int32_t unit_shift;  // log2 of a unit's keys
  int32_t nreq;
  int32_t kv_heads;
  int32_t group_heads; // query heads of a kv head
  int32_t max_pages;
  int32_t page_shift;

  EFIM_HOST_DEVICE int64_t first_unit(int group) const { return group * share + (group < longer ? group : longer); }
};

// Tiles of a request and kv head, the rows of one, the keys that they see and its units.
EFIM_HOST_DEVICE inline int mx4_tiles(const Mx4Req& q, int g, int row_tile) { return (q.new_len * g + row_tile - 1) / row_tile; }
EFIM_HOST_DEVICE inline int mx4_rows_of(const Mx4Req& q, int g, int row_tile, int tile) {
  const int left = q.new_len * g - tile * row_tile;
  return left < row_tile ? left : row_tile;
}
EFIM_HOST_DEVICE inline int mx4_keys_of(const Mx4Req& q, int g, int row_tile, int tile) {
  return q.cached + (tile * row_tile + mx4_rows_of(q, g, row_tile, tile) - 1) / g + 1;
}
EFIM_HOST_DEVICE inline int mx4_units_of(const Mx4Req& q, int g, int row_tile, int unit_shift, int tile) {
  return ((mx4_keys_of(q, g, row_tile, tile) - 1) >> unit_shift) + 1;
}

// Tiles of a request and kv head that have `units` or more: the last ones.  (A tile has c units where its last row's token lies behind
// the keys of c - 1; the first such tile is the one of that token's first row.)
EFIM_HOST_DEVICE inline int mx4_tiles_from(const Mx4Req& q, int g, int row_tile, int unit_shift, int units) {
  const int token = ((units - 1) << unit_shift) - q.cached, tiles = mx4_tiles(q, g, row_tile);
  return token <= 0 ? tiles : token >= q.new_len ? 0 : tiles - token * g / row_tile;
}

// A workgroup has at most two parts of tiles that it does not have whole: one that goes on where another's ends, and one that
// begins its tile.
EFIM_HOST_DEVICE inline int64_t mx4_slot(int group, bool goes_on) { return 2 * (int64_t)group + (goes_on ? 0 : 1); }

struct Mx4ManyPlan {
  bool any = false;
  int places = 0;      // workgroups that the device holds
  size_t slots = 0;    // partial results of the largest launch
};

// Where the next launch of a class begins.
struct Mx4Cursor {
  int req = 0;
  int64_t row = 0;
};

Mx4FewPlan plan_mx4_few(const efim_batch_t* b, int compute_units);
Mx4ManyPlan plan_mx4_many(const efim_batch_t* b, int compute_units);
// Fill the table of the next launch; false where no request of the class is left.
template <int MAXREQ>
bool mx4_next(const efim_batch_t* b, const Mx4FewPlan& plan, Mx4Cursor* at, Mx4FewTable<MAXREQ>* table);
bool mx4_next(const efim_batch_t* b, const Mx4ManyPlan& plan, Mx4Cursor* at, Mx4Table* table);

// Workspace of a class: partial outputs [slots][row tile][head_dim] and two floats (reference, sum) for each row of them.
struct Mx4Bytes {
  size_t off_ml = 0, total = 0;
};
Mx4Bytes mx4_bytes(size_t slots, int row_tile, int head_dim);

}  // namespace efim
