// Device code that both forms of the latent attention use.
#pragma once
#include <hip/hip_runtime.h>

#include "efim_internal.h"
#include "latent_plan.h"
#include "wave_ops.h"

namespace efim {

// The outputs of a wave take most or all of the accumulation registers, which only products and moves can name.  Their
// scaling by a moved reference is written out, element by element through one other register: left to the
// compiler it drew outputs into the other registers for the whole loop, which hold queries and operands, and spilled
// those.  The compiler does not count wait states across written-out instructions, so they are kept here: a product
// of 16 passes is read at the earliest 18 states behind it.
__device__ __forceinline__ void after_products() { asm volatile("s_nop 15\n\ts_nop 7" ::: "memory"); }
__device__ __forceinline__ void before_products() { asm volatile("s_nop 7" ::: "memory"); }
__device__ __forceinline__ float scale_accumulator(float x, float f) {
  float held;
  asm volatile(
      "v_accvgpr_read_b32 %1, %0\n\t"
      "v_mul_f32 %1, %1, %2\n\t"
      "v_accvgpr_write_b32 %0, %1"
      : "+a"(x), "=&v"(held)
      : "v"(f));
  return x;
}

// A lane each (two for each lane), asked for at once: what a unit's request is follows without another load.
struct Requests {
  LatentReq held[kLatentTableReqs / 64];
  int nreq;
  template <typename Table>
  __device__ __forceinline__ Requests(const Table& t, int lane) : nreq(t.nreq) {
#pragma unroll
    for (int i = 0; i < kLatentTableReqs / 64; ++i) held[i] = t.req[min(i * 64 + lane, t.nreq - 1)];
  }
  __device__ __forceinline__ int find(int64_t unit, int lane) const {
    int r = -1;
#pragma unroll
    for (int i = 0; i < kLatentTableReqs / 64; ++i) r += __popcll(__ballot(i * 64 + lane < nreq && held[i].unit_start <= unit));
    return __builtin_amdgcn_readfirstlane(r);
  }
  // the request of a workgroup, dealt by tile
  __device__ __forceinline__ int find_group(int group, int lane) const {
    int r = -1;
#pragma unroll
    for (int i = 0; i < kLatentTableReqs / 64; ++i) r += __popcll(__ballot(i * 64 + lane < nreq && (int)(uint32_t)held[i].unit_start <= group));
    return __builtin_amdgcn_readfirstlane(r);
  }
  // the request of a tile of query rows, and its first tile
  __device__ __forceinline__ int find_row_tile(const ExpandedTable& t, int tile, int lane, int* first) const {
    int starts[kLatentTableReqs / 64], r = -1;
#pragma unroll
    for (int i = 0; i < kLatentTableReqs / 64; ++i) starts[i] = t.row_tile_start[min(i * 64 + lane, nreq - 1)];
#pragma unroll
    for (int i = 0; i < kLatentTableReqs / 64; ++i) r += __popcll(__ballot(i * 64 + lane < nreq && starts[i] <= tile));
    r = __builtin_amdgcn_readfirstlane(r);
    *first = __builtin_amdgcn_readlane(r >= 64 ? starts[1] : starts[0], r & 63);
    return r;
  }
  __device__ __forceinline__ LatentReq get(int r) const {
    static_assert(kLatentTableReqs == 128, "two requests to a lane");
    const bool upper = r >= 64;
    auto of = [&](int low, int high) { return __builtin_amdgcn_readlane(upper ? high : low, r & 63); };
    const uint32_t first = (uint32_t)of((int)held[0].unit_start, (int)held[1].unit_start);
    const uint32_t rest = (uint32_t)of((int)(held[0].unit_start >> 32), (int)(held[1].unit_start >> 32));
    return LatentReq{(int64_t)((uint64_t)rest << 32 | first), of(held[0].req, held[1].req), of(held[0].cached, held[1].cached),
                     of(held[0].new_len, held[1].new_len), of(held[0].row_start, held[1].row_start)};
  }
};

// Torn columns.  A row that sees an unfit key (unfit_keys) at a score of minus infinity has no weight for it, and zero times
// an infinite value is no number; but the key was left out.  So where a wave left a key out its outputs, once formed, lose their
// numbers in the columns in which the value of a key that the row sees is not finite.  (In the weightless key's infinite
// columns, that is; at any other score the whole row has none.)  The marks are laid over outputs: 0x7FFF, no number in
// bf16 as in binary16, for each of eight values that is not finite.
typedef uint32_t torn_words __attribute__((ext_vector_type(4)));
__device__ __forceinline__ torn_words torn_marks(torn_words values) {
  torn_words marks;
#pragma unroll
  for (int c = 0; c < 4; ++c)
    marks[c] = ((values[c] & 0x7F80u) == 0x7F80u ? 0x7FFFu : 0u) | ((values[c] & 0x7F800000u) == 0x7F800000u ? 0x7FFF0000u : 0u);
  return marks;
}

// --- tiles of cache rows in LDS ------------------------------------------------------------------------------------------------
constexpr int kRowBytes = kLatentRow * 2;
constexpr int kRowChunks = kRowBytes / 16;
constexpr int kGroupKeys = 8;                             // rows gathered together
constexpr int kGroupBytes = kGroupKeys * kRowBytes;
constexpr int kGroupLoads = kGroupBytes / 1024;
static_assert(kGroupKeys <= kMinPageSize && kGroupLoads == 9, "a group of rows lies in one page");

// Swizzle of a tile row's chunks (exclusive or on the chunk's low three bits).  A row is 72 chunks, so neighbouring rows
// start half of the 256-byte bank line apart; with these three bits of the row sixteen rows' equal chunks take the sixteen
// places of the line, and so do the four chunks of eight rows that a transposing read takes at a time.
__device__ __forceinline__ int swizzle(int row) { return ((row >> 1) & 1) << 2 | ((row >> 2) & 1) << 1 | ((row >> 3) & 1); }

// Copies of cache rows into a tile, eight rows (a group) at a time: nine loads of 1 KB.
struct Gather {
  const char* cache;
  int k1, page_shift, page_mask;
  uint32_t swizzles;  // two bits from bit 5 on for each of the nine loads: the swizzle of the row that this lane's chunk lies in, halved
  uint32_t lane16;

  __device__ __forceinline__ Gather(const uint16_t* rows, int end, int shift, int lane)
      : cache(reinterpret_cast<const char*>(rows)), k1(end), page_shift(shift), page_mask((1 << shift) - 1), swizzles(0), lane16(lane * 16) {
    asm volatile("" : "+v"(lane));  // (formed where it is used: offsets held from part to part were spilled)
#pragma unroll
    for (int j = 0; j < kGroupLoads; ++j) swizzles |= (uint32_t)(swizzle((j * 64 + lane) / kRowChunks) >> 1) << (5 + 2 * j);
  }
  // (formed again for every tile, as the operands' addresses are)
  __device__ __forceinline__ void forget() { asm volatile("" : "+v"(swizzles), "+v"(lane16)); }
  // byte offset of load j in a group (its multiple of 1 KB aside) whose tile row divided by eight is even or odd
  __device__ __forceinline__ uint32_t offset(int j, int odd) const { return ((swizzles >> (2 * j)) & 0x60) ^ (lane16 ^ (odd << 4)); }
  __device__ __forceinline__ const char* row_at(int32_t page, int key) const {
    return cache + (((int64_t)page << page_shift) + (key & page_mask)) * kRowBytes;
  }
  __device__ __forceinline__ bool whole(int key) const { return key + kGroupKeys <= k1; }
  // loads j and j + 1 of a whole group whose first row is at `base`, or the last one
  __device__ __forceinline__ void pair(const char* base, int j, int odd, uint32_t to) const {
    if (j + 1 < kGroupLoads) load_to_lds_2x16(base + j * 1024, offset(j, odd), offset(j + 1, odd), to + j * 1024);
    else load_to_lds_16(base + j * 1024, offset(j, odd), to + j * 1024);
  }
  // group `key` .. key + 7, which is group g of its tile, to LDS at `to`; rows at or behind k1 become copies of the last one's
  __device__ __forceinline__ void group(int key, int g, int32_t page, uint32_t to) const {
    if (whole(key)) {
      const char* base = row_at(page, key);
      load_to_lds_4x16(base, offset(0, g & 1), offset(1, g & 1), offset(2, g & 1), offset(3, g & 1), to);
      load_to_lds_4x16(base + 4096, offset(4, g & 1), offset(5, g & 1), offset(6, g & 1), offset(7, g & 1), to + 4096);
      load_to_lds_16(base + 8192, offset(8, g & 1), to + 8192);
    } else {
      const int last = k1 - 1, from = min(key, last & ~(kGroupKeys - 1)), most = last - from;
      const char* base = row_at(page, from);
#pragma unroll 1
      for (int j = 0; j < kGroupLoads; ++j) {
        const int n = j * 64 + (int)(lane16 >> 4), row = n / kRowChunks, chunk = n - row * kRowChunks;
        load_to_lds_16(base, (uint32_t)(min(row, most) * kRowBytes + ((chunk ^ swizzle(g * kGroupKeys + row)) << 4)), to + j * 1024);
      }
    }
  }
};

}  // namespace efim
