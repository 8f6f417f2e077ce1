// efim_extend_attention_mx4: causal softmax attention of the new tokens over a paged 4-bit cache.
//   s = scale <q, k_j>,  p = softmax(s),  o = sum_j p_j v_j,   j = 0 .. C_r + i
// Rows are (token, head of the group) pairs, so all query heads of a kv head read its rows once.  What codes stand for is exact
// in bf16, so the products are those of a bf16 cache: bf16 operands, fp32 sums, probabilities rounded to bf16 (as many bits as
// the values that they weigh).  S^T = K Q^T and O^T = V^T P^T: a lane holds scores of ONE query row, and the rounded
// probabilities are the second product's operand as they stand.
//
// Values lie in memory along the head dimension and enter the product along the keys; they go through LDS as bf16 and the
// transposing read turns them.  (The read for 4-bit elements would leave keys with scales of their own in one operand word.)
//
// A value block that is no number must not reach rows that do not see it as zero times no number: such blocks enter the products
// as finite numbers (zeros with few rows, the codes under a scale of one with many), under probabilities that are zero in the rows that
// do not see them, and behind a part's last key the rows that see one lose their numbers in its columns.  For that a thread keeps the
// first such key that it meets, and a workgroup the first one of each block of columns.  (With one such block in the context a token over
// 30000 keys takes 19.7 us, a prompt of 8192 tokens 227, as without; a walk over the part's keys again for each row 59 and 775.)
#include <type_traits>

#include "efim_internal.h"
#include "mx4_math.h"
#include "mx4_plan.h"
#include "wave_ops.h"

namespace efim {
namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;

#define LDS_PTR(T) __attribute__((address_space(3))) T*

constexpr int kXcdCount = 8;  // of the device: workgroup i runs on XCD i % 8
constexpr int kWaves = 4;
constexpr int kThreads = 64 * kWaves;
constexpr float kSlack = 8.f;  // log2 units by which a row's maximum may outgrow its reference
constexpr float kOver = 256.f;  // 2^kSlack: a sum of rounded probabilities is never below its largest one
constexpr float kNoReference = -3.0e38f;  // of a row that has seen no key: any finite score moves it
constexpr uint32_t kTorn = 253;  // scale bytes from here on: values that are not finite
constexpr int32_t kNoKey = INT32_MAX;  // behind every key

struct Mx4Args {
  Mx4Table table;
  float scale_log2;  // sm_scale * log2(e)
  float* part_o;     // partial results of split tiles, [slot][row tile][D]: the unnormalised output
  float* part_ml;    // [slot][row tile][2]: reference in log2 units, sum
  int32_t* splits;   // [workgroup][8]: the tile that its share ends in, for the join: rows (0: ends with a tile, or inside one that began
                     // in front of it), first row, packed row of the request, head, the last workgroup with a part
  uint16_t* out;
};

// A lane each (two for each lane), asked for at once: what a unit's request is follows without another load.  (All of the table,
// whatever it holds: which part of it counts is known at the same time.)
struct Requests {
  Mx4Req held[2];
  int nreq;
  __device__ __forceinline__ Requests(const Mx4Table& t, int lane) : nreq(t.nreq) {
#pragma unroll
    for (int i = 0; i < 2; ++i) held[i] = t.req[min(i * 64 + lane, kMx4TableReqs - 1)];
  }
  __device__ __forceinline__ int find(int64_t unit, int lane) const {
    int r = -1;
#pragma unroll
    for (int i = 0; i < 2; ++i) r += __popcll(__ballot(i * 64 + lane < nreq && held[i].unit_start <= unit));
    return __builtin_amdgcn_readfirstlane(r);
  }
  __device__ __forceinline__ Mx4Req get(int r) const {
    const bool upper = r >= 64;
    auto of = [&](int low, int high) { return __builtin_amdgcn_readlane(upper ? high : low, r & 63); };
    auto of2 = [&](int64_t low, int64_t high) {
      return (int64_t)((uint64_t)(uint32_t)of((int)(low >> 32), (int)(high >> 32)) << 32 | (uint32_t)of((int)low, (int)high));
    };
    return Mx4Req{of2(held[0].unit_start, held[1].unit_start), of2(held[0].units_per_head, held[1].units_per_head),
                  of(held[0].req, held[1].req), of(held[0].cached, held[1].cached), of(held[0].new_len, held[1].new_len),
                  of(held[0].row_start, held[1].row_start)};
  }
};

// The tile that a unit of the launch lies in, by the whole wave.
struct Place {
  int r;          // request of the launch
  int head;
  int tile;       // of the request and head
  int units;      // of the tile
  int64_t first;  // unit of the launch at which it begins
};
template <int TILE>
__device__ __forceinline__ Place find_tile(const Mx4Table& t, const Requests& requests, int64_t unit, int lane) {
  Place at;
  at.r = requests.find(unit, lane);
  const Mx4Req q = requests.get(at.r);
  const int64_t in = unit - q.unit_start;
  // (fewer than 2^32 units in nearly all launches: a 64-bit division takes hundreds of cycles)
  at.head = (in | q.units_per_head) >> 32 == 0 ? (int)((uint32_t)in / (uint32_t)q.units_per_head) : (int)(in / q.units_per_head);
  at.head = __builtin_amdgcn_readfirstlane(at.head);
  at.first = q.unit_start + at.head * q.units_per_head;
  at.tile = 0;
  const int tiles = mx4_tiles(q, t.group_heads, TILE);
  at.units = mx4_units_of(q, t.group_heads, TILE, t.unit_shift, 0);
  if (tiles == 1) return at;
  for (int t0 = 0; t0 < tiles; t0 += 64) {
    const int mine = t0 + lane < tiles ? mx4_units_of(q, t.group_heads, TILE, t.unit_shift, t0 + lane) : 0;
    int upto = mine;  // of the lanes up to this one
#pragma unroll
    for (int by = 1; by < 64; by <<= 1) {
      const int other = __shfl_up(upto, by);
      if (lane >= by) upto += other;
    }
    const uint64_t in_front = __ballot(at.first + upto <= unit);  // tiles that end in front of the unit
    if (in_front != ~0ull) {
      const int k = __popcll(in_front);
      at.tile = t0 + k;
      at.units = __builtin_amdgcn_readlane(mine, k);
      at.first += __builtin_amdgcn_readlane(upto, k) - at.units;
      return at;
    }
    at.first += __builtin_amdgcn_readlane(upto, 63);
  }
  return at;
}

// Sum of a lane's numbers over the wave, in all lanes: exchanges inside rows of sixteen lanes, then of rows and halves.
__device__ __forceinline__ int lanes_sum(int v) {
  auto with = [&](auto ctrl) { return __builtin_amdgcn_update_dpp(0, v, decltype(ctrl)::value, 0xf, 0xf, true); };
  v += with(std::integral_constant<int, 0xB1>{});   // quad_perm [1, 0, 3, 2]
  v += with(std::integral_constant<int, 0x4E>{});   // quad_perm [2, 3, 0, 1]
  v += with(std::integral_constant<int, 0x141>{});  // row_half_mirror
  v += with(std::integral_constant<int, 0x140>{});  // row_mirror
  return __builtin_amdgcn_readlane(v, 0) + __builtin_amdgcn_readlane(v, 16) + __builtin_amdgcn_readlane(v, 32) + __builtin_amdgcn_readlane(v, 48);
}

// The tile that is the n-th in the order of their units, the largest first, by the whole wave: what starts last is then
// short.  Of equally long tiles the heads are next to each other, so that an XCD meets few of them.
template <int TILE>
__device__ __forceinline__ Place nth_tile(const Mx4Table& t, const Requests& requests, int n, int lane) {
  const int g = t.group_heads;
  const auto& q = requests.held;
  auto longer = [&](int c, int i) { return i * 64 + lane < t.nreq ? mx4_tiles_from(q[i], g, TILE, t.unit_shift, c) : 0; };
  auto of_all = [&](int c) { return t.kv_heads * lanes_sum(longer(c, 0) + longer(c, 1)); };
  int low = 1, high = t.most_units + 1;  // the units of the tile: more tiles than n have `low` or more, at most n `high` or more
  while (high - low > 1) {
    const int middle = low + (high - low) / 2;
    (of_all(middle) > n ? low : high) = middle;
  }
  int in = n - of_all(high);
  Place at;
  at.units = low;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int mine = t.kv_heads * (longer(low, i) - longer(high, i));
    int upto = mine;
#pragma unroll
    for (int by = 1; by < 64; by <<= 1) {
      const int other = __shfl_up(upto, by);
      if (lane >= by) upto += other;
    }
    const int k = __popcll(__ballot(upto <= in));
    if (k < 64) {
      in -= __builtin_amdgcn_readlane(upto - mine, k);
      at.r = i * 64 + k;
      at.head = in % t.kv_heads;
      at.tile = mx4_tiles(requests.get(at.r), g, TILE) - __builtin_amdgcn_readlane(longer(low, i), k) + in / t.kv_heads;
      break;
    }
    in -= __builtin_amdgcn_readlane(upto, 63);
  }
  at.first = 0;
  return at;
}

// A workgroup's share of the units, a tile's part at a time.
template <int TILE>
struct Share {
  const Mx4Table& t;
  Place at;
  int group;
  int64_t begin, end;  // units that are left
  // the part at hand
  Mx4Req rq;
  int row0, rows;  // of the request
  int k0, k1;      // keys
  int64_t slot;    // partial result, -1: the workgroup has the whole tile

  __device__ __forceinline__ Share(const Mx4Table& table, int lane) : t(table) {
    const Requests requests(table, lane);
    if (t.by_tile) {
      group = 0;
      at = nth_tile<TILE>(t, requests, blockIdx.x, lane);
      begin = at.first;
      end = begin + at.units;
      rq = requests.get(at.r);
      part();
      return;
    }
    // an XCD takes neighbouring shares, which have rows of the cache in common
    group = (int)(blockIdx.x % kXcdCount) * (int)(gridDim.x / kXcdCount) + (int)(blockIdx.x / kXcdCount);
    begin = end = 0;
    if (group >= t.groups) return;
    begin = t.first_unit(group);
    end = t.first_unit(group + 1);
    at = find_tile<TILE>(t, requests, begin, lane);
    rq = requests.get(at.r);
    part();
  }
  __device__ __forceinline__ bool done() const { return begin >= end; }
  __device__ __forceinline__ bool ends() const { return at.first + at.units >= end; }  // with the part at hand
  __device__ __forceinline__ int last_group() const {  // with a part of the tile at hand
    int last = group;
    while (last + 1 < t.groups && t.first_unit(last + 1) < at.first + at.units) ++last;
    return last;
  }
  __device__ __forceinline__ void part() {
    row0 = at.tile * TILE;
    rows = mx4_rows_of(rq, t.group_heads, TILE, at.tile);
    const int u0 = (int)(begin - at.first);
    const int u1 = (int)min((int64_t)at.units, end - at.first);
    k0 = u0 << t.unit_shift;
    k1 = min((int64_t)u1 << t.unit_shift, (int64_t)mx4_keys_of(rq, t.group_heads, TILE, at.tile));
    slot = u0 == 0 && u1 == at.units ? -1 : mx4_slot(group, u0 > 0);
  }
  __device__ __forceinline__ void advance() {
    begin = at.first + at.units;
    if (done()) return;
    at.first = begin;
    if (++at.tile == mx4_tiles(rq, t.group_heads, TILE)) {
      at.tile = 0;
      if (++at.head == t.kv_heads) {
        at.head = 0;
        rq = t.req[++at.r];
      }
    }
    at.units = mx4_units_of(rq, t.group_heads, TILE, t.unit_shift, at.tile);
    part();
  }
};

// Where the rows of a request's kv head lie.
template <int D>
struct Cache {
  const char* rows;
  const __attribute__((address_space(4))) int32_t* pages;  // (scalar loads)
  int page_shift, kv_heads, head;

  template <typename Table>
  __device__ __forceinline__ Cache(const uint8_t* cache, const int32_t* block_table, const Table& t, int req, int h)
      : rows(reinterpret_cast<const char*>(cache)),
        pages((const __attribute__((address_space(4))) int32_t*)(uintptr_t)(block_table + (int64_t)req * t.max_pages)),
        page_shift(t.page_shift), kv_heads(t.kv_heads), head(h) {}
  // page of a (wave-uniform) key, and where the head's rows of a page begin
  __device__ __forceinline__ int32_t page_id(int key) const { return pages[__builtin_amdgcn_readfirstlane(key >> page_shift)]; }
  __device__ __forceinline__ int64_t page_at(int32_t id) const { return (((int64_t)id * kv_heads + head) << page_shift) * mx4_row_bytes(D); }
  __device__ __forceinline__ int slot_of(int key) const { return key & ((1 << page_shift) - 1); }
  __device__ __forceinline__ uint32_t code_at(int key) const { return (uint32_t)slot_of(key) * mx4_code_bytes(D); }
  __device__ __forceinline__ uint32_t scale_at(int key) const {
    return ((uint32_t)mx4_code_bytes(D) << page_shift) + (uint32_t)slot_of(key) * mx4_scale_bytes(D);
  }
};

__device__ __forceinline__ float add_pair(uint32_t two, float sum) {  // of two probabilities as they were rounded
  const bf16x2 ones = {(__bf16)1.0f, (__bf16)1.0f};
  return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, two), ones, sum, false);
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){lo, hi}, bf16x2));
}

// Chunk swizzles (exclusive or) of a tile's bf16 rows in LDS, of which the bank line holds one (D 128) or two.  Keys (D 64) and values that
// a workgroup shares: eight lanes write two pieces of 32 elements of each of four rows, word by word, and a wave reads sixteen
// neighbouring rows' equal chunks (keys) and four neighbouring chunks of each of four rows (values); all of them take all banks.
template <int D>
__device__ __forceinline__ int key_swizzle(int row) { return row >> 1 & 7; }
template <int D>
__device__ __forceinline__ int value_swizzle(int row) { return D == 128 ? (row & 3) * 5 : (row >> 1 & 3) ^ (row >> 1 & 1) << 2; }
// Values of a wave's own: the same writes, and two neighbouring chunks of each of eight rows, which the transposing read for products of
// 16 rows takes.
template <int D>
__device__ __forceinline__ int value_swizzle16(int row) { return D == 128 ? (row & 7) << 1 | (row >> 1 & 1) : (row >> 1 & 3) << 1 | (row >> 2 & 1); }

// One wave writes and reads its own LDS: the accesses are in order, the compiler is told by the fences.
__device__ __forceinline__ void own_writes() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// --- few rows ---------------------------------------------------------------------------------------------------------------
template <int MAXREQ>
struct Mx4FewArgs {
  Mx4FewTable<MAXREQ> table;
  float scale_log2;
  float* part_o;
  float* part_ml;
  uint16_t* out;
};

// A wave's copy of the table, 64 requests to a load, all asked for at once.
template <int MAXREQ>
struct FewLanes {
  static constexpr int kLoads = (MAXREQ + 63) / 64;
  int group_start[kLoads], parts[kLoads], split_start[kLoads], slot_start[kLoads], req[kLoads], cached[kLoads], new_len[kLoads], row_start[kLoads];
  int nreq, lane;
  __device__ __forceinline__ FewLanes(const Mx4FewTable<MAXREQ>& t, int l) : nreq(t.nreq), lane(l) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int k = min(i * 64 + l, t.nreq - 1);
      group_start[i] = t.group_start[k];
      parts[i] = t.parts[k];
      split_start[i] = t.split_start[k];
      slot_start[i] = t.slot_start[k];
      req[i] = t.req[k];
      cached[i] = t.cached[k];
      new_len[i] = t.new_len[k];
      row_start[i] = t.row_start[k];
    }
  }
  // the last request that starts at or in front of a workgroup or split tile
  __device__ __forceinline__ int find(const int (&starts)[kLoads], int index) const {
    int r = -1;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) r += __popcll(__ballot(i * 64 + lane < nreq && starts[i] <= index));
    return __builtin_amdgcn_readfirstlane(r);
  }
  __device__ __forceinline__ int of(const int (&field)[kLoads], int r) const {
    return __builtin_amdgcn_readlane(kLoads == 2 && r >= 64 ? field[kLoads - 1] : field[0], r & 63);
  }
};

// NB blocks of 16 query rows.  The four waves share the rows: of each 128 keys a wave takes 32, with a maximum and sums of its
// own, and their sums are combined at the part's end.  A wave's keys go from memory to registers, where they are the product's
// operands as they are converted; a lane has 16 (D 128; 8) bytes of a row's codes, all under one scale, and the query operands
// follow that order of elements.
// Bound by HBM where there are many: 32 requests of 2048..8192 keys, one token each, 28/4 heads 20.4 us for 96 MB (4.7 TB/s) and 4.7 for
// the join.  16 requests of 1024..4096 keys and 24 rows 17.8 for 48 MB: the first two units of all waves take 2 us to come, five more as long
// as their conversions and products (37 % and 15 % of the cycles), and the four waves' join 1.5.  One request of 2344 keys: latency,
// 6.1 and 4.1.  Three units in flight instead of two: 4 % slower in the first case, 5 % in the second.
template <int D, int NB, int MAXREQ>
__global__ __launch_bounds__(kThreads, 2) void mx4_few_kernel(
    const Mx4FewArgs<MAXREQ> args, const uint16_t* __restrict__ q, const uint8_t* __restrict__ k_cache,
    const uint8_t* __restrict__ v_cache, const int32_t* __restrict__ block_table) {
  constexpr int kSteps = D / 32;           // products over the head dimension
  constexpr int kBlocks = D / 16;          // output blocks
  constexpr int kKeyBytes = D / 8;         // of a row's codes, in a lane
  constexpr int kValueLanes = D / 32;      // lanes of a value row, 16 bytes of codes each
  constexpr int kValueLoads = 32 * kValueLanes / 64;
  constexpr int kRowBytes = 2 * D;         // of a bf16 row in LDS
  constexpr int kTileBytes = 32 * kRowBytes;
  constexpr int kPitch = D + 4;            // floats from row to row of the sums
  constexpr int kSumBytes = kWaves * 16 * (kPitch + 2) * 4;
  constexpr int kLds = kWaves * kTileBytes > kSumBytes ? kWaves * kTileBytes : kSumBytes;
  __shared__ __attribute__((aligned(1024))) char lds[kLds];
  __shared__ uint32_t s_met[kWaves];                 // whether the wave met a value block that is no number,
  __shared__ int32_t s_torn[kWaves][D / kMx4Block];  // then the first key of which, by columns
  using KeyCodes = std::conditional_t<D == 128, u32x4, u32x2>;

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int i16 = lane & 15, q4 = lane >> 4;
  const auto& t = args.table;
  const int g = t.group_heads, hq = g * t.kv_heads, page_shift = t.page_shift;
  const uint32_t tile = (uint32_t)(uintptr_t)(LDS_PTR(char))lds + wave * kTileBytes;

  // the workgroup's part
  const FewLanes<MAXREQ> requests(t, lane);
  const int group = blockIdx.x;
  const int r = requests.find(requests.group_start, group);
  const int in = group - requests.of(requests.group_start, r), parts = requests.of(requests.parts, r);
  const int head = in / parts, cached = requests.of(requests.cached, r);
  const int rows = requests.of(requests.new_len, r) * g, row_start = requests.of(requests.row_start, r);
  const int all_keys = cached + requests.of(requests.new_len, r);
  const int units = (all_keys + kMx4FewKeys - 1) / kMx4FewKeys;
  const int k0 = mx4_first_of(units, parts, in - head * parts) * kMx4FewKeys;
  const int k1 = min(mx4_first_of(units, parts, in - head * parts + 1) * kMx4FewKeys, all_keys);
  const int slot = parts == 1 ? -1 : requests.of(requests.slot_start, r) + in;
  const Cache<D> keys(k_cache, block_table, t, requests.of(requests.req, r), head);
  const Cache<D> values(v_cache, block_table, t, requests.of(requests.req, r), head);
  const int last = k1 - 1;

  struct Pages {  // of eight keys each
    int32_t id[4];
  };
  auto look_up = [&](int key0) __attribute__((always_inline)) {
    Pages p;
#pragma unroll
    for (int e = 0; e < 4; ++e) p.id[e] = keys.page_id(min(key0 + 8 * e, last));
    return p;
  };
  struct Chunk {  // codes and scales of 32 keys
    KeyCodes k[2];
    uint32_t ks[2];
    u32x4 v[kValueLoads];
    uint32_t vs[kValueLoads];
  };
  const int v_row = D == 128 ? (lane >> 4) * 4 + (lane >> 1 & 3) : (lane >> 4) * 8 + (lane >> 1 & 3) * 2 + (lane >> 3 & 1);
  const int v_piece = D == 128 ? (lane >> 3 & 1) * 2 + (lane & 1) : lane & 1;
  const uint32_t k_code = i16 * mx4_code_bytes(D) + q4 * kKeyBytes, k_scale = i16 * mx4_scale_bytes(D) + (D == 128 ? q4 : q4 >> 1);
  const uint32_t v_code = v_row * mx4_code_bytes(D) + v_piece * 16, v_scale = v_row * mx4_scale_bytes(D) + v_piece;
  auto load = [&](int key0, const Pages& p, Chunk& c) __attribute__((always_inline)) {
    if (page_shift >= 4 && key0 + 32 <= k1) {
      // sixteen rows lie in one page: wave-uniform bases, the lane's place in them is known
      int64_t codes[2], scales[2];
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const int64_t page = keys.page_at(p.id[2 * b]);
        codes[b] = page + keys.code_at(key0 + 16 * b);
        scales[b] = page + keys.scale_at(key0 + 16 * b);
      }
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        c.k[b] = *reinterpret_cast<const KeyCodes*>(keys.rows + codes[b] + k_code);
        c.ks[b] = *reinterpret_cast<const uint8_t*>(keys.rows + scales[b] + k_scale);
      }
#pragma unroll
      for (int j = 0; j < kValueLoads; ++j) {
        int64_t code = codes[j], scale = scales[j];
        if constexpr (kValueLoads == 1) {  // (32 rows to a load, the second sixteen from their own base)
          const int64_t code2 = codes[1] - 16 * mx4_code_bytes(D), scale2 = scales[1] - 16 * mx4_scale_bytes(D);
          code = v_row < 16 ? code : code2;
          scale = v_row < 16 ? scale : scale2;
        }
        c.v[j] = *reinterpret_cast<const u32x4*>(values.rows + code + v_code);
        c.vs[j] = *reinterpret_cast<const uint8_t*>(values.rows + scale + v_scale);
      }
      return;
    }
    int64_t at_page[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) at_page[e] = keys.page_at(p.id[e]);
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const int key = min(key0 + b * 16 + i16, last);
      const int64_t low = at_page[2 * b], high = at_page[2 * b + 1];  // (values: chosen between where they lie they would be memory)
      const char* page = keys.rows + (i16 & 8 ? high : low);
      c.k[b] = *reinterpret_cast<const KeyCodes*>(page + keys.code_at(key) + q4 * kKeyBytes);
      c.ks[b] = *reinterpret_cast<const uint8_t*>(page + keys.scale_at(key) + (D == 128 ? q4 : q4 >> 1));
    }
#pragma unroll
    for (int j = 0; j < kValueLoads; ++j) {
      const int row = j * (64 / kValueLanes) + v_row;
      const int key = min(key0 + row, last);
      const int64_t low = at_page[2 * j], high = at_page[2 * j + 1];
      int64_t at = row & 8 ? high : low;
      if constexpr (kValueLoads == 1) {
        const int64_t low2 = at_page[2], high2 = at_page[3];
        at = row & 16 ? (row & 8 ? high2 : low2) : at;
      }
      const char* page = values.rows + at;
      c.v[j] = *reinterpret_cast<const u32x4*>(page + values.code_at(key) + v_piece * 16);
      c.vs[j] = *reinterpret_cast<const uint8_t*>(page + values.scale_at(key) + v_piece);
    }
  };

  Chunk even, odd;
  int key0 = k0 + wave * 32;
  Pages pages = look_up(min(key0, last & -32));
  // queries
  bf16x8 qb[NB][kSteps];
  int visible[NB];  // keys that the row sees
#pragma unroll
  for (int n = 0; n < NB; ++n) {
    const int row = n * 16 + i16, tok = row / g;
    visible[n] = row < rows ? cached + tok + 1 : 0;
    const uint16_t* src = q + ((int64_t)(row_start + tok) * hq + head * g + (row - tok * g)) * D + q4 * (D / 4);
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      u32x4 v = {0, 0, 0, 0};
      if (row < rows) v = *reinterpret_cast<const u32x4*>(src + 8 * s);
      qb[n][s] = __builtin_bit_cast(bf16x8, v);
    }
  }
  f32x4 o[NB][kBlocks];
  float m_run[NB], l_run[NB];
#pragma unroll
  for (int n = 0; n < NB; ++n) {
#pragma unroll
    for (int d = 0; d < kBlocks; ++d) o[n][d] = f32x4{0.f, 0.f, 0.f, 0.f};
    m_run[n] = kNoReference;
    l_run[n] = 0.f;
  }
  bool met = false;       // a value block that is no number
  int32_t torn = kNoKey;  // the first key of which, of the lane's columns

  auto work = [&](int key0, Chunk& c) __attribute__((always_inline)) {
    // scores
    f32x4 sc[NB][2];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const float scale = mx4_scale_value(c.ks[b]);
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        const bf16x8 ka = __builtin_bit_cast(bf16x8, mx4_decode8(c.k[b][s], scale));
#pragma unroll
        for (int n = 0; n < NB; ++n) {
          if (s == 0) sc[n][b] = f32x4{0.f, 0.f, 0.f, 0.f};
          sc[n][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ka, qb[n][s], sc[n][b], 0, 0, 0);
        }
      }
    }
    // values, as bf16 rows to LDS
    own_writes();
#pragma unroll
    for (int j = 0; j < kValueLoads; ++j) {
      if (__any(c.vs[j] >= kTorn)) {
        met = true;
        if (c.vs[j] >= kTorn) {
          torn = min(torn, min(key0 + j * (64 / kValueLanes) + v_row, last));
          c.v[j] = u32x4{0, 0, 0, 0};
          c.vs[j] = 127;
        }
      }
      const float scale = mx4_scale_value(c.vs[j]);
      const int key = j * (64 / kValueLanes) + v_row;
#pragma unroll
      for (int w = 0; w < 4; ++w)
        *(LDS_PTR(mx4_words))(uintptr_t)(tile + key * kRowBytes + (((v_piece * 4 + w) ^ value_swizzle16<D>(key)) << 4)) = mx4_decode8(c.v[j][w], scale);
    }
    own_writes();
    // Probabilities.  No maximum is formed on the way: the reference of a row is a maximum that was, and a chunk whose weights
    // sum to 2^kSlack in a lane is looked at again.
    bf16x8 pb[NB];
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      if (key0 + 32 > min(cached + 1, k1)) {
        const int end = min(visible[n], k1) - key0 - q4 * 4;
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (b * 16 + e >= end) sc[n][b][e] = -INFINITY;
      }
      u32x4 p;
      auto weigh = [&]() __attribute__((always_inline)) {
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float x = __builtin_amdgcn_exp2f(sc[n][e >> 1][(e & 1) * 2] * args.scale_log2 - m_run[n]);
          const float y = __builtin_amdgcn_exp2f(sc[n][e >> 1][(e & 1) * 2 + 1] * args.scale_log2 - m_run[n]);
          p[e] = pack_bf16(x, y);
          sum = add_pair(p[e], sum);
        }
        return sum;
      };
      float sum = weigh();
      if (__any(sum >= kOver)) {
        float top = max3(max3(sc[n][0][0], sc[n][0][1], sc[n][0][2]), sc[n][0][3], max3(sc[n][1][0], sc[n][1][1], sc[n][1][2]));
        top = cross_half_max(cross_quarter_max(fmaxf(top, sc[n][1][3]))) * args.scale_log2;
        // (a row is moved by its own scores alone, whatever the other rows of the wave hold)
        const float m_next = top > m_run[n] + kSlack ? top : m_run[n];
        const float f = m_next == m_run[n] ? 1.f : __builtin_amdgcn_exp2f(m_run[n] - m_next);
        l_run[n] *= f;
#pragma unroll
        for (int d = 0; d < kBlocks; ++d) o[n][d] *= f;
        m_run[n] = m_next;
        sum = weigh();
      }
      l_run[n] += sum;
      pb[n] = __builtin_bit_cast(bf16x8, p);
    }
    // outputs
    const int v_key = 4 * q4 + (i16 >> 2);
    const uint32_t v_at = tile + v_key * kRowBytes + (i16 & 1) * 8;
#pragma unroll
    for (int d = 0; d < kBlocks; ++d) {
      const uint32_t at = v_at + (((2 * d + ((i16 & 3) >> 1)) ^ value_swizzle16<D>(v_key)) << 4);
      const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((LDS_PTR(bf16x4))(uintptr_t)at);
      const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((LDS_PTR(bf16x4))(uintptr_t)(at + 16 * kRowBytes));
      const bf16x8 va = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
      for (int n = 0; n < NB; ++n) o[n][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, pb[n], o[n][d], 0, 0, 0);
    }
  };
  // (No branch around the loads of a chunk ahead: where the ways meet, they would all be waited for.)
  const int last_chunk = last & -32;
  auto fetch = [&](int key, Chunk& c) __attribute__((always_inline)) {
    load(min(key, last_chunk), pages, c);
    pages = look_up(min(key + kMx4FewKeys, last_chunk));
  };
  fetch(key0, even);
  while (key0 < k1) {
    fetch(key0 + kMx4FewKeys, odd);
    work(key0, even);
    key0 += kMx4FewKeys;
    if (key0 >= k1) break;
    fetch(key0 + kMx4FewKeys, even);
    work(key0, odd);
    key0 += kMx4FewKeys;
  }

  // The waves' sums, rescaled to the largest reference: M = max m,  O = sum 2^(m - M) O_w.  A block of rows at a time.
  if (lane == 0) s_met[wave] = met;
  if (met) {
    if (lane < D / kMx4Block) s_torn[wave][lane] = kNoKey;
    own_writes();
    if (torn != kNoKey) atomicMin(&s_torn[wave][v_piece], torn);
  }
  float* xo = reinterpret_cast<float*>(lds);  // [wave][row] x kPitch
  float* xm = xo + kWaves * 16 * kPitch;      // [wave][row]
  float* xl = xm + kWaves * 16;
#pragma unroll
  for (int n = 0; n < NB; ++n) {
    if (n * 16 >= rows) break;
    __syncthreads();  // every wave is done with its tile, or with the block in front
#pragma unroll
    for (int d = 0; d < kBlocks; ++d) *reinterpret_cast<f32x4*>(xo + (wave * 16 + i16) * kPitch + d * 16 + q4 * 4) = o[n][d];
    const float l_wave = cross_half_sum(cross_quarter_sum(l_run[n]));
    if (q4 == 0) {
      xm[wave * 16 + i16] = m_run[n];
      xl[wave * 16 + i16] = l_wave;
    }
    __syncthreads();
    constexpr int kVec = D / 4;  // threads of a row
    const int c = tid % kVec * 4;
    for (int in_block = tid / kVec; in_block < min(16, rows - n * 16); in_block += kThreads / kVec) {
      const int row = n * 16 + in_block;
      float m[kWaves], top = kNoReference;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        m[w] = xm[w * 16 + in_block];
        top = fmaxf(top, m[w]);
      }
      float l = 0.f;
      f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float f = __builtin_amdgcn_exp2f(m[w] - top);
        l += f * xl[w * 16 + in_block];
        v += f * *reinterpret_cast<const f32x4*>(xo + (w * 16 + in_block) * kPitch + c);
      }
      const int tok = row / g;
      if (s_met[0] | s_met[1] | s_met[2] | s_met[3]) {
#pragma unroll
        for (int w = 0; w < kWaves; ++w)
          if (s_met[w] && s_torn[w][c / kMx4Block] <= cached + tok) v = f32x4{NAN, NAN, NAN, NAN};
      }
      if (slot < 0) {
        const float inv = 1.f / l;
        const u32x2 words = {pack_bf16(v[0] * inv, v[1] * inv), pack_bf16(v[2] * inv, v[3] * inv)};
        *reinterpret_cast<u32x2*>(args.out + ((int64_t)(row_start + tok) * hq + head * g + (row - tok * g)) * D + c) = words;
      } else {
        const int64_t part = (int64_t)slot * (16 * NB) + row;
        *reinterpret_cast<f32x4*>(args.part_o + part * D + c) = v;
        if (c == 0) *reinterpret_cast<f32x2*>(args.part_ml + part * 2) = f32x2{top, l};
      }
    }
  }
}

// The parts of a split tile: with M = max m_s,  out = sum 2^(m_s - M) O_s / sum 2^(m_s - M) l_s.  A workgroup for two rows of each, which
// its threads share by parts and join through LDS.  Bound by latency: four parts at a time.  (us with one, two and four or more rows: 5
// requests of 28 rows and 5300 keys 9.7, 9.4 and 10.6, one of 4 rows and 2344 keys with its first kernel 10.9, 10.6 and 11.4.)
constexpr int kJoinRows = 2;
template <int D, int ROWS, int MAXREQ>
__global__ __launch_bounds__(kThreads) void mx4_few_join_kernel(const Mx4FewArgs<MAXREQ> args) {
  constexpr int kVec = D / 4;                // threads of a row
  constexpr int kPlaces = kThreads / kVec;   // rows (and slices of their parts) at a time
  constexpr int kAtOnce = 4;
  __shared__ __attribute__((aligned(16))) float s_o[kPlaces][D];
  __shared__ float s_m[kPlaces], s_l[kPlaces];
  const auto& t = args.table;
  const int g = t.group_heads, hq = g * t.kv_heads;
  const FewLanes<MAXREQ> requests(t, threadIdx.x & 63);
  const int r = requests.find(requests.split_start, blockIdx.x);
  const int head = blockIdx.x - requests.of(requests.split_start, r), parts = requests.of(requests.parts, r);
  const int rows = requests.of(requests.new_len, r) * g, row_start = requests.of(requests.row_start, r);
  const int64_t first = requests.of(requests.slot_start, r) + (int64_t)head * parts;
  const int c = threadIdx.x % kVec * 4, place = threadIdx.x / kVec;
  const int at_once = rows == 1 ? 1 : kJoinRows;
  const int slices = kPlaces / at_once, slice = place / at_once;
  for (int row0 = blockIdx.y * at_once; row0 < rows; row0 += gridDim.y * at_once) {
    const int row = min(row0 + place % at_once, rows - 1);
    float m = kNoReference, l = 0.f;
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    for (int s0 = slice; s0 < parts; s0 += kAtOnce * slices) {
      f32x2 ml[kAtOnce];
      f32x4 x[kAtOnce];
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        const int64_t part = (first + min(s0 + i * slices, parts - 1)) * ROWS + row;
        ml[i] = *reinterpret_cast<const f32x2*>(args.part_ml + part * 2);
        x[i] = *reinterpret_cast<const f32x4*>(args.part_o + part * D + c);
      }
      float top = m;
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) top = fmaxf(top, ml[i][0]);
      const float back = __builtin_amdgcn_exp2f(m - top);
      l *= back;
      v *= back;
      m = top;
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        if (s0 + i * slices >= parts) break;
        const float f = __builtin_amdgcn_exp2f(ml[i][0] - top);
        l += f * ml[i][1];
        v += f * x[i];
      }
    }
    if (slices > 1) {
      *reinterpret_cast<f32x4*>(&s_o[place][c]) = v;
      if (c == 0) {
        s_m[place] = m;
        s_l[place] = l;
      }
      __syncthreads();
      if (slice > 0) continue;
      float top = m;
      for (int i = 1; i < slices; ++i) top = fmaxf(top, s_m[i * at_once + place]);
      const float back = __builtin_amdgcn_exp2f(m - top);
      l *= back;
      v *= back;
      for (int i = 1; i < slices; ++i) {
        const float f = __builtin_amdgcn_exp2f(s_m[i * at_once + place] - top);
        l += f * s_l[i * at_once + place];
        v += f * *reinterpret_cast<const f32x4*>(&s_o[i * at_once + place][c]);
      }
    }
    if (row0 + place % at_once >= rows) continue;
    const float inv = 1.f / l;
    const int tok = row / g;
    *reinterpret_cast<u32x2*>(args.out + ((int64_t)(row_start + tok) * hq + head * g + (row - tok * g)) * D + c) =
        u32x2{pack_bf16(v[0] * inv, v[1] * inv), pack_bf16(v[2] * inv, v[3] * inv)};
  }
}

// --- many rows --------------------------------------------------------------------------------------------------------------
// Four waves of 32 query rows.  The codes of 64 keys and values are converted once for all of them on their way to LDS (a thread
// takes 16 bytes of a row's codes from memory, two rounds ahead).
//
// A wave works off its keys in halves of 32, three at a time: while the scores of half n are turned into probabilities, the
// products form the scores of n + 1 and add the values of n - 1, and the thread converts its share of what the next round of two
// halves reads.  The waves meet once a round.  A unit holds two workgroups, so that each computes through the other's meetings,
// first loads and last stores.
//
// Bound by the products at the rate that power leaves: 8 prompts of 1024..4096 tokens, 32/8 heads 577 us (931 TFLOP/s that count), products 46 %
// of the cycles at 2.1 GHz.  With nothing beside the products a half of two waves takes 1490 cycles where 1024 are nominal, with
// everything 1750.  One workgroup of eight waves and 256 rows, which converts half as often, 602 (without any conversion 557, without
// exponentials 587): a tile's start and end, 20k of 105k cycles, go by with nothing beside them.  All phases of a tile one
// behind the other 713.  Operands of a third to sixth product ahead: no difference.
//
// SMALL: pages of fewer rows than a wave converts.
template <int D, bool SMALL>
__global__ __launch_bounds__(kThreads, 2) void mx4_many_kernel(const Mx4Args args, const uint16_t* __restrict__ q,
                                                               const uint8_t* __restrict__ k_cache, const uint8_t* __restrict__ v_cache,
                                                               const int32_t* __restrict__ block_table) {
  constexpr int kTile = 32 * kWaves;
  static_assert(kTile == kMx4ManyRows, "the plan's");
  constexpr int kSteps = D / 16, kBlocks = D / 32;
  constexpr int kProducts = kSteps + 2 * kBlocks, kAhead = 4;
  constexpr int kExps = 16 / kProducts;            // probabilities beside a product
  constexpr int kRowBytes = 2 * D;                 // of a bf16 row in LDS
  constexpr int kHalfBytes = 32 * kRowBytes, kStageBytes = 2 * kHalfBytes;
  // (keys, D 128: a chunk more from row to row in place of a swizzle, so that the products' places are offsets of the reads: 22 registers and
  // 1 % of the time less)
  constexpr int kKeyRow = D == 128 ? kRowBytes + 16 : kRowBytes, kKeyHalf = 32 * kKeyRow, kKeyRing = 4 * kKeyHalf;
  constexpr int kPieces = D / 32;                    // of 16 bytes, of a row's codes
  constexpr int kWaveRows = 64 / kPieces;            // that a wave converts
  constexpr int kIds = SMALL ? kWaveRows / 8 : 1;    // of pages, of those
  constexpr int kChunks = 128 * kPieces / kThreads;  // of a thread: both matrices' or one
  constexpr int kWords = 4;                          // of a chunk
  constexpr int kHalfWords = kChunks * kWords / 2;   // of a thread beside a half
  constexpr int kTurn = kProducts / (kHalfWords * 4);  // products for each conversion of two codes
  static_assert(kTurn * kHalfWords * 4 == kProducts && kExps * kProducts == 16, "a half's work is dealt to its products");
  __shared__ __attribute__((aligned(1024))) char lds[kKeyRing + 2 * kStageBytes];
  __shared__ int32_t s_torn[kPieces];  // the part's first key of which a value block, of these columns, is no number

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int i32 = lane & 31, hi = lane >> 5;
  const Mx4Table& t = args.table;
  const int g = t.group_heads, hq = g * t.kv_heads;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(LDS_PTR(char))lds;

  // Operands: the first chunk of the lane's key row, and where a lane of the transposing read begins in the first block.  (The
  // further ones' places differ in bits that the row's place leaves free.)
  const uint32_t key_at = lds0 + i32 * kKeyRow + ((hi ^ (D == 128 ? 0 : key_swizzle<D>(i32))) << 4);
  const int v_key = (lane >> 5) * 4 + ((lane & 15) >> 2), v_chunk = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
  const uint32_t value_at = lds0 + kKeyRing + v_key * kRowBytes + (lane & 1) * 8 + ((v_chunk ^ value_swizzle<D>(v_key)) << 4);
  // what this thread converts
  const int first_matrix = kChunks == 2 ? 0 : wave / (kWaves / 2);
  const int piece = D == 128 ? (lane >> 3 & 1) * 2 + (lane & 1) : lane & 1;
  const int wave_row = D == 128 ? (lane >> 4) * 4 + (lane >> 1 & 3) : (lane >> 4) * 8 + (lane >> 1 & 3) * 2 + (lane >> 3 & 1);
  const int first_row = wave * kWaveRows % 64, in_round = first_row + wave_row;
  const uint32_t put_keys = lds0 + in_round * kKeyRow + (((piece * kWords) ^ (D == 128 ? 0 : key_swizzle<D>(in_round & 31))) << 4);
  const uint32_t put_values = lds0 + kKeyRing + in_round * kRowBytes + (((piece * kWords) ^ value_swizzle<D>(in_round & 31)) << 4);

  for (Share<kTile> it(t, lane); !it.done(); it.advance()) {
    const Cache<D> cache(k_cache, block_table, t, it.rq.req, it.at.head);
    const int local = wave * 32 + i32;
    const bool row_ok = local < it.rows;
    const int row = it.row0 + local, tok = row / g;
    const int visible = min(row_ok ? it.rq.cached + tok + 1 : 0, it.k1);
    const int64_t q_off = ((int64_t)(it.rq.row_start + tok) * hq + it.at.head * g + (row - tok * g)) * D;
    // halves of the part; whether the wave has rows, and the keys that all of them see
    const int rounds = (it.k1 - it.k0 + 31) / 32;
    const bool rows_here = wave * 32 < it.rows;
    const int least = min(it.rq.cached + (it.row0 + wave * 32) / g + 1, it.k1);
    bf16x8 qb[kSteps];
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      u32x4 v = {0, 0, 0, 0};
      if (row_ok) v = *reinterpret_cast<const u32x4*>(q + q_off + 16 * s + 8 * hi);
      qb[s] = __builtin_bit_cast(bf16x8, v);
    }
    f32x16 o[kBlocks];
#pragma unroll
    for (int d = 0; d < kBlocks; ++d)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[d][e] = 0.f;
    float m_run = kNoReference, l_run = 0.f;
    f32x16 s0, s1;                                      // scores of an even and an odd half
    u32x4 p0[2], p1[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};  // and their probabilities, as operands
    int32_t torn = kNoKey;  // the first key of which a block that this thread converts is no number
    if (tid < kPieces) s_torn[tid] = kNoKey;

    // Round u of two halves, 2u and 2u + 1, reads the keys of halves 2u + 1 and 2u + 2 and the values of 2u - 1 and 2u, and converts
    // those of round u + 1.  (In place of groups of rows that are not the part's its first or last group; what of their rows no query
    // sees is masked, and the values of half -1 have no weight.)
    struct Chunk {
      u32x4 codes[kChunks];
      uint32_t scales[kChunks];
      int key[kChunks];  // first of the wave's rows
    };
    auto group_of = [&](int u, int j) {
      return max(min(it.k0 + u * 64 + (first_matrix + j == 0 ? 32 : -32) + first_row, (it.k1 - 1) & -kWaveRows), it.k0);
    };
    struct PageIds {
      int32_t id[kChunks][kIds];
    };
    auto look_up = [&](int u) __attribute__((always_inline)) {
      PageIds p;
#pragma unroll
      for (int j = 0; j < kChunks; ++j)
#pragma unroll
        for (int i = 0; i < kIds; ++i) p.id[j][i] = cache.page_id(min(group_of(u, j) + 8 * i, it.k1 - 1));
      return p;
    };
    auto load = [&](int u, const PageIds& p, Chunk& c) __attribute__((always_inline)) {
#pragma unroll
      for (int j = 0; j < kChunks; ++j) {
        const uint8_t* matrix = first_matrix + j == 0 ? k_cache : v_cache;
        c.key[j] = group_of(u, j);
        if constexpr (SMALL) {
          int64_t at = cache.page_at(p.id[j][0]);
#pragma unroll
          for (int i = 1; i < kIds; ++i) {
            const int64_t other = cache.page_at(p.id[j][i]);
            at = wave_row >= 8 * i ? other : at;
          }
          const int key = c.key[j] + wave_row;
          c.codes[j] = *reinterpret_cast<const u32x4*>(matrix + at + cache.code_at(key) + piece * 16);
          c.scales[j] = matrix[at + cache.scale_at(key) + piece];
        } else {
          const uint8_t* page = matrix + cache.page_at(p.id[j][0]);
          c.codes[j] = *reinterpret_cast<const u32x4*>(page + cache.code_at(c.key[j]) + (uint32_t)(wave_row * kPieces + piece) * 16);
          c.scales[j] = (page + cache.scale_at(c.key[j]))[(uint32_t)(wave_row * kPieces + piece)];
        }
      }
    };
    // Where a round's chunks go, and their scales.  (A value block that is no number: any that are.)
    struct Target {
      uint32_t at[kChunks];
      float scale[kChunks];
    };
    auto target = [&](uint32_t stage, const Chunk& c) __attribute__((always_inline)) {
      Target to;
#pragma unroll
      for (int j = 0; j < kChunks; ++j) {
        to.at[j] = first_matrix + j == 0 ? put_keys + stage * (2 * kKeyHalf) : put_values + stage * kStageBytes;
        const bool bad = first_matrix + j == 1 && c.scales[j] >= kTorn;
        if (first_matrix + j == 1) torn = min(torn, bad && wave_row < it.k1 - c.key[j] ? c.key[j] + wave_row : kNoKey);
        to.scale[j] = mx4_scale_value(bad ? 127u : c.scales[j]);
      }
      return to;
    };
    constexpr auto kFirst = std::integral_constant<int, 0>{};
    constexpr auto kSecond = std::integral_constant<int, 1>{};
    uint32_t here = 0, ahead = 1;  // the stages of the round and the next one
    uint32_t made[4];
    // the n-th conversion of a round
    auto convert = [&](auto n_c, const Chunk& c, const Target& to) __attribute__((always_inline)) {
      constexpr int n = decltype(n_c)::value, word = n / 4, j = word / kWords, w = word % kWords;
      made[n % 4] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c.codes[j][w], to.scale[j], n % 4));
      if constexpr (n % 4 == 3)
        *(LDS_PTR(u32x4))(uintptr_t)(D == 128 && j == 0 ? to.at[j] + w * 16 : to.at[j] ^ (uint32_t)(w << 4)) = u32x4{made[0], made[1], made[2], made[3]};
    };
    auto meet = [&]() __attribute__((always_inline)) { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); };

    auto probability = [&](const f32x16& sc, int e) __attribute__((always_inline)) { return __builtin_amdgcn_exp2f(sc[e] * args.scale_log2 - m_run); };
    auto score_product = [&](u32x4 a, int n, f32x16& sn) __attribute__((always_inline)) {
      f32x16 from = sn;
      if (n == 0) {
#pragma unroll
        for (int e = 0; e < 16; ++e) from[e] = 0.f;
      }
      sn = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), qb[n], from, 0, 0, 0);
    };
    auto key_operand = [&](uint32_t stage, int second, int n) __attribute__((always_inline)) -> u32x4 {
      const uint32_t row = key_at + stage * (2 * kKeyHalf);
      return *(const LDS_PTR(u32x4))(uintptr_t)((D == 128 ? row + n * 32 : row ^ (uint32_t)(n << 5)) + second * kKeyHalf);
    };
    u32x4 staged[kAhead];  // operands of the next products
    // Products of a half, the first or second of its round: the scores of the stage's keys into `sn`, the stage's values under the
    // probabilities `pv`; beside them the probabilities of the scores `sc` into `pn`, whose sum is returned, and conversions.
    auto round = [&](uint32_t stage, auto second, f32x16& sn, const u32x4 (&pv)[2], const f32x16& sc, u32x4 (&pn)[2],
                     const Chunk& c, const Target& to) __attribute__((always_inline)) -> float {
      auto operand = [&](int n) __attribute__((always_inline)) -> u32x4 {
        if (n < kSteps) return key_operand(stage, decltype(second)::value, n);
        if (n >= kProducts) return key_operand(stage, 1, n - kProducts);  // (of the second half)
        const int k = (n - kSteps) / kBlocks, d = (n - kSteps) % kBlocks;
        const uint32_t at = ((value_at + stage * kStageBytes) ^ (uint32_t)(d << 6)) + decltype(second)::value * kHalfBytes;
        const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((LDS_PTR(bf16x4))(uintptr_t)(at + 2 * k * 8 * kRowBytes));
        const bf16x4 up = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((LDS_PTR(bf16x4))(uintptr_t)(at + (2 * k + 1) * 8 * kRowBytes));
        return __builtin_bit_cast(u32x4, __builtin_shufflevector(lo, up, 0, 1, 2, 3, 4, 5, 6, 7));
      };
      __builtin_amdgcn_s_setprio(1);
      __builtin_amdgcn_sched_barrier(0);
      float sum = 0.f, pair[2];
      auto step = [&](auto n_c) __attribute__((always_inline)) {
        constexpr int n = decltype(n_c)::value;
        if constexpr (n < kSteps) {
          score_product(staged[n % kAhead], n, sn);
        } else {
          constexpr int j = n - kSteps;
          o[j % kBlocks] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, staged[n % kAhead]),
                                                                   __builtin_bit_cast(bf16x8, pv[j / kBlocks]), o[j % kBlocks], 0, 0, 0);
        }
        if constexpr (n + kAhead < kProducts || !decltype(second)::value) staged[n % kAhead] = operand(n + kAhead);
#pragma unroll
        for (int i = 0; i < kExps; ++i) {
          const int e = n * kExps + i;
          pair[e & 1] = probability(sc, e);
          if (e & 1) {
            const uint32_t two = pack_bf16(pair[0], pair[1]);
            pn[e >> 3][(e & 7) >> 1] = two;
            sum = add_pair(two, sum);
            asm volatile("" : "+v"(sum));  // (keeps the step in its place)
          }
        }
        if constexpr (n % kTurn == kTurn - 1) convert(std::integral_constant<int, decltype(second)::value * kHalfWords * 4 + n / kTurn>{}, c, to);
        __builtin_amdgcn_sched_barrier(0);
      };
      [&]<int... N>(std::integer_sequence<int, N...>) __attribute__((always_inline)) { (step(std::integral_constant<int, N>{}), ...); }
      (std::make_integer_sequence<int, kProducts>{});
      __builtin_amdgcn_s_setprio(0);
      return sum;
    };
    auto convert_half = [&](auto second, const Chunk& c, const Target& to) __attribute__((always_inline)) {
      [&]<int... N>(std::integer_sequence<int, N...>) __attribute__((always_inline)) {
        (convert(std::integral_constant<int, decltype(second)::value * kHalfWords * 4 + N>{}, c, to), ...);
      }
      (std::make_integer_sequence<int, kHalfWords * 4>{});
    };
    auto row_max = [&](const f32x16& sc) __attribute__((always_inline)) {
      float mx = sc[0];
#pragma unroll
      for (int e = 1; e < 16; ++e) mx = fmaxf(mx, sc[e]);
      return cross_half_max(mx) * args.scale_log2;
    };
    // Where the sum says that a probability may have passed the slack: a reference moves to its row's maximum if that did, and
    // the probabilities are formed again.
    auto settle = [&](const f32x16& sc, u32x4 (&pn)[2], float sum) __attribute__((always_inline)) {
      if (__any(sum >= kOver)) {
        const float mx = row_max(sc);
        const float m_new = mx > m_run + kSlack ? mx : m_run;
        const float f = m_new == m_run ? 1.f : __builtin_amdgcn_exp2f(m_run - m_new);
        l_run *= f;
#pragma unroll
        for (int d = 0; d < kBlocks; ++d)
#pragma unroll
          for (int e = 0; e < 16; ++e) o[d][e] *= f;
        m_run = m_new;
        sum = 0.f;
#pragma unroll
        for (int e = 0; e < 16; e += 2) {
          const uint32_t two = pack_bf16(probability(sc, e), probability(sc, e + 1));
          pn[e >> 3][(e & 7) >> 1] = two;
          sum = add_pair(two, sum);
        }
      }
      l_run += sum;
    };
    // The n-th half: one that every row sees whole,
    auto seen_half = [&](int n, auto second, f32x16& sc, f32x16& sn, u32x4 (&pn)[2], u32x4 (&po)[2], const Chunk& c, const Target& to) __attribute__((always_inline)) {
      if (n == 0) m_run = fmaxf(row_max(sc), kNoReference);
      settle(sc, pn, round(here, second, sn, po, sc, pn, c, to));
    };
    // one that not all rows see, or none (behind the last one there is a round for its values alone),
    auto half = [&](int n, auto second, f32x16& sc, f32x16& sn, u32x4 (&pn)[2], u32x4 (&po)[2], const Chunk& c, const Target& to) __attribute__((always_inline)) {
      if (it.k0 + n * 32 + 32 > least) {
        const int end = visible - it.k0 - n * 32 - hi * 4;
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if ((e >> 2) * 8 + (e & 3) >= end) sc[e] = -INFINITY;
      }
      seen_half(n, second, sc, sn, pn, po, c, to);
    };
    // and one of a wave without rows.
    auto no_half = [&](int, auto second, f32x16&, f32x16&, u32x4 (&)[2], u32x4 (&)[2], const Chunk& c, const Target& to) __attribute__((always_inline)) {
      convert_half(second, c, to);
    };

    Chunk at_hand, next;
    {
      Chunk early[2];
      const PageIds ids[3] = {look_up(-1), look_up(0), look_up(1)};
      load(-1, ids[0], early[0]);
      load(0, ids[1], early[1]);
      load(1, ids[2], at_hand);
#pragma unroll
      for (int u = -1; u < 1; ++u) {
        const Target to = target(u < 0 ? ahead : here, early[u + 1]);
        convert_half(kFirst, early[u + 1], to);
        if (u == 0 || kChunks == 1) convert_half(kSecond, early[u + 1], to);  // (of the round in front of the first one the keys are wanted)
      }
    }
    PageIds pages = look_up(2);
    meet();
    if (rows_here) {
#pragma unroll
      for (int n = 0; n < kSteps; ++n) score_product(key_operand(ahead, 1, n), n, s0);
    }
    auto two_halves = [&](int n, auto&& one) __attribute__((always_inline)) {
      meet();
      load(n / 2 + 2, pages, next);
      pages = look_up(n / 2 + 3);
      const Target to = target(ahead, at_hand);
#pragma unroll
      for (int n = 0; n < kAhead; ++n) staged[n] = key_operand(here, 0, n);
      one(n, kFirst, s0, s1, p0, p1, at_hand, to);
#pragma unroll
      for (int n = 0; n < kAhead; ++n) asm volatile("" : "+v"(staged[n]));
      one(n + 1, kSecond, s1, s0, p1, p0, at_hand, to);
      at_hand = next;
      const uint32_t done = here;
      here = ahead;
      ahead = done;
    };
    // First the halves that all rows of the workgroup see, without masks.
    const int clear = max(0, (min(it.rq.cached + it.row0 / g + 1, it.k1) - it.k0) / 32) & ~1;
    int n = 0;
    if (rows_here) {
      for (; n < clear; n += 2) two_halves(n, seen_half);
      for (; n <= rounds; n += 2) two_halves(n, half);
    } else {
      for (; n <= rounds; n += 2) two_halves(n, no_half);
    }

    if (torn != kNoKey) atomicMin(&s_torn[piece], torn);
    __syncthreads();  // every wave is done with the rings, and the keys are known
    if (row_ok) {
      const float l = cross_half_sum(l_run);
#pragma unroll
      for (int d = 0; d < kBlocks; ++d)
        if (s_torn[d] < visible)
#pragma unroll
          for (int e = 0; e < 16; ++e) o[d][e] = NAN;
      const float inv = 1.f / l;
      const int64_t part = it.slot * kTile + local;
#pragma unroll
      for (int d = 0; d < kBlocks; ++d)
#pragma unroll
        for (int r4 = 0; r4 < 4; ++r4) {
          const f32x4 v = {o[d][4 * r4], o[d][4 * r4 + 1], o[d][4 * r4 + 2], o[d][4 * r4 + 3]};
          const int c = d * 32 + r4 * 8 + hi * 4;
          if (it.slot < 0)
            *reinterpret_cast<u32x2*>(args.out + q_off + c) = u32x2{pack_bf16(v[0] * inv, v[1] * inv), pack_bf16(v[2] * inv, v[3] * inv)};
          else
            *reinterpret_cast<f32x4*>(args.part_o + part * D + c) = v;
        }
      if (it.slot >= 0 && hi == 0) *reinterpret_cast<f32x2*>(args.part_ml + part * 2) = f32x2{m_run, l};
    }
    if (tid == 0 && !t.by_tile && it.ends()) {
      const bool begins = it.slot == mx4_slot(it.group, false);
      *reinterpret_cast<u32x4*>(args.splits + 8 * (int64_t)it.group) =
          u32x4{begins ? (uint32_t)it.rows : 0u, (uint32_t)it.row0, (uint32_t)it.rq.row_start, (uint32_t)it.at.head};
      args.splits[8 * (int64_t)it.group + 4] = begins ? it.last_group() : 0;
    }
    __syncthreads();
  }
}

// --- join -------------------------------------------------------------------------------------------------------------------
// The parts of split tiles: with M = max m_s,  out = sum 2^(m_s - M) O_s / sum 2^(m_s - M) l_s, in the order of the keys.  Workgroup
// i has the tile that begins in share i and ends in a further one.  Bound by latency: what the tile is was left by its first part, and
// four parts are read at a time.
template <int D>
__global__ __launch_bounds__(kThreads) void mx4_join_kernel(const Mx4Args args) {
  constexpr int kAtOnce = 4;
  const int g = args.table.group_heads, hq = g * args.table.kv_heads;
  const auto* split = (const __attribute__((address_space(4))) int32_t*)(uintptr_t)(args.splits + 8 * (int64_t)blockIdx.x);  // (scalar loads)
  const int rows = split[0], row0 = split[1], row_start = split[2], head = split[3], last = split[4];
  const int first = blockIdx.x;
  constexpr int kVec = D / 4;
  const int c = threadIdx.x % kVec * 4;
  for (int r = blockIdx.y * (kThreads / kVec) + threadIdx.x / kVec; r < rows; r += gridDim.y * (kThreads / kVec)) {
    float m = kNoReference, l = 0.f;
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    for (int group = first; group <= last; group += kAtOnce) {
      f32x2 ml[kAtOnce];
      f32x4 x[kAtOnce];
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        const int64_t part = mx4_slot(min(group + i, last), group + i > first) * kMx4ManyRows + r;
        ml[i] = *reinterpret_cast<const f32x2*>(args.part_ml + part * 2);
        x[i] = *reinterpret_cast<const f32x4*>(args.part_o + part * D + c);
      }
      float top = m;
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) top = fmaxf(top, ml[i][0]);
      const float back = __builtin_amdgcn_exp2f(m - top);
      l *= back;
      v *= back;
      m = top;
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        if (group + i > last) break;
        const float f = __builtin_amdgcn_exp2f(ml[i][0] - top);
        l += f * ml[i][1];
        v += f * x[i];
      }
    }
    const float inv = 1.f / l;
    const int row = row0 + r, tok = row / g;
    *reinterpret_cast<u32x2*>(args.out + ((int64_t)(row_start + tok) * hq + head * g + (row - tok * g)) * D + c) =
        u32x2{pack_bf16(v[0] * inv, v[1] * inv), pack_bf16(v[2] * inv, v[3] * inv)};
  }
}

struct Mx4Tensors {
  const uint16_t* q;
  const uint8_t *k_cache, *v_cache;
  const int32_t* block_table;
  uint16_t* out;
  float scale_log2;
};

int last_error() {
  const hipError_t e = hipGetLastError();
  if (e == hipSuccess) return EFIM_OK;
  set_last_hip_error(e);
  return EFIM_ERR_LAUNCH;
}

template <int D, int NB, int MAXREQ>
int launch_few(const efim_batch_t* b, const Mx4FewPlan& plan, const Mx4Tensors& x, char* workspace, hipStream_t stream) {
  Mx4FewArgs<MAXREQ> args;
  args.scale_log2 = x.scale_log2;
  args.part_o = reinterpret_cast<float*>(workspace);
  args.part_ml = reinterpret_cast<float*>(workspace + mx4_bytes(plan.slots, plan.row_tile, D).off_ml);
  args.out = x.out;
  Mx4Cursor at;
  while (mx4_next(b, plan, &at, &args.table)) {
    mx4_few_kernel<D, NB, MAXREQ><<<args.table.groups, kThreads, 0, stream>>>(args, x.q, x.k_cache, x.v_cache, x.block_table);
    if (args.table.splits > 0) mx4_few_join_kernel<D, 16 * NB, MAXREQ><<<dim3((unsigned)args.table.splits, 16 * NB / kJoinRows), kThreads, 0, stream>>>(args);
    const int rc = last_error();
    if (rc != EFIM_OK) return rc;
  }
  return EFIM_OK;
}

template <int D>
int launch_many(const efim_batch_t* b, const Mx4ManyPlan& plan, const Mx4Tensors& x, char* workspace, hipStream_t stream) {
  Mx4Args args;
  args.scale_log2 = x.scale_log2;
  args.part_o = reinterpret_cast<float*>(workspace);
  args.part_ml = reinterpret_cast<float*>(workspace + mx4_bytes(plan.slots, kMx4ManyRows, D).off_ml);
  args.splits = reinterpret_cast<int32_t*>(workspace + mx4_bytes(plan.slots, kMx4ManyRows, D).total);
  args.out = x.out;
  constexpr int kAtOnce = kThreads / (D / 4);
  Mx4Cursor at;
  while (mx4_next(b, plan, &at, &args.table)) {
    const int groups = args.table.groups;
    const int launched = args.table.by_tile ? groups : (groups + kXcdCount - 1) / kXcdCount * kXcdCount;
    auto* kernel = b->page_size < 2048 / D ? mx4_many_kernel<D, true> : mx4_many_kernel<D, false>;
    kernel<<<launched, kThreads, 0, stream>>>(args, x.q, x.k_cache, x.v_cache, x.block_table);
    if (!args.table.by_tile && groups > 1)
      mx4_join_kernel<D>
          <<<dim3((unsigned)groups - 1, kMx4ManyRows / kAtOnce), kThreads, 0, stream>>>(args);
    const int rc = last_error();
    if (rc != EFIM_OK) return rc;
  }
  return EFIM_OK;
}

// The plans of a batch's two classes and where their partial results lie.
struct Mx4Work {
  Mx4FewPlan few;
  Mx4ManyPlan many;
  size_t many_at = 0, total = 0;
  explicit Mx4Work(const efim_batch_t* b) : few(plan_mx4_few(b, compute_units())), many(plan_mx4_many(b, compute_units())) {
    if (few.any) many_at = mx4_bytes(few.slots, few.row_tile, b->head_dim).total;
    total = many_at + (many.any ? mx4_bytes(many.slots, kMx4ManyRows, b->head_dim).total + (many.slots / 2 * 32 + 255) / 256 * 256 : 0);
    if (total < 256) total = 256;
  }
};

int validate(const efim_batch_t* batch, int64_t* total) {
  const int rc = validate_batch(batch, total);
  if (rc != EFIM_OK) return rc;
  // (rows and workgroups are counted in 32 bits)
  return batch->num_kv_heads > 1 << 16 || *total * batch->num_q_heads > (int64_t)1 << 30 ? EFIM_ERR_UNSUPPORTED : EFIM_OK;
}

}  // namespace
}  // namespace efim

extern "C" {

size_t efim_mx4_workspace_bytes(const efim_batch_t* batch) {
  int64_t total = 0;
  if (efim::validate(batch, &total) != EFIM_OK) return 0;
  return efim::Mx4Work(batch).total;
}

int efim_extend_attention_mx4(const efim_batch_t* batch, const void* q, const void* k_cache, const void* v_cache, void* out,
                              float sm_scale, void* workspace, size_t workspace_bytes, void* stream) {
  using namespace efim;
  int64_t total = 0;
  const int rc = validate(batch, &total);
  if (rc != EFIM_OK) return rc;
  if (!(sm_scale >= 0.f) || sm_scale - sm_scale != 0.f) return EFIM_ERR_INVALID_ARG;
  if (total == 0) return EFIM_OK;
  if (!q || !k_cache || !v_cache || !out) return EFIM_ERR_INVALID_ARG;
  for (const void* p : {q, k_cache, v_cache, (const void*)out})
    if (!aligned16(p)) return EFIM_ERR_INVALID_ARG;
  if (!aligned4(batch->block_table)) return EFIM_ERR_INVALID_ARG;
  const Mx4Work work(batch);
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u) || workspace_bytes < work.total) return EFIM_ERR_WORKSPACE;
  const float scale = sm_scale == 0.f ? 1.f / sqrtf((float)batch->head_dim) : sm_scale;
  const Mx4Tensors x{static_cast<const uint16_t*>(q),     static_cast<const uint8_t*>(k_cache), static_cast<const uint8_t*>(v_cache),
                     batch->block_table, static_cast<uint16_t*>(out), scale * 1.4426950408889634f};
  hipStream_t s = static_cast<hipStream_t>(stream);
  char* at = static_cast<char*>(workspace);
  const bool wide = batch->head_dim == 128, small = batch->batch <= 64;
  if (work.few.any) {
    auto* launch = work.few.row_tile == 16 ? (wide ? (small ? launch_few<128, 1, 64> : launch_few<128, 1, kMx4FewReqs>)
                                                   : (small ? launch_few<64, 1, 64> : launch_few<64, 1, kMx4FewReqs>))
                                           : (wide ? (small ? launch_few<128, 2, 64> : launch_few<128, 2, kMx4FewReqs>)
                                                   : (small ? launch_few<64, 2, 64> : launch_few<64, 2, kMx4FewReqs>));
    const int done = launch(batch, work.few, x, at, s);
    if (done != EFIM_OK) return done;
  }
  if (work.many.any) return (wide ? launch_many<128> : launch_many<64>)(batch, work.many, x, at + work.many_at, s);
  return EFIM_OK;
}

}  // extern "C"
