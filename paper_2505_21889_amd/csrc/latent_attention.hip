// efim_latent_attention: causal softmax attention of the new tokens over the paged latent cache, absorbed form: a token's
// row l_t of 576 elements is the key of all heads and its first 512 are their value,
//   s = sm_scale <q, l_t>,  p = softmax(s),  o = sum_t p_t l_t[:512].
// Rows are (token, head) pairs, so all heads of a request read its rows once.  Work items are tiles of rows against
// ranges of keys; partial results of a tile that several ranges share are combined by a second kernel.
//
// A key tile is 32 rows = 36 KB, gathered through the block table straight into LDS (nine 1 KB loads to eight rows, which
// lie in one page) with the 16-byte chunks of a row swizzled, and read twice: row by row as the operand of S^T = L Q^T and
// through the transposing read as the operand of O^T += L^T P^T.  A lane holds scores of ONE query row, so that maximum
// and sum of the softmax are per-lane scalars, and the probabilities, rounded to bf16 (8 significant bits, as the rows that
// they weigh), are the second product's operand as they stand.  Sums are fp32.
#include <cstddef>
#include <type_traits>

#include "efim_internal.h"
#include "latent_plan.h"
#include "latent_device.h"
#include "rope_math.h"
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

constexpr int kTileKeys = kLatentTileKeys;
constexpr int kTileBytes = kTileKeys * kRowBytes;
constexpr int kGroups = kTileKeys / kGroupKeys;
constexpr int kWaves = 4;
constexpr float kSlack = 8.f;            // log2 units by which a row's maximum may outgrow its reference
constexpr float kNoReference = -3.0e38f;  // of a row that has seen no key: any finite score moves it

struct LatentArgs {
  LatentTable table;
  float scale_log2;  // sm_scale * log2(e)
  // Partial results of the ranges of split tiles, [slot][row tile]: the unnormalised output O as binary16 values O / a with
  // a = 2^-15 max |O| over the row (2^-126 at least), and (reference in log2 units, sum, a, -).  Half the bytes of fp32; what
  // is within 2^-29 of the row's largest keeps 11 significant bits, a fraction of what the output's own rounding to bf16 costs.
  uint16_t* part_o;
  float* part_ml;
};

// The tile that a unit lies in, by the whole wave: 64 tiles of the request at a time.
struct Place {
  int r;           // request of the launch
  int tile;
  int units;       // of the tile
  int64_t first;   // unit of the launch at which the tile begins
};
template <int TILE>
__device__ __forceinline__ Place find_tile(const LatentTable& t, const Requests& requests, int64_t unit, int lane) {
  Place at;
  at.r = requests.find(unit, lane);
  const LatentReq q = requests.get(at.r);
  at.first = q.unit_start;
  at.tile = 0;
  at.units = latent_units_of(q, t.heads, TILE, 0);
  const int tiles = latent_tiles(q, t.heads, TILE);
  if (tiles == 1) return at;
  for (int t0 = 0; t0 < tiles; t0 += kLatentWaveTiles) {
    const int mine = t0 + lane < tiles ? latent_units_of(q, t.heads, TILE, t0 + lane) : 0;
    LatentWaveUnits upto = mine;  // of the lanes up to this one
#pragma unroll
    for (int by = 1; by < 64; by <<= 1) {
      const LatentWaveUnits other = __shfl_up(upto, by);
      if (lane >= by) upto += other;
    }
    const uint64_t in_front = __ballot(at.first + upto <= unit);  // tiles that end in front of the unit
    if (in_front != ~0ull) {
      const int k = __popcll(in_front);
      at.tile = t0 + k;
      at.units = __builtin_amdgcn_readlane(mine, k);
      at.first += (int64_t)(LatentWaveUnits)__builtin_amdgcn_readlane(upto, k) - at.units;
      return at;
    }
    at.first += (LatentWaveUnits)__builtin_amdgcn_readlane(upto, 63);
  }
  return at;
}

// A workgroup's share of the units, a tile's part at a time, the last one first: where a share is about a tile, its last part
// begins at its tile's first key and its first part goes on from about the key where that one ends, so that the workgroups of
// a request are at the same keys at a time and gather them from their XCD's L2.
template <int TILE>
struct Share {
  const LatentTable& t;
  Place at;
  int group;
  int64_t begin, end;  // units that are left
  int64_t next;        // the part's first
  // the part at hand
  LatentReq rq;
  int row0, rows;      // of the request
  int k0, k1;          // keys
  int slot;            // partial result, -1: the workgroup has the whole tile
  int64_t packed;      // packed query row of the tile's first row

  __device__ __forceinline__ Share(const LatentTable& table, int lane) : t(table) {
    const Requests requests(table, lane);
    // an XCD takes neighbouring shares, which have rows of the cache in common
    group = (int)(blockIdx.x % kXcds) * (int)(gridDim.x / kXcds) + (int)(blockIdx.x / kXcds);
    begin = end = 0;
    if (group >= t.groups) return;
    if (t.by_tile) {
      at.r = requests.find_group(group, lane);
      rq = requests.get(at.r);
      const int n = (int)(rq.unit_start >> 32), k = group - (int)(uint32_t)rq.unit_start;
      at.tile = k / n;
      at.units = latent_units_of(rq, t.heads, TILE, at.tile);
      at.first = 0;
      begin = LatentTable::first_of(at.units, n, k - at.tile * n);
      end = LatentTable::first_of(at.units, n, k - at.tile * n + 1);
    } else {
      begin = t.first_unit(group);
      end = t.first_unit(group + 1);
      at = find_tile<TILE>(t, requests, end - 1, lane);
      rq = requests.get(at.r);
    }
    part();
  }
  __device__ __forceinline__ bool done() const { return end <= begin; }
  __device__ __forceinline__ void part() {
    row0 = at.tile * TILE;
    rows = latent_rows_of(rq, t.heads, TILE, at.tile);
    const bool first = begin >= at.first;
    const int u0 = first ? (int)(begin - at.first) : 0, u1 = (int)(end - at.first);
    next = at.first + u0;
    k0 = u0 * kTileKeys;
    k1 = min(u1 * kTileKeys, latent_keys_of(rq, t.heads, TILE, at.tile));
    slot = u0 == 0 && u1 == at.units ? -1 : latent_slot(group, first);
    packed = (int64_t)rq.row_start * t.heads + row0;
  }
  __device__ __forceinline__ void advance() {
    end = at.first;
    if (done()) return;
    if (at.tile == 0) {
      rq = t.req[--at.r];
      at.tile = latent_tiles(rq, t.heads, TILE);
    }
    --at.tile;
    at.units = latent_units_of(rq, t.heads, TILE, at.tile);
    at.first = end - at.units;
    part();
  }
};

// The scale of a partial result whose largest magnitude is `top`: never below fp32's least normal number, so that its
// reciprocal is finite.  Rows of less than 2^-111 are then stored as less than 2^15; fp32's normal numbers keep their 11 bits.
constexpr float kPartScale = 0x1p-15f;
__device__ __forceinline__ float part_scale(float top) { return fmaxf(top * kPartScale, 0x1p-126f); }
constexpr float kOver = 256.f;  // 2^kSlack: a sum of rounded probabilities is never below its largest one
constexpr int kZeros = kWaves * kTileBytes;  // 1 KB of zeros behind the tiles, in place of values that are not finite
constexpr int kTornAt = kZeros + 1024;      // a word for each wave: whether it left a key out
constexpr int kLdsBytes = kTornAt + 4 * kWaves;

// LDS addresses of a wave's operands in a tile at 0.  The low bits of a chunk take part in the swizzle and need an address
// each, all else goes into the offset field of the read.
template <int ROWS>
struct Operands {
  static constexpr bool R32 = ROWS == 32;
  static constexpr int kSteps = R32 ? kLatentRow / 16 : kLatentRow / 32;  // products along a row
  static constexpr int kBlocks = kLatentRank / ROWS;                       // output blocks
  static constexpr int kKeyBlocks = kTileKeys / ROWS;                      // of a tile
  static constexpr int kKeyAddrs = R32 ? 4 : 2, kValueAddrs = R32 ? 2 : 4;
  static constexpr int kKeyGroups = R32 ? 4 : 2, kGroupRows = R32 ? 8 : 16;  // rows of a value operand: value_key + multiples
  using Acc = std::conditional_t<R32, f32x16, f32x4>;
  static constexpr int kAcc = R32 ? 16 : 4;
  static constexpr int kScores = kAcc * kKeyBlocks;
  uint32_t key_at, value_at;  // of the first; the others differ in the swizzled bits, 4 to 6
  int value_key;

  __device__ __forceinline__ explicit Operands(int lane) {
    const int i = lane % ROWS, part = lane / ROWS;
    key_at = i * kRowBytes + ((part ^ swizzle(i)) << 4);
    const int w16 = lane & 15, blk = lane >> 4;
    value_key = (R32 ? (blk >> 1) * 4 : blk * 4) + (w16 >> 2);
    const int chunk = (R32 ? 2 * (blk & 1) : 0) + ((w16 & 3) >> 1);
    value_at = value_key * kRowBytes + ((chunk ^ swizzle(value_key)) << 4) + (w16 & 1) * 8;
  }
  // (formed again in every tile: held through the loop the derived addresses cost the registers that operands wait in)
  __device__ __forceinline__ void forget() { asm volatile("" : "+v"(key_at), "+v"(value_at)); }
  static_assert(kRowBytes % 128 == 0, "rows leave the swizzled bits alone");
  static __device__ __forceinline__ Acc product(bf16x8 a, bf16x8 b, Acc c) {
    if constexpr (R32) return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
  }
  static constexpr int kKeyProducts = kSteps * kKeyBlocks, kValueProducts = kScores / 8 * kBlocks;
};

// Addresses of the key operands of the tile at `buf`.
template <int ROWS>
struct Keys {
  using Op = Operands<ROWS>;
  uint32_t at[Op::kKeyAddrs];
  __device__ __forceinline__ Keys(const Op& op, uint32_t buf) {
#pragma unroll
    for (int s = 0; s < Op::kKeyAddrs; ++s) at[s] = buf + (op.key_at ^ (s * (Op::R32 ? 32 : 64)));
  }
  // operand of score product n
  __device__ __forceinline__ bf16x8 read(int n) const {
    const int s = n / Op::kKeyBlocks, b = n % Op::kKeyBlocks;
    return *(const LDS_PTR(bf16x8))(uintptr_t)(at[s % Op::kKeyAddrs] + (s / Op::kKeyAddrs) * 128 + b * 16 * kRowBytes);
  }
};

// Addresses of the value operands of the tile at `buf`, without the rows of its keys named in `unfit`.
template <int ROWS>
struct Values {
  using Op = Operands<ROWS>;
  uint32_t at[Op::kKeyGroups][Op::kValueAddrs];
  // addresses of one of the key groups
  __device__ __forceinline__ void set(const Op& op, uint32_t buf, int g) {
    // (the swizzle of a row eight further on differs in its lowest bit, sixteen further on it is the same)
#pragma unroll
    for (int d = 0; d < Op::kValueAddrs; ++d)
      at[g][d] = buf + ((op.value_at ^ (d * (Op::R32 ? 64 : 32)) ^ (Op::R32 ? (g & 1) * 16 : 0)) + g * Op::kGroupRows * kRowBytes);
  }
  // zeros in place of the keys named in `unfit`
  __device__ __forceinline__ void drop(const Op& op, uint32_t unfit, uint32_t zeros) {
    if (unfit) {
#pragma unroll
      for (int g = 0; g < Op::kKeyGroups; ++g)
#pragma unroll
        for (int d = 0; d < Op::kValueAddrs; ++d)
          if (unfit >> (op.value_key + g * Op::kGroupRows) & 1) at[g][d] = zeros;
    }
  }
  __device__ __forceinline__ void set(const Op& op, uint32_t buf, uint32_t unfit, uint32_t zeros) {
#pragma unroll
    for (int g = 0; g < Op::kKeyGroups; ++g) set(op, buf, g);
    drop(op, unfit, zeros);
  }
  // operand of value product n
  __device__ __forceinline__ bf16x8 read(int n) const {
    const int k = n / Op::kBlocks, d = n % Op::kBlocks, c = (d / Op::kValueAddrs) * 128;
    const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((LDS_PTR(bf16x4))(uintptr_t)(at[2 * k][d % Op::kValueAddrs] + c));
    const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((LDS_PTR(bf16x4))(uintptr_t)(at[2 * k + 1][d % Op::kValueAddrs] + c));
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  }
};

// Scores of 32 keys for 32 rows: the sum of the products over the steps; `ahead` holds the first operands of the keys,
// `key(n)` is the n-th, `query(n)` the other one, `beside(n)` what goes along with a product.  Written out, because the
// compiler gives every product accumulation registers once some have them, and the outputs take all of those.  It counts no
// wait states for it: a product's sum goes straight into the next, and the last one may be read kScoreStates behind it.
constexpr int kScoreStates = 12;
template <int AHEAD, int STEPS, typename Key, typename Query, typename Beside>
__device__ __forceinline__ f32x16 score_products(bf16x8 (&ahead)[AHEAD], Key key, Query query, Beside beside) {
  f32x16 acc;
#pragma unroll
  for (int n = 0; n < STEPS; ++n) {
    if (n == 0) asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, 0" : "=&v"(acc) : "v"(ahead[0]), "v"(query(0)));
    else asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+v"(acc) : "v"(ahead[n % AHEAD]), "v"(query(n)));
    if (n + AHEAD < STEPS) ahead[n % AHEAD] = key(n + AHEAD);
    beside(n);
    __builtin_amdgcn_sched_barrier(0);
  }
  return acc;
}
// Lets the scores be read.
__device__ __forceinline__ void await_scores(f32x16& acc) { asm volatile("s_nop %1" : "+v"(acc) : "n"(kScoreStates)); }

// Masks the scores of the tile whose first key is key0 for a row that sees keys in front of `visible`; returns its unfit keys.
// Where there are some, sets the word at `torn`.
// R32: element r of lane i, half `part` is key (r / 4) * 8 + part * 4 + r % 4; R16: (r / 4) * 16 + part * 4 + r % 4.
template <int ROWS, int N>
__device__ __forceinline__ uint32_t mask_scores(float (&sc)[N], int key0, int visible, int part, uint32_t torn) {
  const uint32_t unfit = unfit_keys<ROWS>(sc);
  auto place = [&](int r) { return (r >> 2) * (ROWS == 32 ? 8 : 16) + part * 4 + (r & 3); };
  if (unfit) *(LDS_PTR(uint32_t))(uintptr_t)torn = 1;
#pragma unroll
  for (int r = 0; r < N; ++r) sc[r] = key0 + place(r) < visible ? sc[r] : -__builtin_inff();
  return unfit;
}

// Marks of eight columns of a key.
__device__ __forceinline__ u32x4 torn_columns(const Gather& gather, const int32_t* pages, int key, int column) {
  return torn_marks(*reinterpret_cast<const u32x4*>(gather.row_at(pages[key >> gather.page_shift], key) + column * 2));
}
template <int ROWS, int N>
__device__ __forceinline__ float row_max(const float (&sc)[N]) {
  float mx = sc[0];
#pragma unroll
  for (int r = 1; r < N; ++r) mx = fmaxf(mx, sc[r]);
  if constexpr (ROWS == 16) mx = cross_quarter_max(mx);
  return cross_half_max(mx);
}

__device__ __forceinline__ float add_pair(uint32_t two, float sum) {  // of two probabilities as they were rounded
  const bf16x2 ones = {(__bf16)1.0f, (__bf16)1.0f};
  return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, two), ones, sum, false);
}

__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){lo, hi}, f16x2));
}

// Writes a wave's rows of outputs times `factor`: column d * 32 + r / 4 * 8 + part * 4 + r % 4 is element r of block d.  They go
// through the wave's LDS at `staged` and out a row at a time; written from where they are, 32 bytes of each of 32 rows
// at a time, they took 43 cycles a store.
constexpr int kStagedPitch = kLatentRank * 2 + 16;  // so that sixteen rows' equal chunks take all banks
static_assert(32 * kStagedPitch <= kTileBytes, "a wave's rows take a tile's place");
template <typename Pack>
__device__ __forceinline__ void write_rows(const f32x16 (&o)[16], char* staged, uint16_t* to, float factor, int lane, int rows, Pack pack) {
  const int i = lane & 31, part = lane >> 5;
#pragma unroll
  for (int d = 0; d < 16; ++d)
#pragma unroll
    for (int r4 = 0; r4 < 4; ++r4) {
      const u32x2 words = {pack(o[d][4 * r4] * factor, o[d][4 * r4 + 1] * factor), pack(o[d][4 * r4 + 2] * factor, o[d][4 * r4 + 3] * factor)};
      *reinterpret_cast<u32x2*>(staged + i * kStagedPitch + (d * 32 + r4 * 8 + part * 4) * 2) = words;
    }
#pragma unroll 8
  for (int row = 0; row < rows; ++row)
    *reinterpret_cast<u32x4*>(to + (int64_t)row * kLatentRank + lane * 8) = *reinterpret_cast<const u32x4*>(staged + row * kStagedPitch + lane * 16);
}

// Tiles of 128 query rows: a wave takes 32 of them and the four share the key tiles, three ahead.  One wave runs on a SIMD (256
// registers of outputs, 144 of queries), so whatever is not a product has to go out beside one.  Of key tile h a wave
//   * forms the scores; beside the products go the gather of tile h + 2, a quarter each wave, and the first reads of the
//     values of h - 1,
//   * adds the value product of h - 1 and beside it turns the scores of h into probabilities; behind the last read of
//     values, six products before the end, the waves meet: the buffer of h - 1 is free and tile h + 1 is there for all, and
//     beside the six go the first reads of its keys.
// No maximum is formed on the way: the reference is the row's maximum over the part's first key tile.  A tile of which a lane's
// sixteen probabilities sum to 2^kSlack is looked at again, and the references of rows move whose maximum is beyond 2^kSlack.  Rows
// whose keys lie 4 to kSlack log2 units above the part's first are thus looked at in every tile without moving; it costs
// about the time of a tile.  1014 tokens of 28 heads over 164k keys: level scores 327 us, 2 units more every 1000 keys 437, 16 more
// 530, all behind a request's first 32 keys higher by 5 480.
// A tile takes 3.7k cycles, 2.2k of them products; a part's queries in and outputs out 20 to 25k, reloads of 35 spilled
// registers among them (the tile loop's common path has none).  32 requests of 128 rows, 88k keys: 43 us; the 1014 tokens above 320 to
// 350 us (the kernel alone) = 0.90 to 0.98 PFLOP/s, products 49 % of the cycles.
__global__ __launch_bounds__(64 * kWaves, 1) void latent_rows_kernel(const LatentArgs args, const uint16_t* __restrict__ q,
                                                                     const uint16_t* __restrict__ cache,
                                                                     const int32_t* __restrict__ block_table,
                                                                     uint16_t* __restrict__ out) {
  using Op = Operands<32>;
  constexpr int TILE = 32 * kWaves;
  constexpr int kAhead = 6;  // operands read in front of their products
  __shared__ __attribute__((aligned(1024))) char lds[kLdsBytes];
  const uint32_t lds0 = (uint32_t)(uintptr_t)(LDS_PTR(char))lds;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int heads = args.table.heads, page_shift = args.table.page_shift;
  *reinterpret_cast<u32x4*>(lds + kZeros + lane * 16) = u32x4{0, 0, 0, 0};  // (by every wave: it reads behind its own writes)
  Op op(lane);

  for (Share<TILE> it(args.table, lane); !it.done(); it.advance()) {
    const int32_t* pages = block_table + (int64_t)it.rq.req * args.table.max_pages;
    const int ntiles = (it.k1 - it.k0 + kTileKeys - 1) / kTileKeys;
    const int i = lane & 31, part = lane >> 5;
    const int row = min(wave * 32 + i, it.rows - 1);
    // The wave's queries, through a tile's place: read from memory as operands, 16 bytes of each of 32 rows at a time, they
    // took 55 cycles a load.  Rows behind the tile's last are copies of it.
    const Gather queries(q + it.packed * kLatentRow, it.rows, 30, lane);
#pragma unroll
    for (int g = 0; g < kGroups; ++g)
      queries.group(wave * 32 + g * kGroupKeys, g, 0, lds0 + wave * kTileBytes + g * kGroupBytes);
    // the wave gathers a quarter of each key tile; lane t holds the page of its rows in tile held_from + t
    Gather gather(cache, it.k1, page_shift, lane);
    auto key_of = [&](int tile) { return it.k0 + tile * kTileKeys + wave * kGroupKeys; };
    auto pages_from = [&](int tile) { return pages[min(key_of(tile + lane), it.k1 - 1) >> page_shift]; };
    int held_from = 0;
    int32_t held = pages_from(0);
    auto page_of = [&](int tile) { return __builtin_amdgcn_readlane(held, tile - held_from); };
    auto buffer = [&](int tile) { return lds0 + (tile & (kWaves - 1)) * kTileBytes; };
    // (the gathers in flight are counted here: everything the compiler knows of is waited for)
    __builtin_amdgcn_s_waitcnt(0x0F70);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    bf16x8 qb[Op::kSteps];
    {
      const Keys<32> rows(op, lds0 + wave * kTileBytes);
#pragma unroll
      for (int s = 0; s < Op::kSteps; ++s) qb[s] = rows.read(s);
    }
    __syncthreads();
#pragma unroll
    for (int a = 0; a < kWaves - 1; ++a)
      if (a < ntiles) gather.group(key_of(a), wave, page_of(a), buffer(a) + wave * kGroupBytes);
    if (ntiles > 2) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * kGroupLoads) : "memory");
    else if (ntiles > 1) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kGroupLoads) : "memory");
    else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();

    const int visible = it.rq.cached + (it.row0 + row) / heads + 1;
    const int least = it.rq.cached + (it.row0 + min(wave * 32, it.rows - 1)) / heads + 1;  // of the wave's first row
    f32x16 o[Op::kBlocks];
#pragma unroll
    for (int d = 0; d < Op::kBlocks; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[d][r] = 0.f;
    const uint32_t torn = lds0 + kTornAt + 4 * wave;
    *(LDS_PTR(uint32_t))(uintptr_t)torn = 0;
    float m_run = kNoReference, l_run = 0.f;
    u32x4 pb[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}}, pn[2];  // probabilities of the tile in front and of the one at hand, as operands
    uint32_t unfit = 0, pb_unfit = ~0u;                  // (in front of the first there is none)
    f32x16 sc;
    auto probability = [&](int e) __attribute__((always_inline)) { return __builtin_amdgcn_exp2f(sc[e] * args.scale_log2 - m_run); };
    bf16x8 ka[kAhead], va[kAhead];
    {
      const Keys<32> keys(op, buffer(0));
#pragma unroll
      for (int n = 0; n < kAhead; ++n) ka[n] = keys.read(n);
    }

    // One copy of each product: a second one for the first or the last tile makes the compiler move the outputs between
    // registers.  So the last round forms the value product of the last tile beside probabilities that nobody takes.
    for (int tile = 0;; ++tile) {
      Values<32> v;
      const uint32_t values_at = buffer(tile + kWaves - 1);
      if (tile < ntiles) {
        const int next = tile + kWaves - 2;
        bool fetch = tile > 0 && next < ntiles;
        const char* from = nullptr;
        const uint32_t to = buffer(next) + wave * kGroupBytes;
        if (fetch) {
          if (next - held_from >= 64) {
            held_from = next;
            held = pages_from(next);
            __builtin_amdgcn_s_waitcnt(0x0F70);
          }
          const int key = key_of(next);
          fetch = gather.whole(key);
          if (fetch) from = gather.row_at(page_of(next), key);
          else gather.group(key, wave, page_of(next), to);
        }
        op.forget();
        gather.forget();
        const Keys<32> keys(op, buffer(tile));
        constexpr int kLast = Op::kKeyProducts;
        sc = score_products<kAhead, kLast>(
            ka, [&](int n) { return keys.read(n); }, [&](int n) { return qb[n]; },
            [&](int n) __attribute__((always_inline)) {
              if (n % 4 == 1 && n / 2 < kGroupLoads && fetch) gather.pair(from, n / 2, wave & 1, to);
              if (n >= kLast - kAhead - 4 && n < kLast - kAhead) v.set(op, values_at, n - (kLast - kAhead - 4));
              if (n == kLast - kAhead - 1) v.drop(op, pb_unfit, lds0 + kZeros);
              if (n >= kLast - kAhead) va[n - (kLast - kAhead)] = v.read(n - (kLast - kAhead));
            });
        unfit = 0;
        const int key0 = it.k0 + tile * kTileKeys;
        if (tile == 0 || key0 + kTileKeys > least) {
          await_scores(sc);
          float x[16];
#pragma unroll
          for (int r = 0; r < 16; ++r) x[r] = sc[r];
          unfit = mask_scores<32>(x, key0, visible, part, torn);
          if (tile == 0) m_run = fmaxf(row_max<32>(x) * args.scale_log2, kNoReference);
#pragma unroll
          for (int r = 0; r < 16; ++r) sc[r] = x[r];
        }
      } else {
        v.set(op, values_at, pb_unfit, lds0 + kZeros);
#pragma unroll
        for (int n = 0; n < kAhead; ++n) va[n] = v.read(n);
      }
      __builtin_amdgcn_sched_barrier(0);
      constexpr int kMeet = Op::kValueProducts - kAhead;
      float sum = 0.f, pair[2];
      const Keys<32> next_keys(op, buffer(tile + 1));
#pragma unroll
      for (int n = 0; n < Op::kValueProducts; ++n) {
        o[n % Op::kBlocks] = Op::product(va[n % kAhead], __builtin_bit_cast(bf16x8, pb[n / Op::kBlocks]), o[n % Op::kBlocks]);
        if (n < kMeet) va[n % kAhead] = v.read(n + kAhead);
        if (n == kMeet - 1 && tile + 1 < ntiles) {
          if (tile + 2 < ntiles) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kGroupLoads) : "memory");
          else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
          __syncthreads();
        }
        if (n >= kMeet) ka[n - kMeet] = next_keys.read(n - kMeet);  // (behind the last tile: whatever is there, for nobody)
        // the scores are read two products and some states behind the last of theirs, then an element to two products
        if (n == 1) await_scores(sc);
        const int e = n < 2 ? -1 : n == 31 ? 15 : n % 2 == 0 ? n / 2 - 1 : -1;
        if (e >= 0) {
          pair[e & 1] = probability(e);
          if (e & 1) {
            const uint32_t two = pack_bf16(pair[0], pair[1]);
            pn[e >> 3][(e & 7) >> 1] = two;
            sum = add_pair(two, sum);
            asm volatile("" : "+v"(sum));  // (keeps the step in its place)
          }
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      if (tile == ntiles) break;
      // where the sum says that a probability may have passed the slack: a reference moves to its row's maximum if that did, and the
      // probabilities are formed again
      if (__any(sum >= kOver)) {
        float x[16];
#pragma unroll
        for (int r = 0; r < 16; ++r) x[r] = sc[r];
        const float mx = row_max<32>(x) * args.scale_log2;
        const float m_new = mx > m_run + kSlack ? mx : m_run;
        const float f = m_new == m_run ? 1.f : __builtin_amdgcn_exp2f(m_run - m_new);
        l_run *= f;
        after_products();
#pragma unroll
        for (int d = 0; d < Op::kBlocks; ++d)
#pragma unroll
          for (int r = 0; r < 16; ++r) o[d][r] = scale_accumulator(o[d][r], f);
        before_products();
        m_run = m_new;
        sum = 0.f;
#pragma unroll
        for (int e = 0; e < 16; e += 2) {
          const uint32_t two = pack_bf16(probability(e), probability(e + 1));
          pn[e >> 3][(e & 7) >> 1] = two;
          sum = add_pair(two, sum);
        }
      }
      l_run += sum;
      pb[0] = pn[0];
      pb[1] = pn[1];
      pb_unfit = unfit;
    }
    l_run = cross_half_sum(l_run);

    __syncthreads();  // every wave is done with the part's tiles
    const int mine = max(0, min(32, it.rows - wave * 32));
    char* const staged = lds + wave * kTileBytes;
    if (it.slot >= 0) {
      float top = 0.f;
#pragma unroll
      for (int d = 0; d < Op::kBlocks; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) top = fmaxf(top, fabsf(o[d][r]));
      top = cross_half_max(top);
      const int64_t at = (int64_t)it.slot * TILE + wave * 32;
      if (i < mine && part == 0) *reinterpret_cast<f32x4*>(args.part_ml + (at + i) * 4) = f32x4{m_run, l_run, part_scale(top), 0.f};
      write_rows(o, staged, args.part_o + at * kLatentRank, 1.f / part_scale(top), lane, mine,
                 [](float a, float b) { return pack_f16(a, b); });
    } else {
      write_rows(o, staged, out + (it.packed + wave * 32) * kLatentRank, 1.f / l_run, lane, mine,
                 [](float a, float b) { return pack_bf16(a, b); });
    }
    // torn columns, over what was written
    if (__builtin_expect(__builtin_amdgcn_readfirstlane(*(LDS_PTR(uint32_t))(uintptr_t)torn) != 0, 0)) {
      int own = lane;
      asm volatile("" : "+v"(own));  // (its addresses are formed here: held from part to part they were spilled)
      uint16_t* const to = it.slot >= 0 ? args.part_o + ((int64_t)it.slot * TILE + wave * 32) * kLatentRank : out + (it.packed + wave * 32) * kLatentRank;
      u32x4 marks = {0, 0, 0, 0};
      int key = it.k0;
#pragma unroll 1
      for (int n = 0; n < mine; ++n) {
        const int end = min(it.k1, it.rq.cached + (it.row0 + wave * 32 + n) / heads + 1);
        while (key < end) {
          marks |= torn_columns(gather, pages, key, own * 8);
          // (the tiles that were masked: the first and those that some row does not see whole)
          ++key;
          if (key == it.k0 + kTileKeys) key = max(key, least & -kTileKeys);
        }
        *reinterpret_cast<u32x4*>(to + (int64_t)n * kLatentRank + own * 8) |= marks;
      }
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the wave's place is read
    __syncthreads();
  }
}

// Items of at most ROWS (16 or 32) query rows: all waves take the same rows, the key tiles in turn, in LDS of their own, and join
// their results at the end.  Such a step is bound by reading the cache; the waves wait for nothing but their own gathers, so
// that some load while others compute; two waves have a second place each and load while they compute.  The reference follows
// the maximum, so the time does not depend on the scores.  32 requests, 176k keys, 16 heads: 39 us = 5.3 TB/s (45 where the
// cache comes from HBM); one request of 2345 keys 11 us.
template <int ROWS, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 1) void latent_keys_kernel(const LatentArgs args, const uint16_t* __restrict__ q,
                                                                     const uint16_t* __restrict__ cache,
                                                                     const int32_t* __restrict__ block_table,
                                                                     uint16_t* __restrict__ out) {
  using Op = Operands<ROWS>;
  using Acc = typename Op::Acc;
  constexpr int kAcc = Op::kAcc, kBuffers = kWaves / WAVES;  // of a wave
  __shared__ __attribute__((aligned(1024))) char lds[kLdsBytes];
  const uint32_t lds0 = (uint32_t)(uintptr_t)(LDS_PTR(char))lds;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int heads = args.table.heads, page_shift = args.table.page_shift;
  *reinterpret_cast<u32x4*>(lds + kZeros + lane * 16) = u32x4{0, 0, 0, 0};  // (by every wave: it reads behind its own writes)
  Op op(lane);

  for (Share<ROWS> it(args.table, lane); !it.done(); it.advance()) {
    const int32_t* pages = block_table + (int64_t)it.rq.req * args.table.max_pages;
    const int ntiles = (it.k1 - it.k0 + kTileKeys - 1) / kTileKeys;
    // (the units are dealt to the waves in turn from one part to the next)
    const int turn = (wave - (int)(it.next & (WAVES - 1))) & (WAVES - 1);
    // the n-th tile of the wave; lane 4 n + g holds the page of group g of its tile held_from + n
    const Gather gather(cache, it.k1, page_shift, lane);
    auto buffer = [&](int n) { return lds0 + (wave * kBuffers + n % kBuffers) * kTileBytes; };
    auto key_of = [&](int n, int g) { return it.k0 + (turn + n * WAVES) * kTileKeys + g * kGroupKeys; };
    auto pages_from = [&](int n) { return pages[min(key_of(n + (lane >> 2), lane & 3), it.k1 - 1) >> page_shift]; };
    int held_from = 0;
    int32_t held = pages_from(0);
    auto fetch = [&](int n) __attribute__((always_inline)) {
#pragma unroll
      for (int g = 0; g < kGroups; ++g)
        gather.group(key_of(n, g), g, __builtin_amdgcn_readlane(held, (n - held_from) * 4 + g), buffer(n) + g * kGroupBytes);
    };
    const int mine = (ntiles - turn + WAVES - 1) / WAVES;
    if (mine > 0) fetch(0);

    const int i = lane % ROWS, part = lane / ROWS;
    const int row = min(i, it.rows - 1);
    const uint16_t* q_row = q + (it.packed + row) * kLatentRow + part * 8;
    bf16x8 qb[Op::kSteps];
#pragma unroll
    for (int s = 0; s < Op::kSteps; ++s) qb[s] = *reinterpret_cast<const bf16x8*>(q_row + s * (Op::R32 ? 16 : 32));
    const int visible = it.rq.cached + (it.row0 + row) / heads + 1;
    const int least = it.rq.cached + it.row0 / heads + 1;  // of the first row
    Acc o[Op::kBlocks];
#pragma unroll
    for (int d = 0; d < Op::kBlocks; ++d)
#pragma unroll
      for (int r = 0; r < kAcc; ++r) o[d][r] = 0.f;
    const uint32_t torn = lds0 + kTornAt;
    *(LDS_PTR(uint32_t))(uintptr_t)(torn + 4 * wave) = 0;
    float m_run = kNoReference, l_run = 0.f;
    constexpr int kAhead = 6;
    __builtin_amdgcn_s_waitcnt(0x0F70);

    for (int n = 0; n < mine; ++n) {
      if (n + 1 - held_from >= 16 && n + 1 < mine) {
        held_from = n + 1;
        held = pages_from(n + 1);
        __builtin_amdgcn_s_waitcnt(0x0F70);
      }
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      if (kBuffers > 1 && n + 1 < mine) fetch(n + 1);
      op.forget();
      const uint32_t buf = buffer(n);
      const Keys<ROWS> keys(op, buf);
      float sc[Op::kScores];
      if constexpr (Op::R32) {
        bf16x8 ka[kAhead];
#pragma unroll
        for (int p = 0; p < kAhead; ++p) ka[p] = keys.read(p);
        f32x16 acc = score_products<kAhead, Op::kSteps>(ka, [&](int p) { return keys.read(p); }, [&](int p) { return qb[p]; }, [](int) {});
        await_scores(acc);
#pragma unroll
        for (int r = 0; r < Op::kScores; ++r) sc[r] = acc[r];
      } else {
        bf16x8 ka[kAhead];
#pragma unroll
        for (int p = 0; p < kAhead; ++p) ka[p] = keys.read(p);
        Acc acc[Op::kKeyBlocks];
#pragma unroll
        for (int b = 0; b < Op::kKeyBlocks; ++b)
#pragma unroll
          for (int r = 0; r < kAcc; ++r) acc[b][r] = 0.f;
#pragma unroll
        for (int p = 0; p < Op::kKeyProducts; ++p) {
          acc[p % Op::kKeyBlocks] = Op::product(ka[p % kAhead], qb[p / Op::kKeyBlocks], acc[p % Op::kKeyBlocks]);
          if (p + kAhead < Op::kKeyProducts) ka[p % kAhead] = keys.read(p + kAhead);
          __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int r = 0; r < Op::kScores; ++r) sc[r] = acc[r / kAcc][r % kAcc];
      }
      uint32_t unfit = 0;
      const int key0 = key_of(n, 0);
      if (key0 + kTileKeys > least) unfit = mask_scores<ROWS>(sc, key0, visible, part, torn + 4 * wave);
      const float mx = row_max<ROWS>(sc) * args.scale_log2;
      if (__any(mx > m_run + kSlack)) {
        const float m_new = mx > m_run + kSlack ? mx : m_run;
        const float f = m_new == m_run ? 1.f : __builtin_amdgcn_exp2f(m_run - m_new);
        l_run *= f;
        after_products();
#pragma unroll
        for (int d = 0; d < Op::kBlocks; ++d)
#pragma unroll
          for (int r = 0; r < kAcc; ++r) o[d][r] = scale_accumulator(o[d][r], f);
        before_products();
        m_run = m_new;
      }
      Values<ROWS> v;
      v.set(op, buf, unfit, lds0 + kZeros);
      bf16x8 va[kAhead];
#pragma unroll
      for (int p = 0; p < kAhead; ++p) va[p] = v.read(p);
      u32x4 pb[Op::kScores / 8];
#pragma unroll
      for (int e = 0; e < Op::kScores; e += 2) {
        const uint32_t two = pack_bf16(__builtin_amdgcn_exp2f(sc[e] * args.scale_log2 - m_run),
                                       __builtin_amdgcn_exp2f(sc[e + 1] * args.scale_log2 - m_run));
        pb[e >> 3][(e & 7) >> 1] = two;
        l_run = add_pair(two, l_run);
      }
#pragma unroll
      for (int p = 0; p < Op::kValueProducts; ++p) {
        o[p % Op::kBlocks] = Op::product(va[p % kAhead], __builtin_bit_cast(bf16x8, pb[p / Op::kBlocks]), o[p % Op::kBlocks]);
        if (p + kAhead < Op::kValueProducts) va[p % kAhead] = v.read(p + kAhead);
        __builtin_amdgcn_sched_barrier(0);
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the tile has been read
      if (kBuffers == 1 && n + 1 < mine) fetch(n + 1);
    }
    if constexpr (!Op::R32) l_run = cross_quarter_sum(l_run);
    l_run = cross_half_sum(l_run);

    // join of the waves, kStage columns at a time (more of 32 rows cost registers): [wave][row][kStage + 4], and behind them
    // [wave][row] (reference, sum, largest magnitude, -)
    constexpr int kCols = 128, kStage = ROWS == 16 ? 512 : 128, kPitch = kStage + 4;
    static_assert(WAVES * ROWS * (kPitch + 4) * 4 <= kZeros, "the join fits the tiles' place");
    float* const joined = reinterpret_cast<float*>(lds);
    f32x4* const s_ml = reinterpret_cast<f32x4*>(joined + WAVES * ROWS * kPitch);
    float top = 0.f;
    if (it.slot >= 0) {
#pragma unroll
      for (int d = 0; d < Op::kBlocks; ++d)
#pragma unroll
        for (int r = 0; r < kAcc; ++r) top = fmaxf(top, fabsf(o[d][r]));
      if constexpr (!Op::R32) top = cross_quarter_max(top);
      top = cross_half_max(top);
    }
    __syncthreads();  // the tiles are read
    if (part == 0) s_ml[wave * ROWS + i] = f32x4{m_run, l_run, top, 0.f};
    __syncthreads();
    float m = kNoReference;
#pragma unroll
    for (int k = 0; k < WAVES; ++k) m = fmaxf(m, s_ml[k * ROWS + i][0]);
    const float f = __builtin_amdgcn_exp2f(m_run - m);
    constexpr int kThreadsPerRow = 64 * WAVES / ROWS, kPer = kCols / kThreadsPerRow;  // 8 columns, or 16
    const int my_row = tid / kThreadsPerRow, my_col = tid % kThreadsPerRow * kPer;
    float my_m = kNoReference, my_l = 0.f, my_top = 0.f;
#pragma unroll
    for (int k = 0; k < WAVES; ++k) my_m = fmaxf(my_m, s_ml[k * ROWS + my_row][0]);
#pragma unroll
    for (int k = 0; k < WAVES; ++k) {
      const f32x4 ml = s_ml[k * ROWS + my_row];
      const float weight = __builtin_amdgcn_exp2f(ml[0] - my_m);
      my_l += ml[1] * weight;
      my_top += ml[2] * weight;  // (no sum over the waves is larger)
    }
    const int64_t at = (int64_t)it.slot * ROWS + my_row;
    if (it.slot >= 0 && my_col == 0 && my_row < it.rows) *reinterpret_cast<f32x4*>(args.part_ml + at * 4) = f32x4{my_m, my_l, part_scale(my_top), 0.f};
    const float inv = 1.f / (it.slot < 0 ? my_l : part_scale(my_top));
    uint16_t* const dst = (it.slot < 0 ? out + (it.packed + my_row) * kLatentRank : args.part_o + at * kLatentRank) + my_col;
    constexpr int kBlocksPerRound = kStage / ROWS;
#pragma unroll
    for (int round = 0; round < kLatentRank / kStage; ++round) {
      if (round) __syncthreads();
#pragma unroll
      for (int b = 0; b < kBlocksPerRound; ++b)
#pragma unroll
        for (int r4 = 0; r4 < kAcc / 4; ++r4) {
          const int d = round * kBlocksPerRound + b;
          const f32x4 x = {o[d][4 * r4] * f, o[d][4 * r4 + 1] * f, o[d][4 * r4 + 2] * f, o[d][4 * r4 + 3] * f};
          *reinterpret_cast<f32x4*>(joined + (wave * ROWS + i) * kPitch + b * ROWS + r4 * 8 + part * 4) = x;
        }
      __syncthreads();
      if (my_row < it.rows) {
#pragma unroll
        for (int n = 0; n < kStage / kCols * kPer; n += 8) {
          const int c = n / kPer * kCols + n % kPer;
          f32x4 x[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
          for (int k = 0; k < WAVES; ++k)
#pragma unroll
            for (int h = 0; h < 2; ++h)
              x[h] += *reinterpret_cast<const f32x4*>(joined + (k * ROWS + my_row) * kPitch + my_col + c + 4 * h);
          u32x4 words;
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const float a = x[k >> 1][2 * (k & 1)] * inv, b = x[k >> 1][2 * (k & 1) + 1] * inv;
            words[k] = it.slot < 0 ? pack_bf16(a, b) : pack_f16(a, b);
          }
          *reinterpret_cast<u32x4*>(dst + round * kStage + c) = words;
        }
      }
    }
    // torn columns, over what this thread wrote
    uint32_t some = 0;
#pragma unroll
    for (int k = 0; k < WAVES; ++k) some |= *(LDS_PTR(uint32_t))(uintptr_t)(torn + 4 * k);
    if (__builtin_amdgcn_readfirstlane(some) && my_row < it.rows) {
      const int end = min(it.k1, it.rq.cached + (it.row0 + my_row) / heads + 1);
#pragma unroll 1
      for (int n = 0; n < kLatentRank / kCols * kPer; n += 8) {
        const int c = n / kPer * kCols + n % kPer;
        u32x4 marks = {0, 0, 0, 0};
#pragma unroll 1
        for (int key = max(it.k0, least & -kTileKeys); key < end; ++key) marks |= torn_columns(gather, pages, key, my_col + c);
        *reinterpret_cast<u32x4*>(dst + c) |= marks;
      }
    }
    __syncthreads();  // what was joined has been read
  }
}

// Joins the parts of a tile that several workgroups share: with M = max m, out = sum 2^(m - M) O / sum 2^(m - M) l, in the parts'
// order.  blockIdx.y stands for the first workgroup whose share begins inside the tile; a wave takes every
// 4 gridDim.x-th row, eight columns to a lane, eight parts' loads at a time.  A launch and 33 MB of parts 10 us, 67 MB and as many
// outputs 18 us, 4 MB 5 us.
template <int TILE>
__global__ __launch_bounds__(256) void latent_join_kernel(const LatentArgs args, uint16_t* __restrict__ out) {
  const LatentTable& t = args.table;
  const int lane = threadIdx.x & 63;
  const int group = blockIdx.y + 1;
  const Requests requests(t, lane);
  Place at;
  LatentReq q;
  int parts = 2;
  bool together = true;
  if (t.by_tile) {
    q = requests.get(requests.find_group(group, lane));
    const int k = group - (int)(uint32_t)q.unit_start;
    parts = (int)(q.unit_start >> 32);
    at.tile = k / parts;
    if (k - at.tile * parts != 1) return;
  } else {
    const int64_t cut = t.first_unit(group);
    at = find_tile<TILE>(t, requests, cut, lane);
    if (cut == at.first || t.first_unit(group - 1) > at.first) return;
    q = requests.get(at.r);
    while (group - 1 + parts < t.groups && t.first_unit(group - 1 + parts) < at.first + at.units) ++parts;
    // the first part is its workgroup's first too where the two begin together, the others are
    together = t.first_unit(group - 1) == at.first;
  }
  const int rows = latent_rows_of(q, t.heads, TILE, at.tile);
  auto slot_of = [&](int s) { return latent_slot(group - 1 + s, s > 0 || together); };
  for (int row = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6)); row < rows; row += 4 * gridDim.x) {
    float m = kNoReference, l = 0.f, v[8] = {};
    auto add = [&](int s0, auto count) __attribute__((always_inline)) {
      constexpr int kGroup = decltype(count)::value;  // parts, asked for at once
      f32x4 ml[kGroup];
      u32x4 h[kGroup];
#pragma unroll
      for (int s = 0; s < kGroup; ++s) {
        const int64_t from = (int64_t)slot_of(min(s0 + s, parts - 1)) * TILE + row;
        ml[s] = *reinterpret_cast<const f32x4*>(args.part_ml + from * 4);
        h[s] = *reinterpret_cast<const u32x4*>(args.part_o + from * kLatentRank + lane * 8);
      }
      float m_new = m;
#pragma unroll
      for (int s = 0; s < kGroup; ++s)
        if (s0 + s < parts) m_new = fmaxf(m_new, ml[s][0]);
      const float f = __builtin_amdgcn_exp2f(m - m_new);
      m = m_new;
      l *= f;
#pragma unroll
      for (int c = 0; c < 8; ++c) v[c] *= f;
#pragma unroll
      for (int s = 0; s < kGroup; ++s) {
        if (s0 + s >= parts) continue;
        const float w = __builtin_amdgcn_exp2f(ml[s][0] - m), scale = w * ml[s][2];
        l += w * ml[s][1];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
          const uint32_t word = h[s][c];
          const f16x2 two = __builtin_bit_cast(f16x2, word);
          v[2 * c] += (float)two[0] * scale;
          v[2 * c + 1] += (float)two[1] * scale;
        }
      }
    };
    if (parts == 2) add(0, std::integral_constant<int, 2>());
    else
      for (int s0 = 0; s0 < parts; s0 += 8) add(s0, std::integral_constant<int, 8>());
    const float inv = 1.f / l;
    u32x4 words;
#pragma unroll
    for (int c = 0; c < 4; ++c) words[c] = pack_bf16(v[2 * c] * inv, v[2 * c + 1] * inv);
    *reinterpret_cast<u32x4*>(out + ((int64_t)q.row_start * t.heads + at.tile * TILE + row) * kLatentRank + lane * 8) = words;
  }
}

int latent_attention(const efim_batch_t* b, const void* q, const void* cache, void* out, float sm_scale,
                     void* workspace, size_t workspace_bytes, hipStream_t stream) {
  int64_t total = 0;
  const int rc = validate_latent_batch(b, &total);
  if (rc != EFIM_OK) return rc;
  if (!(sm_scale > 0.f) || sm_scale - sm_scale != 0.f) return EFIM_ERR_INVALID_ARG;
  if (total == 0) return EFIM_OK;
  if (!q || !cache || !out || q == out || out == cache) return EFIM_ERR_INVALID_ARG;
  if (!aligned16(q) || !aligned16(cache) || !aligned16(out) || !aligned4(b->block_table)) return EFIM_ERR_INVALID_ARG;
  const LatentPlan plan = plan_latent(b, compute_units());
  const LatentBytes bytes = latent_bytes(plan);
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u) || workspace_bytes < bytes.total) return EFIM_ERR_WORKSPACE;
  LatentArgs args;
  args.scale_log2 = sm_scale * 1.44269504088896340736f;
  args.part_o = static_cast<uint16_t*>(workspace);
  args.part_ml = reinterpret_cast<float*>(static_cast<char*>(workspace) + bytes.off_ml);
  LatentCursor at;
  while (latent_next(b, plan, &at, &args.table)) {
    const unsigned groups = (unsigned)(args.table.groups + kXcds - 1) / kXcds * kXcds;
    auto launch = [&](auto* kernel, int waves, auto* join, int join_groups) {
      kernel<<<groups, 64 * waves, 0, stream>>>(args, static_cast<const uint16_t*>(q), static_cast<const uint16_t*>(cache),
                                                 b->block_table, static_cast<uint16_t*>(out));
      if (args.table.groups > 1)
        join<<<dim3(join_groups, args.table.groups - 1), 256, 0, stream>>>(args, static_cast<uint16_t*>(out));
    };
    // 32 rows: four waves where no workgroup has many units, else two that gather a tile while they compute another.  us with four
    // and two: 32 requests of 1k to 8k keys 58.7 / 56.4, 8 of 4k to 16k 47.7 / 45.1, 200 of 100 to 600 67.9 / 64.4; with
    // four units one of 2344 keys 23.4 / 24.2, one of 300 20.3 / 21.7.  16 rows compute so little that four are ahead there too (45.8 / 47.7).
    constexpr int kUnitsForTwo = 6;
    if (plan.row_tile == 16) launch(latent_keys_kernel<16, 4>, 4, latent_join_kernel<16>, 4);
    else if (plan.row_tile == 32 && args.table.longest < kUnitsForTwo) launch(latent_keys_kernel<32, 4>, 4, latent_join_kernel<32>, 8);
    else if (plan.row_tile == 32) launch(latent_keys_kernel<32, 2>, 2, latent_join_kernel<32>, 8);
    else launch(latent_rows_kernel, kWaves, latent_join_kernel<128>, args.table.by_tile ? 32 : 16);  // (many parts of few tiles, or two of each)
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) { set_last_hip_error(e); return EFIM_ERR_LAUNCH; }
  }
  return EFIM_OK;
}

}  // namespace
}  // namespace efim

extern "C" {

size_t efim_latent_workspace_bytes(const efim_batch_t* batch) {
  int64_t total = 0;
  if (efim::validate_latent_batch(batch, &total) != EFIM_OK) return 0;
  if (total == 0) return 256;
  const size_t bytes = efim::latent_bytes(efim::plan_latent(batch, efim::compute_units())).total;
  return bytes < 256 ? 256 : bytes;
}

int efim_latent_attention(const efim_batch_t* batch, const void* q, const void* latent_cache, void* out, float sm_scale,
                          void* workspace, size_t workspace_bytes, void* stream) {
  return efim::latent_attention(batch, q, latent_cache, out, sm_scale, workspace, workspace_bytes,
                                static_cast<hipStream_t>(stream));
}

}  // extern "C"
