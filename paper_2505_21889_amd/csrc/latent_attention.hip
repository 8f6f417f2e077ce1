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

constexpr int kRowBytes = kLatentRow * 2;
constexpr int kRowChunks = kRowBytes / 16;
constexpr int kTileKeys = kLatentTileKeys;
constexpr int kTileBytes = kTileKeys * kRowBytes;
constexpr int kGroupKeys = 8;  // rows that nine 1 KB loads hold
constexpr int kGroupLoads = kGroupKeys * kRowBytes / 1024;
constexpr int kGroups = kTileKeys / kGroupKeys;
constexpr int kWaves = 4;
constexpr float kSlack = 8.f;            // log2 units by which a row's maximum may outgrow its reference
constexpr float kNoReference = -3.0e38f;  // of a row that has seen no key: any finite score moves it
static_assert(kGroupKeys <= kMinPageSize && kGroupLoads == 9, "a group of rows lies in one page");

struct LatentArgs {
  LatentTable table;
  float scale_log2;  // sm_scale * log2(e)
  float* part_o;     // [slot][row tile][512] unnormalised outputs of the ranges of split tiles
  float* part_ml;    // [slot][row tile][2] reference (log2 units) and sum
};

// Swizzle of a tile row's chunks (exclusive or on the chunk's low three bits).  A row is 72 chunks, so neighbouring rows
// start half of the 256-byte bank line apart; with these three bits of the row sixteen rows' equal chunks take the sixteen
// places of the line, and so do the four chunks of eight rows that a transposing read takes at a time.
__device__ __forceinline__ int swizzle(int row) { return ((row >> 1) & 1) << 2 | ((row >> 2) & 1) << 1 | ((row >> 3) & 1); }

// The outputs of a wave of 32 rows are 256 registers: all of the accumulation registers, which only products and moves
// can name.  Their scaling by a moved reference is written out, element by element through one other register: left to the
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

// The request of a work item.
__device__ __forceinline__ LatentReq find_request(const LatentTable& t, int item, int lane) {
  int r = -1;
#pragma unroll
  for (int i = 0; i < kLatentTableReqs / 64; ++i) {
    const int at = i * 64 + lane;
    r += __popcll(__ballot(at < t.nreq && t.req[min(at, t.nreq - 1)].item_start <= item));
  }
  return t.req[__builtin_amdgcn_readfirstlane(r)];
}

// ROWS: query rows of a wave, 32 or 16, which is also the shape of its products.  KEYS: the four waves take the same rows and
// every fourth key tile each, in LDS of their own, and join their results at the end; else they take rows of their own and
// share the tiles, three ahead.
template <int ROWS, bool KEYS>
__global__ __launch_bounds__(64 * kWaves, 1) void latent_attention_kernel(
    const LatentArgs args, const uint16_t* __restrict__ q, const uint16_t* __restrict__ cache,
    const int32_t* __restrict__ block_table, uint16_t* __restrict__ out) {
  constexpr int TILE = KEYS ? ROWS : ROWS * kWaves;
  constexpr bool R32 = ROWS == 32;
  constexpr int kSteps = R32 ? kLatentRow / 16 : kLatentRow / 32;  // products along a row
  constexpr int kBlocks = kLatentRank / (R32 ? 32 : 16);           // output blocks
  constexpr int kZeros = kWaves * kTileBytes;  // 1 KB of zeros, in place of values that are not finite
  __shared__ __attribute__((aligned(1024))) char lds[kZeros + 1024];
  const uint32_t lds0 = (uint32_t)(uintptr_t)(LDS_PTR(char))lds;

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const LatentTable& t = args.table;
  const LatentReq rq = find_request(t, blockIdx.x, lane);
  const LatentItem it = latent_item(t, rq, blockIdx.x, TILE);
  const int heads = t.heads;
  const int64_t first = (int64_t)rq.row_start * heads;  // packed query row of the request's row 0
  if (it.k0 >= it.k1) {
    // a range behind the tile's last key: no weight in the join
    if (it.slot >= 0 && tid < TILE) {
      float* ml = args.part_ml + ((int64_t)it.slot * TILE + tid) * 2;
      ml[0] = kNoReference;
      ml[1] = 0.f;
    }
    return;
  }
  const int32_t* pages = block_table + (int64_t)rq.req * t.max_pages;
  const int page_shift = t.page_shift, page_mask = (1 << page_shift) - 1;
  const int ntiles = (it.k1 - it.k0 + kTileKeys - 1) / kTileKeys;

  // the lane's place in the nine loads of a group whose rows have an even eighth
  uint32_t off[kGroupLoads];
#pragma unroll
  for (int j = 0; j < kGroupLoads; ++j) off[j] = (uint32_t)((lane ^ swizzle((j * 64 + lane) / kRowChunks)) << 4);
  auto page_of = [&](int tile, int g) { return pages[min(it.k0 + tile * kTileKeys + g * kGroupKeys, it.k1 - 1) >> page_shift]; };
  // group g of a tile into LDS at `to`; rows behind the range are copies of its last row
  auto gather = [&](int tile, int g, int32_t page, uint32_t to) __attribute__((always_inline)) {
    const int key = it.k0 + tile * kTileKeys + g * kGroupKeys;
    if (key + kGroupKeys <= it.k1) {
      const char* base = reinterpret_cast<const char*>(cache) + (((int64_t)page << page_shift) + (key & page_mask)) * kRowBytes;
      const uint32_t flip = (g & 1) << 4;
      load_to_lds_4x16(base, off[0] ^ flip, off[1] ^ flip, off[2] ^ flip, off[3] ^ flip, to);
      load_to_lds_4x16(base + 4096, off[4] ^ flip, off[5] ^ flip, off[6] ^ flip, off[7] ^ flip, to + 4096);
      load_to_lds_16(base + 8192, off[8] ^ flip, to + 8192);
    } else {
      const int last = it.k1 - 1, from = min(key, last & ~(kGroupKeys - 1));
      const char* base = reinterpret_cast<const char*>(cache) + (((int64_t)page << page_shift) + (from & page_mask)) * kRowBytes;
      const int most = last - from;
#pragma unroll 1
      for (int j = 0; j < kGroupLoads; ++j) {
        const int n = j * 64 + lane, row = n / kRowChunks, chunk = n - row * kRowChunks;
        load_to_lds_16(base, (uint32_t)(min(row, most) * kRowBytes + ((chunk ^ swizzle(g * kGroupKeys + row)) << 4)), to + j * 1024);
      }
    }
  };

  // (every wave writes all the zeros: it reads them behind its own writes)
  *reinterpret_cast<u32x4*>(lds + kZeros + lane * 16) = u32x4{0, 0, 0, 0};

  // first tiles
  const int step = KEYS ? kWaves : 1;
  int32_t ids[kGroups];
  if constexpr (KEYS) {
    if (wave < ntiles) {
#pragma unroll
      for (int g = 0; g < kGroups; ++g) ids[g] = page_of(wave, g);
#pragma unroll
      for (int g = 0; g < kGroups; ++g) gather(wave, g, ids[g], lds0 + wave * kTileBytes + g * (kGroupKeys * kRowBytes));
    }
  } else {
#pragma unroll
    for (int a = 0; a < kWaves - 1; ++a)
      if (a < ntiles) gather(a, wave, page_of(a, wave), lds0 + a * kTileBytes + wave * (kGroupKeys * kRowBytes));
    ids[0] = page_of(kWaves - 1, wave);
  }

  // the wave's query rows as operands; rows behind the tile's last are copies of it
  const int i = lane % ROWS, part = lane / ROWS;
  const int row = min((KEYS ? 0 : wave * ROWS) + i, it.rows - 1);
  const uint16_t* q_row = q + (first + it.row0 + row) * kLatentRow + part * 8;
  bf16x8 qb[kSteps];
#pragma unroll
  for (int s = 0; s < kSteps; ++s) qb[s] = *reinterpret_cast<const bf16x8*>(q_row + s * (R32 ? 16 : 32));
  const int visible = rq.cached + (it.row0 + row) / heads + 1;
  const int least = rq.cached + (it.row0 + min((KEYS ? 0 : wave * ROWS), it.rows - 1)) / heads + 1;  // of the wave's first row

  // LDS addresses of the operands, in a tile at 0: the chunk's low bits take part in the swizzle and need an address each,
  // all else goes into the offset field of the read
  constexpr int kKeyAddrs = R32 ? 4 : 2, kValueAddrs = R32 ? 2 : 4;
  uint32_t key_at[kKeyAddrs], value_at[kValueAddrs], value_at8[kValueAddrs];
  const int value_key = R32 ? (lane >> 5) * 4 + ((lane & 15) >> 2) : (lane >> 4) * 4 + ((lane & 15) >> 2);
#pragma unroll
  for (int s = 0; s < kKeyAddrs; ++s)
    key_at[s] = i * kRowBytes + ((((R32 ? 2 : 4) * s + part) ^ swizzle(i)) << 4);
  {
    const int w16 = lane & 15, blk = lane >> 4;
    const int key = value_key;
    const int chunk = (R32 ? 2 * (blk & 1) : 0) + ((w16 & 3) >> 1);
#pragma unroll
    for (int d = 0; d < kValueAddrs; ++d) {
      const int c = (R32 ? 4 : 2) * d + chunk;
      value_at[d] = key * kRowBytes + ((c ^ swizzle(key)) << 4) + (w16 & 1) * 8;
      value_at8[d] = (key + 8) * kRowBytes + ((c ^ swizzle(key + 8)) << 4) + (w16 & 1) * 8;
    }
  }

  using Acc = std::conditional_t<R32, f32x16, f32x4>;
  constexpr int kAcc = R32 ? 16 : 4;
  Acc o[kBlocks];
#pragma unroll
  for (int d = 0; d < kBlocks; ++d)
#pragma unroll
    for (int r = 0; r < kAcc; ++r) o[d][r] = 0.f;
  float m_run = kNoReference, l_run = 0.f;
  auto product = [](bf16x8 a, bf16x8 b, Acc c) __attribute__((always_inline)) {
    if constexpr (R32) return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
  };
  constexpr int kAhead = 4;  // operands read in front of their products

  for (int tile = KEYS ? wave : 0; tile < ntiles; tile += step) {
    uint32_t buf;
    if constexpr (KEYS) {
      buf = lds0 + wave * kTileBytes;
#pragma unroll
      for (int g = 0; g < kGroups; ++g) ids[g] = page_of(tile + kWaves, g);
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    } else {
      buf = lds0 + (tile % kWaves) * kTileBytes;
      const int ahead = min(ntiles - 1 - tile, kWaves - 2);
      if (ahead == 2) asm volatile("s_waitcnt vmcnt(18)" ::: "memory");
      else if (ahead == 1) asm volatile("s_waitcnt vmcnt(9)" ::: "memory");
      else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __syncthreads();
      const int next = tile + kWaves - 1;
      if (next < ntiles)
        gather(next, wave, ids[0], lds0 + (next % kWaves) * kTileBytes + wave * (kGroupKeys * kRowBytes));
      ids[0] = page_of(next + 1, wave);
    }
    const int key0 = it.k0 + tile * kTileKeys;

    // scores: R32 lane i, half `part`: element r is key (r / 4) * 8 + part * 4 + r % 4; R16 lane i, quarter `part`: element r of
    // block b is key b * 16 + part * 4 + r
    float sc[R32 ? 16 : 8];
    constexpr int kKeyBlocks = R32 ? 1 : 2;  // of a tile
    bf16x8 ka[kAhead];
    auto read_key = [&](int n) __attribute__((always_inline)) {  // operand of product n
      const int s = n / kKeyBlocks, b = n % kKeyBlocks;
      ka[n % kAhead] = *(const LDS_PTR(bf16x8))(uintptr_t)(buf + key_at[s % kKeyAddrs] + (s / kKeyAddrs) * 128 + b * 16 * kRowBytes);
    };
    Acc acc[kKeyBlocks];
#pragma unroll
    for (int b = 0; b < kKeyBlocks; ++b)
#pragma unroll
      for (int r = 0; r < kAcc; ++r) acc[b][r] = 0.f;
#pragma unroll
    for (int n = 0; n < kAhead; ++n) read_key(n);
#pragma unroll
    for (int n = 0; n < kSteps * kKeyBlocks; ++n) {
      acc[n % kKeyBlocks] = product(ka[n % kAhead], qb[n / kKeyBlocks], acc[n % kKeyBlocks]);
      if (n + kAhead < kSteps * kKeyBlocks) read_key(n + kAhead);
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int r = 0; r < kAcc * kKeyBlocks; ++r) sc[r] = acc[r / kAcc][r % kAcc];
    constexpr int kScores = R32 ? 16 : 8;
    uint32_t unfit = 0;
    if (key0 + kTileKeys > least) {
      unfit = unfit_keys<ROWS>(sc);
#pragma unroll
      for (int r = 0; r < kScores; ++r) {
        const int key = key0 + (R32 ? (r >> 2) * 8 : (r >> 2) * 16) + part * 4 + (r & 3);
        sc[r] = key < visible ? sc[r] : -__builtin_inff();
      }
    }
    float mx = sc[0];
#pragma unroll
    for (int r = 1; r < kScores; ++r) mx = fmaxf(mx, sc[r]);
    if constexpr (!R32) mx = cross_quarter_max(mx);
    mx = cross_half_max(mx) * args.scale_log2;
    if (__any(mx > m_run + kSlack)) {
      const float m_new = mx > m_run + kSlack ? mx : m_run;
      const float f = m_new == m_run ? 1.f : __builtin_amdgcn_exp2f(m_run - m_new);
      l_run *= f;
      after_products();
#pragma unroll
      for (int d = 0; d < kBlocks; ++d)
#pragma unroll
        for (int r = 0; r < kAcc; ++r) o[d][r] = scale_accumulator(o[d][r], f);
      before_products();
      m_run = m_new;
    }
    u32x4 pb[kScores / 8];
#pragma unroll
    for (int r = 0; r < kScores; r += 2) {
      const float p0 = __builtin_amdgcn_exp2f(sc[r] * args.scale_log2 - m_run);
      const float p1 = __builtin_amdgcn_exp2f(sc[r + 1] * args.scale_log2 - m_run);
      const uint32_t two = pack_bf16(p0, p1);
      pb[r >> 3][(r & 7) >> 1] = two;
      l_run += __uint_as_float(two << 16) + __uint_as_float(two & 0xFFFF0000u);
    }
    // values: the addresses of the operands' keys `group` eighths (R32) or halves (R16) into the tile
    constexpr int kKeyGroups = R32 ? 4 : 2, kGroupRows = R32 ? 8 : 16;
    uint32_t at[kKeyGroups][kValueAddrs];
#pragma unroll
    for (int g = 0; g < kKeyGroups; ++g)
#pragma unroll
      for (int d = 0; d < kValueAddrs; ++d)
        at[g][d] = buf + (R32 && (g & 1) ? value_at8[d] + (g - 1) * kGroupRows * kRowBytes : value_at[d] + g * kGroupRows * kRowBytes);
    if (unfit) {
#pragma unroll
      for (int g = 0; g < kKeyGroups; ++g)
#pragma unroll
        for (int d = 0; d < kValueAddrs; ++d)
          if (unfit >> (value_key + g * kGroupRows) & 1) at[g][d] = lds0 + kZeros;
    }
    bf16x8 va[kAhead];
    auto read_value = [&](int n) __attribute__((always_inline)) {
      const int k = n / kBlocks, d = n % kBlocks, c = (d / kValueAddrs) * 128;
      const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((LDS_PTR(bf16x4))(uintptr_t)(at[2 * k][d % kValueAddrs] + c));
      const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((LDS_PTR(bf16x4))(uintptr_t)(at[2 * k + 1][d % kValueAddrs] + c));
      va[n % kAhead] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    };
    constexpr int kValueSteps = kScores / 8 * kBlocks;
#pragma unroll
    for (int n = 0; n < kAhead; ++n) read_value(n);
#pragma unroll
    for (int n = 0; n < kValueSteps; ++n) {
      o[n % kBlocks] = product(va[n % kAhead], __builtin_bit_cast(bf16x8, pb[n / kBlocks]), o[n % kBlocks]);
      if (n + kAhead < kValueSteps) read_value(n + kAhead);
      __builtin_amdgcn_sched_barrier(0);
    }
    if constexpr (KEYS) {
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the tile has been read
      if (tile + kWaves < ntiles)
#pragma unroll
        for (int g = 0; g < kGroups; ++g) gather(tile + kWaves, g, ids[g], buf + g * (kGroupKeys * kRowBytes));
    }
  }
  if constexpr (!R32) l_run = cross_quarter_sum(l_run);
  l_run = cross_half_sum(l_run);

  // Element r of block d is column d * ROWS + column(r) .. + 3 of row i.
  auto column = [&](int d, int r4) { return R32 ? d * 32 + r4 * 8 + part * 4 : d * 16 + part * 4; };
  auto write4 = [&](int tile_row, int col, f32x4 v, float inv) {
    if (it.slot >= 0) {
      *reinterpret_cast<f32x4*>(args.part_o + ((int64_t)it.slot * TILE + tile_row) * kLatentRank + col) = v;
    } else {
      const u32x2 w = {pack_bf16(v[0] * inv, v[1] * inv), pack_bf16(v[2] * inv, v[3] * inv)};
      *reinterpret_cast<u32x2*>(out + (first + it.row0 + tile_row) * kLatentRank + col) = w;
    }
  };

  if constexpr (!KEYS) {
    const int tile_row = wave * ROWS + i;
    if (tile_row < it.rows) {
      if (it.slot >= 0 && part == 0) {
        float* ml = args.part_ml + ((int64_t)it.slot * TILE + tile_row) * 2;
        ml[0] = m_run;
        ml[1] = l_run;
      }
      const float inv = 1.f / l_run;
#pragma unroll
      for (int d = 0; d < kBlocks; ++d)
#pragma unroll
        for (int r4 = 0; r4 < kAcc / 4; ++r4)
          write4(tile_row, column(d, r4), f32x4{o[d][4 * r4], o[d][4 * r4 + 1], o[d][4 * r4 + 2], o[d][4 * r4 + 3]}, inv);
    }
  } else {
    // join of the four waves, 128 columns at a time: [wave][row][128 + 4]
    constexpr int kCols = 128, kPitch = kCols + 4;
    static_assert(kWaves * ROWS * (kPitch + 2) * 4 <= kWaves * kTileBytes, "the join fits the tiles' place");
    float* const joined = reinterpret_cast<float*>(lds);
    float* const s_ml = joined + kWaves * ROWS * kPitch;  // [wave][row][2]
    __syncthreads();  // the tiles are read
    if (part == 0) {
      s_ml[(wave * ROWS + i) * 2] = m_run;
      s_ml[(wave * ROWS + i) * 2 + 1] = l_run;
    }
    __syncthreads();
    float m = kNoReference;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) m = fmaxf(m, s_ml[(w * ROWS + i) * 2]);
    const float f = __builtin_amdgcn_exp2f(m_run - m);
    constexpr int kThreadsPerRow = 64 * kWaves / ROWS, kPer = kCols / kThreadsPerRow;
    const int my_row = tid / kThreadsPerRow, my_col = tid % kThreadsPerRow * kPer;
    float my_m = kNoReference, my_l = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) my_m = fmaxf(my_m, s_ml[(w * ROWS + my_row) * 2]);
#pragma unroll
    for (int w = 0; w < kWaves; ++w)
      my_l += s_ml[(w * ROWS + my_row) * 2 + 1] * __builtin_amdgcn_exp2f(s_ml[(w * ROWS + my_row) * 2] - my_m);
    if (it.slot >= 0 && my_col == 0) {
      float* ml = args.part_ml + ((int64_t)it.slot * TILE + my_row) * 2;
      ml[0] = my_m;
      ml[1] = my_l;
    }
    const float inv = 1.f / my_l;
    constexpr int kBlocksPerRound = kCols / ROWS;
#pragma unroll
    for (int round = 0; round < kLatentRank / kCols; ++round) {
      if (round) __syncthreads();
#pragma unroll
      for (int b = 0; b < kBlocksPerRound; ++b)
#pragma unroll
        for (int r4 = 0; r4 < kAcc / 4; ++r4) {
          const int d = round * kBlocksPerRound + b;
          const f32x4 v = {o[d][4 * r4] * f, o[d][4 * r4 + 1] * f, o[d][4 * r4 + 2] * f, o[d][4 * r4 + 3] * f};
          *reinterpret_cast<f32x4*>(joined + (wave * ROWS + i) * kPitch + column(b, r4)) = v;
        }
      __syncthreads();
      if (my_row < it.rows) {
#pragma unroll
        for (int c = 0; c < kPer; c += 4) {
          f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int w = 0; w < kWaves; ++w) v += *reinterpret_cast<const f32x4*>(joined + (w * ROWS + my_row) * kPitch + my_col + c);
          write4(my_row, round * kCols + my_col + c, v, inv);
        }
      }
    }
  }
}

// Joins the ranges of split tiles: with M = max m, out = sum 2^(m - M) O / sum 2^(m - M) l, in the ranges' order.  Two rows to a
// workgroup, 128 threads each; blockIdx.y is the request.
__global__ __launch_bounds__(256) void latent_join_kernel(const LatentArgs args, int row_tile, uint16_t* __restrict__ out) {
  const LatentTable& t = args.table;
  const LatentReq q = t.req[blockIdx.y];
  const int splits = latent_splits(q.cached + q.new_len, t.range);
  const int row = blockIdx.x * 2 + (threadIdx.x >> 7), col = (threadIdx.x & 127) * 4;
  if (splits < 2 || row >= q.new_len * t.heads) return;
  const int tile = row / row_tile, in_tile = row - tile * row_tile;
  const int64_t first = ((int64_t)q.slot_start + (int64_t)tile * splits) * row_tile + in_tile;
  float m = kNoReference;
  for (int s = 0; s < splits; ++s) m = fmaxf(m, args.part_ml[(first + (int64_t)s * row_tile) * 2]);
  float l = 0.f;
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
  for (int s = 0; s < splits; ++s) {
    const int64_t at = first + (int64_t)s * row_tile;
    const float part = args.part_ml[at * 2 + 1];
    if (part == 0.f) continue;  // (its output may never have been written)
    const float w = __builtin_amdgcn_exp2f(args.part_ml[at * 2] - m);
    l += w * part;
    v += *reinterpret_cast<const f32x4*>(args.part_o + at * kLatentRank + col) * w;
  }
  const float inv = 1.f / l;
  const u32x2 w = {pack_bf16(v[0] * inv, v[1] * inv), pack_bf16(v[2] * inv, v[3] * inv)};
  *reinterpret_cast<u32x2*>(out + ((int64_t)q.row_start * t.heads + row) * kLatentRank + col) = w;
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
  args.part_o = reinterpret_cast<float*>(static_cast<char*>(workspace) + bytes.off_o);
  args.part_ml = reinterpret_cast<float*>(static_cast<char*>(workspace) + bytes.off_ml);
  LatentCursor at;
  while (latent_next(b, plan, &at, &args.table)) {
    auto* kernel = plan.row_tile == 16 ? latent_attention_kernel<16, true>
                   : plan.row_tile == 32 ? latent_attention_kernel<32, true> : latent_attention_kernel<32, false>;
    kernel<<<args.table.items, 64 * kWaves, 0, stream>>>(args, static_cast<const uint16_t*>(q), static_cast<const uint16_t*>(cache),
                                                        b->block_table, static_cast<uint16_t*>(out));
    if (args.table.split_rows > 0)
      latent_join_kernel<<<dim3((unsigned)((args.table.split_rows + 1) / 2), args.table.nreq), 256, 0, stream>>>(
          args, plan.row_tile, static_cast<uint16_t*>(out));
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
  const size_t bytes = efim::latent_bytes(efim::plan_latent(batch, efim::compute_units())).total;
  return bytes < 256 ? 256 : bytes;
}

int efim_latent_attention(const efim_batch_t* batch, const void* q, const void* latent_cache, void* out, float sm_scale,
                          void* workspace, size_t workspace_bytes, void* stream) {
  return efim::latent_attention(batch, q, latent_cache, out, sm_scale, workspace, workspace_bytes,
                                static_cast<hipStream_t>(stream));
}

}  // extern "C"
