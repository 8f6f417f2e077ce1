// efim_latent_attention_expanded: causal attention over the paged latent cache with keys and values per head, expanded from
// the latents by the caller's weight:
//   key [ W_uk,h c | r ],  value W_uv,h c,  s = sm_scale <q, key>,  p = softmax(s),  o = sum p value.
// A pair of a query row and a key costs 192 + 128 multiplications in place of the absorbed form's 576 + 512, and every
// key 512 * 256 a head for its expansion: cheaper from some 170 new tokens a request on.
//
// Two kernels.  The first is a product of the gathered latents with the weight, whose results it leaves in the workspace
// as the second one's LDS tiles: of 64 keys and a head, 24 KB of keys and 16 KB of values, chunks swizzled, so that the
// second gathers a tile with plain 1 KB loads.  The second is the attention, 32 query rows to a wave: scores and values as in the
// absorbed form, sums fp32, expanded keys, values and probabilities bf16 (as the weight and the latents are).
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
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;

#define LDS_PTR(T) __attribute__((address_space(3))) T*

constexpr int kQueryRow = kLatentNope + kLatentRope;  // 192
constexpr int kHeadOut = kLatentNope + kLatentValue;  // rows of the weight a head
constexpr int kTileKeys = kExpandedTileKeys;
constexpr int kKeyBytes = kQueryRow * 2;              // a key row of a tile
constexpr int kValueBytes = kLatentValue * 2;
constexpr int kKeysBytes = kTileKeys * kKeyBytes;
constexpr int kTileBytes = kExpandedTileBytes;
static_assert(kTileBytes == kTileKeys * (kKeyBytes + kValueBytes), "keys, then values");
constexpr float kSlack = 8.f;    // log2 units by which a row's maximum may outgrow its reference
constexpr float kOver = 256.f;   // 2^kSlack: a sum of rounded probabilities is never below its largest one
constexpr float kNoReference = -3.0e38f;

// Swizzles of a tile row's 16-byte chunks.  Keys: 24 chunks, so neighbouring rows start half of the 256-byte bank line
// apart; the three bits spread sixteen rows' equal chunks over its sixteen places.  Values: 16 chunks, the two bits spread
// the four chunks that a transposing read takes of each of eight rows.
__device__ __forceinline__ int key_swizzle(int row) { return (row >> 1) & 7; }
__device__ __forceinline__ int value_swizzle(int row) { return (row & 3) << 2; }

// The request that a tile of keys, or of query rows, lies in.
template <bool KEYS>
__device__ __forceinline__ int find_request(const ExpandedTable& t, int tile, int lane) {
  int r = -1;
#pragma unroll
  for (int i = 0; i < kLatentTableReqs / 64; ++i) {
    const int k = min(i * 64 + lane, t.nreq - 1);
    r += __popcll(__ballot(i * 64 + lane < t.nreq && (KEYS ? (int)t.req[k].unit_start : t.row_tile_start[k]) <= tile));
  }
  return __builtin_amdgcn_readfirstlane(r);
}

// --- expansion -----------------------------------------------------------------------------------------------------------

constexpr int kTokens = 2 * kTileKeys;  // of a workgroup: two tiles
constexpr int kDepth = 32;              // elements of the latent staged at a time
constexpr int kDepthBytes = kDepth * 2;
constexpr int kStageBytes = (kTokens + kHeadOut) * kDepthBytes;
constexpr int kStageCount = 3;
constexpr int kExpandWaves = 4;

// Swizzle of a staged row's four 16-byte chunks: sixteen rows' equal chunks take the sixteen places of the bank line.
__device__ __forceinline__ int stage_swizzle(int row) { return (row >> 2) & 3; }

// blockIdx.x: head (fastest, so that an XCD meets few heads' weights) and pair of tiles.  A wave forms 64 tokens x 128
// outputs as W C^T: a lane's results are four neighbouring outputs of one token, and an operand of either side serves two or
// four products.  Two workgroups share a unit, so that one multiplies while the other writes its tiles; the loads are two
// stages ahead.
__global__ __launch_bounds__(64 * kExpandWaves, 2) void expand_kernel(const ExpandedTable t, const uint16_t* __restrict__ cache,
                                                                      const uint16_t* __restrict__ w_kv,
                                                                      const int32_t* __restrict__ block_table,
                                                                      char* __restrict__ tiles) {
  constexpr int kLdsBytes = 2 * kTileBytes;
  static_assert(kStageCount * kStageBytes <= kLdsBytes, "the finished tiles take the stages' place");
  __shared__ __attribute__((aligned(1024))) char lds[kLdsBytes];
  const uint32_t lds0 = (uint32_t)(uintptr_t)(LDS_PTR(char))lds;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int pair = blockIdx.x / t.heads, head = blockIdx.x - pair * t.heads;
  const LatentReq rq = t.req[find_request<true>(t, 2 * pair, lane)];
  const int keys = rq.cached + rq.new_len;
  const int key0 = (2 * pair - (int)rq.unit_start) * kTileKeys;  // first token of the pair
  const int32_t* pages = block_table + (int64_t)rq.req * t.max_pages;
  const int page_shift = t.page_shift, page_mask = (1 << page_shift) - 1;
  const char* w = reinterpret_cast<const char*>(w_kv) + (int64_t)head * kHeadOut * kLatentRank * 2;
  // Tokens behind the request's last are copies of it (their scores are masked).
  auto token_row = [&](int token) {
    const int key = min(key0 + token, keys - 1);
    const int64_t page = pages[key >> page_shift];
    return reinterpret_cast<const char*>(cache) + ((page << page_shift) + (key & page_mask)) * (kLatentRow * 2);
  };

  // 1 KB loads of sixteen rows by 64 bytes, eight of tokens and sixteen of weight rows: two and four a wave; lane l fetches row
  // l / 4, its chunk l % 4 swizzled.
  constexpr int kLoadRows = 1024 / kDepthBytes;
  constexpr int kTokenLoads = kTokens / kLoadRows / kExpandWaves, kWeightLoads = kHeadOut / kLoadRows / kExpandWaves;
  static_assert(kTokenLoads == 2 && kWeightLoads == 4, "loads of a wave and stage");
  const char* token_src[kTokenLoads];
  uint32_t weight_src[kWeightLoads];
#pragma unroll
  for (int j = 0; j < kTokenLoads; ++j) {
    const int row = (wave * kTokenLoads + j) * kLoadRows + (lane >> 2);
    token_src[j] = token_row(row) + (((lane & 3) ^ stage_swizzle(row)) << 4);
  }
#pragma unroll
  for (int j = 0; j < kWeightLoads; ++j) {
    const int row = (wave * kWeightLoads + j) * kLoadRows + (lane >> 2);
    weight_src[j] = (uint32_t)(row * (kLatentRank * 2) + (((lane & 3) ^ stage_swizzle(row)) << 4));
  }
  auto stage = [&](int step) { return lds0 + (uint32_t)(step % kStageCount) * kStageBytes; };
  auto fetch = [&](int step) __attribute__((always_inline)) {
    const uint32_t to = stage(step);
#pragma unroll
    for (int j = 0; j < kTokenLoads; ++j)
      load_to_lds_16(token_src[j] + step * kDepthBytes, to + (wave * kTokenLoads + j) * 1024);
#pragma unroll
    for (int j = 0; j < kWeightLoads; ++j)
      load_to_lds_16(w + step * kDepthBytes, weight_src[j], to + kTokens * kDepthBytes + (wave * kWeightLoads + j) * 1024);
  };
  fetch(0);
  fetch(1);

  const int i = lane & 31, part = lane >> 5;
  const int token_half = wave & 1, out_half = wave >> 1;
  f32x16 acc[2][4];  // [token block][output block]
#pragma unroll
  for (int a = 0; a < 2; ++a)
#pragma unroll
    for (int b = 0; b < 4; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[a][b][r] = 0.f;
  uint32_t at[2];  // of an operand in a staged row
#pragma unroll
  for (int s = 0; s < 2; ++s) at[s] = i * kDepthBytes + (((2 * s + part) ^ stage_swizzle(i)) << 4);
  constexpr int kSteps = kLatentRank / kDepth;
  for (int step = 0; step < kSteps; ++step) {
    if (step + 1 < kSteps) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kTokenLoads + kWeightLoads) : "memory");
    else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (step + 2 < kSteps) fetch(step + 2);
    const uint32_t tok = stage(step) + token_half * 64 * kDepthBytes;
    const uint32_t wgt = stage(step) + kTokens * kDepthBytes + out_half * 128 * kDepthBytes;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      bf16x8 x[2], y[4];
#pragma unroll
      for (int a = 0; a < 2; ++a) x[a] = *(const LDS_PTR(bf16x8))(uintptr_t)(tok + at[s] + a * 32 * kDepthBytes);
#pragma unroll
      for (int b = 0; b < 4; ++b) y[b] = *(const LDS_PTR(bf16x8))(uintptr_t)(wgt + at[s] + b * 32 * kDepthBytes);
#pragma unroll
      for (int b = 0; b < 4; ++b)
#pragma unroll
        for (int a = 0; a < 2; ++a) acc[a][b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(y[b], x[a], acc[a][b], 0, 0, 0);
    }
  }
  __syncthreads();
  // the tiles as the attention takes them, in LDS, then out in whole lines
  char* const tile = lds + token_half * kTileBytes;
#pragma unroll
  for (int a = 0; a < 2; ++a)
#pragma unroll
    for (int b = 0; b < 4; ++b)
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4) {
        const int row = a * 32 + i;
        const int col = b * 32 + r4 * 8 + part * 4;  // of the keys (out_half 0) or of the values
        const u32x2 v = {pack_bf16(acc[a][b][4 * r4], acc[a][b][4 * r4 + 1]), pack_bf16(acc[a][b][4 * r4 + 2], acc[a][b][4 * r4 + 3])};
        char* to = out_half == 0 ? tile + row * kKeyBytes + (((col >> 3) ^ key_swizzle(row)) << 4)
                                 : tile + kKeysBytes + row * kValueBytes + (((col >> 3) ^ value_swizzle(row)) << 4);
        *reinterpret_cast<u32x2*>(to + part * 8) = v;
      }
  // rotated part of the keys: 8 chunks a token, of the cache
#pragma unroll
  for (int j = 0; j < kTokens * 8 / (64 * kExpandWaves); ++j) {
    const int n = j * 64 * kExpandWaves + tid, token = n >> 3, chunk = n & 7;
    const u32x4 v = *reinterpret_cast<const u32x4*>(token_row(token) + kLatentRank * 2 + chunk * 16);
    const int row = token & (kTileKeys - 1);
    *reinterpret_cast<u32x4*>(lds + (token / kTileKeys) * kTileBytes + row * kKeyBytes + ((16 + (chunk ^ key_swizzle(row))) << 4)) = v;
  }
  __syncthreads();
  char* dst = tiles + ((int64_t)head * t.key_tiles + 2 * pair) * kTileBytes;
#pragma unroll
  for (int j = 0; j < 2 * kTileBytes / (64 * kExpandWaves * 16); ++j) {
    const int n = (j * 64 * kExpandWaves + tid) * 16;
    *reinterpret_cast<u32x4*>(dst + n) = *reinterpret_cast<const u32x4*>(lds + n);
  }
}

// --- attention -----------------------------------------------------------------------------------------------------------

struct ExpandedArgs {
  ExpandedTable table;
  float scale_log2;
};

// blockIdx.x: head (fastest: an XCD meets few heads, whose tiles its workgroups share) and tile of query rows, the request's
// last rows, which see most keys, first.  Eight waves of 32 rows each: SETS 8 takes 256 rows; SETS 4 takes 128 and
// divides the keys, the first halves of the key tiles to four waves and the second ones to the others, which join at the end.
//
// A wave works off its halves three at a time: while the scores of half n are turned into probabilities, the products form the
// scores of n + 1 and add the values of n - 1.  The waves meet where one of the three enters another tile.  Keys are
// gathered three tiles ahead and values, which are wanted two halves later, two tiles.  No maximum is formed on the way: the
// reference is the row's maximum over the first half and moves where a half's sum of probabilities tells that one of
// them passed 2^kSlack.
constexpr int kAttendWaves = 8;
constexpr int kKeyStages = 4, kValueStages = 3;
constexpr int kValuesAt = kKeyStages * kKeysBytes;                           // in LDS
constexpr int kZeros = kValuesAt + kValueStages * (kTileBytes - kKeysBytes);  // the values in front of the first half

template <int SETS>
__global__ __launch_bounds__(64 * kAttendWaves, 2) void expanded_attention_kernel(const ExpandedArgs args,
                                                                                  const uint16_t* __restrict__ q,
                                                                                  const char* __restrict__ tiles,
                                                                                  uint16_t* __restrict__ out) {
  constexpr int TILE = 32 * SETS;
  constexpr bool kDivided = SETS < kAttendWaves;
  constexpr int kKeyLoads = kKeysBytes / 1024 / kAttendWaves, kValueLoads = (kTileBytes - kKeysBytes) / 1024 / kAttendWaves;  // a wave's, of a tile
  __shared__ __attribute__((aligned(1024))) char lds[kZeros + 32 * kValueBytes];
  const uint32_t lds0 = (uint32_t)(uintptr_t)(LDS_PTR(char))lds;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int set = wave % SETS, group = wave / SETS;
  static_assert(32 * kValueBytes == 64 * kAttendWaves * 16, "a piece of the zeros each");
  *reinterpret_cast<u32x4*>(lds + kZeros + tid * 16) = u32x4{0, 0, 0, 0};
  const ExpandedTable& t = args.table;
  const int heads = t.heads;
  const int at = blockIdx.x / heads, head = blockIdx.x - at * heads;
  const int r = find_request<false>(t, at, lane);
  const LatentReq rq = t.req[r];
  const int row_tiles = (rq.new_len + TILE - 1) / TILE;
  const int row0 = (row_tiles - 1 - (at - t.row_tile_start[r])) * TILE;
  const int rows = min(TILE, rq.new_len - row0);
  const int keys = rq.cached + row0 + rows;
  const int ntiles = (keys + kTileKeys - 1) / kTileKeys;
  const char* src = tiles + ((int64_t)head * t.key_tiles + rq.unit_start) * kTileBytes;
  // (a tile in front of the first, or behind the last, stands for whatever lies in its place)
  auto keys_at = [&](int tile) { return lds0 + (uint32_t)(tile & (kKeyStages - 1)) * kKeysBytes; };
  auto values_of = [&](int tile) {
    return lds0 + kValuesAt + (uint32_t)((tile + kValueStages) % kValueStages) * (kTileBytes - kKeysBytes);
  };
  auto fetch_keys = [&](int tile) __attribute__((always_inline)) {
    const char* from = src + (int64_t)tile * kTileBytes + wave * (kKeyLoads * 1024);
    load_to_lds_run<kKeyLoads>(from, (uint32_t)lane * 16, keys_at(tile) + wave * (kKeyLoads * 1024));
  };
  auto fetch_values = [&](int tile) __attribute__((always_inline)) {
    const char* from = src + (int64_t)tile * kTileBytes + kKeysBytes + wave * (kValueLoads * 1024);
    load_to_lds_run<kValueLoads>(from, (uint32_t)lane * 16, values_of(tile) + wave * (kValueLoads * 1024));
  };

  const int i = lane & 31, part = lane >> 5;
  const int row = min(set * 32 + i, rows - 1);
  const int64_t packed = (int64_t)rq.row_start + row0 + row;
  constexpr int kSteps = kQueryRow / 16, kBlocks = kLatentValue / 32, kValueProducts = 2 * kBlocks;
  bf16x8 qb[kSteps];
#pragma unroll
  for (int s = 0; s < kSteps; ++s)
    qb[s] = *reinterpret_cast<const bf16x8*>(q + (packed * heads + head) * kQueryRow + s * 16 + part * 8);
  fetch_keys(0);
  fetch_values(0);
  if (1 < ntiles) fetch_keys(1);
  // (the loop below counts the gathers in flight itself: everything the compiler knows of is waited for here)
  __builtin_amdgcn_s_waitcnt(0x0F70);
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  if (!kDivided && 1 < ntiles) fetch_values(1);
  if (2 < ntiles) fetch_keys(2);
  if (3 < ntiles) fetch_keys(3);
  __syncthreads();
  const int visible = rq.cached + row0 + row + 1;
  const int least = rq.cached + row0 + set * 32 + 1;  // of the wave's first row
  // halves of which the wave's last row sees a part, counted in its own; none where the wave has no rows
  const int seen = set * 32 >= rows ? 0 : (rq.cached + row0 + min(set * 32 + 31, rows - 1) + 32) / 32;
  const int halves = kDivided ? (seen + 1 - group) / 2 : seen;

  uint32_t key_at[4], value_at[kBlocks];
#pragma unroll
  for (int s = 0; s < 4; ++s) key_at[s] = i * kKeyBytes + (((2 * s + part) ^ key_swizzle(i)) << 4);
  {
    const int w16 = lane & 15, blk = lane >> 4;
    const int key = (blk >> 1) * 4 + (w16 >> 2), chunk = 2 * (blk & 1) + ((w16 & 3) >> 1);
#pragma unroll
    for (int d = 0; d < kBlocks; ++d)
      value_at[d] = key * kValueBytes + (((4 * d + chunk) ^ value_swizzle(key)) << 4) + (w16 & 1) * 8;
  }
  f32x16 o[kBlocks];
#pragma unroll
  for (int d = 0; d < kBlocks; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[d][r] = 0.f;
  float m_run = kNoReference, l_run = 0.f;
  f32x16 s0, s1;                  // scores of an even and an odd half
  u32x4 p0[2], p1[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};  // and their probabilities, as operands

  // Products of a round: the scores of the 32 keys at `ks` into `sn`, the values of the 32 keys at `vs` under the
  // probabilities `pv`; beside them the probabilities of the scores `sc` into `pn`, whose sum is returned.
  constexpr int kProducts = kSteps + kValueProducts, kAhead = 4;
  auto probability = [&](const f32x16& sc, int e) __attribute__((always_inline)) { return __builtin_amdgcn_exp2f(sc[e] * args.scale_log2 - m_run); };
  auto add_pair = [&](uint32_t two, float sum) __attribute__((always_inline)) {  // of two probabilities as they were rounded
    typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
    const bf16x2 ones = {(__bf16)1.0f, (__bf16)1.0f};
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, two), ones, sum, false);
  };
  auto key_operand = [&](uint32_t ks, int n) __attribute__((always_inline)) {
    return *(const LDS_PTR(u32x4))(uintptr_t)(ks + key_at[n & 3] + (n >> 2) * 128);
  };
  auto score_product = [&](u32x4 a, int n, f32x16& sn) __attribute__((always_inline)) {
    f32x16 from = sn;
    if (n == 0) {
#pragma unroll
      for (int r = 0; r < 16; ++r) from[r] = 0.f;
    }
    sn = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), qb[n], from, 0, 0, 0);
  };
  auto round = [&](f32x16& sn, uint32_t ks, const u32x4 (&pv)[2], uint32_t vs, const f32x16& sc, u32x4 (&pn)[2]) __attribute__((always_inline)) -> float {
    u32x4 staged[kAhead];
    auto operand = [&](int n) __attribute__((always_inline)) -> u32x4 {
      if (n < kSteps) return key_operand(ks, n);
      const int k = (n - kSteps) / kBlocks, d = (n - kSteps) % kBlocks;
      const uint32_t v = vs + value_at[d] + k * 16 * kValueBytes;
      const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((LDS_PTR(bf16x4))(uintptr_t)(v));
      const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((LDS_PTR(bf16x4))(uintptr_t)(v + 8 * kValueBytes));
      return __builtin_bit_cast(u32x4, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    };
#pragma unroll
    for (int n = 0; n < kAhead; ++n) staged[n] = operand(n);
    __builtin_amdgcn_sched_barrier(0);
    float sum = 0.f, pair[2];
#pragma unroll
    for (int n = 0; n < kProducts; ++n) {
      if (n < kSteps) {
        score_product(staged[n % kAhead], n, sn);
      } else {
        const int j = n - kSteps;
        o[j % kBlocks] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, staged[n % kAhead]),
                                                                 __builtin_bit_cast(bf16x8, pv[j / kBlocks]), o[j % kBlocks], 0, 0, 0);
      }
      if (n + kAhead < kProducts) staged[n % kAhead] = operand(n + kAhead);
      if (n < 16) {
        pair[n & 1] = probability(sc, n);
        if (n & 1) {
          const uint32_t two = pack_bf16(pair[0], pair[1]);
          pn[n >> 3][(n & 7) >> 1] = two;
          sum = add_pair(two, sum);
          asm volatile("" : "+v"(sum));  // (keeps the step in its place)
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    return sum;
  };
  auto row_max = [&](const f32x16& sc) __attribute__((always_inline)) {
    float mx = sc[0];
#pragma unroll
    for (int r = 1; r < 16; ++r) mx = fmaxf(mx, sc[r]);
    return cross_half_max(mx) * args.scale_log2;
  };
  // The waves meet in front of the round that enters key tile `next`: it is there then, as are the values of the tile
  // `kLate` tiles in front of it, and what the rounds so far read is free for those further on.
  constexpr int kLate = kDivided ? 2 : 1;
  auto meet = [&](int next) __attribute__((always_inline)) {
    // (in flight may be what the meeting in front sent for: keys three tiles on, values)
    if (next + 2 < ntiles) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kKeyLoads + kValueLoads) : "memory");
    else if (next + 1 - kLate < ntiles) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kValueLoads) : "memory");
    else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (next + 3 < ntiles) fetch_keys(next + 3);
    if (next + 2 - kLate < ntiles) fetch_values(next + 2 - kLate);
  };

  // The wave's n-th half: scores `sc`, probabilities to `pn`.  The round's products are those of its neighbours.  Behind the
  // last half there is a round for its values alone: what it does beside them is for nobody, as are the scores behind
  // the last half.
  auto tile_of = [&](int n) { return kDivided ? n : n >> 1; };
  auto half_of = [&](int n) { return kDivided ? group : n & 1; };
  auto half = [&](int n, f32x16& sc, f32x16& sn, u32x4 (&pn)[2], u32x4 (&po)[2]) __attribute__((always_inline)) {
    if (n > halves || halves == 0) return;
    const bool last = n == halves;
    const int key0 = tile_of(n) * kTileKeys + half_of(n) * 32;
    if (!last && key0 + 32 > least) {
      float raw[16];
#pragma unroll
      for (int r = 0; r < 16; ++r) raw[r] = sc[r];
      uint32_t unfit = unfit_keys<32>(raw);
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (key0 + (r >> 2) * 8 + part * 4 + (r & 3) >= visible) sc[r] = -__builtin_inff();
      // Their values become zeros where they lie: the weight of a row that sees such a key is no number, so that any wave may
      // take either.
      while (unfit) {
        const int key = half_of(n) * 32 + __builtin_ctz(unfit);
        unfit &= unfit - 1;
        if (lane < kValueBytes / 16)
          *(LDS_PTR(u32x4))(uintptr_t)(values_of(tile_of(n)) + key * kValueBytes + lane * 16) = u32x4{0, 0, 0, 0};
      }
    }
    if (n == 0) m_run = fmaxf(row_max(sc), kNoReference);
    const uint32_t front = n == 0 ? lds0 + kZeros : values_of(tile_of(n - 1)) + half_of(n - 1) * 32 * kValueBytes;
    float sum = round(sn, keys_at(tile_of(n + 1)) + half_of(n + 1) * 32 * kKeyBytes, po, front, sc, pn);
    if (last) return;
    if (__any(sum >= kOver)) {
      const float mx = row_max(sc);
      const float m_new = mx > m_run + kSlack ? mx : m_run;
      const float f = m_new == m_run ? 1.f : __builtin_amdgcn_exp2f(m_run - m_new);
      l_run *= f;
#pragma unroll
      for (int d = 0; d < kBlocks; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[d][r] *= f;
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
  if (halves > 0) {
#pragma unroll
    for (int n = 0; n < kSteps; ++n) score_product(key_operand(keys_at(0) + half_of(0) * 32 * kKeyBytes, n), n, s0);
  }
  if constexpr (kDivided) {
    for (int n = 0; n <= ntiles; n += 2) {
      meet(n + 1);
      half(n, s0, s1, p0, p1);
      if (n + 1 > ntiles) break;
      meet(n + 2);
      half(n + 1, s1, s0, p1, p0);
    }
  } else {
    for (int tile = 0; tile <= ntiles; ++tile) {
      half(2 * tile, s0, s1, p0, p1);
      if (tile == ntiles) break;
      meet(tile + 1);
      half(2 * tile + 1, s1, s0, p1, p0);
    }
  }
  l_run = cross_half_sum(l_run);
  if constexpr (kDivided) {
    // join: the second four waves leave their outputs, references and sums, a row to a lane, the first four add them
    constexpr int kPitch = 33;  // words of a lane's 32 and one, so that the lanes' words take all banks
    float* const left = reinterpret_cast<float*>(lds) + set * (64 * kPitch * 2 + 2 * 64);
    static_assert(SETS * (64 * kPitch * 2 + 2 * 64) * 4 <= kZeros, "the join takes the tiles' place");
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (group == 1) {
#pragma unroll
      for (int d = 0; d < kBlocks; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) left[(d >> 1) * 64 * kPitch + lane * kPitch + (d & 1) * 16 + r] = o[d][r];
      left[64 * kPitch * 2 + lane] = m_run;
      left[64 * kPitch * 2 + 64 + lane] = l_run;
    }
    __syncthreads();
    if (group == 1) return;
    const float m_other = left[64 * kPitch * 2 + lane], l_other = left[64 * kPitch * 2 + 64 + lane];
    const float m = fmaxf(m_run, m_other);
    const float f = __builtin_amdgcn_exp2f(m_run - m), f_other = __builtin_amdgcn_exp2f(m_other - m);
    l_run = l_run * f + l_other * f_other;
#pragma unroll
    for (int d = 0; d < kBlocks; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[d][r] = o[d][r] * f + left[(d >> 1) * 64 * kPitch + lane * kPitch + (d & 1) * 16 + r] * f_other;
  }
  const float inv = 1.f / l_run;
  uint16_t* dst = out + (packed * heads + head) * kLatentValue;
  // the two halves of the wave exchange four columns each, so that a lane writes eight in a row
#pragma unroll
  for (int d = 0; d < kBlocks; ++d)
#pragma unroll
    for (int r8 = 0; r8 < 2; ++r8) {
      u32x2 x[2];
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int k = 0; k < 2; ++k)
          x[h][k] = pack_bf16(o[d][r8 * 8 + h * 4 + 2 * k] * inv, o[d][r8 * 8 + h * 4 + 2 * k + 1] * inv);
      u32x4 words;
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const auto both = __builtin_amdgcn_permlane32_swap(x[0][k], x[1][k], false, false);
        words[k] = both[0];
        words[2 + k] = both[1];
      }
      if (set * 32 + i < rows) *reinterpret_cast<u32x4*>(dst + d * 32 + r8 * 16 + part * 8) = words;
    }
}

int latent_attention_expanded(const efim_batch_t* b, const void* q, const void* cache, const void* w_kv, void* out,
                              float sm_scale, void* workspace, size_t workspace_bytes, hipStream_t stream) {
  int64_t total = 0;
  const int rc = validate_latent_batch(b, &total);
  if (rc != EFIM_OK) return rc;
  if (!(sm_scale > 0.f) || sm_scale - sm_scale != 0.f) return EFIM_ERR_INVALID_ARG;
  if (total == 0) return EFIM_OK;
  if (!q || !cache || !w_kv || !out || q == out || out == cache || out == w_kv) return EFIM_ERR_INVALID_ARG;
  if (!aligned16(q) || !aligned16(cache) || !aligned16(w_kv) || !aligned16(out) || !aligned4(b->block_table))
    return EFIM_ERR_INVALID_ARG;
  const ExpandedPlan plan = plan_expanded(b, compute_units());
  if (!plan.ok) return EFIM_ERR_UNSUPPORTED;
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u) || workspace_bytes < plan.bytes) return EFIM_ERR_WORKSPACE;
  ExpandedArgs args;
  args.scale_log2 = sm_scale * 1.44269504088896340736f;
  char* tiles = static_cast<char*>(workspace);
  LatentCursor at;
  while (expanded_next(b, plan, &at, &args.table)) {
    const unsigned heads = (unsigned)b->num_q_heads;
    expand_kernel<<<(unsigned)args.table.key_tiles / 2 * heads, 64 * kExpandWaves, 0, stream>>>(
        args.table, static_cast<const uint16_t*>(cache), static_cast<const uint16_t*>(w_kv), b->block_table, tiles);
    if (plan.row_tile == 256)
      expanded_attention_kernel<8><<<(unsigned)args.table.row_tiles * heads, 512, 0, stream>>>(args, static_cast<const uint16_t*>(q), tiles,
                                                                                    static_cast<uint16_t*>(out));
    else
      expanded_attention_kernel<4><<<(unsigned)args.table.row_tiles * heads, 512, 0, stream>>>(args, static_cast<const uint16_t*>(q), tiles,
                                                                                    static_cast<uint16_t*>(out));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) { set_last_hip_error(e); return EFIM_ERR_LAUNCH; }
  }
  return EFIM_OK;
}

}  // namespace
}  // namespace efim

extern "C" {

size_t efim_latent_expanded_workspace_bytes(const efim_batch_t* batch) {
  int64_t total = 0;
  if (efim::validate_latent_batch(batch, &total) != EFIM_OK) return 0;
  const efim::ExpandedPlan plan = efim::plan_expanded(batch, efim::compute_units());
  return !plan.ok ? 0 : plan.bytes < 256 ? 256 : plan.bytes;
}

int efim_latent_attention_expanded(const efim_batch_t* batch, const void* q, const void* latent_cache, const void* w_kv,
                                   void* out, float sm_scale, void* workspace, size_t workspace_bytes, void* stream) {
  return efim::latent_attention_expanded(batch, q, latent_cache, w_kv, out, sm_scale, workspace, workspace_bytes,
                                         static_cast<hipStream_t>(stream));
}

}  // extern "C"
