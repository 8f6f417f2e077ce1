// efim_latent_attention_expanded: causal attention over the paged latent cache with keys and values per head, expanded from
// the latents by the caller's weight:
//   key [ W_uk,h c | r ],  value W_uv,h c,  s = sm_scale <q, key>,  p = softmax(s),  o = sum p value.
// A pair of a query row and a key costs 192 + 128 multiplications in place of the absorbed form's 576 + 512, and every
// key 512 * 256 a head for its expansion: cheaper from some 170 new tokens a request on.
//
// Two kernels.  The first is a product of the gathered latents with the weight, whose results it leaves in the workspace
// as the second one's LDS tiles: of 64 keys and a head, 24 KB of keys and 16 KB of values, chunks swizzled, so that the
// second gathers a tile with plain 1 KB loads.  The second is the attention, 32 query rows to a wave: scores and values as in the
// absorbed form, sums fp32, expanded keys, values and probabilities bf16 (as the weight and the latents are, and with their range):
// 2.8e-3 of the result's norm from the exact one, where its own rounding alone leaves 1.7e-3.
// 12 prompts of 20k new tokens, 26k keys and 32 heads: 228 to 240 us (214 GFLOP, 523 MB written) and 590 to 630 us (536 GFLOP that count).
#include <cstddef>
#include <type_traits>
#include <utility>

#include "efim_internal.h"
#include "latent_plan.h"
#include "latent_device.h"
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

// --- expansion -----------------------------------------------------------------------------------------------------------

constexpr int kUnitKeys = 32;                             // half a tile
constexpr int kLatentBytes = kLatentRank * 2;
constexpr int kStageBytes = kUnitKeys * kRowBytes;        // rows of the cache, as the absorbed form's tiles have them
constexpr int kStageCount = 3;
constexpr int kExpandWaves = 8, kWaveOuts = kHeadOut / kExpandWaves;
constexpr int kPlacePitch = kWaveOuts * 2 + 16;           // of a wave's outputs on their way out
constexpr int kPlacesAt = kStageCount * kStageBytes;
constexpr int kWeightBytes = kWaveOuts * kLatentBytes / 2;  // half of a wave's weight on its way in
constexpr int kExpandLds = kPlacesAt + kExpandWaves * kUnitKeys * kPlacePitch;
static_assert(kExpandWaves * kWeightBytes <= kExpandLds && kLatentBytes == 1024 && kWaveOuts == 32, "sizes");
static_assert(kExpandWaves / 2 * kGroupKeys == kUnitKeys, "two waves gather a group");

// f(0), f(1), .. with the number as a type: a loop of so long a body is not unrolled.
template <int... N, typename F>
__device__ __forceinline__ void each(std::integer_sequence<int, N...>, F f) {
  (f(std::integral_constant<int, N>()), ...);
}
template <int COUNT, typename F>
__device__ __forceinline__ void each(F f) {
  each(std::make_integer_sequence<int, COUNT>(), f);
}

// The compiler gives such products accumulation registers, which the weight takes, and counts no states behind written-out ones.
__device__ __forceinline__ void first_expand_product(f32x16& acc, bf16x8 weight, bf16x8 token) {
  asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, 0" : "=&v"(acc) : "a"(weight), "v"(token));
}
__device__ __forceinline__ void expand_product(f32x16& acc, bf16x8 weight, bf16x8 token) {
  asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+v"(acc) : "a"(weight), "v"(token));
}

// blockIdx.x: head and slice of the launch's keys.  A workgroup keeps the head's whole weight in registers, 32 of its 256 rows
// in each of eight waves, and the slice's latents pass by in LDS, 32 at a time: so a latent is fetched once a head.  A wave's
// results W C^T are, a lane, four neighbouring outputs of one token; beside the products of a unit those of the unit in front
// go out through LDS, in runs of 64 bytes, and the gather of the unit two further on.  Without the gathers and the stores the
// products take 160 us of the 228 above, alone 110.  (Four waves of 64 rows, for which an operand read from LDS serves
// two products, measured the same; tiles of 128 tokens and 256 outputs with the weight in LDS, 2.5 GB gathered, 290 us.)
__global__ __launch_bounds__(64 * kExpandWaves, 2) void expand_kernel(const ExpandedTable t, const uint16_t* __restrict__ cache,
                                                                      const uint16_t* __restrict__ w_kv,
                                                                      const int32_t* __restrict__ block_table,
                                                                      char* __restrict__ tiles) {
  __shared__ __attribute__((aligned(1024))) char lds[kExpandLds];
  const uint32_t lds0 = (uint32_t)(uintptr_t)(LDS_PTR(char))lds;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int head = blockIdx.x / t.slices, slice = blockIdx.x - head * t.slices;
  const int units = t.key_tiles * (kTileKeys / kUnitKeys);
  const int begin = (int)((int64_t)units * slice / t.slices), end = (int)((int64_t)units * (slice + 1) / t.slices);
  if (begin == end) return;
  const int i = lane & 31, part = lane >> 5;
  constexpr int kSteps = kLatentRank / 16;
  bf16x8 weight[kSteps];
  {
    // Through LDS, half of the depth at a time: chunk c of row r lies at c exclusive or the row's low four bits.
    const char* from = reinterpret_cast<const char*>(w_kv) + ((int64_t)head * kHeadOut + wave * kWaveOuts) * kLatentBytes;
    const uint32_t place = lds0 + wave * kWeightBytes;
#pragma unroll
    for (int b = 0; b < 2; ++b) {
#pragma unroll
      for (int r = 0; r < kWaveOuts; r += 2) {
        const int row = r + part;
        load_to_lds_16(from + b * (kLatentBytes / 2), (uint32_t)(row * kLatentBytes + ((i ^ (row & 15)) << 4)), place + r * (kLatentBytes / 2));
      }
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
      for (int s = 0; s < kSteps / 2; ++s)
        weight[b * (kSteps / 2) + s] =
            *(const LDS_PTR(bf16x8))(uintptr_t)(place + i * (kLatentBytes / 2) + (((2 * (s & 7) + part) ^ (i & 15)) << 4) + (s >> 3) * 256);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }
  }
  __syncthreads();

  // Lane l holds where the wave's group of unit held_from + l lies: its row's address, its first key in its request, the request's
  // keys, the page.  (Keys behind the last become copies of it; their scores are masked.)
  Gather rows(cache, 0, t.page_shift, lane);
  // A group's nine loads are shared by two waves: five and four.
  const int group = wave & 3, first_piece = wave < 4 ? 0 : 5;
  uint32_t piece_at[5];
#pragma unroll
  for (int n = 0; n < 5; ++n) piece_at[n] = rows.offset(min(first_piece + n, kGroupLoads - 1), group & 1);
  int held_from = begin, held_key, held_keys;
  int32_t held_page;
  uint64_t held_row;
  auto look = [&](int from) __attribute__((always_inline)) {
    const Requests requests(t, lane);  // (seldom wanted: not held meanwhile)
    const int u = min(from + lane, end - 1);
    int r = 0;
    for (int k = 1; k < t.nreq; ++k) r += u >= 2 * (int)requests.get(k).unit_start;
    auto of = [&](int low, int high) {
      const int a = __shfl(low, r & 63), b = __shfl(high, r & 63);
      return r >= 64 ? b : a;
    };
    const int start = of((int)requests.held[0].unit_start, (int)requests.held[1].unit_start);
    const int req = of(requests.held[0].req, requests.held[1].req);
    held_from = from;
    held_keys = of(requests.held[0].cached + requests.held[0].new_len, requests.held[1].cached + requests.held[1].new_len);
    held_key = (u - 2 * start) * kUnitKeys + group * kGroupKeys;
    held_page = block_table[(int64_t)req * t.max_pages + (min(held_key, held_keys - 1) >> t.page_shift)];
    __builtin_amdgcn_s_waitcnt(0x0F70);
    held_row = reinterpret_cast<uint64_t>(rows.row_at(held_page, held_key));
  };
  // Where unit u's group comes from; one that the request's end cuts off is gathered at once.
  struct Source {
    const char* base;
    bool whole;
  };
  auto source = [&](int u, uint32_t to) __attribute__((always_inline)) {
    Source from = {nullptr, false};
    if (u < end) {
      if (u - held_from >= 64) look(u);
      const int l = u - held_from, key = __builtin_amdgcn_readlane(held_key, l);
      rows.k1 = __builtin_amdgcn_readlane(held_keys, l);
      from.whole = rows.whole(key);
      const uint32_t low = __builtin_amdgcn_readlane((uint32_t)held_row, l), high = __builtin_amdgcn_readlane((uint32_t)(held_row >> 32), l);
      from.base = reinterpret_cast<const char*>((uint64_t)high << 32 | low) + first_piece * 1024;
      if (!from.whole && wave < 4) rows.group(key, group, __builtin_amdgcn_readlane(held_page, l), to);
    }
    return from;
  };
  // the wave's loads of a whole group: two, two and for the first waves one
  auto gather = [&](const char* base, int n, uint32_t to) __attribute__((always_inline)) {
    if (n < 4) load_to_lds_2x16(base + n * 1024, piece_at[n], piece_at[n < 4 ? n + 1 : n], to + (first_piece + n) * 1024);
    else if (wave < 4) load_to_lds_16(base + n * 1024, piece_at[n], to + (first_piece + n) * 1024);
  };
  // places of the units u, u + 1 and u + 2, in turn
  uint32_t now = lds0, next = lds0 + kStageBytes, later = lds0 + 2 * kStageBytes;
  look(begin);
#pragma unroll
  for (int ahead = 0; ahead < 2; ++ahead) {
    const uint32_t to = (ahead ? next : now) + group * kGroupBytes;
    const Source from = source(begin + ahead, to);
    if (from.whole) {
#pragma unroll
      for (int n = 0; n <= 4; n += 2) gather(from.base, n, to);
    }
  }

  // An operand's address, as the absorbed form's keys have it.
  uint32_t operand_at[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) operand_at[k] = i * kRowBytes + (((2 * k + part) ^ swizzle(i)) << 4);
  struct Addresses {
    uint32_t at[4];
  };
  auto addresses = [&](uint32_t from) __attribute__((always_inline)) {
    Addresses a;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      a.at[k] = from + operand_at[k];
      asm volatile("" : "+v"(a.at[k]));  // (the steps' offsets then go into the reads)
    }
    return a;
  };
  auto operand = [&](const Addresses& a, int s) __attribute__((always_inline)) {
    return *(const LDS_PTR(bf16x8))(uintptr_t)(a.at[s & 3] + (s >> 2) * 128);
  };
  // Outputs leave a lane's 16 bytes at a time: row lane / 4 of sixteen, chunk lane % 4 of the wave's, to its place in the tile.
  // The values' waves bring the rotated parts from a group of rows to the keys too.
  const uint32_t place = lds0 + kPlacesAt + wave * (kUnitKeys * kPlacePitch);
  const bool of_keys = wave < 4;
  const int row16 = lane >> 2, chunk4 = group * 4 + (lane & 3);
  const uint32_t out_at = of_keys ? row16 * kKeyBytes + ((chunk4 ^ key_swizzle(row16)) << 4)
                                  : kKeysBytes + row16 * kValueBytes + ((chunk4 ^ value_swizzle(row16)) << 4);
  // (the row sixteen further on has the same swizzle)
  const uint32_t store_at[2] = {out_at, out_at + 16u * (of_keys ? kKeyBytes : kValueBytes)};
  const int rope_row = group * kGroupKeys + (lane >> 3), rope_chunk = lane & 7;
  const uint32_t rope_from = rope_row * kRowBytes + kLatentBytes + ((rope_chunk ^ swizzle(rope_row)) << 4);
  const uint32_t rope_at = rope_row * kKeyBytes + ((16 + (rope_chunk ^ key_swizzle(rope_row))) << 4);
  char* const head_tiles = tiles + (int64_t)head * t.key_tiles * kTileBytes;
  auto tile_of = [&](int u) { return head_tiles + (int64_t)(u >> 1) * kTileBytes; };
  const int half_bytes = kUnitKeys * (of_keys ? kKeyBytes : kValueBytes);
  auto write_place = [&](u32x2 words, int r4) __attribute__((always_inline)) {
    *(LDS_PTR(u32x2))(uintptr_t)(place + i * kPlacePitch + (r4 * 8 + part * 4) * 2) = words;
  };
  auto read_place = [&](int k) __attribute__((always_inline)) {
    return *(const LDS_PTR(u32x4))(uintptr_t)(place + (k * 16 + row16) * kPlacePitch + (lane & 3) * 16);
  };
  auto store = [&](char* half, uint32_t at, u32x4 v) __attribute__((always_inline)) { *reinterpret_cast<u32x4*>(half + at) = v; };

  // Products of unit u; beside them the results of the one in front go out (in front of the first there is none: what
  // is written for it goes to the first one's place, which is written again) and unit u + 2 comes in.  Some products in front
  // of the end, with its last operand read, the waves meet: unit u + 1 is there, its first operands are read beside the rest, and
  // the place of u is free for u + 3.
  constexpr int kAhead = 8, kMeet = 26;
  bf16x8 staged[kAhead];
  Addresses here = addresses(now);
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
#pragma unroll
  for (int s = 0; s < kAhead; ++s) staged[s] = operand(here, s);
  u32x2 done[4] = {{0, 0}, {0, 0}, {0, 0}, {0, 0}};  // outputs of the unit in front
  for (int u = begin; u < end; ++u) {
    const uint32_t to = later + group * kGroupBytes;
    const Source source2 = source(u + 2, to);
    const int in_front = max(u - 1, begin);
    char* const front = tile_of(in_front) + (in_front & 1) * half_bytes;
    char* const ropes = tile_of(u) + (u & 1) * (kUnitKeys * kKeyBytes);
    const uint32_t rope = now + rope_from;
    const Addresses from = here;
    here = addresses(next);
    u32x4 leaving[3];
    f32x16 acc;
    __builtin_amdgcn_s_setprio(1);
    __builtin_amdgcn_sched_barrier(0);
    each<kSteps>([&](auto index) __attribute__((always_inline)) {
      constexpr int p = decltype(index)::value;
      if constexpr (p == 0) first_expand_product(acc, weight[0], staged[0]);
      else expand_product(acc, weight[p], staged[p % kAhead]);
      if constexpr (p + kAhead < kSteps) staged[p % kAhead] = operand(from, p + kAhead);
      if constexpr (p == 1 || p == 3 || p == 5) {
        if (source2.whole) gather(source2.base, p - 1, to);
      }
      if constexpr (p % 2 == 0 && p >= 4 && p <= 10) write_place(done[(p - 4) / 2], (p - 4) / 2);
      if constexpr (p == 12 || p == 13) leaving[p - 12] = read_place(p - 12);
      if constexpr (p == 14) {
        if (!of_keys) leaving[2] = *(const LDS_PTR(u32x4))(uintptr_t)rope;
      }
      if constexpr (p == 18 || p == 20) store(front, store_at[(p - 18) / 2], leaving[(p - 18) / 2]);
      if constexpr (p == 22) {
        if (!of_keys) store(ropes, rope_at, leaving[2]);
      }
      if constexpr (p == kMeet) {
        // (in flight may be the stores of the unit in front, at least two, the gather of unit u + 2 and the stores behind it, five
        // and two or four and three)
        if (u + 2 < end && source2.whole) asm volatile("s_waitcnt vmcnt(9)" ::: "memory");
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_setprio(0);
        __syncthreads();
        __builtin_amdgcn_s_setprio(1);
      }
      // the next unit's operand k takes the place of the one of step kSteps - kAhead + k
      if constexpr (p > kMeet && p <= kMeet + 3) {
        constexpr int k = 2 * (p - kMeet - 1);
        staged[k] = operand(here, k), staged[k + 1] = operand(here, k + 1);
      }
      if constexpr (p > kMeet + 3) staged[p - (kSteps - kAhead)] = operand(here, p - (kSteps - kAhead));
      __builtin_amdgcn_sched_barrier(0);
    });
    __builtin_amdgcn_s_setprio(0);
    asm volatile("s_nop 15" : "+v"(acc));  // (the last product's result may be read 12 states behind it)
#pragma unroll
    for (int r4 = 0; r4 < 4; ++r4)
      done[r4] = u32x2{pack_bf16(acc[4 * r4], acc[4 * r4 + 1]), pack_bf16(acc[4 * r4 + 2], acc[4 * r4 + 3])};
    const uint32_t place0 = now;
    now = next, next = later, later = place0;
  }
  static_assert(kSteps == 32 && kAhead == 8 && kMeet == 26, "as the places above are counted");
#pragma unroll
  for (int r4 = 0; r4 < 4; ++r4) write_place(done[r4], r4);
#pragma unroll
  for (int k = 0; k < 2; ++k) store(tile_of(end - 1) + ((end - 1) & 1) * half_bytes, store_at[k], read_place(k));
}

// --- attention -----------------------------------------------------------------------------------------------------------

struct ExpandedArgs {
  ExpandedTable table;
  float scale_log2;
};

// blockIdx.x: head (fastest: an XCD meets few heads, whose tiles its workgroups share) and tile of 128 query rows, the
// request's last rows, which see most keys, first.  A team of four waves, one on each SIMD, takes the rows, 32 each.  GROUPS 1: a
// workgroup is one team and a unit holds two workgroups, so that each computes through the other's meetings, first loads
// and last stores.  GROUPS 2: it is two teams, which divide the keys and join at the end.  Bound by the products and what has to
// be issued beside them (49 % of the cycles are products), at a clock that their power sets.  One workgroup of eight waves
// and 256 rows to a unit took 2 % more, four waves of 64 rows, whose operands serve two products, 15 % more.
//
// A wave works off its keys in halves of tiles, three at a time: while the scores of half n are turned into probabilities, the
// products form the scores of n + 1 and add the values of n - 1.  The waves meet in front of every round.  Keys are
// gathered three halves ahead and values, which are wanted two halves later, two.  No maximum is formed on the way: the
// reference is the row's maximum over the first half.  A half of which a lane's sixteen probabilities sum to 2^kSlack is looked at
// again, and the references of rows move whose maximum is beyond 2^kSlack.  Rows whose keys lie 4 to kSlack log2 units above the
// first half's are thus looked at in every half without moving: the prompts above 839 us level (both kernels), 930 where scores rise
// by 8 units every 1000 keys, 1001 where all behind the first 32 keys are higher by 6.
constexpr int kTeam = 4;                              // waves
constexpr int kHalfKeys = kKeysBytes / 2, kHalfValues = (kTileBytes - kKeysBytes) / 2;
constexpr int kKeyStages = 4, kValueStages = 3;       // halves in a team's LDS
constexpr int kValuesAt = kKeyStages * kHalfKeys;
constexpr int kTeamBytes = kValuesAt + kValueStages * kHalfValues;
static_assert(kExpandedRowTile == kTeam * 32 && kTeam * 32 * kKeyBytes == kValuesAt, "the queries are first gathered to the keys' place");
// The outputs leave through LDS too, in rows of 256 bytes and 16 more, so that sixteen rows' equal chunks take all banks.
constexpr int kOutPitch = kValueBytes + 16;
constexpr int kJoinPitch = 33;  // words: 32 outputs of a lane and one, so that the lanes' words take all banks
constexpr int kJoinWords = 2 * 64 * kJoinPitch + 2 * 64;
static_assert(32 * kOutPitch <= kHalfKeys && kTeam * kJoinWords * 4 <= kTeamBytes, "place for the outputs and a join");

template <int GROUPS>
__global__ __launch_bounds__(64 * kTeam * GROUPS, 2) void expanded_attention_kernel(const ExpandedArgs args,
                                                                                    const uint16_t* __restrict__ q,
                                                                                    const char* __restrict__ tiles,
                                                                                    uint16_t* __restrict__ out) {
  constexpr int kKeyLoads = kHalfKeys / 1024 / kTeam, kValueLoads = kHalfValues / 1024 / kTeam;  // a wave's, of a half
  constexpr int kZeros = GROUPS * kTeamBytes;  // what a key that is to be left out has for a value
  constexpr int kTornAt = kZeros + 1024;       // a word for each wave: whether it left a key out
  __shared__ __attribute__((aligned(1024))) char lds[kTornAt + 4 * kTeam * GROUPS];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int set = wave % kTeam, group = wave / kTeam;
  const uint32_t zeros = (uint32_t)(uintptr_t)(LDS_PTR(char))lds + kZeros;
  const uint32_t base = (uint32_t)(uintptr_t)(LDS_PTR(char))lds + group * kTeamBytes;
  *reinterpret_cast<u32x4*>(lds + kZeros + lane * 16) = u32x4{0, 0, 0, 0};  // (by every wave: it reads behind its own writes)
  const uint32_t torn = zeros + 1024;
  *(LDS_PTR(uint32_t))(uintptr_t)(torn + 4 * wave) = 0;
  const ExpandedTable& t = args.table;
  const int heads = t.heads;
  const int at = blockIdx.x / heads, head = blockIdx.x - at * heads;
  const Requests requests(t, lane);
  int start;
  const int r = requests.find_row_tile(t, at, lane, &start);
  const LatentReq rq = requests.get(r);
  const int row_tiles = (rq.new_len + kExpandedRowTile - 1) / kExpandedRowTile;
  const int row0 = (row_tiles - 1 - (at - start)) * kExpandedRowTile;
  const int rows = min(kExpandedRowTile, rq.new_len - row0);
  // halves that some row sees: the team's begin at `first`, `count` of them
  const int whole = (rq.cached + row0 + rows + 31) / 32, middle = (whole + 1) / 2;
  const int first = GROUPS == 1 || group == 0 ? 0 : middle;
  const int count = GROUPS == 1 ? whole : group == 0 ? middle : whole - middle;
  const int rounds = GROUPS == 1 ? whole : middle;  // of the longer team
  const char* src = tiles + ((int64_t)head * t.key_tiles + rq.unit_start) * kTileBytes;
  // (halves are counted from the team's first; one in front of it, or behind the last, stands for whatever lies in its place)
  auto keys_at = [&](int n) { return base + (uint32_t)(n & (kKeyStages - 1)) * kHalfKeys; };
  auto values_at = [&](int n) { return base + kValuesAt + (uint32_t)((n + kValueStages) % kValueStages) * kHalfValues; };
  auto tile_of = [&](int n) { return src + (int64_t)((first + n) >> 1) * kTileBytes; };
  auto fetch_keys = [&](int n) __attribute__((always_inline)) {
    const int piece = set * (kKeyLoads * 1024);
    load_to_lds_run<kKeyLoads>(tile_of(n) + ((first + n) & 1) * kHalfKeys + piece, (uint32_t)lane * 16, keys_at(n) + piece);
  };
  auto fetch_values = [&](int n) __attribute__((always_inline)) {
    const int piece = set * (kValueLoads * 1024);
    load_to_lds_run<kValueLoads>(tile_of(n) + kKeysBytes + ((first + n) & 1) * kHalfValues + piece, (uint32_t)lane * 16, values_at(n) + piece);
  };

  const int i = lane & 31, part = lane >> 5;
  const int64_t packed = (int64_t)rq.row_start + row0;  // the workgroup's first row
  // the values in front of the first half
#pragma unroll
  for (int n = 0; n < kHalfValues / (64 * kTeam * 16); ++n)
    *(LDS_PTR(u32x4))(uintptr_t)(values_at(-1) + (n * 64 * kTeam + set * 64 + lane) * 16) = u32x4{0, 0, 0, 0};
  constexpr int kSteps = kQueryRow / 16, kBlocks = kLatentValue / 32, kValueProducts = 2 * kBlocks;
  // The wave's queries, swizzled as keys are: eight rows are three loads.  Rows behind the last are copies of it.
  const uint32_t own_place = base + set * kHalfKeys;
  {
    const char* from = reinterpret_cast<const char*>(q + (packed * heads + head) * kQueryRow);
    const uint32_t pitch = (uint32_t)heads * kKeyBytes;
#pragma unroll
    for (int j = 0; j < 3; ++j) {
      const int n = j * 64 + lane, of8 = n / 24, chunk = n - of8 * 24;
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int row = g * 8 + of8;
        const int64_t off = (int64_t)(uint32_t)min(set * 32 + row, rows - 1) * pitch + ((chunk ^ key_swizzle(row)) << 4);
        load_to_lds_16(from + off, own_place + (g * 3 + j) * 1024);
      }
    }
  }
  if (0 < count) {
    fetch_values(0);
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kValueLoads) : "memory");
  } else {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  }
  uint32_t key_at[4], value_at[kBlocks];
#pragma unroll
  for (int s = 0; s < 4; ++s) key_at[s] = i * kKeyBytes + (((2 * s + part) ^ key_swizzle(i)) << 4);
  const int value_key = part * 4 + ((lane & 15) >> 2);  // and 8, 16, 24 further on
  {
    const int w16 = lane & 15, chunk = 2 * ((lane >> 4) & 1) + ((w16 & 3) >> 1);
#pragma unroll
    for (int d = 0; d < kBlocks; ++d)
      value_at[d] = value_key * kValueBytes + (((4 * d + chunk) ^ value_swizzle(value_key)) << 4) + (w16 & 1) * 8;
  }
  auto key_operand = [&](uint32_t ks, int n) __attribute__((always_inline)) {
    return *(const LDS_PTR(u32x4))(uintptr_t)(ks + key_at[n & 3] + (n >> 2) * 128);
  };
  bf16x8 qb[kSteps];
#pragma unroll
  for (int s = 0; s < kSteps; ++s) qb[s] = __builtin_bit_cast(bf16x8, key_operand(own_place, s));
  __syncthreads();
#pragma unroll
  for (int n = 0; n < kKeyStages; ++n)
    if (n < count) fetch_keys(n);
  if (kKeyStages <= count) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * kKeyLoads) : "memory");
  else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  const int visible = rq.cached + row0 + min(set * 32 + i, rows - 1) + 1;
  const int least = rq.cached + row0 + set * 32 + 1;  // of the wave's first row
  // of the team's halves those of which the wave's last row sees a part; none where the wave has no rows
  const int seen = set * 32 >= rows ? 0 : (rq.cached + row0 + min(set * 32 + 31, rows - 1) + 32) / 32;
  const int halves = max(0, min(seen - first, count));

  f32x16 o[kBlocks];
#pragma unroll
  for (int d = 0; d < kBlocks; ++d)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[d][e] = 0.f;
  float m_run = kNoReference, l_run = 0.f;
  f32x16 s0, s1;                                      // scores of an even and an odd half
  u32x4 p0[2], p1[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};  // and their probabilities, as operands
  uint32_t dropped = 0;  // keys of the half in front that count for nothing

  // Products of a round: the scores of the 32 keys at `ks` into `sn`, the values of the 32 keys at `vs` under the
  // probabilities `pv`; beside them the probabilities of the scores `sc` into `pn`, whose sum is returned.
  constexpr int kProducts = kSteps + kValueProducts, kAhead = 4;
  auto probability = [&](const f32x16& sc, int e) __attribute__((always_inline)) { return __builtin_amdgcn_exp2f(sc[e] * args.scale_log2 - m_run); };
  auto add_pair = [&](uint32_t two, float sum) __attribute__((always_inline)) {  // of two probabilities as they were rounded
    typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
    const bf16x2 ones = {(__bf16)1.0f, (__bf16)1.0f};
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, two), ones, sum, false);
  };
  auto score_product = [&](u32x4 a, int n, f32x16& sn) __attribute__((always_inline)) {
    f32x16 from = sn;
    if (n == 0) {
#pragma unroll
      for (int e = 0; e < 16; ++e) from[e] = 0.f;
    }
    sn = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), qb[n], from, 0, 0, 0);
  };
  auto round = [&](f32x16& sn, uint32_t ks, const u32x4 (&pv)[2], uint32_t vs, const f32x16& sc, u32x4 (&pn)[2], auto drops) __attribute__((always_inline)) -> float {
    u32x4 staged[kAhead];
    uint32_t va[4][kBlocks];
#pragma unroll
    for (int d = 0; d < kBlocks; ++d) {
      va[0][d] = vs + value_at[d];
      if constexpr (!decltype(drops)::value) asm volatile("" : "+v"(va[0][d]));  // (the other rows' offsets then go into the reads)
#pragma unroll
      for (int g = 1; g < 4; ++g) va[g][d] = va[0][d] + g * 8 * kValueBytes;
    }
    if (decltype(drops)::value && dropped) {
#pragma unroll
      for (int g = 0; g < 4; ++g)
#pragma unroll
        for (int d = 0; d < kBlocks; ++d)
          if (dropped >> (value_key + g * 8) & 1) va[g][d] = zeros;
    }
    auto operand = [&](int n) __attribute__((always_inline)) -> u32x4 {
      if (n < kSteps) return key_operand(ks, n);
      const int k = (n - kSteps) / kBlocks, d = (n - kSteps) % kBlocks;
      const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((LDS_PTR(bf16x4))(uintptr_t)(va[2 * k][d]));
      const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((LDS_PTR(bf16x4))(uintptr_t)(va[2 * k + 1][d]));
      return __builtin_bit_cast(u32x4, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    };
#pragma unroll
    for (int n = 0; n < kAhead; ++n) staged[n] = operand(n);
    // (a wave with operands goes in front of one that looks after meetings and gathers: 10 % fewer cycles)
    __builtin_amdgcn_s_setprio(1);
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
    __builtin_amdgcn_s_setprio(0);
    return sum;
  };
  auto row_max = [&](const f32x16& sc) __attribute__((always_inline)) {
    float mx = sc[0];
#pragma unroll
    for (int e = 1; e < 16; ++e) mx = fmaxf(mx, sc[e]);
    return cross_half_max(mx) * args.scale_log2;
  };
  // In front of round n: the keys of half n + 1 and the values of n - 1 are there, and the places of the keys of n and of the
  // values of n - 2 are free.
  auto meet = [&](int n) __attribute__((always_inline)) {
    // (in flight may be, in this order: keys n + 2, values n, keys n + 3)
    if (n + 3 < count) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * kKeyLoads + kValueLoads) : "memory");
    else if (n + 2 < count) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kKeyLoads + kValueLoads) : "memory");
    else if (n < count) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kValueLoads) : "memory");
    else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (n + 1 < count) fetch_values(n + 1);
    if (n + 4 < count) fetch_keys(n + 4);
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
  // A half that every row sees whole; each wave with rows has a further one behind it.
  auto seen_half = [&](int n, f32x16& sc, f32x16& sn, u32x4 (&pn)[2], u32x4 (&po)[2]) __attribute__((always_inline)) {
    if (halves == 0) return;
    if (n == 0) m_run = fmaxf(row_max(sc), kNoReference);
    settle(sc, pn, round(sn, keys_at(n + 1), po, values_at(n - 1), sc, pn, std::false_type()));
  };
  // The wave's n-th half: scores `sc`, probabilities to `pn`.  The round's products are those of its neighbours.  Behind the
  // last half there is a round for its values alone: what it does beside them is for nobody, as are the scores behind
  // the last half.
  auto half = [&](int n, f32x16& sc, f32x16& sn, u32x4 (&pn)[2], u32x4 (&po)[2]) __attribute__((always_inline)) {
    if (n > halves || halves == 0) return;
    const bool last = n == halves;
    const int key0 = (first + n) * 32;
    uint32_t unfit = 0;
    if (!last && key0 + 32 > least) {
      float raw[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) raw[e] = sc[e];
      unfit = unfit_keys<32>(raw);
      if (unfit) *(LDS_PTR(uint32_t))(uintptr_t)(torn + 4 * wave) = 1;
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (key0 + (e >> 2) * 8 + part * 4 + (e & 3) >= visible) sc[e] = -__builtin_inff();
    }
    if (n == 0) m_run = fmaxf(row_max(sc), kNoReference);
    const float sum = round(sn, keys_at(n + 1), po, values_at(n - 1), sc, pn, std::true_type());
    dropped = unfit;
    if (last) return;
    settle(sc, pn, sum);
  };
  if (halves > 0) {
#pragma unroll
    for (int n = 0; n < kSteps; ++n) score_product(key_operand(keys_at(0), n), n, s0);
  }
  // First the halves in front of the workgroup's first row, in pairs, without masks and what they bring with them: a prompt of 2355
  // tokens and 16 heads 73.5 -> 69 us.  (Both kinds of round in one loop make the compiler spill.)
  const int clear = max(0, min((rq.cached + row0 + 1) / 32 - first, count)) & ~1;
  int n = 0;
  for (; n < clear; n += 2) {
    meet(n);
    seen_half(n, s0, s1, p0, p1);
    meet(n + 1);
    seen_half(n + 1, s1, s0, p1, p0);
  }
  for (; n <= rounds; n += 2) {
    meet(n);
    half(n, s0, s1, p0, p1);
    meet(n + 1);
    half(n + 1, s1, s0, p1, p0);
  }
  __syncthreads();  // the tiles' place is free
  l_run = cross_half_sum(l_run);
  float own = 1.f / l_run, other = 0.f;
  // Two teams: the second one leaves its outputs, references and sums, the first one adds them.
  float* const left = reinterpret_cast<float*>(lds + kTeamBytes) + set * kJoinWords;
  float* const stats = left + 2 * 64 * kJoinPitch;
  auto place = [&](int d, int e) { return ((d >> 1) * 64 + lane) * kJoinPitch + (d & 1) * 16 + e; };
  if constexpr (GROUPS == 2) {
    if (group == 1) {
#pragma unroll
      for (int d = 0; d < kBlocks; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e) left[place(d, e)] = o[d][e];
      stats[lane] = m_run;
      stats[64 + lane] = l_run;
    }
    __syncthreads();
    if (group == 1) return;
    const float m_other = stats[lane], l_other = stats[64 + lane], m = fmaxf(m_run, m_other);
    own = __builtin_amdgcn_exp2f(m_run - m), other = __builtin_amdgcn_exp2f(m_other - m);
    const float inv = 1.f / (l_run * own + l_other * other);
    own *= inv, other *= inv;
  }
  // out through LDS, sixteen lanes to a row
  char* const staged = lds + set * kHalfKeys;
#pragma unroll
  for (int d = 0; d < kBlocks; ++d)
#pragma unroll
    for (int e4 = 0; e4 < 4; ++e4) {
      float v[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        v[k] = o[d][4 * e4 + k] * own;
        if constexpr (GROUPS == 2) v[k] = __builtin_fmaf(left[place(d, 4 * e4 + k)], other, v[k]);
      }
      *reinterpret_cast<u32x2*>(staged + i * kOutPitch + (d * 32 + e4 * 8 + part * 4) * 2) = u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
    }
  // torn columns
  uint32_t some = *(LDS_PTR(uint32_t))(uintptr_t)(torn + 4 * set);
  if constexpr (GROUPS == 2) some |= *(LDS_PTR(uint32_t))(uintptr_t)(torn + 4 * (kTeam + set));
  if (__builtin_expect(__builtin_amdgcn_readfirstlane(some) != 0, 0)) {
    const int chunk = lane & 15;
    u32x4 marks = {0, 0, 0, 0};
    int key = least & -32;  // (the halves that were masked)
#pragma unroll 1
    for (int row = lane >> 4; row < 32; row += 4) {
      const int end = rq.cached + row0 + min(set * 32 + row, rows - 1) + 1;
      for (; key < end; ++key) {
        const char* const value = src + (int64_t)(key / kTileKeys) * kTileBytes + kKeysBytes + (key % kTileKeys) * kValueBytes;
        marks |= torn_marks(*reinterpret_cast<const u32x4*>(value + ((chunk ^ value_swizzle(key)) << 4)));
      }
      *reinterpret_cast<u32x4*>(staged + row * kOutPitch + chunk * 16) |= marks;
    }
  }
  uint16_t* dst = out + ((packed + set * 32) * heads + head) * kLatentValue;
#pragma unroll
  for (int row4 = 0; row4 < 32; row4 += 4) {
    const int row = row4 + (lane >> 4);
    if (set * 32 + row < rows)
      *reinterpret_cast<u32x4*>(dst + (int64_t)row * heads * kLatentValue + (lane & 15) * 8) =
          *reinterpret_cast<const u32x4*>(staged + row * kOutPitch + (lane & 15) * 16);
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
    expand_kernel<<<(unsigned)args.table.slices * heads, 64 * kExpandWaves, 0, stream>>>(
        args.table, static_cast<const uint16_t*>(cache), static_cast<const uint16_t*>(w_kv), b->block_table, tiles);
    const unsigned groups = (unsigned)args.table.row_tiles * heads;
    if (plan.teams == 1)
      expanded_attention_kernel<1><<<groups, 64 * kTeam, 0, stream>>>(args, static_cast<const uint16_t*>(q), tiles, static_cast<uint16_t*>(out));
    else
      expanded_attention_kernel<2><<<groups, 128 * kTeam, 0, stream>>>(args, static_cast<const uint16_t*>(q), tiles, static_cast<uint16_t*>(out));
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
