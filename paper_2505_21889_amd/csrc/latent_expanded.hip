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
constexpr float kSlack = 8.f;
constexpr float kNoReference = -3.0e38f;

// Swizzles of a tile row's 16-byte chunks.  Keys: 24 chunks, so neighbouring rows start half of the 256-byte bank line
// apart; the three bits spread sixteen rows' equal chunks over its sixteen places.  Values: 16 chunks, the two bits spread
// the four chunks that a transposing read takes of each of eight rows.
__device__ __forceinline__ int key_swizzle(int row) { return (row >> 1) & 7; }
__device__ __forceinline__ int value_swizzle(int row) { return (row & 3) << 2; }

// An operand of the value product without the keys named in `unfit`, by the bits of its elements 0..3 and 8 on.
__device__ __forceinline__ bf16x8 without_keys(bf16x8 x, uint32_t unfit) {
  u32x4 w = __builtin_bit_cast(u32x4, x);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t two = unfit >> (j < 2 ? 2 * j : 2 * j + 4);
    w[j] &= (two & 1 ? 0u : 0xFFFFu) | (two & 2 ? 0u : 0xFFFF0000u);
  }
  return __builtin_bit_cast(bf16x8, w);
}

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
constexpr int kDepth = 64;              // elements of the latent staged at a time
constexpr int kStageBytes = (kTokens + kHeadOut) * kDepth * 2;
constexpr int kExpandWaves = 8;

// blockIdx.x: head (fastest, so that an XCD meets few heads' weights) and pair of tiles.  A wave forms 64 tokens x 64
// outputs as W C^T: a lane's results are four neighbouring outputs of one token.
__global__ __launch_bounds__(64 * kExpandWaves, 2) void expand_kernel(const ExpandedTable t, const uint16_t* __restrict__ cache,
                                                                      const uint16_t* __restrict__ w_kv,
                                                                      const int32_t* __restrict__ block_table,
                                                                      char* __restrict__ tiles) {
  __shared__ __attribute__((aligned(1024))) char lds[2 * kStageBytes];
  static_assert(2 * kStageBytes >= 2 * kTileBytes, "the finished tiles take the stages' place");
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

  // 1 KB loads of eight rows by 128 bytes: 16 of tokens, 32 of weight rows; lane l fetches row l / 8, its chunk l % 8
  // swizzled.  Tokens behind the request's last are copies of it (their scores are masked).
  constexpr int kTokenLoads = kTokens / 8, kLoads = kTokenLoads + kHeadOut / 8, kPerWave = kLoads / kExpandWaves;
  static_assert(kTokenLoads == 2 * kExpandWaves && kPerWave == 6, "two loads of tokens, four of the weight a wave");
  const char* src[kPerWave];
#pragma unroll
  for (int j = 0; j < kPerWave; ++j) {
    const int row = (j < 2 ? wave * 2 + j : wave * 4 + j - 2) * 8 + (lane >> 3);
    const int chunk = (lane & 7) ^ key_swizzle(row);
    if (j < 2) {
      const int key = min(key0 + row, keys - 1);
      const int64_t page = pages[key >> page_shift];
      src[j] = reinterpret_cast<const char*>(cache) + ((page << page_shift) + (key & page_mask)) * (kLatentRow * 2) + chunk * 16;
    } else {
      src[j] = w + (int64_t)row * (kLatentRank * 2) + chunk * 16;
    }
  }
  auto fetch = [&](int step) {
    const uint32_t to = lds0 + (step & 1) * kStageBytes;
#pragma unroll
    for (int j = 0; j < kPerWave; ++j)
      load_to_lds_16(src[j] + step * (kDepth * 2), to + (j < 2 ? wave * 2 + j : kTokenLoads + wave * 4 + j - 2) * 1024);
  };
  fetch(0);

  const int i = lane & 31, part = lane >> 5;
  const int token_half = wave & 1, out_quarter = wave >> 1;
  f32x16 acc[2][2];  // [token block][output block]
#pragma unroll
  for (int a = 0; a < 2; ++a)
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[a][b][r] = 0.f;
  uint32_t at[4];  // of an operand's step in a row of 128 bytes
#pragma unroll
  for (int s = 0; s < 4; ++s) at[s] = i * (kDepth * 2) + (((2 * s + part) ^ key_swizzle(i)) << 4);
  constexpr int kStepCount = kLatentRank / kDepth;
  for (int step = 0; step < kStepCount; ++step) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (step + 1 < kStepCount) fetch(step + 1);
    const uint32_t tok = lds0 + (step & 1) * kStageBytes + token_half * 64 * (kDepth * 2);
    const uint32_t wgt = lds0 + (step & 1) * kStageBytes + kTokens * (kDepth * 2) + out_quarter * 64 * (kDepth * 2);
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      bf16x8 x[2], y[2];
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        x[b] = *(const LDS_PTR(bf16x8))(uintptr_t)(tok + at[s] + b * 32 * (kDepth * 2));
        y[b] = *(const LDS_PTR(bf16x8))(uintptr_t)(wgt + at[s] + b * 32 * (kDepth * 2));
      }
#pragma unroll
      for (int a = 0; a < 2; ++a)
#pragma unroll
        for (int b = 0; b < 2; ++b) acc[a][b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(y[b], x[a], acc[a][b], 0, 0, 0);
    }
  }
  __syncthreads();
  // the tiles as the attention takes them, in LDS, then out in whole lines
#pragma unroll
  for (int a = 0; a < 2; ++a)
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4) {
        const int row = a * 32 + i;  // of tile `token_half`
        const int col = out_quarter * 64 + b * 32 + r4 * 8 + part * 4;
        const u32x2 v = {pack_bf16(acc[a][b][4 * r4], acc[a][b][4 * r4 + 1]), pack_bf16(acc[a][b][4 * r4 + 2], acc[a][b][4 * r4 + 3])};
        char* tile = lds + token_half * kTileBytes;
        char* to = col < kLatentNope ? tile + row * kKeyBytes + (((col >> 3) ^ key_swizzle(row)) << 4)
                                     : tile + kKeysBytes + row * kValueBytes + ((((col - kLatentNope) >> 3) ^ value_swizzle(row)) << 4);
        *reinterpret_cast<u32x2*>(to + (col & 4) * 2) = v;
      }
  // rotated part of the keys: 8 chunks a token, of the cache
#pragma unroll
  for (int j = 0; j < kTokens * 8 / (64 * kExpandWaves); ++j) {
    const int n = j * 64 * kExpandWaves + tid, token = n >> 3, chunk = n & 7;
    const int key = min(key0 + token, keys - 1);
    const int64_t page = pages[key >> page_shift];
    const u32x4 v = *reinterpret_cast<const u32x4*>(cache + ((page << page_shift) + (key & page_mask)) * kLatentRow + kLatentRank + chunk * 8);
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

// blockIdx.x: head (fastest: an XCD meets few heads, whose tiles its workgroups share) and tile of 32 * WAVES query rows,
// the request's last rows, which see most keys, first.
template <int WAVES>
__global__ __launch_bounds__(64 * WAVES, 2) void expanded_attention_kernel(const ExpandedArgs args,
                                                                           const uint16_t* __restrict__ q,
                                                                           const char* __restrict__ tiles,
                                                                           uint16_t* __restrict__ out) {
  constexpr int TILE = 32 * WAVES;
  constexpr int kStages = WAVES == 8 ? 3 : 2;
  constexpr int kLoads = kTileBytes / 1024 / WAVES;  // a wave's, of a tile
  __shared__ __attribute__((aligned(1024))) char lds[kStages * kTileBytes];
  const uint32_t lds0 = (uint32_t)(uintptr_t)(LDS_PTR(char))lds;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
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
  const char* src = tiles + ((int64_t)head * t.key_tiles + rq.unit_start) * kTileBytes + wave * (kLoads * 1024);
  auto fetch = [&](int tile) __attribute__((always_inline)) {
    const char* from = src + (int64_t)tile * kTileBytes;
    const uint32_t to = lds0 + (tile % kStages) * kTileBytes + wave * (kLoads * 1024);
#pragma unroll
    for (int j = 0; j < kLoads; ++j) load_to_lds_16(from + j * 1024, (uint32_t)lane * 16, to + j * 1024);
  };
#pragma unroll
  for (int a = 0; a < kStages - 1; ++a)
    if (a < ntiles) fetch(a);

  const int i = lane & 31, part = lane >> 5;
  const int row = min(wave * 32 + i, rows - 1);
  const int64_t packed = (int64_t)rq.row_start + row0 + row;
  constexpr int kSteps = kQueryRow / 16, kBlocks = kLatentValue / 32;
  bf16x8 qb[kSteps];
#pragma unroll
  for (int s = 0; s < kSteps; ++s)
    qb[s] = *reinterpret_cast<const bf16x8*>(q + (packed * heads + head) * kQueryRow + s * 16 + part * 8);
  const int visible = rq.cached + row0 + row + 1;
  const int least = rq.cached + row0 + min(wave * 32, rows - 1) + 1;

  uint32_t key_at[4], value_at[kBlocks];
#pragma unroll
  for (int s = 0; s < 4; ++s) key_at[s] = i * kKeyBytes + (((2 * s + part) ^ key_swizzle(i)) << 4);
  {
    const int w16 = lane & 15, blk = lane >> 4;
    const int key = (blk >> 1) * 4 + (w16 >> 2), chunk = 2 * (blk & 1) + ((w16 & 3) >> 1);
#pragma unroll
    for (int d = 0; d < kBlocks; ++d)
      value_at[d] = kKeysBytes + key * kValueBytes + (((4 * d + chunk) ^ value_swizzle(key)) << 4) + (w16 & 1) * 8;
  }
  f32x16 o[kBlocks];
#pragma unroll
  for (int d = 0; d < kBlocks; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[d][r] = 0.f;
  float m_run = kNoReference, l_run = 0.f;

  auto work_off = [&](int tile, auto masked) __attribute__((always_inline)) {
    constexpr bool kMasked = decltype(masked)::value;
    if (kStages == 3 && tile + 1 < ntiles) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kLoads) : "memory");
    else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (tile + kStages - 1 < ntiles) fetch(tile + kStages - 1);
    const uint32_t buf = lds0 + (tile % kStages) * kTileBytes;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int key0 = tile * kTileKeys + half * 32;
      f32x16 sc;
#pragma unroll
      for (int r = 0; r < 16; ++r) sc[r] = 0.f;
#pragma unroll
      for (int s = 0; s < kSteps; ++s)
        sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
            *(const LDS_PTR(bf16x8))(uintptr_t)(buf + key_at[s & 3] + (s >> 2) * 128 + half * 32 * kKeyBytes), qb[s], sc, 0, 0, 0);
      uint32_t unfit = 0;
      if constexpr (kMasked) {
        float raw[16];
#pragma unroll
        for (int r = 0; r < 16; ++r) raw[r] = sc[r];
        unfit = unfit_keys<32>(raw);
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (key0 + (r >> 2) * 8 + part * 4 + (r & 3) >= visible) sc[r] = -__builtin_inff();
      }
      float mx = sc[0];
#pragma unroll
      for (int r = 1; r < 16; ++r) mx = fmaxf(mx, sc[r]);
      mx = cross_half_max(mx) * args.scale_log2;
      if (__any(mx > m_run + kSlack)) {
        const float m_new = mx > m_run + kSlack ? mx : m_run;
        const float f = m_new == m_run ? 1.f : __builtin_amdgcn_exp2f(m_run - m_new);
        l_run *= f;
#pragma unroll
        for (int d = 0; d < kBlocks; ++d)
#pragma unroll
          for (int r = 0; r < 16; ++r) o[d][r] *= f;
        m_run = m_new;
      }
      u32x4 pb[2];
#pragma unroll
      for (int r = 0; r < 16; r += 2) {
        const uint32_t two = pack_bf16(__builtin_amdgcn_exp2f(sc[r] * args.scale_log2 - m_run),
                                       __builtin_amdgcn_exp2f(sc[r + 1] * args.scale_log2 - m_run));
        pb[r >> 3][(r & 7) >> 1] = two;
        l_run += __uint_as_float(two << 16) + __uint_as_float(two & 0xFFFF0000u);
      }
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int d = 0; d < kBlocks; ++d) {
          const uint32_t v = buf + value_at[d] + (half * 32 + k * 16) * kValueBytes;
          const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((LDS_PTR(bf16x4))(uintptr_t)(v));
          const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((LDS_PTR(bf16x4))(uintptr_t)(v + 8 * kValueBytes));
          bf16x8 a = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
          if constexpr (kMasked)
            if (unfit) a = without_keys(a, unfit >> (16 * k + 4 * part));
          o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, __builtin_bit_cast(bf16x8, pb[k]), o[d], 0, 0, 0);
        }
    }
  };
  // Tiles that all rows of the wave see, then those that some see a part of.
  const int plain = min(ntiles, least / kTileKeys);
  for (int tile = 0; tile < plain; ++tile) work_off(tile, std::false_type{});
  for (int tile = plain; tile < ntiles; ++tile) work_off(tile, std::true_type{});
  const float inv = 1.f / cross_half_sum(l_run);
  if (wave * 32 + i >= rows) return;
  uint16_t* dst = out + (packed * heads + head) * kLatentValue;
#pragma unroll
  for (int d = 0; d < kBlocks; ++d)
#pragma unroll
    for (int r4 = 0; r4 < 4; ++r4) {
      const u32x2 v = {pack_bf16(o[d][4 * r4] * inv, o[d][4 * r4 + 1] * inv), pack_bf16(o[d][4 * r4 + 2] * inv, o[d][4 * r4 + 3] * inv)};
      *reinterpret_cast<u32x2*>(dst + d * 32 + r4 * 8 + part * 4) = v;
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
      expanded_attention_kernel<4><<<(unsigned)args.table.row_tiles * heads, 256, 0, stream>>>(args, static_cast<const uint16_t*>(q), tiles,
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
