// efim_latent_append: the new tokens' latent vectors normed, the rotary part of keys and queries rotated at the tokens'
// positions, latent and rotated key written as one row of the paged latent cache.
//   row = [ c * (mean(c^2) + eps)^(-1/2) * w | rot(k_r) ],  q_r -> rot(q_r), each rounded once to bf16
// Streaming kernel, bound by HBM bandwidth: 4 * 576 + 256 * Hq bytes per token, 795 MB in 170 to 177 us = 4.6 TB/s read and written (a copy's
// rate); two tokens 3.7 us.  Squares, norm and rotation are fp32, the angle fp64.
#include <type_traits>

#include "append_table.h"
#include "efim_internal.h"
#include "rope_math.h"

namespace efim {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

template <int MAXREQ>
struct LatentAppendArgs {
  AppendTable<MAXREQ> table;
  int32_t num_q_heads;  // 0 where there are no queries
  float eps;
  int64_t q_stride;     // elements between the query rows of neighbouring heads; a token has Hq of them
  int64_t q_out_stride;
  int64_t kv_stride;    // elements between the rows of neighbouring tokens
  double inv_freq[kLatentRope / 2];
};

constexpr int kUnits = kLatentRope / 16;          // lanes of a rotated row, two chunks of 16 bytes each
constexpr int kRowsPerPass = 64 / kUnits;
constexpr int kRowsPerWave = 2 * kRowsPerPass;
static_assert(kLatentRank == 64 * 8, "a lane holds eight elements of the latent");

// A wave takes one token: of blockIdx.y 0 its latent (a 16-byte chunk per lane), of the others 32 of its rotated rows, the
// queries' and behind them the key's.
template <bool INTERLEAVED, int MAXREQ>
__global__ __launch_bounds__(kAppendThreads) void latent_append_kernel(
    const LatentAppendArgs<MAXREQ> args, const uint16_t* q, uint16_t* q_out, const uint16_t* __restrict__ kv_new,
    const uint16_t* __restrict__ weight, uint16_t* __restrict__ cache, const int32_t* __restrict__ block_table) {
  __shared__ __attribute__((aligned(16))) float s_cs[kAppendThreads / 64][2][kLatentRope / 2];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int tok = blockIdx.x * (kAppendThreads / 64) + wave;
  if (tok >= args.table.tokens) return;
  const int64_t row = args.table.row_start[0] + tok;
  TableLanes<MAXREQ> lanes;
  lanes.load(args.table, lane);
  const uint16_t* kv = kv_new + row * args.kv_stride;
  const int page_shift = args.table.page_shift;
  auto place = [&](int* pos) {  // the token's row in the cache
    int req;
    lanes.find(args.table, lane, (int)row, &req, pos);
    const int32_t page = block_table[(int64_t)(args.table.req_base + req) * args.table.max_pages + (*pos >> page_shift)];
    return cache + (((int64_t)page << page_shift) + (*pos & ((1 << page_shift) - 1))) * kLatentRow;
  };

  if (blockIdx.y == 0) {
    const u32x4 raw = *reinterpret_cast<const u32x4*>(kv + lane * 8);
    u32x4 wraw = {0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u};  // ones
    if (weight) wraw = *reinterpret_cast<const u32x4*>(weight + lane * 8);
    int pos;
    uint16_t* dst = place(&pos);
    float x[8], w[8];
    widen(raw, x);
    widen(wraw, w);
    float sum = 0.f;
#pragma unroll
    for (int t = 0; t < 8; ++t) sum += x[t] * x[t];
    sum = group_sum<64>(sum);
    const float r = 1.0f / sqrtf(sum * (1.0f / kLatentRank) + args.eps);
#pragma unroll
    for (int t = 0; t < 8; ++t) x[t] = x[t] * r * w[t];
    *reinterpret_cast<u32x4*>(dst + lane * 8) = narrow(x);
    return;
  }

  const double freq = args.inv_freq[lane % (kLatentRope / 2)];
  const int hq = args.num_q_heads;
  const int cp = lane % kUnits;
  const int e0 = INTERLEAVED ? cp * 16 : cp * 8, e1 = INTERLEAVED ? cp * 16 + 8 : cp * 8 + kLatentRope / 2;
  const int hr0 = (blockIdx.y - 1) * kRowsPerWave + lane / kUnits;
  u32x4 a[2], b[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int hr = min(hr0 + i * kRowsPerPass, hq);
    const uint16_t* src = hr < hq ? q + (row * hq + hr) * args.q_stride : kv + kLatentRank;
    a[i] = *reinterpret_cast<const u32x4*>(src + e0);
    b[i] = *reinterpret_cast<const u32x4*>(src + e1);
  }
  int pos;
  uint16_t* key = place(&pos) + kLatentRank;
  if (lane < kLatentRope / 2) {
    double s, c;
    sincos((double)pos * freq, &s, &c);
    s_cs[wave][0][lane] = (float)c;
    s_cs[wave][1][lane] = (float)s;
  }
  // (one wave writes and reads: its LDS accesses are in order, the compiler is told by the fence)
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  float cs[8], sn[8];
#pragma unroll
  for (int t = 0; t < 8; ++t) {
    cs[t] = s_cs[wave][0][cp * 8 + t];
    sn[t] = s_cs[wave][1][cp * 8 + t];
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int hr = hr0 + i * kRowsPerPass;
    if (hr > hq) continue;
    float x[8], y[8];
    widen(a[i], x);
    widen(b[i], y);
    if constexpr (INTERLEAVED) rotate_interleaved_f32(x, y, cs, sn);
    else rotate_pairs_f32(x, y, cs, sn);
    uint16_t* dst = hr < hq ? q_out + (row * hq + hr) * args.q_out_stride : key;
    *reinterpret_cast<u32x4*>(dst + e0) = narrow(x);
    *reinterpret_cast<u32x4*>(dst + e1) = narrow(y);
  }
}

struct LatentTensors {
  const uint16_t *q, *kv_new, *weight;
  uint16_t *q_out, *cache;
  int64_t q_stride, q_out_stride, kv_stride;
};

template <int MAXREQ>
int launch_with(const efim_batch_t* b, const LatentTensors& t, float eps, const double* inv_freq, int interleaved,
                hipStream_t stream) {
  LatentAppendArgs<MAXREQ> args;
  for (int j = 0; j < kLatentRope / 2; ++j) args.inv_freq[j] = inv_freq[j];
  args.num_q_heads = t.q ? b->num_q_heads : 0;
  args.eps = eps;
  args.q_stride = t.q_stride;
  args.q_out_stride = t.q_out_stride;
  args.kv_stride = t.kv_stride;
  int64_t row = 0;
  for (int r0 = 0; r0 < b->batch;) {
    r0 = fill_table(b, r0, &row, &args.table);
    if (args.table.tokens == 0) continue;
    constexpr int kTokens = kAppendThreads / 64;
    const dim3 grid((unsigned)((args.table.tokens + kTokens - 1) / kTokens), 1 + args.num_q_heads / kRowsPerWave + 1);
    if (interleaved)
      latent_append_kernel<true, MAXREQ><<<grid, kAppendThreads, 0, stream>>>(args, t.q, t.q_out, t.kv_new, t.weight, t.cache, b->block_table);
    else
      latent_append_kernel<false, MAXREQ><<<grid, kAppendThreads, 0, stream>>>(args, t.q, t.q_out, t.kv_new, t.weight, t.cache, b->block_table);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) { set_last_hip_error(e); return EFIM_ERR_LAUNCH; }
  }
  return EFIM_OK;
}

// Rows of 16-byte chunks: a stride is a multiple of eight elements and no row runs into the next.
bool stride_ok(int64_t stride, int width) { return stride >= width && stride % 8 == 0 && stride <= (int64_t)1 << 31; }

}  // namespace
}  // namespace efim

extern "C" int efim_latent_append(const efim_batch_t* batch, const void* q_rope, int64_t q_stride, void* q_out,
                                  int64_t q_out_stride, const void* kv_new, int64_t kv_stride, const void* norm_weight,
                                  float norm_eps, void* latent_cache, const double* inv_freq, int rope_interleaved,
                                  void* stream) {
  using namespace efim;
  int64_t total = 0;
  const int rc = validate_latent_batch(batch, &total);
  if (rc != EFIM_OK) return rc;
  if (!(norm_eps >= 0.f) || norm_eps - norm_eps != 0.f || (rope_interleaved != 0 && rope_interleaved != 1) ||
      !frequencies_ok(inv_freq, kLatentRope))
    return EFIM_ERR_INVALID_ARG;
  if (!stride_ok(kv_stride, kLatentRow)) return EFIM_ERR_INVALID_ARG;
  if (!q_rope != !q_out) return EFIM_ERR_INVALID_ARG;
  if (q_rope && (!stride_ok(q_stride, kLatentRope) || !stride_ok(q_out_stride, kLatentRope) ||
                 (q_rope == q_out && q_stride != q_out_stride)))
    return EFIM_ERR_INVALID_ARG;
  if (total >= kMaxAppendTokens) return EFIM_ERR_UNSUPPORTED;
  if (total == 0) return EFIM_OK;
  if (!kv_new || !latent_cache) return EFIM_ERR_INVALID_ARG;
  for (const void* p : {q_rope, (const void*)q_out, kv_new, norm_weight, (const void*)latent_cache})
    if (!aligned16(p)) return EFIM_ERR_INVALID_ARG;
  if (!aligned4(batch->block_table)) return EFIM_ERR_INVALID_ARG;
  const LatentTensors t{static_cast<const uint16_t*>(q_rope), static_cast<const uint16_t*>(kv_new),
                        static_cast<const uint16_t*>(norm_weight), static_cast<uint16_t*>(q_out),
                        static_cast<uint16_t*>(latent_cache), q_stride, q_out_stride, kv_stride};
  auto* launch = batch->batch <= 64 ? launch_with<64> : launch_with<kMaxReqPerAppend>;
  return launch(batch, t, norm_eps, inv_freq, rope_interleaved, static_cast<hipStream_t>(stream));
}
