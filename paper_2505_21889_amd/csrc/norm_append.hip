// efim_norm_rope_append: root-mean-square norm of every query and key head row, rotary embedding at the tokens' positions
// and append of keys and values to the paged cache, in one pass over the new tokens' rows.
//   y = x * (mean(x^2) + eps)^(-1/2) * w,  rotated, rounded once to bf16
// Streaming kernel, bound by HBM bandwidth: 2 * (2 Hq + 4 Hkv) * D bytes per token.  80k tokens of 32/8 heads 353 us = 5.6 TB/s
// read and written; three tokens 4.6 us, one latency behind the other.
//
// Squares, their sum, the norm and the rotation are fp32; the angle is fp64, since a position in the ten thousands
// leaves an fp32 angle three decimal digits behind the point.
#include <type_traits>

#include "append_table.h"
#include "efim_internal.h"
#include "fp8_math.h"
#include "rope_math.h"

namespace efim {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

template <int MAXREQ>
struct NormArgs {
  AppendTable<MAXREQ> table;
  int32_t tok_shift;              // log2 of the tokens of a workgroup
  int32_t parts;                  // waves per token in a workgroup
  int32_t num_q_heads;            // 0 where there are no queries
  int32_t num_kv_heads;
  int32_t rotary_dim;             // leading elements of a head row that are rotated
  float eps;
  double inv_freq[64];            // rotation frequency of pair j (rotary_dim/2 entries)
  double k_inv;                   // 8-bit caches: 1 / scale (code = value / scale)
  double v_inv;
};

// A wave takes one token and kAppendPasses passes of 64 / (D / 16) head rows of it.  A lane holds two chunks of 16 bytes
// of a row, so that D / 16 neighbouring lanes hold a row and its sum of squares is formed by lane exchanges alone;
// inside the rotated part the two chunks are each other's partners (rotate-half: rotary_dim / 2 elements apart).  As in
// the append that only rotates, all loads that need no answer of another go out first.
template <int D, bool INTERLEAVED, bool KV8, int MAXREQ>
__global__ __launch_bounds__(kAppendThreads) void norm_append_kernel(
    const NormArgs<MAXREQ> args, const uint16_t* q, uint16_t* q_out, const uint16_t* __restrict__ k_new,
    const uint16_t* __restrict__ v_new, const uint16_t* __restrict__ q_weight, const uint16_t* __restrict__ k_weight,
    void* __restrict__ k_cache_raw, void* __restrict__ v_cache_raw, const int32_t* __restrict__ block_table) {
  constexpr int HALF = D / 2;
  constexpr int UNITS_PER_ROW = D / 16;
  constexpr int ROWS_PER_PASS = 64 / UNITS_PER_ROW;
  __shared__ __attribute__((aligned(16))) float s_cs[kAppendThreads / 64][2][HALF];  // cosines and sines of the wave's token

  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int tok = (blockIdx.x << args.tok_shift) + (wave & ((1 << args.tok_shift) - 1));
  if (tok >= args.table.tokens) return;
  const int part = blockIdx.y * args.parts + (wave >> args.tok_shift);
  const int row = args.table.row_start[0] + tok;
  const int rot_half = args.rotary_dim / 2;

  TableLanes<MAXREQ> lanes;
  lanes.load(args.table, lane);
  const double freq = args.inv_freq[lane % HALF];

  const int hq = args.num_q_heads, hkv = args.num_kv_heads;
  const int rows_per_tok = hq + 2 * hkv;
  const int cp = lane % UNITS_PER_ROW;
  const bool in_rotary = cp * 16 < args.rotary_dim;
  const bool apart = !INTERLEAVED && in_rotary;
  const int e0 = apart ? cp * 8 : cp * 16, e1 = apart ? cp * 8 + rot_half : cp * 16 + 8;
  const int hr0 = part * (kAppendPasses * ROWS_PER_PASS) + lane / UNITS_PER_ROW;
  u32x4 a[kAppendPasses], b[kAppendPasses], wa[kAppendPasses], wb[kAppendPasses];
#pragma unroll
  for (int i = 0; i < kAppendPasses; ++i) {
    // (0..Hq-1: q heads, then Hkv k heads, then Hkv v heads)
    const int hr = min(hr0 + i * ROWS_PER_PASS, rows_per_tok - 1);
    const uint16_t* src = k_new + ((int64_t)row * hkv + (hr - hq)) * D;
    if (hr < hq) src = q + ((int64_t)row * hq + hr) * D;
    if (hr >= hq + hkv) src = v_new + ((int64_t)row * hkv + (hr - hq - hkv)) * D;
    a[i] = *reinterpret_cast<const u32x4*>(src + e0);
    b[i] = *reinterpret_cast<const u32x4*>(src + e1);
    const uint16_t* w = hr < hq ? q_weight : k_weight;
    wa[i] = wb[i] = u32x4{0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u};  // ones
    if (w) {
      wa[i] = *reinterpret_cast<const u32x4*>(w + e0);
      wb[i] = *reinterpret_cast<const u32x4*>(w + e1);
    }
  }

  int req, pos;
  lanes.find(args.table, lane, row, &req, &pos);
  const int page_shift = args.table.page_shift;
  const int32_t page_id = block_table[(int64_t)(args.table.req_base + req) * args.table.max_pages + (pos >> page_shift)];
  if (lane < rot_half) {
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
  // element offset of (page, head 0, slot, 0) in the caches
  const int64_t slot = ((((int64_t)page_id * hkv) << page_shift) + (pos & ((1 << page_shift) - 1))) * D;

#pragma unroll
  for (int i = 0; i < kAppendPasses; ++i) {
    const int hr = hr0 + i * ROWS_PER_PASS;
    const bool is_q = hr < hq, is_k = !is_q && hr < hq + hkv;
    float x[8], y[8];
    widen(a[i], x);
    widen(b[i], y);
    float sum = 0.f;
#pragma unroll
    for (int t = 0; t < 8; ++t) sum += x[t] * x[t] + y[t] * y[t];
    sum = group_sum<UNITS_PER_ROW>(sum);
    if (is_q || is_k) {
      const float r = 1.0f / sqrtf(sum * (1.0f / D) + args.eps);
      float w[8];
      widen(wa[i], w);
#pragma unroll
      for (int t = 0; t < 8; ++t) x[t] = x[t] * r * w[t];
      widen(wb[i], w);
#pragma unroll
      for (int t = 0; t < 8; ++t) y[t] = y[t] * r * w[t];
      if (in_rotary) {
        if constexpr (INTERLEAVED) rotate_interleaved_f32(x, y, cs, sn);
        else rotate_pairs_f32(x, y, cs, sn);
      }
      a[i] = narrow(x);
      b[i] = narrow(y);
    }
    if (hr >= rows_per_tok) continue;
    const int64_t cache_off = slot + (((int64_t)(hr - hq - (is_k ? 0 : hkv)) * D) << page_shift);
    if (KV8 && !is_q) {
      uint8_t* row8 = static_cast<uint8_t*>(is_k ? k_cache_raw : v_cache_raw) + cache_off;
      const double inv = is_k ? args.k_inv : args.v_inv;
      *reinterpret_cast<u32x2*>(row8 + e0) = quantize8(a[i], inv);
      *reinterpret_cast<u32x2*>(row8 + e1) = quantize8(b[i], inv);
    } else {
      uint16_t* dst = is_q ? q_out + ((int64_t)row * hq + hr) * D
                           : static_cast<uint16_t*>(is_k ? k_cache_raw : v_cache_raw) + cache_off;
      *reinterpret_cast<u32x4*>(dst + e0) = a[i];
      *reinterpret_cast<u32x4*>(dst + e1) = b[i];
    }
  }
}

struct NormTensors {
  const uint16_t *q, *k_new, *v_new, *q_weight, *k_weight;
  uint16_t* q_out;
  void *k_cache, *v_cache;
};

template <int MAXREQ>
int launch_with(const efim_batch_t* b, const NormTensors& t, float eps, const double* inv_freq, int rotary_dim,
                int interleaved, const CacheFormat& fmt, hipStream_t stream) {
  const int D = b->head_dim;
  NormArgs<MAXREQ> args;
  for (int j = 0; j < 64; ++j) args.inv_freq[j] = j < rotary_dim / 2 ? inv_freq[j] : 0.0;
  args.rotary_dim = rotary_dim;
  args.eps = eps;
  args.num_q_heads = t.q ? b->num_q_heads : 0;
  args.num_kv_heads = b->num_kv_heads;
  args.k_inv = 1.0 / (double)fmt.k_scale;
  args.v_inv = 1.0 / (double)fmt.v_scale;
  int64_t row = 0;
  for (int r0 = 0; r0 < b->batch;) {
    r0 = fill_table(b, r0, &row, &args.table);
    if (args.table.tokens == 0) continue;
    const AppendShape shape = append_shape(args.table.tokens, args.num_q_heads + 2 * b->num_kv_heads, D);
    args.parts = shape.parts;
    args.tok_shift = shape.tok_shift;
    const dim3 grid(shape.x, shape.y);
    auto launch = [&](auto d, auto il, auto f8) {
      norm_append_kernel<decltype(d)::value, decltype(il)::value, decltype(f8)::value, MAXREQ>
          <<<grid, 64 * args.parts << args.tok_shift, 0, stream>>>(args, t.q, t.q_out, t.k_new, t.v_new, t.q_weight,
                                                                   t.k_weight, t.k_cache, t.v_cache, b->block_table);
    };
    auto by_format = [&](auto d, auto il) { fmt.fp8 ? launch(d, il, std::true_type{}) : launch(d, il, std::false_type{}); };
    auto by_pairing = [&](auto d) { interleaved ? by_format(d, std::true_type{}) : by_format(d, std::false_type{}); };
    if (D == 128) by_pairing(std::integral_constant<int, 128>{});
    else by_pairing(std::integral_constant<int, 64>{});
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) { set_last_hip_error(e); return EFIM_ERR_LAUNCH; }
  }
  return EFIM_OK;
}

int norm_append(const efim_batch_t* b, const void* q, void* q_out, const void* k_new, const void* v_new,
                const void* q_weight, const void* k_weight, float eps, void* k_cache, void* v_cache,
                const double* inv_freq, int rotary_dim, int interleaved, const CacheFormat& fmt, void* stream) {
  int64_t total = 0;
  const int rc = validate_batch(b, &total);
  if (rc != EFIM_OK) return rc;
  if (!(eps >= 0.f) || eps - eps != 0.f || (interleaved != 0 && interleaved != 1)) return EFIM_ERR_INVALID_ARG;
  if (rotary_dim < 16 || rotary_dim > b->head_dim || rotary_dim % 16 != 0) return EFIM_ERR_INVALID_ARG;
  if (!frequencies_ok(inv_freq, rotary_dim)) return EFIM_ERR_INVALID_ARG;
  if (total >= kMaxAppendTokens) return EFIM_ERR_UNSUPPORTED;
  if (total == 0) return EFIM_OK;
  if (!k_new || !v_new || !k_cache || !v_cache || !q != !q_out) return EFIM_ERR_INVALID_ARG;
  for (const void* p : {q, (const void*)q_out, k_new, v_new, q_weight, k_weight, (const void*)k_cache, (const void*)v_cache})
    if (!aligned16(p)) return EFIM_ERR_INVALID_ARG;
  if (!aligned4(b->block_table)) return EFIM_ERR_INVALID_ARG;
  const NormTensors t{static_cast<const uint16_t*>(q), static_cast<const uint16_t*>(k_new), static_cast<const uint16_t*>(v_new),
                      static_cast<const uint16_t*>(q_weight), static_cast<const uint16_t*>(k_weight),
                      static_cast<uint16_t*>(q_out), k_cache, v_cache};
  auto* launch = b->batch <= 64 ? launch_with<64> : launch_with<kMaxReqPerAppend>;
  return launch(b, t, eps, inv_freq, rotary_dim, interleaved, fmt, static_cast<hipStream_t>(stream));
}

}  // namespace
}  // namespace efim

extern "C" {

int efim_norm_rope_append(const efim_batch_t* batch, const void* q, void* q_out, const void* k_new, const void* v_new,
                          const void* q_weight, const void* k_weight, float norm_eps, void* k_cache, void* v_cache,
                          const double* inv_freq, int rotary_dim, int rope_interleaved, void* stream) {
  return efim::norm_append(batch, q, q_out, k_new, v_new, q_weight, k_weight, norm_eps, k_cache, v_cache, inv_freq,
                           rotary_dim, rope_interleaved, efim::CacheFormat(), stream);
}

int efim_norm_rope_append_fp8(const efim_batch_t* batch, const void* q, void* q_out, const void* k_new,
                              const void* v_new, const void* q_weight, const void* k_weight, float norm_eps,
                              void* k_cache, void* v_cache, const double* inv_freq, int rotary_dim,
                              int rope_interleaved, float k_scale, float v_scale, void* stream) {
  if (!efim::scale_ok(k_scale) || !efim::scale_ok(v_scale)) return EFIM_ERR_INVALID_ARG;
  efim::CacheFormat fmt;
  fmt.fp8 = true;
  fmt.k_scale = k_scale;
  fmt.v_scale = v_scale;
  return efim::norm_append(batch, q, q_out, k_new, v_new, q_weight, k_weight, norm_eps, k_cache, v_cache, inv_freq,
                           rotary_dim, rope_interleaved, fmt, stream);
}

}  // extern "C"
