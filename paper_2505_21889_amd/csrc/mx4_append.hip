// efim_rope_append_mx4: rotary embedding of the new tokens and append of their keys and values to a 4-bit cache, in one pass
// over the tokens' rows.  The rotation is the bf16 append's (fp64, rounded once), so the queries are the same bits; what that
// append would have stored is rounded block by block to 4 bits.
// Streaming kernel, bound by HBM bandwidth: (4 Hq + 2 Hkv (2 + 17/32 + 2 where the stored rows are asked for)) D bytes a token.
// 64 requests, half of them whole prompts of 1024..4096 tokens, 32/8 heads: 2054 MB in 363 us, 5.7 TB/s (a copy: 5.1); 16 single tokens: 4.5 us.
#include <type_traits>

#include "append_table.h"
#include "efim_internal.h"
#include "mx4_math.h"
#include "rope_math.h"

namespace efim {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

template <int MAXREQ>
struct Mx4Args {
  AppendTable<MAXREQ> table;
  int32_t tok_shift;     // log2 of the tokens of a workgroup
  int32_t parts;         // waves per token in a workgroup
  int32_t num_q_heads;   // 0 where there are no queries
  int32_t num_kv_heads;
  int32_t rotary_dim;    // leading elements of a head row that are rotated
  double inv_freq[64];   // rotation frequency of pair j (rotary_dim/2 entries)
};

// A wave takes one token and kAppendPasses passes of 64 / (D / 16) head rows of it; a lane has two chunks of eight elements of a
// row, partners under the rotation (see the bf16 append).  Blocks of 32 elements need neighbours instead: rotate-half rows change
// their lanes through LDS inside the wave, behind which a lane has 16 consecutive elements and its neighbour the block's others.
template <int D, bool INTERLEAVED, int MAXREQ>
__global__ __launch_bounds__(kAppendThreads) void mx4_append_kernel(
    const Mx4Args<MAXREQ> args, const uint16_t* q, uint16_t* q_out, const uint16_t* __restrict__ k_new,
    const uint16_t* __restrict__ v_new, uint8_t* __restrict__ k_cache, uint8_t* __restrict__ v_cache,
    uint16_t* __restrict__ k_stored, uint16_t* __restrict__ v_stored, const int32_t* __restrict__ block_table) {
  constexpr int HALF = D / 2;
  constexpr int UNITS_PER_ROW = D / 16;
  constexpr int ROWS_PER_PASS = 64 / UNITS_PER_ROW;
  __shared__ __attribute__((aligned(16))) double s_cs[kAppendThreads / 64][HALF][2];  // (cos, sin) of the wave's token
  __shared__ __attribute__((aligned(16))) u32x4 s_rows[INTERLEAVED ? 1 : kAppendThreads / 64][128];  // a pass's rows

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
  u32x4 a[kAppendPasses], b[kAppendPasses];
#pragma unroll
  for (int i = 0; i < kAppendPasses; ++i) {
    // (0..Hq-1: q heads, then Hkv k heads, then Hkv v heads)
    const int hr = min(hr0 + i * ROWS_PER_PASS, rows_per_tok - 1);
    const uint16_t* src = k_new + ((int64_t)row * hkv + (hr - hq)) * D;
    if (hr < hq) src = q + ((int64_t)row * hq + hr) * D;
    if (hr >= hq + hkv) src = v_new + ((int64_t)row * hkv + (hr - hq - hkv)) * D;
    a[i] = *reinterpret_cast<const u32x4*>(src + e0);
    b[i] = *reinterpret_cast<const u32x4*>(src + e1);
  }

  int req, pos;
  lanes.find(args.table, lane, row, &req, &pos);
  const int page_shift = args.table.page_shift;
  const int32_t page_id = block_table[(int64_t)(args.table.req_base + req) * args.table.max_pages + (pos >> page_shift)];
  if (lane < rot_half) {
    double s, c;
    sincos((double)pos * freq, &s, &c);
    s_cs[wave][lane][0] = c;
    s_cs[wave][lane][1] = s;
  }
  // (one wave writes and reads: its LDS accesses are in order, the compiler is told by the fences)
  auto own_writes = [] {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  };
  own_writes();
  double cs[8], sn[8];
#pragma unroll
  for (int t = 0; t < 8; ++t) {
    cs[t] = s_cs[wave][cp * 8 + t][0];
    sn[t] = s_cs[wave][cp * 8 + t][1];
  }
  const int slot = pos & ((1 << page_shift) - 1);

#pragma unroll
  for (int i = 0; i < kAppendPasses; ++i) {
    const int hr = hr0 + i * ROWS_PER_PASS;
    const bool is_q = hr < hq, is_k = !is_q && hr < hq + hkv;
    if (in_rotary && hr < hq + hkv) rotate_units<INTERLEAVED>(a[i], b[i], cs, sn);
    if (is_q) {
      uint16_t* dst = q_out + ((int64_t)row * hq + hr) * D;
      *reinterpret_cast<u32x4*>(dst + e0) = a[i];
      *reinterpret_cast<u32x4*>(dst + e1) = b[i];
    }
    if (hr0 - lane / UNITS_PER_ROW + (i + 1) * ROWS_PER_PASS <= hq) continue;  // (wave-uniform: query rows alone)
    if constexpr (!INTERLEAVED) {
      char* mine = reinterpret_cast<char*>(s_rows[wave]) + lane / UNITS_PER_ROW * (2 * D);
      own_writes();
      *reinterpret_cast<u32x4*>(mine + 2 * e0) = a[i];
      *reinterpret_cast<u32x4*>(mine + 2 * e1) = b[i];
      own_writes();
      a[i] = s_rows[wave][2 * lane];
      b[i] = s_rows[wave][2 * lane + 1];
    }
    // largest magnitude of the block, by its bit pattern
    u16x2 top = {0, 0};
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, a[i][t] & 0x7FFF7FFFu));
      top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, b[i][t] & 0x7FFF7FFFu));
    }
    uint32_t largest = max((uint32_t)top[0], (uint32_t)top[1]);
    largest = max(largest, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)largest, 0xB1, 0xf, 0xf, true));  // quad_perm [1, 0, 3, 2]
    if (is_q || hr >= rows_per_tok) continue;
    const uint32_t byte = mx4_scale_of(largest);
    const float scale = mx4_scale_value(byte);
    u32x2 codes = {mx4_encode8(a[i], scale), mx4_encode8(b[i], scale)};
    if (byte == kMx4Nan) codes = u32x2{0, 0};
    const int head = hr - hq - (is_k ? 0 : hkv);
    uint8_t* page = (is_k ? k_cache : v_cache) + (((int64_t)page_id * hkv + head) << page_shift) * mx4_row_bytes(D);
    *reinterpret_cast<u32x2*>(page + slot * mx4_code_bytes(D) + cp * 8) = codes;
    if ((cp & 1) == 0) page[(mx4_code_bytes(D) << page_shift) + slot * mx4_scale_bytes(D) + cp / 2] = (uint8_t)byte;
    uint16_t* stored = is_k ? k_stored : v_stored;
    if (stored) {
      uint16_t* dst = stored + ((int64_t)row * hkv + head) * D + cp * 16;
      *reinterpret_cast<u32x4*>(dst) = mx4_decode8(codes[0], scale);
      *reinterpret_cast<u32x4*>(dst + 8) = mx4_decode8(codes[1], scale);
    }
  }
}

struct Mx4Tensors {
  const uint16_t *q, *k_new, *v_new;
  uint16_t *q_out, *k_stored, *v_stored;
  uint8_t *k_cache, *v_cache;
};

template <int MAXREQ>
int launch_with(const efim_batch_t* b, const Mx4Tensors& t, const double* inv_freq, int rotary_dim, int interleaved,
                hipStream_t stream) {
  const int D = b->head_dim;
  Mx4Args<MAXREQ> args;
  for (int j = 0; j < 64; ++j) args.inv_freq[j] = j < rotary_dim / 2 ? inv_freq[j] : 0.0;
  args.rotary_dim = rotary_dim;
  args.num_q_heads = t.q ? b->num_q_heads : 0;
  args.num_kv_heads = b->num_kv_heads;
  int64_t row = 0;
  for (int r0 = 0; r0 < b->batch;) {
    r0 = fill_table(b, r0, &row, &args.table);
    if (args.table.tokens == 0) continue;
    const AppendShape shape = append_shape(args.table.tokens, args.num_q_heads + 2 * b->num_kv_heads, D);
    args.parts = shape.parts;
    args.tok_shift = shape.tok_shift;
    const dim3 grid(shape.x, shape.y);
    auto launch = [&](auto d, auto il) {
      mx4_append_kernel<decltype(d)::value, decltype(il)::value, MAXREQ><<<grid, 64 * args.parts << args.tok_shift, 0, stream>>>(
          args, t.q, t.q_out, t.k_new, t.v_new, t.k_cache, t.v_cache, t.k_stored, t.v_stored, b->block_table);
    };
    auto by_pairing = [&](auto d) { interleaved ? launch(d, std::true_type{}) : launch(d, std::false_type{}); };
    if (D == 128) by_pairing(std::integral_constant<int, 128>{});
    else by_pairing(std::integral_constant<int, 64>{});
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) { set_last_hip_error(e); return EFIM_ERR_LAUNCH; }
  }
  return EFIM_OK;
}

}  // namespace
}  // namespace efim

extern "C" {

size_t efim_mx4_cache_bytes(int64_t num_pages, int num_kv_heads, int page_size, int head_dim) {
  if (num_pages < 0 || num_kv_heads < 1 || page_size < efim::kMinPageSize || page_size > efim::kMaxPageSize ||
      (page_size & (page_size - 1)) != 0 || (head_dim != 64 && head_dim != 128))
    return 0;
  // (a size that does not fit the type is no size)
  size_t bytes = (size_t)efim::mx4_row_bytes(head_dim) * (size_t)page_size;
  if (__builtin_mul_overflow(bytes, (size_t)num_kv_heads, &bytes) || __builtin_mul_overflow(bytes, (size_t)num_pages, &bytes)) return 0;
  return bytes;
}

int efim_rope_append_mx4(const efim_batch_t* batch, const void* q, void* q_out, const void* k_new, const void* v_new, void* k_cache,
                         void* v_cache, void* k_stored, void* v_stored, const double* inv_freq, int rotary_dim,
                         int rope_interleaved, void* stream) {
  using namespace efim;
  int64_t total = 0;
  const int rc = validate_batch(batch, &total);
  if (rc != EFIM_OK) return rc;
  if (rope_interleaved != 0 && rope_interleaved != 1) return EFIM_ERR_INVALID_ARG;
  if (rotary_dim < 16 || rotary_dim > batch->head_dim || rotary_dim % 16 != 0) return EFIM_ERR_INVALID_ARG;
  if (!frequencies_ok(inv_freq, rotary_dim)) return EFIM_ERR_INVALID_ARG;
  if (total >= kMaxAppendTokens) return EFIM_ERR_UNSUPPORTED;
  if (total == 0) return EFIM_OK;
  if (!k_new || !v_new || !k_cache || !v_cache || !q != !q_out) return EFIM_ERR_INVALID_ARG;
  for (const void* p : {q, (const void*)q_out, k_new, v_new, (const void*)k_cache, (const void*)v_cache, (const void*)k_stored,
                        (const void*)v_stored})
    if (!aligned16(p)) return EFIM_ERR_INVALID_ARG;
  if (!aligned4(batch->block_table)) return EFIM_ERR_INVALID_ARG;
  const Mx4Tensors t{static_cast<const uint16_t*>(q), static_cast<const uint16_t*>(k_new), static_cast<const uint16_t*>(v_new),
                     static_cast<uint16_t*>(q_out), static_cast<uint16_t*>(k_stored), static_cast<uint16_t*>(v_stored),
                     static_cast<uint8_t*>(k_cache), static_cast<uint8_t*>(v_cache)};
  auto* launch = batch->batch <= 64 ? launch_with<64> : launch_with<kMaxReqPerAppend>;
  return launch(batch, t, inv_freq, rotary_dim, rope_interleaved, static_cast<hipStream_t>(stream));
}

}  // extern "C"
