// efim_verify_drafts: drafted tokens accepted or refused against the target's probabilities, and the token that follows
// the accepted ones, from given random numbers.
//   x_i stays while u_i q_i(x_i) < p_i(x_i).  Behind a accepted tokens the next is drawn from p_a (all stayed) or from
//   max(p_a - q_a, 0) (x_a was refused): the first token j with w_0 + .. + w_j > u w_total.
// Weights are whole numbers of 2^-40: their sums are exact, so the answer does not depend on the order of summation, and
// with it not on the launch.  The product in the comparison is exact in fp64.
//
// Bound by reading one row of p, and of q where a token was refused, per request.  A first kernel sums the weights of
// chunks of a row, a second finds the chunk and the token in it.  64 requests and 128003 tokens: 15.6 us for 60 MB (3 of them the
// judging's chain of loads) and 5; chunks of twice and four times the size 14.6 and 14.0, but 6.9 and 10.3 to draw from.
// One request of 32004 tokens: 4.5 and 4.5.
#include <cstdint>

#include "efim_internal.h"

namespace efim {
namespace {

constexpr int kMaxDrafts = 63;        // of a request: a lane each
constexpr int kReqPerLaunch = 512;
constexpr int kThreads = 256;
constexpr int kPerThread = 8;
constexpr int kBlock = kThreads * kPerThread;  // elements that a workgroup takes at a time
constexpr int kMaxChunks = kThreads;  // of a row: the second kernel has a thread for each
constexpr int kMaxVocab = 1 << 22;

struct VerifyArgs {
  int32_t first[kReqPerLaunch + 1];  // drafted tokens in front of each request of the launch, and the end
  int32_t req_base;
  int32_t vocab;
  int32_t chunks;                    // of a row
  int32_t chunk;                     // elements, a multiple of kBlock
  const float* target;
  const float* draft;                // nullptr: the draft is certain of its tokens
  int64_t target_stride, draft_stride;
  const int32_t* draft_tokens;
  const float* uniforms;
  int32_t* tokens;
  int32_t* accepted;
  uint64_t* sums;                    // [request][chunk][2]: of the weights, and of p alone
};

struct Verdict {
  int accepted;
  const float* p;  // the row to draw from
  const float* q;  // the row to take off, or nullptr
  int without;     // token whose weight is zero (a refused token of a draft that was certain of it), or -1
};

// The drafted tokens of request r, a lane each; every lane gets the answer.
__device__ __forceinline__ Verdict judge(const VerifyArgs& a, int r, int lane) {
  const int d0 = a.first[r], n = a.first[r + 1] - d0;
  const int64_t t0 = (int64_t)d0 + a.req_base + r;
  int token = -1;
  bool stays = true;
  if (lane < n) {
    token = a.draft_tokens[d0 + lane];
    stays = token >= 0 && token < a.vocab;
    if (stays) {
      const double p = a.target[(t0 + lane) * a.target_stride + token];
      const double q = a.draft ? a.draft[(int64_t)(d0 + lane) * a.draft_stride + token] : 1.0f;
      stays = (double)a.uniforms[t0 + lane] * q < p;
    }
  }
  const uint64_t refused = __ballot(!stays);
  Verdict v;
  v.accepted = refused ? __builtin_ctzll(refused) : n;
  v.p = a.target + (t0 + v.accepted) * a.target_stride;
  v.q = v.accepted < n && a.draft ? a.draft + (int64_t)(d0 + v.accepted) * a.draft_stride : nullptr;
  v.without = v.accepted < n && !a.draft ? __builtin_amdgcn_readlane(token, v.accepted) : -1;
  return v;
}

// A probability in whole numbers of 2^-40; what is negative or no number counts as nothing, what is above one as one.
__device__ __forceinline__ uint64_t weight_of(float p) { return p > 0.f ? (uint64_t)(fminf(p, 1.f) * 0x1p40f) : 0; }

typedef float f32x4 __attribute__((ext_vector_type(4), aligned(4)));  // (rows of an odd vocabulary start anywhere)

// Weights of the elements from `at` on, past the row's end none.  w: of the draw; p: of the target alone.
__device__ __forceinline__ void weights(const Verdict& v, int vocab, int at, uint64_t (&w)[kPerThread], uint64_t (&whole)[kPerThread]) {
  float p[kPerThread], q[kPerThread];
  if (at + kPerThread <= vocab) {
#pragma unroll
    for (int j = 0; j < kPerThread; j += 4) {
      const f32x4 x = *reinterpret_cast<const f32x4*>(v.p + at + j);
#pragma unroll
      for (int k = 0; k < 4; ++k) p[j + k] = x[k];
    }
    if (v.q) {
#pragma unroll
      for (int j = 0; j < kPerThread; j += 4) {
        const f32x4 x = *reinterpret_cast<const f32x4*>(v.q + at + j);
#pragma unroll
        for (int k = 0; k < 4; ++k) q[j + k] = x[k];
      }
    }
  } else {
#pragma unroll
    for (int j = 0; j < kPerThread; ++j) {
      p[j] = at + j < vocab ? v.p[at + j] : 0.f;
      q[j] = v.q && at + j < vocab ? v.q[at + j] : 0.f;
    }
  }
#pragma unroll
  for (int j = 0; j < kPerThread; ++j) {
    whole[j] = weight_of(p[j]);
    const uint64_t off = v.q ? weight_of(q[j]) : at + j == v.without ? (uint64_t)1 << 40 : 0;
    w[j] = whole[j] > off ? whole[j] - off : 0;
  }
}

__device__ __forceinline__ uint64_t shuffle_up(uint64_t v, int by) {
  return (uint64_t)(uint32_t)__shfl_up((int)(uint32_t)v, by) | (uint64_t)(uint32_t)__shfl_up((int)(v >> 32), by) << 32;
}

// Sum of v over the threads in front of this one; *total: over all of them.  `held`: LDS of kThreads / 64 numbers.
__device__ __forceinline__ uint64_t sum_in_front(uint64_t v, uint64_t* held, uint64_t* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint64_t sum = v;
#pragma unroll
  for (int by = 1; by < 64; by <<= 1) {
    const uint64_t other = shuffle_up(sum, by);
    if (lane >= by) sum += other;
  }
  __syncthreads();  // (of the use before)
  if (lane == 63) held[wave] = sum;
  __syncthreads();
  uint64_t front = sum - v, all = 0;
#pragma unroll
  for (int k = 0; k < kThreads / 64; ++k) {
    if (k < wave) front += held[k];
    all += held[k];
  }
  *total = all;
  return front;
}

__global__ __launch_bounds__(kThreads) void verify_sums_kernel(const VerifyArgs a) {
  __shared__ uint64_t held[2][kThreads / 64];
  const int r = blockIdx.y, lane = threadIdx.x & 63;
  const Verdict v = judge(a, r, lane);
  uint64_t sum = 0, sum_p = 0;
  const int end = min((int)(blockIdx.x + 1) * a.chunk, a.vocab);
  for (int at = blockIdx.x * a.chunk + threadIdx.x * kPerThread; at < end; at += kBlock) {
    uint64_t w[kPerThread], p[kPerThread];
    weights(v, a.vocab, at, w, p);
#pragma unroll
    for (int j = 0; j < kPerThread; ++j) {
      sum += w[j];
      sum_p += p[j];
    }
  }
  uint64_t total, total_p;
  sum_in_front(sum, held[0], &total);
  sum_in_front(sum_p, held[1], &total_p);
  if (threadIdx.x == 0) {
    uint64_t* to = a.sums + ((int64_t)r * a.chunks + blockIdx.x) * 2;
    to[0] = total;
    to[1] = total_p;
  }
}

__global__ __launch_bounds__(kThreads) void verify_draw_kernel(const VerifyArgs a) {
  __shared__ uint64_t held[kThreads / 64];
  __shared__ uint64_t s_front;
  __shared__ int s_chunk;
  const int r = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
  Verdict v = judge(a, r, lane);
  const int d0 = a.first[r], n = a.first[r + 1] - d0;
  const int64_t t0 = (int64_t)d0 + a.req_base + r;
  // accepted tokens; what is behind the drawn one holds none
  if (tid <= n && tid != v.accepted) a.tokens[t0 + tid] = tid < v.accepted ? a.draft_tokens[d0 + tid] : -1;
  if (tid == 0) a.accepted[a.req_base + r] = v.accepted;
  const uint64_t* sums = a.sums + (int64_t)r * a.chunks * 2;
  uint64_t mine = tid < a.chunks ? sums[2 * tid] : 0, total;
  uint64_t front = sum_in_front(mine, held, &total);
  if (total == 0) {  // nothing is left of p where q is taken off: p itself
    v.q = nullptr;
    v.without = -1;
    mine = tid < a.chunks ? sums[2 * tid + 1] : 0;
    front = sum_in_front(mine, held, &total);
    if (total == 0) {
      if (tid == 0) a.tokens[t0 + v.accepted] = -1;
      return;
    }
  }
  // floor(u total), u in whole numbers of 2^-24 (total is below 2^62)
  const float u = a.uniforms[t0 + n];
  const uint64_t part = u > 0.f ? (uint64_t)fminf(u * 0x1p24f, 0x1.fffffep23f) : 0;
  const uint64_t below = part * (total >> 24) + ((part * (total & 0xFFFFFF)) >> 24);
  if (below >= front && below < front + mine) {
    s_chunk = tid;
    s_front = front;
  }
  __syncthreads();
  uint64_t before = s_front;
  const int begin = s_chunk * a.chunk;
  for (int at0 = begin; at0 < begin + a.chunk; at0 += kBlock) {
    const int at = at0 + tid * kPerThread;
    uint64_t w[kPerThread] = {}, p[kPerThread];
    if (at < a.vocab) weights(v, a.vocab, at, w, p);
    uint64_t sum = 0, block;
#pragma unroll
    for (int j = 0; j < kPerThread; ++j) sum += w[j];
    uint64_t upto = before + sum_in_front(sum, held, &block);
    if (below >= upto && below < upto + sum) {
#pragma unroll
      for (int j = 0; j < kPerThread; ++j) {
        if (below >= upto && below < upto + w[j]) a.tokens[t0 + v.accepted] = at + j;
        upto += w[j];
      }
    }
    before += block;
    if (below < before) return;
  }
}

int chunk_of(int vocab) {
  const int blocks = (vocab + kBlock - 1) / kBlock;
  return (blocks + kMaxChunks - 1) / kMaxChunks * kBlock;
}
int chunks_of(int vocab) { return (vocab + chunk_of(vocab) - 1) / chunk_of(vocab); }

bool sizes_ok(int batch, int vocab) { return batch >= 0 && vocab > 0; }

}  // namespace
}  // namespace efim

extern "C" {

size_t efim_verify_workspace_bytes(int batch, int vocab) {
  if (!efim::sizes_ok(batch, vocab) || vocab > efim::kMaxVocab) return 0;
  const int reqs = batch < efim::kReqPerLaunch ? batch : efim::kReqPerLaunch;
  const size_t bytes = (size_t)reqs * efim::chunks_of(vocab) * 2 * sizeof(uint64_t);
  return bytes < 256 ? 256 : bytes;
}

int efim_verify_drafts(int batch, const int32_t* num_drafts, int vocab, const void* target_probs, int64_t target_stride,
                       const void* draft_probs, int64_t draft_stride, const int32_t* draft_tokens,
                       const void* uniforms, int32_t* tokens, int32_t* accepted, void* workspace,
                       size_t workspace_bytes, void* stream) {
  using namespace efim;
  if (!sizes_ok(batch, vocab) || target_stride < vocab || (draft_probs && draft_stride < vocab)) return EFIM_ERR_INVALID_ARG;
  if (vocab > kMaxVocab) return EFIM_ERR_UNSUPPORTED;
  if (batch == 0) return EFIM_OK;
  if (!num_drafts) return EFIM_ERR_INVALID_ARG;
  int64_t drafts = 0;
  for (int r = 0; r < batch; ++r) {
    if (num_drafts[r] < 0) return EFIM_ERR_INVALID_ARG;
    if (num_drafts[r] > kMaxDrafts) return EFIM_ERR_UNSUPPORTED;
    drafts += num_drafts[r];
  }
  if (drafts + batch > INT32_MAX) return EFIM_ERR_UNSUPPORTED;
  if (!target_probs || !uniforms || !tokens || !accepted || (drafts > 0 && !draft_tokens)) return EFIM_ERR_INVALID_ARG;
  for (const void* p : {target_probs, draft_probs, (const void*)draft_tokens, uniforms, (const void*)tokens, (const void*)accepted})
    if (!aligned4(p)) return EFIM_ERR_INVALID_ARG;
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u) || workspace_bytes < efim_verify_workspace_bytes(batch, vocab))
    return EFIM_ERR_WORKSPACE;
  VerifyArgs a;
  a.vocab = vocab;
  a.chunk = chunk_of(vocab);
  a.chunks = chunks_of(vocab);
  a.target = static_cast<const float*>(target_probs);
  a.draft = static_cast<const float*>(draft_probs);
  a.target_stride = target_stride;
  a.draft_stride = draft_stride;
  a.draft_tokens = draft_tokens;
  a.uniforms = static_cast<const float*>(uniforms);
  a.tokens = tokens;
  a.accepted = accepted;
  a.sums = static_cast<uint64_t*>(workspace);
  int32_t first = 0;
  hipStream_t s = static_cast<hipStream_t>(stream);
  for (int r0 = 0; r0 < batch; r0 += kReqPerLaunch) {
    const int n = batch - r0 < kReqPerLaunch ? batch - r0 : kReqPerLaunch;
    a.req_base = r0;
    for (int i = 0; i < n; ++i) {
      a.first[i] = first;
      first += num_drafts[r0 + i];
    }
    a.first[n] = first;
    verify_sums_kernel<<<dim3(a.chunks, n), kThreads, 0, s>>>(a);
    verify_draw_kernel<<<n, kThreads, 0, s>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) { set_last_hip_error(e); return EFIM_ERR_LAUNCH; }
  }
  return EFIM_OK;
}

}  // extern "C"
