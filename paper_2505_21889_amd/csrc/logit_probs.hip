// efim_logit_probs: the logits of a step's rows to the probabilities that efim_verify_drafts takes.  Row i of request r has seen the
// request's history and the drafted tokens in front of it:
//   z = x;  seen:  z = z > 0 ? z / repetition : z * repetition;  made k > 0 times behind the prompt:  z -= k frequency + presence;
//   z += bias;  not allowed by the row's mask: none of the probability;  p = softmax(z / temperature)
// fp32, each operation rounded by itself; a temperature that is not above zero gives the first of the largest z all of it.
//
// Bound by reading the logits and writing the probabilities.  A workgroup has a chunk of the vocabulary for some rows of a request:
// it counts the history's tokens in its chunk once, in LDS (whole numbers: no order of theirs changes the result).  A first
// kernel leaves maximum, sum and place of the maximum of every chunk, a second forms the probabilities.
#include <cstdint>
#include <type_traits>

#include "efim_internal.h"

namespace efim {
namespace {

constexpr int kMaxDrafts = 63;  // of a request, as the verification's
constexpr int kReqPerLaunch = 512;
constexpr int kThreads = 256;
constexpr int kPerThread = 8;                   // neighbouring elements
constexpr int kBlock = kThreads * kPerThread;
constexpr int kBlocks = 2;                      // of a chunk
constexpr int kChunk = kBlocks * kBlock;
constexpr int kMaxVocab = 1 << 22;
constexpr uint32_t kSeen = 1u << 31;            // a token of the prompt; the bits below count those made behind it

struct ChunkStats {
  float top;      // largest z
  float sum;      // of exp((z - top) / temperature)
  int32_t place;  // of the first largest, in the vocabulary
  int32_t pad;
};

struct ProbsArgs {
  int32_t first[kReqPerLaunch + 1];  // drafted tokens in front of each request of the launch, and the end
  int32_t req_base;
  int32_t vocab;
  int32_t chunks;                    // of a row
  int32_t slice;                     // rows of a request that a workgroup takes
  efim_logits_t in;                  // (the host array in it is not looked at here)
  float* probs;
  int64_t probs_stride;
  ChunkStats* stats;                 // [row of the launch][chunk]
};

typedef float f32x4 __attribute__((ext_vector_type(4), aligned(4)));  // (rows of an odd vocabulary start anywhere)
typedef uint16_t u16x8 __attribute__((ext_vector_type(8), aligned(2)));

template <int N>
__device__ __forceinline__ float lanes_max(float v) {
#pragma unroll
  for (int by = 1; by < N; by <<= 1) v = fmaxf(v, __shfl_xor(v, by));
  return v;
}
__device__ __forceinline__ float lanes_sum(float v) {
#pragma unroll
  for (int by = 1; by < 64; by <<= 1) v += __shfl_xor(v, by);
  return v;
}
__device__ __forceinline__ int lanes_min(int v) {
#pragma unroll
  for (int by = 1; by < 64; by <<= 1) v = min(v, __shfl_xor(v, by));
  return v;
}

// WRITE: the second kernel.
template <bool BF16, bool WRITE>
__global__ __launch_bounds__(kThreads) void probs_kernel(const ProbsArgs a) {
#pragma clang fp contract(off)
  __shared__ __attribute__((aligned(16))) uint32_t s_count[kChunk];
  __shared__ __attribute__((aligned(16))) int32_t s_bias[kChunk];  // number of the entry that counts, from one
  __shared__ float s_top[kThreads / 64], s_sum[kThreads / 64];
  __shared__ int32_t s_place[kThreads / 64];

  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int r = blockIdx.y, request = a.req_base + r;
  const int d0 = a.first[r], n = a.first[r + 1] - d0;
  const int i0 = blockIdx.z * a.slice, i1 = min(i0 + a.slice, n + 1);
  if (i0 >= i1) return;
  const int base = blockIdx.x * kChunk;  // first token of the chunk
  const int width = min(kChunk, a.vocab - base);
  const int64_t row0 = (int64_t)d0 + request;          // the request's first row
  const int64_t launch_row0 = (int64_t)(d0 - a.first[0]) + r;

  efim_sampling_t how = {1.f, 1.f, 0.f, 0.f, 0, 0, 0, 0};
  if (a.in.params) how = a.in.params[request];
  const int64_t past = a.in.history ? min(max((int64_t)how.history_len, (int64_t)0), a.in.history_stride) : 0;
  const int64_t prompt = min(max((int64_t)how.prompt_len, (int64_t)0), past);
  const int biases = a.in.bias_tokens ? min(max(how.num_biases, 0), a.in.bias_stride) : 0;

  for (int e = tid; e < kChunk; e += kThreads) {
    s_count[e] = 0;
    s_bias[e] = 0;
  }
  __syncthreads();
  const int32_t* history = a.in.history + (int64_t)request * a.in.history_stride;
  for (int64_t j = tid; j < past; j += kThreads) {
    const uint32_t e = (uint32_t)(history[j] - base);
    if (e < (uint32_t)width) {
      if (j < prompt) atomicOr(&s_count[e], kSeen);
      else atomicAdd(&s_count[e], 1u);
    }
  }
  for (int j = tid; j < i0; j += kThreads) {
    const uint32_t e = (uint32_t)(a.in.draft_tokens[d0 + j] - base);
    if (e < (uint32_t)width) atomicAdd(&s_count[e], 1u);
  }
  for (int j = tid; j < biases; j += kThreads) {
    const uint32_t e = (uint32_t)(a.in.bias_tokens[(int64_t)request * a.in.bias_stride + j] - base);
    if (e < (uint32_t)width) atomicMax(&s_bias[e], j + 1);
  }
  const bool greedy = !(how.temperature > 0.f);
  const float to_log2 = greedy ? 1.4426950408889634f : 1.4426950408889634f / fmaxf(how.temperature, 0x1p-100f);

  for (int i = i0; i < i1; ++i) {
    __syncthreads();  // the counts are there
    const int64_t row = row0 + i;
    const int mask_row = a.in.masks && a.in.mask_rows ? a.in.mask_rows[row] : -1;
    const bool none = mask_row >= a.in.num_masks && mask_row >= 0;  // nothing is allowed
    const uint32_t* mask = mask_row >= 0 && !none ? a.in.masks + mask_row * a.in.mask_stride : nullptr;
    float z[kBlocks][kPerThread];
    uint32_t allowed[kBlocks];
#pragma unroll
    for (int b = 0; b < kBlocks; ++b) {
      const int e0 = b * kBlock + tid * kPerThread;
      allowed[b] = 0;
      if (e0 >= width) {
#pragma unroll
        for (int k = 0; k < kPerThread; ++k) z[b][k] = -INFINITY;
        continue;
      }
      const int64_t at = row * a.in.logits_stride + base + e0;
      if (e0 + kPerThread <= width) {
        if constexpr (BF16) {
          const u16x8 x = *reinterpret_cast<const u16x8*>(static_cast<const uint16_t*>(a.in.logits) + at);
#pragma unroll
          for (int k = 0; k < kPerThread; ++k) z[b][k] = __uint_as_float((uint32_t)x[k] << 16);
        } else {
          const f32x4 x = *reinterpret_cast<const f32x4*>(static_cast<const float*>(a.in.logits) + at);
          const f32x4 y = *reinterpret_cast<const f32x4*>(static_cast<const float*>(a.in.logits) + at + 4);
#pragma unroll
          for (int k = 0; k < 4; ++k) z[b][k] = x[k], z[b][4 + k] = y[k];
        }
        allowed[b] = 0xFF;
      } else {
#pragma unroll
        for (int k = 0; k < kPerThread; ++k) {
          z[b][k] = -INFINITY;
          if (e0 + k < width) {
            if constexpr (BF16) z[b][k] = __uint_as_float((uint32_t)static_cast<const uint16_t*>(a.in.logits)[at + k] << 16);
            else z[b][k] = static_cast<const float*>(a.in.logits)[at + k];
            allowed[b] |= 1u << k;
          }
        }
      }
      if (none) allowed[b] = 0;
      if (mask) allowed[b] &= mask[(base + e0) >> 5] >> ((base + e0) & 31);
#pragma unroll
      for (int k = 0; k < kPerThread; ++k) {
        const uint32_t count = s_count[e0 + k];
        const int bias = s_bias[e0 + k];
        if (count) z[b][k] = z[b][k] > 0.f ? z[b][k] / how.repetition : z[b][k] * how.repetition;
        if (count & ~kSeen) {
          const float often = how.frequency * (float)(count & ~kSeen);
          z[b][k] = z[b][k] - often - how.presence;
        }
        if (bias) z[b][k] = z[b][k] + a.in.bias_values[(int64_t)request * a.in.bias_stride + bias - 1];
        if (!(allowed[b] >> k & 1)) z[b][k] = -INFINITY;
      }
    }
    ChunkStats* stats = a.stats + (launch_row0 + i) * a.chunks;
    if constexpr (!WRITE) {
      float top = -INFINITY;
#pragma unroll
      for (int b = 0; b < kBlocks; ++b)
#pragma unroll
        for (int k = 0; k < kPerThread; ++k) top = fmaxf(top, z[b][k]);
      top = lanes_max<64>(top);
      if (lane == 0) s_top[wave] = top;
      __syncthreads();
      // (a thread that has read the counts of this row: the token drafted behind it may join them)
      if (tid == 0 && i + 1 < i1) {
        const uint32_t e = (uint32_t)(a.in.draft_tokens[d0 + i] - base);
        if (e < (uint32_t)width) s_count[e] += 1;
      }
#pragma unroll
      for (int w = 0; w < kThreads / 64; ++w) top = fmaxf(top, s_top[w]);
      float sum = 0.f;
      int place = INT32_MAX;
#pragma unroll
      for (int b = 0; b < kBlocks; ++b)
#pragma unroll
        for (int k = 0; k < kPerThread; ++k) {
          if (z[b][k] != -INFINITY) sum += __builtin_amdgcn_exp2f((z[b][k] - top) * to_log2);
          if (z[b][k] == top) place = min(place, base + b * kBlock + tid * kPerThread + k);
        }
      sum = lanes_sum(sum);
      place = lanes_min(place);
      if (lane == 0) {
        s_sum[wave] = sum;
        s_place[wave] = place;
      }
      __syncthreads();
      if (tid == 0) {
        float all = 0.f;
        int first = INT32_MAX;
#pragma unroll
        for (int w = 0; w < kThreads / 64; ++w) {
          all += s_sum[w];
          first = min(first, s_place[w]);
        }
        stats[blockIdx.x] = ChunkStats{top, all, first, 0};
      }
    } else {
      // the whole row's, by every wave
      float top = -INFINITY;
      for (int c = lane; c < a.chunks; c += 64) top = fmaxf(top, stats[c].top);
      top = lanes_max<64>(top);
      float sum = 0.f;
      int place = INT32_MAX;
      for (int c = lane; c < a.chunks; c += 64) {
        const ChunkStats s = stats[c];
        sum += s.sum * (s.top == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((s.top - top) * to_log2));
        if (s.top == top) place = min(place, s.place);
      }
      sum = lanes_sum(sum);
      place = lanes_min(place);
      __syncthreads();
      if (tid == 0 && i + 1 < i1) {
        const uint32_t e = (uint32_t)(a.in.draft_tokens[d0 + i] - base);
        if (e < (uint32_t)width) s_count[e] += 1;
      }
      const float part = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
      for (int b = 0; b < kBlocks; ++b) {
        const int e0 = b * kBlock + tid * kPerThread;
        if (e0 >= width) continue;
        float p[kPerThread];
#pragma unroll
        for (int k = 0; k < kPerThread; ++k) {
          const float e = z[b][k] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((z[b][k] - top) * to_log2);
          p[k] = greedy ? (base + e0 + k == place && top > -INFINITY ? 1.f : 0.f) : e * part;
          if (!(allowed[b] >> k & 1)) p[k] = 0.f;
        }
        float* to = a.probs + row * a.probs_stride + base + e0;
        if (e0 + kPerThread <= width) {
          *reinterpret_cast<f32x4*>(to) = f32x4{p[0], p[1], p[2], p[3]};
          *reinterpret_cast<f32x4*>(to + 4) = f32x4{p[4], p[5], p[6], p[7]};
        } else {
#pragma unroll
          for (int k = 0; k < kPerThread; ++k)
            if (e0 + k < width) to[k] = p[k];
        }
      }
    }
  }
}

int chunks_of(int vocab) { return (vocab + kChunk - 1) / kChunk; }

// Rows of a launch, and what of a description can be checked on the host.
int checked(const efim_logits_t* in, int64_t* rows) {
  *rows = 0;
  if (!in || in->batch < 0 || in->vocab <= 0) return EFIM_ERR_INVALID_ARG;
  if (in->vocab > kMaxVocab) return EFIM_ERR_UNSUPPORTED;
  if (in->batch == 0) return EFIM_OK;
  if (!in->num_drafts) return EFIM_ERR_INVALID_ARG;
  int64_t all = 0, launch = 0;
  for (int r = 0; r < in->batch; ++r) {
    if (in->num_drafts[r] < 0) return EFIM_ERR_INVALID_ARG;
    if (in->num_drafts[r] > kMaxDrafts) return EFIM_ERR_UNSUPPORTED;
    if (r % kReqPerLaunch == 0) launch = 0;
    launch += in->num_drafts[r] + 1;
    all += in->num_drafts[r] + 1;
    if (launch > *rows) *rows = launch;
  }
  return all > INT32_MAX ? EFIM_ERR_UNSUPPORTED : EFIM_OK;
}

size_t bytes_for(const efim_logits_t* in, int64_t rows) {
  const size_t bytes = (size_t)rows * chunks_of(in->vocab) * sizeof(ChunkStats);
  return bytes < 256 ? 256 : bytes;
}

}  // namespace
}  // namespace efim

extern "C" {

size_t efim_logit_workspace_bytes(const efim_logits_t* in) {
  int64_t rows = 0;
  return efim::checked(in, &rows) == EFIM_OK ? efim::bytes_for(in, rows) : 0;
}

int efim_logit_probs(const efim_logits_t* in, void* probs, int64_t probs_stride, void* workspace, size_t workspace_bytes, void* stream) {
  using namespace efim;
  int64_t rows = 0;
  const int rc = checked(in, &rows);
  if (rc != EFIM_OK) return rc;
  if (in->batch == 0) return EFIM_OK;
  if (in->logits_bf16 != 0 && in->logits_bf16 != 1) return EFIM_ERR_INVALID_ARG;
  if (in->logits_stride < in->vocab || probs_stride < in->vocab) return EFIM_ERR_INVALID_ARG;
  int64_t drafts = 0;
  for (int r = 0; r < in->batch; ++r) drafts += in->num_drafts[r];
  if (!in->logits || !probs || (drafts > 0 && !in->draft_tokens)) return EFIM_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(in->logits) & (in->logits_bf16 ? 1u : 3u)) || !aligned4(probs)) return EFIM_ERR_INVALID_ARG;
  if (in->history && in->history_stride < 0) return EFIM_ERR_INVALID_ARG;
  if (!in->bias_tokens != !in->bias_values || (in->bias_tokens && in->bias_stride < 0)) return EFIM_ERR_INVALID_ARG;
  if (in->masks && (in->num_masks < 0 || in->mask_stride < (in->vocab + 31) / 32)) return EFIM_ERR_INVALID_ARG;
  for (const void* p : {(const void*)in->params, (const void*)in->history, (const void*)in->draft_tokens, (const void*)in->bias_tokens,
                        (const void*)in->bias_values, (const void*)in->masks, (const void*)in->mask_rows})
    if (!aligned4(p)) return EFIM_ERR_INVALID_ARG;
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u) || workspace_bytes < bytes_for(in, rows)) return EFIM_ERR_WORKSPACE;
  ProbsArgs a;
  a.vocab = in->vocab;
  a.chunks = chunks_of(in->vocab);
  a.in = *in;
  a.probs = static_cast<float*>(probs);
  a.probs_stride = probs_stride;
  a.stats = static_cast<ChunkStats*>(workspace);
  int32_t first = 0;
  hipStream_t s = static_cast<hipStream_t>(stream);
  for (int r0 = 0; r0 < in->batch; r0 += kReqPerLaunch) {
    const int n = in->batch - r0 < kReqPerLaunch ? in->batch - r0 : kReqPerLaunch;
    a.req_base = r0;
    int most = 0;
    for (int i = 0; i < n; ++i) {
      a.first[i] = first;
      first += in->num_drafts[r0 + i];
      if (in->num_drafts[r0 + i] + 1 > most) most = in->num_drafts[r0 + i] + 1;
    }
    a.first[n] = first;
    a.slice = (int64_t)a.chunks * n >= 4 * compute_units() ? most : 1;
    const dim3 grid((unsigned)a.chunks, (unsigned)n, (unsigned)((most + a.slice - 1) / a.slice));
    if (in->logits_bf16) {
      probs_kernel<true, false><<<grid, kThreads, 0, s>>>(a);
      probs_kernel<true, true><<<grid, kThreads, 0, s>>>(a);
    } else {
      probs_kernel<false, false><<<grid, kThreads, 0, s>>>(a);
      probs_kernel<false, true><<<grid, kThreads, 0, s>>>(a);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) { set_last_hip_error(e); return EFIM_ERR_LAUNCH; }
  }
  return EFIM_OK;
}

}  // extern "C"
