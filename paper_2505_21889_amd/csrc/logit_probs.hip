// efim_logit_probs: the logits of a step's rows to the probabilities that efim_verify_drafts takes.  Row i of request r has seen the
// request's history and the drafted tokens in front of it:
//   z = x;  seen:  z = z > 0 ? z / repetition : z * repetition;  made k > 0 times behind the prompt:  z -= k frequency + presence;
//   z += bias;  not allowed by the row's mask: none of the probability;  p = softmax(z / temperature)
// fp32, each operation rounded by itself; a temperature that is not above zero gives the first of the largest z all of it.
//
// Few tokens of the vocabulary have anything done to them, the same ones in all rows of a request.  A first kernel marks them in a
// bit for each token and lists them, with how often they were made and their bias (counted in whole numbers: no order changes the
// result).  Behind it the others are taken as they are, and an element costs two bits and the exponential.  A second kernel leaves
// maximum, sum and place of the maximum of every chunk of a row, a third forms the probabilities from them; in both a wave has a chunk
// of a row to itself and waits for no other.  Bound by the instructions of the statistics, by reading the logits a second time and by
// writing the probabilities.
// us for 6 rows of 32004 / for 64 requests with 1 to 15 drafts and 128003: 18.0 / 178, of the latter 13 list, 70 statistics (their
// instructions, 22 an element, take three quarters of the issue cycles; 196 MB come from memory, 2.8 TB/s) and 104 probabilities (212 MB from
// memory and 329 MB to it, 5.2 TB/s: a copy's rate).  A workgroup for each row and slice that makes its own list, two kernels: 15.7 / 271.  Listed tokens gone through behind the others instead of through LDS: 20.4 / 194.  A wave for a
// chunk of four rows that loads the list once: 18.5 / 248 (half as many waves at a time).
#include <cstdint>
#include <type_traits>

#include "efim_internal.h"

namespace efim {
namespace {

constexpr int kMaxDrafts = 63;  // of a request, as the verification's
constexpr int kReqPerLaunch = 512;
constexpr int kMaxVocab = 1 << 22;
constexpr uint32_t kSeen = 1u << 31;     // a token of the prompt
constexpr uint32_t kDrafted = 1u << 30;  // a drafted token; the bits below count those made behind the prompt
constexpr int64_t kMaxHistory = kDrafted - 64;

constexpr int kListThreads = 1024;
constexpr int kListWords = 4 * kListThreads;  // of the marks that the first kernel holds at a time
constexpr int kListHeld = 8192;               // listed tokens of those that it counts in LDS

constexpr int kThreads = 256;
constexpr int kPerLane = 4;           // neighbouring elements of a lane: a wave's loads and stores are whole lines
constexpr int kStep = 64 * kPerLane;  // elements that a wave takes at a time
constexpr int kSteps = 4;             // asked for together
constexpr int kChunk = kSteps * kStep;  // of a wave
constexpr int kListed = 4;            // entries of a long list that a lane takes at a time

struct PartStats {  // of a chunk of a row
  float top;      // largest z
  float sum;      // of exp((z - top) / temperature)
  int32_t place;  // of the first largest, in the vocabulary
  int32_t pad;
};

struct RowInfo {
  int32_t request, place;  // the row's request, and how many drafted tokens it has seen
  int32_t first_draft;
  int32_t mask;            // number of its mask, negative: none
  float to_log2;           // log2(e) / temperature
  int32_t greedy;
  int32_t pad[2];
};

struct ProbsArgs {
  const void* logits;
  int64_t logits_stride;
  const efim_sampling_t* params;
  const int32_t* history;
  int64_t history_stride;
  const int32_t* draft_tokens;
  const int32_t* bias_tokens;
  const float* bias_values;
  const uint32_t* masks;
  int64_t mask_stride;
  const int32_t* mask_rows;
  float* probs;
  int64_t probs_stride;
  PartStats* stats;    // [row of the launch][chunks]
  RowInfo* rows;       // [row of the launch]
  uint32_t* touched;   // [request of the launch][words]: a bit for each listed token
  int32_t* listed;     // [request of the launch][most_listed]: the tokens, in their order
  uint32_t* counts;    // how often each was made, kSeen, kDrafted
  int32_t* biases;     // the number, from one, of the entry with its bias
  int32_t* starts;     // [request of the launch][chunks + 1]: listed tokens in front of each chunk, and all of them
  int32_t bias_stride, num_masks;
  int32_t vocab;
  int32_t words;       // ceil(vocab / 32)
  int32_t most_listed;
  int32_t chunks;      // of a row
  int32_t total;       // rows of the launch
  int32_t req_base;
  int64_t row_base;    // rows in front of the launch
  int32_t first[kReqPerLaunch + 1];  // (the first kernel's) drafted tokens in front of each request of the launch, and the end
};

typedef float f32x4 __attribute__((ext_vector_type(4), aligned(4)));     // (rows of an odd vocabulary start anywhere)
typedef uint32_t u32x2 __attribute__((ext_vector_type(2), aligned(2)));  // four bf16 values
typedef int32_t i32x4 __attribute__((ext_vector_type(4), aligned(4)));

// A value with those of the other lanes, in all of them: exchanges inside rows of sixteen lanes, then of rows and halves.
template <typename Join>
__device__ __forceinline__ uint32_t lanes_join(uint32_t v, Join join) {
  auto with = [&](auto ctrl) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, decltype(ctrl)::value, 0xf, 0xf, true); };
  v = join(v, with(std::integral_constant<int, 0xB1>{}));   // quad_perm [1, 0, 3, 2]
  v = join(v, with(std::integral_constant<int, 0x4E>{}));   // quad_perm [2, 3, 0, 1]
  v = join(v, with(std::integral_constant<int, 0x141>{}));  // row_half_mirror
  v = join(v, with(std::integral_constant<int, 0x140>{}));  // row_mirror
  const auto rows = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  v = join(rows[0], rows[1]);
  const auto halves = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return join(halves[0], halves[1]);
}
__device__ __forceinline__ float lanes_max(float v) {
  return __uint_as_float(lanes_join(__float_as_uint(v), [](uint32_t x, uint32_t y) { return __float_as_uint(fmaxf(__uint_as_float(x), __uint_as_float(y))); }));
}
__device__ __forceinline__ float lanes_sum(float v) {
  return __uint_as_float(lanes_join(__float_as_uint(v), [](uint32_t x, uint32_t y) { return __float_as_uint(__uint_as_float(x) + __uint_as_float(y)); }));
}
__device__ __forceinline__ int lanes_min(int v) {
  return (int)lanes_join((uint32_t)v, [](uint32_t x, uint32_t y) { return (uint32_t)min((int)x, (int)y); });
}
template <bool BF16>
__device__ __forceinline__ float load_logit(const void* logits, int64_t at) {
  if constexpr (BF16) return __uint_as_float((uint32_t)static_cast<const uint16_t*>(logits)[at] << 16);
  else return static_cast<const float*>(logits)[at];
}

// Four logits of a row.  (bf16 in whole words: neighbouring halves apart would take a register each.)
template <bool BF16>
struct Four {
  using Words = std::conditional_t<BF16, u32x2, f32x4>;
  static constexpr uint32_t kBytes = BF16 ? 2 : 4;  // of a logit
  Words x;
  __device__ __forceinline__ float operator[](int k) const {
    if constexpr (BF16) return __uint_as_float(k & 1 ? x[k / 2] & 0xFFFF0000u : x[k / 2] << 16);
    else return x[k];
  }
};

// --- the list -----------------------------------------------------------------------------------------------------------------
// A workgroup for each request, kListWords * 32 tokens of the vocabulary at a time.  A token's place in the list is the number of
// marks in front of it.
__global__ __launch_bounds__(kListThreads) void probs_list_kernel(const ProbsArgs a) {
  __shared__ uint32_t s_marks[kListWords];
  __shared__ int32_t s_front[kListWords];  // marks in front of a word
  __shared__ int32_t s_wave[4 * (kListThreads / 64)];
  __shared__ uint32_t s_counts[kListHeld];
  __shared__ int32_t s_biases[kListHeld];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int r = blockIdx.x, request = a.req_base + r;
  const int d0 = a.first[r], n = a.first[r + 1] - d0;
  efim_sampling_t how = {1.f, 1.f, 0.f, 0.f, 0, 0, 0, 0};
  if (a.params) how = a.params[request];
  const int past = a.history ? min(max(how.history_len, 0), (int)a.history_stride) : 0;
  const int prompt = min(max(how.prompt_len, 0), past);
  const int entries = a.bias_tokens ? min(max(how.num_biases, 0), a.bias_stride) : 0;
  const int32_t* history = a.history + (int64_t)request * a.history_stride;
  const int32_t* bias_tokens = a.bias_tokens + (int64_t)request * a.bias_stride;
  int32_t* listed = a.listed + (int64_t)r * a.most_listed;
  uint32_t* counts = a.counts + (int64_t)r * a.most_listed;
  int32_t* biases = a.biases + (int64_t)r * a.most_listed;

  // what(token, its place in the history); a thread's first eight tokens are asked for once
  const int fours = past & ~3;
  i32x4 held0 = {-1, -1, -1, -1}, held1 = held0;
  if (tid * 4 < fours) {
    held0 = *reinterpret_cast<const i32x4*>(history + tid * 4);
    held1 = *reinterpret_cast<const i32x4*>(history + min(tid * 4 + 4 * kListThreads, fours - 4));
  }
  const int draft = tid < n ? a.draft_tokens[d0 + tid] : -1;
  auto for_history = [&](auto what) __attribute__((always_inline)) {
    for (int j0 = tid * 4; j0 < fours; j0 += 2 * 4 * kListThreads) {
      const int j1 = j0 + 4 * kListThreads;
      i32x4 x = held0, y = held1;
      if (j0 != tid * 4) {
        x = *reinterpret_cast<const i32x4*>(history + j0);
        y = *reinterpret_cast<const i32x4*>(history + min(j1, fours - 4));
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) what(x[k], j0 + k);
      if (j1 < fours)
#pragma unroll
        for (int k = 0; k < 4; ++k) what(y[k], j1 + k);
    }
    if (tid < past - fours) what(history[fours + tid], fours + tid);
  };
  int before = 0;  // listed tokens of the words in front
  for (int w0 = 0; w0 < a.words; w0 += kListWords) {
    const int base = w0 * 32, width = min(kListWords * 32, a.vocab - base);
    auto inside = [&](int token) { return (uint32_t)(token - base) < (uint32_t)width; };
#pragma unroll
    for (int k = 0; k < 4; ++k) s_marks[k * kListThreads + tid] = 0;
    __syncthreads();
    auto mark = [&](int token, int) {
      if (inside(token)) atomicOr(&s_marks[(token - base) >> 5], 1u << (token & 31));
    };
    for_history(mark);
    if (tid < n) mark(draft, 0);
    for (int j = tid; j < entries; j += kListThreads) mark(bias_tokens[j], 0);
    __syncthreads();
    // (a thread has words that are far apart: neighbouring ones may hold all of the frequent tokens)
    uint32_t marks[4];
    int upto[4], mine[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int w = k * kListThreads + tid;
      marks[k] = s_marks[w];
      mine[k] = upto[k] = __popc(marks[k]);
      if (w0 + w < a.words) a.touched[(int64_t)r * a.words + w0 + w] = marks[k];
    }
#pragma unroll
    for (int by = 1; by < 64; by <<= 1)
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int other = __shfl_up(upto[k], by);
        if (lane >= by) upto[k] += other;
      }
    if (lane == 63)
#pragma unroll
      for (int k = 0; k < 4; ++k) s_wave[k * (kListThreads / 64) + wave] = upto[k];
    __syncthreads();
    const int in_front = before;
    static_assert(4 * (kListThreads / 64) == 64, "a sum for each lane");
    int sums = s_wave[lane];
#pragma unroll
    for (int by = 1; by < 64; by <<= 1) {
      const int other = __shfl_up(sums, by);
      if (lane >= by) sums += other;
    }
    int at[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int slot = k * (kListThreads / 64) + __builtin_amdgcn_readfirstlane(wave);
      at[k] = before + (slot > 0 ? __builtin_amdgcn_readlane(sums, max(slot - 1, 0)) : 0) + upto[k] - mine[k];
    }
    before += __builtin_amdgcn_readlane(sums, 63);
    const int here = before - in_front;
    // (more than are held: counted where they lie)
    const bool held = here <= kListHeld;
    static_assert(kChunk % 32 == 0 && kListWords * 32 % kChunk == 0, "chunks begin with words of the same time");
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int w = k * kListThreads + tid;
      if ((w0 + w) % (kChunk / 32) == 0 && w0 + w < a.words) a.starts[(int64_t)r * (a.chunks + 1) + (w0 + w) / (kChunk / 32)] = at[k];
      s_front[w] = at[k] - in_front;
      for (uint32_t bits = marks[k]; bits; bits &= bits - 1) {
        listed[at[k]] = base + w * 32 + __builtin_ctz(bits);
        if (!held) counts[at[k]] = biases[at[k]] = 0;
        ++at[k];
      }
    }
    if (held)
      for (int j = tid; j < here; j += kListThreads) s_counts[j] = s_biases[j] = 0;
    __syncthreads();
    auto place_of = [&](int token) {
      const int e = token - base;
      return s_front[e >> 5] + __popc(s_marks[e >> 5] & ((1u << (e & 31)) - 1u));
    };
    auto fill = [&](auto* to_counts, auto* to_biases) __attribute__((always_inline)) {
      for_history([&](int token, int j) {
        if (!inside(token)) return;
        if (j < prompt) atomicOr(&to_counts[place_of(token)], kSeen);
        else atomicAdd(&to_counts[place_of(token)], 1u);
      });
      if (tid < n && inside(draft)) atomicOr(&to_counts[place_of(draft)], kDrafted);
      // of several biases of a token the last: the largest number of an entry
      for (int j = tid; j < entries; j += kListThreads)
        if (inside(bias_tokens[j])) atomicMax(&to_biases[place_of(bias_tokens[j])], j + 1);
    };
    if (held) {
      fill(s_counts, s_biases);
      __syncthreads();
      for (int j = tid; j < here; j += kListThreads) {
        counts[in_front + j] = s_counts[j];
        biases[in_front + j] = s_biases[j];
      }
    } else {
      fill(counts + in_front, biases + in_front);
    }
    __syncthreads();  // (the marks are used again)
  }
  if (tid == 0) a.starts[(int64_t)r * (a.chunks + 1) + a.chunks] = before;
  // the rows of the request
  if (tid <= n) {
    const bool greedy = !(how.temperature > 0.f);
    const int64_t row = (int64_t)d0 + request + tid;
    RowInfo info;
    info.request = r;
    info.place = tid;
    info.first_draft = d0;
    info.mask = a.masks && a.mask_rows ? a.mask_rows[row] : -1;
    info.to_log2 = greedy ? 1.4426950408889634f : 1.4426950408889634f / fminf(fmaxf(how.temperature, 0x1p-100f), 0x1p100f);
    info.greedy = greedy;
    info.pad[0] = info.pad[1] = 0;
    a.rows[row - a.row_base] = info;
  }
}

// --- the rows -----------------------------------------------------------------------------------------------------------------
// What a wave knows of its row.
struct Row {
  RowInfo info;
  int64_t at;             // element of its first logit
  const uint32_t* mask;   // words of its mask (of some mask, where it has none)
  const uint32_t* marks;  // words of its request's marks
  uint32_t all, some;     // all bits where it has no mask; no bit where nothing is allowed
  float* probs;

  template <bool MASKED>
  __device__ __forceinline__ void load(const ProbsArgs& a, int row) {
    const auto* from = (const __attribute__((address_space(4))) int32_t*)(uintptr_t)(a.rows + row);  // (scalar loads)
    int32_t words[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) words[k] = from[k];
    info = RowInfo{words[0], words[1], words[2], words[3], __int_as_float(words[4]), words[5], {0, 0}};
    at = (a.row_base + row) * a.logits_stride;
    probs = a.probs + (a.row_base + row) * a.probs_stride;
    marks = a.touched + (int64_t)info.request * a.words;
    all = info.mask < 0 ? ~0u : 0u;
    some = info.mask >= 0 && info.mask >= a.num_masks ? 0u : ~0u;
    mask = nullptr;
    if constexpr (MASKED) mask = a.masks + max(min(info.mask, a.num_masks - 1), 0) * a.mask_stride;
  }
  // (one load for rows with a mask and without: a branch around it would be waited for)
  template <bool MASKED>
  __device__ __forceinline__ uint32_t allowed_word(int word) const {
    if constexpr (MASKED) return (mask[word] | all) & some;
    else return some;
  }
};

// The whole row's maximum, the reciprocal of its sum and its greedy token (-1: none), from its parts.
struct Whole {
  float top, part;
  int place;
  __device__ __forceinline__ void load(const ProbsArgs& a, int row, const RowInfo& info, int lane) {
    const PartStats* stats = a.stats + (int64_t)row * a.chunks;
    float all = -INFINITY, sum = 0.f;
    int first = INT32_MAX;
    for (int c = lane; c < a.chunks; c += 64) {
      const PartStats s = stats[c];
      const float next = fmaxf(all, s.top), from = next == -INFINITY ? 0.f : next;
      const int others = all == next ? first : INT32_MAX;
      first = s.top == next ? min(others, s.place) : others;
      sum = sum * __builtin_amdgcn_exp2f((all - from) * info.to_log2) + s.sum * __builtin_amdgcn_exp2f((s.top - from) * info.to_log2);
      all = next;
    }
    const float largest = lanes_max(all);
    top = largest == -INFINITY ? 0.f : largest;
    sum = lanes_sum(sum * __builtin_amdgcn_exp2f((all - top) * info.to_log2));
    part = sum == 0.f ? 0.f : 1.f / sum;
    place = largest > -INFINITY ? lanes_min(all == largest ? first : INT32_MAX) : -1;
  }
  __device__ __forceinline__ float probability(const RowInfo& info, float z, int token) const {
    if (info.greedy) return token == place ? 1.f : 0.f;
    return __builtin_amdgcn_exp2f((z - top) * info.to_log2) * part;
  }
};

// Maximum and sum of what a lane has seen of a row.
struct Seen {
  float top = -INFINITY, sum = 0.f;
  int place = INT32_MAX;
  template <int N>
  __device__ __forceinline__ void take(const RowInfo& info, const float (&z)[N], const int (&token)[N]) {
    if (info.greedy) {
#pragma unroll
      for (int k = 0; k < N; ++k)
        if (z[k] > top || (z[k] == top && z[k] > -INFINITY && token[k] < place)) top = z[k], place = token[k];
    } else {
      float next = top;
#pragma unroll
      for (int k = 0; k < N; ++k) next = fmaxf(next, z[k]);
      const float from = next == -INFINITY ? 0.f : next;
      sum *= __builtin_amdgcn_exp2f((top - from) * info.to_log2);
#pragma unroll
      for (int k = 0; k < N; ++k) sum += __builtin_amdgcn_exp2f((z[k] - from) * info.to_log2);
      top = next;
    }
  }
  __device__ __forceinline__ void leave(PartStats* to, const RowInfo& info, int lane) {
    const float all = lanes_max(top);
    if (info.greedy) place = lanes_min(top == all ? place : INT32_MAX);
    else sum = lanes_sum(sum * (top == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((top - all) * info.to_log2)));
    if (lane == 0) *to = PartStats{all, sum, place, 0};
  }
};

// A wave for each chunk of each row.  What its listed tokens' logits become goes through LDS to the lanes that have their places.  WRITE: the
// third kernel.  MASKED: there is a mask at least, and a number of one for each row.
template <bool BF16, bool MASKED, bool WRITE>
__global__ __launch_bounds__(kThreads) void probs_rows_kernel(const ProbsArgs a) {
#pragma clang fp contract(off)
  __shared__ __attribute__((aligned(16))) float s_z[kThreads / 64][kChunk];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int task = blockIdx.x * (kThreads / 64) + wave;
  const int index = task / a.chunks, part = task - index * a.chunks;
  if (index >= a.total) return;
  const int first = part * kChunk, end = min(first + kChunk, a.vocab);
  const bool full = end - first == kChunk;
  float* const touched = s_z[wave];
  struct Group {
    Four<BF16> x[kSteps];
    uint32_t marks[kSteps], allowed[kSteps];
  };
  Group group;
  if (full) {  // (in front of all else: nothing else has to be known for it)
    // (a wave-uniform address and the lane's place behind it)
    const char* from = static_cast<const char*>(a.logits) + ((a.row_base + index) * a.logits_stride + first) * Four<BF16>::kBytes;
#pragma unroll
    for (int s = 0; s < kSteps; ++s)
      group.x[s].x = *reinterpret_cast<const typename Four<BF16>::Words*>(from + s * (kStep * Four<BF16>::kBytes) + lane * (kPerLane * Four<BF16>::kBytes));
  }
  Row row;
  row.load<MASKED>(a, index);
  const RowInfo& info = row.info;
  Whole whole = {};
  Seen seen;

  // The chunk's listed tokens, N to a lane from entry j0 of the list on.
  const auto* starts = (const __attribute__((address_space(4))) int32_t*)(uintptr_t)(a.starts + (int64_t)info.request * (a.chunks + 1) + part);
  const int list_begin = starts[0], list_end = starts[1];
  const int64_t list_base = (int64_t)info.request * a.most_listed;
  const int request = a.req_base + info.request;
  efim_sampling_t how = {1.f, 1.f, 0.f, 0.f, 0, 0, 0, 0};
  if (a.params) how = a.params[request];
  const float* biases = a.bias_values ? a.bias_values + (int64_t)request * a.bias_stride : reinterpret_cast<const float*>(a.listed);
  auto entries_of = [](auto n) {
    struct Entries {
      int token[decltype(n)::value], entry[decltype(n)::value];
      uint32_t count[decltype(n)::value];
      float z[decltype(n)::value], bias[decltype(n)::value];
    };
    return Entries{};
  };
  constexpr auto kOne = std::integral_constant<int, 1>{};
  constexpr auto kMore = std::integral_constant<int, kListed>{};
  auto load_listed = [&](auto n_c, int j0, auto& l) __attribute__((always_inline)) {
#pragma unroll
    for (int k = 0; k < decltype(n_c)::value; ++k) {
      const int64_t j = list_base + max(min(j0 + k * 64 + lane, list_end - 1), 0);
      l.token[k] = a.listed[j];
      l.count[k] = a.counts[j];
      l.entry[k] = a.biases[j];
    }
  };
  auto load_logits = [&](auto n_c, auto& l) __attribute__((always_inline)) {
#pragma unroll
    for (int k = 0; k < decltype(n_c)::value; ++k) {
      l.z[k] = load_logit<BF16>(a.logits, row.at + l.token[k]);
      l.bias[k] = biases[max(l.entry[k] - 1, 0)];
    }
  };
  auto work_listed = [&](auto n_c, int j0, auto& l) __attribute__((always_inline)) {
#pragma unroll
    for (int k = 0; k < decltype(n_c)::value; ++k) {
      float z = l.z[k];
      uint32_t count = l.count[k];
      if (count & kDrafted) {
        count -= kDrafted;
        for (int d = 0; d < info.place; ++d) count += a.draft_tokens[info.first_draft + d] == l.token[k];
      }
      if (how.repetition != 1.f && count) z = z > 0.f ? z / how.repetition : z * how.repetition;
      count &= ~kSeen;
      const float often = how.frequency * (float)count;
      z = count ? z - often - how.presence : z;
      z = l.entry[k] ? z + l.bias[k] : z;
      if (j0 + k * 64 + lane < list_end) touched[l.token[k] - first] = z;
    }
  };
  // (what the list's first entries need is on its way beside the rest)
  auto entries = entries_of(kOne);
  if (list_begin < list_end) load_listed(kOne, list_begin, entries);
  if (full) {
    const char* marks = reinterpret_cast<const char*>(row.marks) + first / 8;
    const char* masks = reinterpret_cast<const char*>(row.mask) + first / 8;
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      group.marks[s] = *reinterpret_cast<const uint32_t*>(marks + s * (kStep / 8) + (lane / 8u) * 4u);
      if constexpr (MASKED) group.allowed[s] = *reinterpret_cast<const uint32_t*>(masks + s * (kStep / 8) + (lane / 8u) * 4u);
      else group.allowed[s] = 0;
    }
  }
  if (list_begin < list_end) load_logits(kOne, entries);
  if constexpr (WRITE) whole.load(a, index, info, lane);
  if (list_begin < list_end) work_listed(kOne, list_begin, entries);
  for (int j0 = list_begin + 64; j0 < list_end; j0 += kListed * 64) {
    auto more = entries_of(kMore);
    load_listed(kMore, j0, more);
    load_logits(kMore, more);
    work_listed(kMore, j0, more);
  }
  // (a wave's own places: the accesses are in order, the compiler is told)
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");

  if (full) {
    // (bit selects: a condition for each of the elements would be more than there are registers for conditions)
    auto all_ones = [](uint32_t bits, int k) { return (uint32_t)__builtin_amdgcn_sbfe((int)bits, k, 1); };
    const int shift = lane * kPerLane & 31;
    float z[kSteps * kPerLane];
    int tokens[kSteps * kPerLane];
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      const int token = first + s * kStep + lane * kPerLane;
      const uint32_t marked = group.marks[s] >> shift;
      const uint32_t in = MASKED ? ((group.allowed[s] | row.all) & row.some) >> shift : row.some;
      const f32x4 other = *reinterpret_cast<const f32x4*>(touched + s * kStep + lane * kPerLane);  // (whatever it is where there are no marks)
      const Four<BF16> own = group.x[s];
      uint32_t in_bits[kPerLane];
#pragma unroll
      for (int k = 0; k < kPerLane; ++k) {
        const uint32_t m = all_ones(marked, k);
        in_bits[k] = all_ones(in, k);
        const uint32_t y = (m & __float_as_uint(other[k])) | (~m & __float_as_uint(own[k]));
        z[s * kPerLane + k] = __uint_as_float((in_bits[k] & y) | (~in_bits[k] & 0xFF800000u));
        tokens[s * kPerLane + k] = token + k;
      }
      if constexpr (WRITE) {
        float p[kPerLane];
#pragma unroll
        for (int k = 0; k < kPerLane; ++k) p[k] = __uint_as_float(in_bits[k] & __float_as_uint(whole.probability(info, z[s * kPerLane + k], token + k)));
        *reinterpret_cast<f32x4*>(reinterpret_cast<char*>(row.probs + first + s * kStep) + lane * (kPerLane * 4u)) = f32x4{p[0], p[1], p[2], p[3]};
      }
    }
    if constexpr (!WRITE) seen.take(info, z, tokens);
  }
  // the vocabulary's last chunk, an element to a lane
  constexpr int kTail = 4;
  for (int at = full ? end : first + lane; at < end; at += kTail * 64) {
    float z[kTail];
    uint32_t marks[kTail], words[kTail];
    int tokens[kTail];
#pragma unroll
    for (int k = 0; k < kTail; ++k) {
      tokens[k] = min(at + k * 64, end - 1);
      z[k] = load_logit<BF16>(a.logits, row.at + tokens[k]);
      marks[k] = row.marks[tokens[k] >> 5];
      words[k] = row.allowed_word<MASKED>(tokens[k] >> 5);
    }
    bool in[kTail];
#pragma unroll
    for (int k = 0; k < kTail; ++k) {
      if (marks[k] >> (tokens[k] & 31) & 1) z[k] = touched[tokens[k] - first];
      in[k] = (words[k] >> (tokens[k] & 31) & 1) != 0;
      if (!in[k] || at + k * 64 >= end) z[k] = -INFINITY;
    }
    if constexpr (!WRITE) {
      seen.take(info, z, tokens);
    } else {
#pragma unroll
      for (int k = 0; k < kTail; ++k)
        if (at + k * 64 < end) row.probs[tokens[k]] = in[k] ? whole.probability(info, z[k], tokens[k]) : 0.f;
    }
  }
  if constexpr (!WRITE) seen.leave(a.stats + (int64_t)index * a.chunks + part, info, lane);
}

// Rows and requests of the largest launch, and what of a description can be checked on the host.
struct Sizes {
  int64_t rows = 0;
  int requests = 0, words = 0, most_listed = 0, chunks = 0;
  size_t off_rows = 0, off_touched = 0, off_listed = 0, off_counts = 0, off_biases = 0, off_starts = 0, total = 256;
};

int checked(const efim_logits_t* in, Sizes* z) {
  if (!in || in->batch < 0 || in->vocab <= 0) return EFIM_ERR_INVALID_ARG;
  if (in->vocab > kMaxVocab) return EFIM_ERR_UNSUPPORTED;
  if (in->history && in->history_stride < 0) return EFIM_ERR_INVALID_ARG;
  if (in->history && in->history_stride > kMaxHistory) return EFIM_ERR_UNSUPPORTED;
  if (!in->bias_tokens != !in->bias_values || (in->bias_tokens && in->bias_stride < 0)) return EFIM_ERR_INVALID_ARG;
  if (in->batch == 0) return EFIM_OK;
  if (!in->num_drafts) return EFIM_ERR_INVALID_ARG;
  int64_t all = 0, launch = 0;
  for (int r = 0; r < in->batch; ++r) {
    if (in->num_drafts[r] < 0) return EFIM_ERR_INVALID_ARG;
    if (in->num_drafts[r] > kMaxDrafts) return EFIM_ERR_UNSUPPORTED;
    if (r % kReqPerLaunch == 0) launch = 0;
    launch += in->num_drafts[r] + 1;
    all += in->num_drafts[r] + 1;
    if (launch > z->rows) z->rows = launch;
  }
  if (all > INT32_MAX) return EFIM_ERR_UNSUPPORTED;
  z->requests = in->batch < kReqPerLaunch ? in->batch : kReqPerLaunch;
  z->words = (in->vocab + 31) / 32;
  const int64_t most = kMaxDrafts + (in->history ? in->history_stride : 0) + (in->bias_tokens ? in->bias_stride : 0);
  z->most_listed = (int)(most < in->vocab ? most : in->vocab);
  z->chunks = (in->vocab + kChunk - 1) / kChunk;
  auto room = [&](size_t bytes) {
    const size_t at = z->total;
    z->total += (bytes + 255) / 256 * 256;
    return at;
  };
  z->total = 0;
  room((size_t)z->rows * z->chunks * sizeof(PartStats));
  z->off_rows = room((size_t)z->rows * sizeof(RowInfo));
  z->off_touched = room((size_t)z->requests * z->words * sizeof(uint32_t));
  z->off_listed = room((size_t)z->requests * z->most_listed * sizeof(int32_t));
  z->off_counts = room((size_t)z->requests * z->most_listed * sizeof(uint32_t));
  z->off_biases = room((size_t)z->requests * z->most_listed * sizeof(int32_t));
  z->off_starts = room((size_t)z->requests * (z->chunks + 1) * sizeof(int32_t));
  return EFIM_OK;
}

}  // namespace
}  // namespace efim

extern "C" {

size_t efim_logit_workspace_bytes(const efim_logits_t* in) {
  efim::Sizes sizes;
  return efim::checked(in, &sizes) == EFIM_OK ? sizes.total : 0;
}

int efim_logit_probs(const efim_logits_t* in, void* probs, int64_t probs_stride, void* workspace, size_t workspace_bytes, void* stream) {
  using namespace efim;
  Sizes sizes;
  const int rc = checked(in, &sizes);
  if (rc != EFIM_OK) return rc;
  if (in->batch == 0) return EFIM_OK;
  if (in->logits_bf16 != 0 && in->logits_bf16 != 1) return EFIM_ERR_INVALID_ARG;
  if (in->logits_stride < in->vocab || probs_stride < in->vocab) return EFIM_ERR_INVALID_ARG;
  int64_t drafts = 0;
  for (int r = 0; r < in->batch; ++r) drafts += in->num_drafts[r];
  if (!in->logits || !probs || (drafts > 0 && !in->draft_tokens)) return EFIM_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(in->logits) & (in->logits_bf16 ? 1u : 3u)) || !aligned4(probs)) return EFIM_ERR_INVALID_ARG;
  if (in->masks && (in->num_masks < 0 || in->mask_stride < (in->vocab + 31) / 32)) return EFIM_ERR_INVALID_ARG;
  for (const void* p : {(const void*)in->params, (const void*)in->history, (const void*)in->draft_tokens, (const void*)in->bias_tokens,
                        (const void*)in->bias_values, (const void*)in->masks, (const void*)in->mask_rows})
    if (!aligned4(p)) return EFIM_ERR_INVALID_ARG;
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u) || workspace_bytes < sizes.total) return EFIM_ERR_WORKSPACE;
  char* const ws = static_cast<char*>(workspace);
  ProbsArgs a;
  a.logits = in->logits;
  a.logits_stride = in->logits_stride;
  a.params = in->params;
  a.history = in->history;
  a.history_stride = in->history_stride;
  a.draft_tokens = in->draft_tokens;
  a.bias_tokens = in->bias_tokens;
  a.bias_values = in->bias_stride > 0 ? in->bias_values : nullptr;
  a.bias_stride = in->bias_stride;
  a.masks = in->masks;
  a.mask_stride = in->mask_stride;
  a.num_masks = in->num_masks;
  a.mask_rows = in->mask_rows;
  a.probs = static_cast<float*>(probs);
  a.probs_stride = probs_stride;
  a.stats = reinterpret_cast<PartStats*>(ws);
  a.rows = reinterpret_cast<RowInfo*>(ws + sizes.off_rows);
  a.touched = reinterpret_cast<uint32_t*>(ws + sizes.off_touched);
  a.listed = reinterpret_cast<int32_t*>(ws + sizes.off_listed);
  a.counts = reinterpret_cast<uint32_t*>(ws + sizes.off_counts);
  a.biases = reinterpret_cast<int32_t*>(ws + sizes.off_biases);
  a.starts = reinterpret_cast<int32_t*>(ws + sizes.off_starts);
  a.vocab = in->vocab;
  a.words = sizes.words;
  a.most_listed = sizes.most_listed;
  a.chunks = sizes.chunks;
  int32_t first = 0;
  hipStream_t s = static_cast<hipStream_t>(stream);
  for (int r0 = 0; r0 < in->batch; r0 += kReqPerLaunch) {
    const int n = in->batch - r0 < kReqPerLaunch ? in->batch - r0 : kReqPerLaunch;
    a.req_base = r0;
    a.row_base = (int64_t)first + r0;
    for (int i = 0; i < n; ++i) {
      a.first[i] = first;
      first += in->num_drafts[r0 + i];
    }
    a.first[n] = first;
    a.total = (int32_t)((int64_t)first + r0 + n - a.row_base);
    const unsigned waves = (unsigned)(a.total * a.chunks);
    const unsigned groups = (waves + kThreads / 64 - 1) / (kThreads / 64);
    probs_list_kernel<<<n, kListThreads, 0, s>>>(a);
    auto launch = [&](auto bf16, auto masked) {
      probs_rows_kernel<decltype(bf16)::value, decltype(masked)::value, false><<<groups, kThreads, 0, s>>>(a);
      probs_rows_kernel<decltype(bf16)::value, decltype(masked)::value, true><<<groups, kThreads, 0, s>>>(a);
    };
    auto by_masks = [&](auto bf16) { in->masks && in->mask_rows && in->num_masks > 0 ? launch(bf16, std::true_type{}) : launch(bf16, std::false_type{}); };
    in->logits_bf16 ? by_masks(std::true_type{}) : by_masks(std::false_type{});
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) { set_last_hip_error(e); return EFIM_ERR_LAUNCH; }
  }
  return EFIM_OK;
}

}  // extern "C"
