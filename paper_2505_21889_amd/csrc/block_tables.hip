// efim_block_tables: the block tables and the slot map of a step from its requests' lengths, which lie on the device.  Pages behind
// a request's end go back onto the stack of free pages, missing ones are taken from its top.
//
// Bound by latency: a scan over the requests, and behind it the entries, which depend on each other only through the stack.  One launch
// for up to 64 requests: 16 of them with a token each 3.5 us (6.3 with the call), 64 with whole prompts among them 4.8 (6.4); as the scan
// and the filling apart 14.1 and 17.6 with the call.  More requests, the scan and the filling: 65 to 256 with a token each 11.1 with the
// call, 1024 12.3, 96 with 24 prompts among them 14.6.  (The scan's workgroup filling too takes 10.2 for 65, 11.1 for 96 and 12.3 for 128: not
// worth a kernel.)
#include <cstdint>

#include "efim_internal.h"

namespace efim {
namespace {

constexpr int kScanThreads = 1024;
constexpr int kFillThreads = 256;

struct TablesArgs {
  const int32_t *held, *cached, *new_len;
  int32_t batch, page_shift, max_pages;
  int64_t capacity;        // of the stack
  int32_t* block_table;
  int32_t* free_pages;
  const int32_t* free_count;
  int32_t* free_count_out;
  int64_t* slots;
  int64_t slot_capacity;
  int32_t* row_start;
  int32_t* status;
  int64_t* plan;           // [0] pages on the stack before any is taken, or -1: nothing changes; [1 + r] pages taken in front of request r,
                           // [1 + batch + r] pages returned in front of it
};

struct Request {
  int64_t held, wanted;  // pages
  int64_t cached, new_len;
  bool ok;
  __device__ __forceinline__ Request(const TablesArgs& a, int r) {
    const int64_t h = a.held[r];
    cached = a.cached[r];
    new_len = a.new_len[r];
    const int64_t round = (1 << a.page_shift) - 1;
    held = (h + round) >> a.page_shift;
    wanted = (cached + new_len + round) >> a.page_shift;
    ok = h >= 0 && cached >= 0 && new_len >= 0 && held <= a.max_pages && wanted <= a.max_pages;
  }
  __device__ __forceinline__ int64_t taken() const { return wanted > held ? wanted - held : 0; }
  __device__ __forceinline__ int64_t returned() const { return held > wanted ? held - wanted : 0; }
};

struct Sums {
  int64_t taken, returned, tokens;
};
__device__ __forceinline__ int64_t shuffle_up(int64_t v, int by) {
  return (int64_t)((uint64_t)(uint32_t)__shfl_up((int)(uint32_t)v, by) | (uint64_t)(uint32_t)__shfl_up((int)(v >> 32), by) << 32);
}

// Entries and slots of a request, by `threads` threads of which this is number `t`.
__device__ __forceinline__ void fill_request(const TablesArgs& a, int r, int64_t stacked, int64_t taken_before, int64_t first, int t, int threads) {
  const Request q(a, r);
  int32_t* row = a.block_table + (int64_t)r * a.max_pages;
  const int64_t top = stacked - 1 - taken_before;  // of the stack for this request
  for (int64_t j = t; j < q.taken(); j += threads) row[q.held + j] = a.free_pages[top - j];
  if (!a.slots) return;
  for (int64_t j = t; j < q.new_len; j += threads) {
    const int64_t pos = q.cached + j, column = pos >> a.page_shift;
    const int64_t page = column < q.held ? row[column] : a.free_pages[top - (column - q.held)];
    a.slots[first + j] = (page << a.page_shift) + (pos & ((1 << a.page_shift) - 1));
  }
}

__global__ __launch_bounds__(kScanThreads) void tables_scan_kernel(const TablesArgs a) {
  __shared__ Sums s_wave[kScanThreads / 64];
  __shared__ int32_t s_bad;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  if (tid == 0) s_bad = 0;
  const int64_t count = *a.free_count;
  __syncthreads();
  // Two rounds over the requests: the sums decide whether anything changes, then the places.
  Sums all = {0, 0, 0};
  bool ok = true, counted = true;
  for (int round = 0; round < 2; ++round) {
    int64_t missing = 0;
    if (round == 1) {
      counted = !s_bad && all.tokens <= INT32_MAX;
      ok = counted && count >= 0 && count + all.returned <= a.capacity && (!a.slots || all.tokens <= a.slot_capacity);
      missing = all.taken - count - all.returned;
      if (tid == 0) {
        *a.status = !ok ? EFIM_ERR_INVALID_ARG : missing > 0 ? (int32_t)min(missing, (int64_t)INT32_MAX) : 0;
        ok = ok && missing <= 0;
        a.plan[0] = ok ? count + all.returned : -1;
        *a.free_count_out = (int32_t)(ok ? count + all.returned - all.taken : count);
      }
      ok = ok && missing <= 0;
    }
    Sums front = {0, 0, 0};
    for (int r0 = 0; r0 < a.batch; r0 += kScanThreads) {
      const int r = r0 + tid;
      Sums mine = {0, 0, 0};
      if (r < a.batch) {
        const Request q(a, r);
        if (q.ok) mine = Sums{q.taken(), q.returned(), q.new_len};
        else s_bad = 1;
      }
      Sums upto = mine;
#pragma unroll
      for (int by = 1; by < 64; by <<= 1) {
        const Sums other = {shuffle_up(upto.taken, by), shuffle_up(upto.returned, by), shuffle_up(upto.tokens, by)};
        if (lane >= by) {
          upto.taken += other.taken;
          upto.returned += other.returned;
          upto.tokens += other.tokens;
        }
      }
      __syncthreads();
      if (lane == 63) s_wave[wave] = upto;
      __syncthreads();
      Sums before = front;
#pragma unroll 4  // (all sixteen waves' sums at once do not fit the registers of so many threads)
      for (int w = 0; w < kScanThreads / 64; ++w) {
        if (w < wave) {
          before.taken += s_wave[w].taken;
          before.returned += s_wave[w].returned;
          before.tokens += s_wave[w].tokens;
        }
        front.taken += s_wave[w].taken;
        front.returned += s_wave[w].returned;
        front.tokens += s_wave[w].tokens;
      }
      if (round == 1 && r < a.batch) {
        a.plan[1 + r] = before.taken + upto.taken - mine.taken;
        a.plan[1 + a.batch + r] = before.returned + upto.returned - mine.returned;
        a.row_start[r] = counted ? (int32_t)(before.tokens + upto.tokens - mine.tokens) : 0;
      }
    }
    all = front;
    __syncthreads();
  }
  if (tid == 0) a.row_start[a.batch] = counted ? (int32_t)all.tokens : 0;
  // returned pages, a request to a wave at a time
  __threadfence_block();
  __syncthreads();
  if (ok && all.returned > 0)
    for (int r = wave; r < a.batch; r += kScanThreads / 64) {
      const Request q(a, r);
      const int32_t* row = a.block_table + (int64_t)r * a.max_pages + q.wanted;
      int32_t* to = a.free_pages + count + a.plan[1 + a.batch + r];
      for (int64_t j = lane; j < q.returned(); j += 64) to[j] = row[j];
    }
}

// Workgroup x of the first `batch` has a request; the others the slots behind the last token.
__global__ __launch_bounds__(kFillThreads) void tables_fill_kernel(const TablesArgs a) {
  const int64_t stacked = a.plan[0];
  const int r = blockIdx.x, t = blockIdx.y * kFillThreads + threadIdx.x, threads = gridDim.y * kFillThreads;
  if (r < a.batch) {
    if (stacked >= 0) fill_request(a, r, stacked, a.plan[1 + r], a.row_start[r], t, threads);
  } else if (a.slots) {
    for (int64_t at = (stacked >= 0 ? a.row_start[a.batch] : 0) + t; at < a.slot_capacity; at += threads) a.slots[at] = -1;
  }
}

// Up to 64 requests, one launch: every wave reads all lengths, a lane each, and sums them by lane exchanges, so that a workgroup
// (a request's, in slices; the last ones have the slots behind the last token) needs no answer of another.  A page that is taken in
// the step in which it comes back is looked up in the row that gives it.  The counts are two words: workgroups read the one while
// another writes the other.
__global__ __launch_bounds__(kFillThreads) void tables_small_kernel(const TablesArgs a) {
  __shared__ int64_t s_taken[64], s_returned[64], s_first[65];
  __shared__ int64_t s_wanted[64];
  const int lane = threadIdx.x & 63;
  const int64_t count = *a.free_count;
  const int r = min(lane, a.batch - 1);
  const Request q(a, r);
  const bool mine = lane < a.batch;
  const bool bad = __any(mine && !q.ok);
  int64_t taken = mine && q.ok ? q.taken() : 0, returned = mine && q.ok ? q.returned() : 0, tokens = mine && q.ok ? q.new_len : 0;
  const int64_t own_taken = taken, own_returned = returned, own_tokens = tokens;
  // (sums of 64 numbers below 2^24 stay within 32 bits: three exchanges a step instead of six)
  if (!__any((taken | returned | tokens) >> 24)) {
    uint32_t x = (uint32_t)taken, y = (uint32_t)returned, z = (uint32_t)tokens;
#pragma unroll
    for (int by = 1; by < 64; by <<= 1) {
      const uint32_t u = __shfl_up(x, by), v = __shfl_up(y, by), w = __shfl_up(z, by);
      if (lane >= by) x += u, y += v, z += w;
    }
    taken = x, returned = y, tokens = z;
  } else {
#pragma unroll
    for (int by = 1; by < 64; by <<= 1) {
      const int64_t u = shuffle_up(taken, by), v = shuffle_up(returned, by), w = shuffle_up(tokens, by);
      if (lane >= by) taken += u, returned += v, tokens += w;
    }
  }
  auto last = [](int64_t v) {
    return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, 63) | (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), 63) << 32);
  };
  const int64_t all_taken = last(taken), all_returned = last(returned), all_tokens = last(tokens);
  const bool counted = !bad && all_tokens <= INT32_MAX;
  const bool fits = counted && count >= 0 && count + all_returned <= a.capacity && (!a.slots || all_tokens <= a.slot_capacity);
  const int64_t missing = all_taken - count - all_returned;
  const bool ok = fits && missing <= 0;
  if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x < 64) {
    if (mine) a.row_start[lane] = counted ? (int32_t)(tokens - own_tokens) : 0;
    if (lane == 0) {
      a.row_start[a.batch] = counted ? (int32_t)all_tokens : 0;
      *a.status = !fits ? EFIM_ERR_INVALID_ARG : missing > 0 ? (int32_t)min(missing, (int64_t)INT32_MAX) : 0;
      *a.free_count_out = (int32_t)(ok ? count + all_returned - all_taken : count);
    }
  }
  const int t = blockIdx.y * kFillThreads + threadIdx.x, threads = gridDim.y * kFillThreads;
  if ((int)blockIdx.x == a.batch || !ok) {
    if (a.slots && (int)blockIdx.x == a.batch)
      for (int64_t at = (ok ? all_tokens : 0) + t; at < a.slot_capacity; at += threads) a.slots[at] = -1;
    return;
  }
  if (threadIdx.x < 64) {
    s_taken[lane] = taken - own_taken;
    s_returned[lane] = returned - own_returned;
    s_first[lane] = tokens - own_tokens;
    s_wanted[lane] = q.wanted;
  }
  __syncthreads();
  const int me = blockIdx.x;
  const Request my(a, me);
  int32_t* row = a.block_table + (int64_t)me * a.max_pages;
  int32_t* to = a.free_pages + count + s_returned[me];
  for (int64_t j = t; j < my.returned(); j += threads) to[j] = row[my.wanted + j];
  // the page at a place of the stack as it is when all have come back
  auto stacked = [&](int64_t place) {
    if (place < count) return a.free_pages[place];
    int from = 0;  // the last request with pages in front of or at the place
    for (int by = 32; by > 0; by >>= 1)
      if (from + by < a.batch && s_returned[from + by] <= place - count) from += by;
    return a.block_table[(int64_t)from * a.max_pages + s_wanted[from] + (place - count - s_returned[from])];
  };
  const int64_t top = count + all_returned - 1 - s_taken[me];
  for (int64_t j = t; j < my.taken(); j += threads) row[my.held + j] = stacked(top - j);
  if (!a.slots) return;
  for (int64_t j = t; j < my.new_len; j += threads) {
    const int64_t pos = my.cached + j, column = pos >> a.page_shift;
    const int64_t page = column < my.held ? row[column] : stacked(top - (column - my.held));
    a.slots[s_first[me] + j] = (page << a.page_shift) + (pos & ((1 << a.page_shift) - 1));
  }
}

__global__ void tables_count_kernel(const int32_t* from, int32_t* to) { *to = *from; }

size_t tables_bytes(int batch) {
  const size_t bytes = (2 * (size_t)batch + 1) * sizeof(int64_t);
  return bytes < 256 ? 256 : bytes;
}

}  // namespace
}  // namespace efim

extern "C" {

size_t efim_block_tables_workspace_bytes(int batch) { return batch < 0 ? 0 : efim::tables_bytes(batch); }

int efim_block_tables(int batch, const int32_t* held_len, const int32_t* cached_len, const int32_t* new_len, int page_size,
                      int32_t* block_table, int max_pages_per_req, int32_t* free_pages, int64_t free_capacity,
                      const int32_t* free_count, int32_t* free_count_out, int64_t* slot_map, int64_t slot_capacity,
                      int32_t* row_start, int32_t* status, void* workspace, size_t workspace_bytes, void* stream) {
  using namespace efim;
  if (batch < 0 || max_pages_per_req < 0 || free_capacity < 0 || free_capacity > INT32_MAX || (slot_map && slot_capacity < 0))
    return EFIM_ERR_INVALID_ARG;
  if (page_size < kMinPageSize || page_size > kMaxPageSize || (page_size & (page_size - 1)) != 0) return EFIM_ERR_UNSUPPORTED;
  if (batch > (1 << 20)) return EFIM_ERR_UNSUPPORTED;
  if (!free_count || !free_count_out || !row_start || !status || (batch > 0 && (!held_len || !cached_len || !new_len)) ||
      (batch > 0 && max_pages_per_req > 0 && !block_table) || (free_capacity > 0 && !free_pages))
    return EFIM_ERR_INVALID_ARG;
  for (const void* p : {(const void*)held_len, (const void*)cached_len, (const void*)new_len, (const void*)block_table, (const void*)free_pages,
                        (const void*)free_count, (const void*)free_count_out, (const void*)row_start, (const void*)status})
    if (!aligned4(p)) return EFIM_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(slot_map) & 7u) return EFIM_ERR_INVALID_ARG;
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u) || workspace_bytes < tables_bytes(batch)) return EFIM_ERR_WORKSPACE;
  TablesArgs a;
  a.held = held_len;
  a.cached = cached_len;
  a.new_len = new_len;
  a.batch = batch;
  a.page_shift = 0;
  while ((1 << a.page_shift) < page_size) ++a.page_shift;
  a.max_pages = max_pages_per_req;
  a.capacity = free_capacity;
  a.block_table = block_table;
  a.free_pages = free_pages;
  a.free_count = free_count;
  a.free_count_out = free_count_out;
  a.slots = slot_map;
  a.slot_capacity = slot_map ? slot_capacity : 0;
  a.row_start = row_start;
  a.status = status;
  a.plan = static_cast<int64_t*>(workspace);
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (batch > 0 && batch <= 64) {
    // (one word for both counts: the new one waits in the workspace until all have read the old one)
    const bool same = free_count == free_count_out;
    if (same) a.free_count_out = static_cast<int32_t*>(workspace);
    // two of the mean request's tokens to a thread at most (a thread's slots wait for their pages one behind the other: 80k tokens
    // of 64 requests with eight to a thread 10 us)
    const int64_t slices = (a.slot_capacity / batch * 2 + kFillThreads - 1) / kFillThreads;
    tables_small_kernel<<<dim3((unsigned)batch + 1, (unsigned)(slices < 1 ? 1 : slices > 16 ? 16 : slices)), kFillThreads, 0, s>>>(a);
    if (same) tables_count_kernel<<<1, 1, 0, s>>>(static_cast<const int32_t*>(workspace), free_count_out);
  } else {
    tables_scan_kernel<<<1, kScanThreads, 0, s>>>(a);
    tables_fill_kernel<<<dim3((unsigned)batch + 1, 4), kFillThreads, 0, s>>>(a);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) { set_last_hip_error(e); return EFIM_ERR_LAUNCH; }
  return EFIM_OK;
}

}  // extern "C"
