// What the kernels that append new tokens to a paged cache share: the requests of a launch as kernel arguments, and the
// place of a token in them.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "efim_internal.h"
#include "rope_math.h"
#include "wave_ops.h"

namespace efim {

constexpr int kMaxReqPerAppend = 384;  // more requests take another launch (kernel arguments end at 4 KB)

constexpr int64_t kMaxAppendTokens = (int64_t)1 << 26;  // a launch along x has fewer than 2^32 threads, 64 to a token

template <int MAXREQ>
struct AppendTable {
  int32_t cached[MAXREQ];         // C_r of the requests of this launch
  int32_t row_start[MAXREQ + 1];  // first packed row of each request, and the end
  int32_t nreq;
  int32_t tokens;                 // new tokens of this launch
  int32_t req_base;               // index of the first request (block_table row)
  int32_t max_pages;
  int32_t page_shift;             // log2 of the page size (tokens per page)
};

inline int log2_of(int power) {
  int shift = 0;
  while ((1 << shift) < power) ++shift;
  return shift;
}

// Fills the table with the requests from r0 on that fit it; *row: first packed row, moved behind them.  Returns the
// index of the first request that is left.
template <int MAXREQ>
int fill_table(const efim_batch_t* b, int r0, int64_t* row, AppendTable<MAXREQ>* t) {
  const int n = b->batch - r0 < MAXREQ ? b->batch - r0 : MAXREQ;
  const int64_t first = *row;
  for (int i = 0; i < n; ++i) {
    t->cached[i] = b->cached_len[r0 + i];
    t->row_start[i] = (int32_t)*row;
    *row += b->new_len[r0 + i];
  }
  t->row_start[n] = (int32_t)*row;
  t->nreq = n;
  t->tokens = (int32_t)(*row - first);
  t->req_base = r0;
  t->max_pages = b->max_pages_per_req;
  t->page_shift = log2_of(b->page_size);
  return r0 + n;
}

// A wave's copy of the table, 64 requests to a load: asked for early, looked into when the rows are on their way.
template <int MAXREQ>
struct TableLanes {
  int32_t starts[MAXREQ / 64], lens[MAXREQ / 64];

  __device__ __forceinline__ void load(const AppendTable<MAXREQ>& t, int lane) {
#pragma unroll
    for (int i = 0; i < MAXREQ / 64; ++i) {
      const int r = i * 64 + lane;
      starts[i] = t.row_start[min(r, t.nreq)];
      lens[i] = t.cached[min(r, t.nreq - 1)];
    }
  }
  // Request (of the launch) of a packed row -- the last one that starts at or in front of it -- and its position.
  __device__ __forceinline__ void find(const AppendTable<MAXREQ>& t, int lane, int row, int* req_out, int* pos_out) const {
    int req = -1;
#pragma unroll
    for (int i = 0; i < MAXREQ / 64; ++i)
      req += __popcll(__ballot(i * 64 + lane < t.nreq && starts[i] <= row));
    int pos = 0;
#pragma unroll
    for (int i = 0; i < MAXREQ / 64; ++i)
      if (MAXREQ == 64 || req >> 6 == i)
        pos = __builtin_amdgcn_readlane(lens[i], req & 63) + row - __builtin_amdgcn_readlane(starts[i], req & 63);
    *req_out = req;
    *pos_out = pos;
  }
};

typedef uint32_t append_chunk __attribute__((ext_vector_type(4)));  // eight bf16 values

// The eight values of a chunk (two to a word, the lower half first), and back.
__device__ __forceinline__ void widen(append_chunk w, float (&x)[8]) {
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    x[2 * t] = __uint_as_float(w[t] << 16);
    x[2 * t + 1] = __uint_as_float(w[t] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ append_chunk narrow(const float (&x)[8]) {
  append_chunk w;
#pragma unroll
  for (int t = 0; t < 4; ++t) w[t] = pack_bf16(x[2 * t], x[2 * t + 1]);
  return w;
}

// Rotation in fp32 of the eight pairs of a unit, in place: (x[t], y[t]) by the angle with cosine c[t] and sine s[t].
__device__ __forceinline__ void rotate_pairs_f32(float (&x)[8], float (&y)[8], const float (&c)[8], const float (&s)[8]) {
#pragma unroll
  for (int t = 0; t < 8; ++t) {
    const float a = x[t], b = y[t];
    x[t] = a * c[t] - b * s[t];
    y[t] = b * c[t] + a * s[t];
  }
}

// The same for interleaved pairs: x and y are 16 consecutive elements, pair t the elements 2t and 2t + 1.
__device__ __forceinline__ void rotate_interleaved_f32(float (&x)[8], float (&y)[8], const float (&c)[8], const float (&s)[8]) {
  float u[8], v[8];
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    u[t] = x[2 * t];
    v[t] = x[2 * t + 1];
    u[t + 4] = y[2 * t];
    v[t + 4] = y[2 * t + 1];
  }
  rotate_pairs_f32(u, v, c, s);
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    x[2 * t] = u[t];
    x[2 * t + 1] = v[t];
    y[2 * t] = u[t + 4];
    y[2 * t + 1] = v[t + 4];
  }
}

// Sum over N (4, 8 or 64) neighbouring lanes, in all of them and in one order.
template <int N>
__device__ __forceinline__ float group_sum(float v) {
  auto with = [&](auto ctrl) {
    return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), decltype(ctrl)::value, 0xf, 0xf, true));
  };
  v += with(std::integral_constant<int, 0xB1>{});                        // quad_perm [1, 0, 3, 2]
  v += with(std::integral_constant<int, 0x4E>{});                        // quad_perm [2, 3, 0, 1]
  if constexpr (N >= 8) v += with(std::integral_constant<int, 0x141>{});  // row_half_mirror
  if constexpr (N == 64) {
    v += with(std::integral_constant<int, 0x140>{});                     // row_mirror
    v = cross_half_sum(cross_quarter_sum(v));
  }
  return v;
}

}  // namespace efim
