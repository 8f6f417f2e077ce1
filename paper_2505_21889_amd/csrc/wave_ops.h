// Lane exchanges, direct copies to LDS and device-coherent accesses shared by the attention kernels.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace efim {

__device__ __forceinline__ float max3(float a, float b, float c) {
  return __builtin_fmaxf(__builtin_fmaxf(a, b), c);
}

// max / sum of a value with the one held by the lane 32 positions away (the two halves of a
// wave hold the two key halves of the same query row): one lane-swap instruction instead of
// a round trip through the LDS crossbar.
__device__ __forceinline__ float cross_half_max(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
// the same between neighbouring quarters (16 lanes) of a wave
__device__ __forceinline__ float cross_quarter_max(float v) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float cross_quarter_sum(float v) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float cross_half_sum(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Direct HBM -> LDS copy of 16 bytes per lane: lane l's data lands at lds_addr + 16 * l
// (lds_addr, the wave-uniform LDS byte address, travels in M0).  Issued as inline assembly so that the
// compiler does not order LDS reads of OTHER buffers behind it; completion is awaited
// explicitly with s_waitcnt vmcnt before the workgroup barrier that publishes the buffer.
// M0 is a reserved register that cannot be named as a clobber, so every block puts back the
// value it found: whatever the compiler keeps in M0 around the block survives it.
__device__ __forceinline__ void load_to_lds_16(const void* gptr, uint32_t lds_addr) {
  uint32_t saved_m0;
  asm volatile(
      "s_mov_b32 %0, m0\n\t"
      "s_mov_b32 m0, %1\n\t"
      "s_nop 0\n\t"
      "global_load_lds_dwordx4 %2, off\n\t"
      "s_mov_b32 m0, %0"
      : "=&s"(saved_m0)
      : "s"(__builtin_amdgcn_readfirstlane(lds_addr)), "v"(gptr)
      : "memory");
}

// The same with the address split into a wave-uniform base (scalar registers) and a 32-bit
// per-lane offset: no vector arithmetic on 64-bit addresses in front of the load.
__device__ __forceinline__ void load_to_lds_16(const void* base, uint32_t lane_off, uint32_t lds_addr) {
  uint32_t saved_m0;
  asm volatile(
      "s_mov_b32 %0, m0\n\t"
      "s_mov_b32 m0, %1\n\t"
      "s_nop 0\n\t"
      "global_load_lds_dwordx4 %2, %3\n\t"
      "s_mov_b32 m0, %0"
      : "=&s"(saved_m0)
      : "s"(__builtin_amdgcn_readfirstlane(lds_addr)), "v"(lane_off), "s"(base)
      : "memory");
}

// Four such loads of consecutive 1 KB pieces: the instruction's offset field moves both the
// global address and the LDS address, so one base and one M0 serve all four.
__device__ __forceinline__ void load_to_lds_4x16(const void* base, uint32_t off0, uint32_t off1, uint32_t off2,
                                                 uint32_t off3, uint32_t lds_addr) {
  uint32_t saved_m0;
  asm volatile(
      "s_mov_b32 %0, m0\n\t"
      "s_mov_b32 m0, %1\n\t"
      "s_nop 0\n\t"
      "global_load_lds_dwordx4 %2, %6\n\t"
      "global_load_lds_dwordx4 %3, %6 offset:1024\n\t"
      "global_load_lds_dwordx4 %4, %6 offset:2048\n\t"
      "global_load_lds_dwordx4 %5, %6 offset:3072\n\t"
      "s_mov_b32 m0, %0"
      : "=&s"(saved_m0)
      : "s"(__builtin_amdgcn_readfirstlane(lds_addr)), "v"(off0), "v"(off1), "v"(off2), "v"(off3), "s"(base)
      : "memory");
}

// N (2 or 3) such loads with one offset for all: N KB that lie as they go.
template <int N>
__device__ __forceinline__ void load_to_lds_run(const void* base, uint32_t lane_off, uint32_t lds_addr) {
  static_assert(N == 2 || N == 3, "the two forms that are written out");
  uint32_t saved_m0;
  if constexpr (N == 2)
    asm volatile(
        "s_mov_b32 %0, m0\n\t"
        "s_mov_b32 m0, %1\n\t"
        "s_nop 0\n\t"
        "global_load_lds_dwordx4 %2, %3\n\t"
        "global_load_lds_dwordx4 %2, %3 offset:1024\n\t"
        "s_mov_b32 m0, %0"
        : "=&s"(saved_m0)
        : "s"(__builtin_amdgcn_readfirstlane(lds_addr)), "v"(lane_off), "s"(base)
        : "memory");
  if constexpr (N == 3)
    asm volatile(
        "s_mov_b32 %0, m0\n\t"
        "s_mov_b32 m0, %1\n\t"
        "s_nop 0\n\t"
        "global_load_lds_dwordx4 %2, %3\n\t"
        "global_load_lds_dwordx4 %2, %3 offset:1024\n\t"
        "global_load_lds_dwordx4 %2, %3 offset:2048\n\t"
        "s_mov_b32 m0, %0"
        : "=&s"(saved_m0)
        : "s"(__builtin_amdgcn_readfirstlane(lds_addr)), "v"(lane_off), "s"(base)
        : "memory");
}

__device__ __forceinline__ void load_to_lds_2x16(const void* base, uint32_t off0, uint32_t off1, uint32_t lds_addr) {
  uint32_t saved_m0;
  asm volatile(
      "s_mov_b32 %0, m0\n\t"
      "s_mov_b32 m0, %1\n\t"
      "s_nop 0\n\t"
      "global_load_lds_dwordx4 %2, %4\n\t"
      "global_load_lds_dwordx4 %3, %4 offset:1024\n\t"
      "s_mov_b32 m0, %0"
      : "=&s"(saved_m0)
      : "s"(__builtin_amdgcn_readfirstlane(lds_addr)), "v"(off0), "v"(off1), "s"(base)
      : "memory");
}

// Two floats as one 8-byte access that is coherent across the whole device.
__device__ __forceinline__ void store_coherent(float* at, float a, float b) {
  const uint64_t bits = (uint64_t)__float_as_uint(a) | ((uint64_t)__float_as_uint(b) << 32);
  __hip_atomic_store(reinterpret_cast<uint64_t*>(at), bits, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ void store_coherent_bits(void* at, uint64_t bits) {
  __hip_atomic_store(reinterpret_cast<uint64_t*>(at), bits, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ uint64_t load_coherent_bits(const void* at) {
  return __hip_atomic_load(reinterpret_cast<const uint64_t*>(at), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ void load_coherent(const float* at, float* a, float* b) {
  const uint64_t bits = __hip_atomic_load(reinterpret_cast<const uint64_t*>(at), __ATOMIC_RELAXED,
                                          __HIP_MEMORY_SCOPE_AGENT);
  *a = __uint_as_float((uint32_t)bits);
  *b = __uint_as_float((uint32_t)(bits >> 32));
}

// A key whose row is not finite must not reach, as zero times infinity, the outputs of rows that do not see it.  Where a
// tile holds keys that some row of the wave does not see, `unfit_keys` names those whose scores are finite for none of
// the rows (as bits of the tile's 32 keys; a query row that is not finite makes its own scores so, not the others').  The
// value product then takes zeros in place of their rows.  A row that does see such a key and has it at plus infinity or no
// number gets a weight that is no number, and keeps that.  At minus infinity its weight is zero: the caller has to see to it
// that the key's infinite values still leave the row no numbers.
// ROWS 32: element r is key (r / 4) * 8 + lane / 32 * 4 + r % 4; ROWS 16: key (r / 4) * 16 + lane / 16 * 4 + r % 4.
template <int ROWS, int N>
__device__ __forceinline__ uint32_t unfit_keys(const float (&scores)[N]) {
  float probe = 0.f;
#pragma unroll
  for (int r = 0; r < N; ++r) probe = __builtin_fmaf(scores[r], 0.f, probe);
  uint32_t unfit = 0;
  if (__any(probe != probe)) {
    constexpr uint64_t kAll = ROWS == 32 ? 0xFFFFFFFFull : 0xFFFFull;
#pragma unroll
    for (int r = 0; r < N; ++r) {
      const uint64_t lanes = __ballot(!__builtin_isfinite(scores[r]));
#pragma unroll
      for (int part = 0; part < 64 / ROWS; ++part)
        if ((lanes >> (ROWS * part) & kAll) == kAll) unfit |= 1u << ((r >> 2) * (ROWS == 32 ? 8 : 16) + part * 4 + (r & 3));
    }
  }
  return unfit;
}

}  // namespace efim
