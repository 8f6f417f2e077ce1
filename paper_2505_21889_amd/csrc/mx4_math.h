// 4-bit floating point in blocks (OCP MXFP4) as used for the 4-bit KV cache: 32 neighbouring elements of a head row share a scale
// 2^s, stored as the byte s + 127, and are 2^s times an E2M1 number (0, 0.5, 1, 1.5, 2, 3, 4, 6 and a sign), two to a byte, the
// first in the lower half.
#pragma once
#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

namespace efim {

constexpr int kMx4Block = 32;
constexpr int kMx4Nan = 255;  // scale byte of a block whose elements are no numbers

// Bytes of a head row's codes, of its scales, and of both.  A page of one head is its rows' codes and behind them their scales.
__host__ __device__ constexpr int mx4_code_bytes(int head_dim) { return head_dim / 2; }
__host__ __device__ constexpr int mx4_scale_bytes(int head_dim) { return head_dim / kMx4Block; }
__host__ __device__ constexpr int mx4_row_bytes(int head_dim) { return mx4_code_bytes(head_dim) + mx4_scale_bytes(head_dim); }

// Scale byte of a block from the bit pattern of its largest bf16 magnitude: the least s with max <= 7 * 2^s.  7 is the middle
// between the largest code, 6, and the 8 that would follow it, so the largest element too is at most half a step off.  (With
// max < 8 * 2^s, the format's plain rule, it is up to a whole one.)  Kept where every product of a code and the scale is a normal
// bf16 number.
__device__ __forceinline__ uint32_t mx4_scale_of(uint32_t largest) {
  if (largest >= 0x7F80u) return kMx4Nan;
  const int s = (int)(largest >> 7) - 2 + ((largest & 0x7Fu) > 0x60u);
  return (uint32_t)min(max(s, 2), 252);
}
__device__ __forceinline__ float mx4_scale_value(uint32_t byte) { return __uint_as_float(byte << 23); }

// Codes of eight bf16 values under a scale: nearest, ties to the even code, saturating (the instruction's own rounding, which
// was compared with the definition on every bf16 number).
typedef uint32_t mx4_words __attribute__((ext_vector_type(4)));
__device__ __forceinline__ uint32_t mx4_encode8(mx4_words x, float scale) {
  typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
  const bf16x8 v = __builtin_bit_cast(bf16x8, x);
  uint32_t codes = 0;
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, __builtin_shufflevector(v, v, 0, 1), scale, 0);
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, __builtin_shufflevector(v, v, 2, 3), scale, 1);
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, __builtin_shufflevector(v, v, 4, 5), scale, 2);
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, __builtin_shufflevector(v, v, 6, 7), scale, 3);
  return codes;
}

// What eight codes stand for, in bf16, exactly; a scale of byte 255 makes them no numbers.
__device__ __forceinline__ mx4_words mx4_decode8(uint32_t codes, float scale) {
  mx4_words x;
  x[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0));
  x[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1));
  x[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2));
  x[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3));
  return x;
}

}  // namespace efim
