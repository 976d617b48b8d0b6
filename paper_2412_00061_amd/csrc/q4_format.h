// The 4-bit cache's rows: dh elements in blocks of 32 (the last one filled up with zeros), an element as sign and one of
// 0 0.5 1 1.5 2 3 4 6 in four bits, the even element in the low half of its byte; for each block one byte s: the scale 2^(s - 127), or 255
// for a block that holds no numbers.  s is the smallest with |x| <= 7 * 2^(s - 127) in the block: then every element is off by at most
// half a step of the grid, the largest ones (6 to 7) included.  From 2 to 252: every value but 0 is a normal number, exact in bf16.
#pragma once

#include "common.h"

namespace ctcspec {

constexpr int kQ4Block = 32;               // elements that share a scale
constexpr int kQ4BlockBytes = kQ4Block / 2;
constexpr int kQ4NoNumber = 255;
constexpr int kQ4MinScale = 2, kQ4MaxScale = 252;

__host__ __device__ inline int q4_blocks(int dh) { return (dh + kQ4Block - 1) / kQ4Block; }
inline bool q4_scales_aligned(const ctcspec_q4_cache* cache) {
  return ((reinterpret_cast<uintptr_t>(cache->k_scales) | reinterpret_cast<uintptr_t>(cache->v_scales)) & 3u) == 0;
}

#if defined(__HIP_DEVICE_COMPILE__)

// scale byte of a block whose largest magnitude has these bits: 7 * 2^e = 1.75 * 2^(e + 2)
__device__ __forceinline__ int q4_scale(unsigned int amax) {
  const int exponent = (int)(amax >> 23);
  if (exponent == 255) return kQ4NoNumber;
  const int s = exponent - ((amax & 0x7fffffu) <= 0x600000u ? 2 : 1);
  return s < kQ4MinScale ? kQ4MinScale : (s > kQ4MaxScale ? kQ4MaxScale : s);
}
// 2^(s - 127); for 255 an infinity, with which the conversions below give NaN
__device__ __forceinline__ float q4_scale_value(int s) { return __uint_as_float((unsigned)s << 23); }

// eight elements: nearest on the grid, of two the even code, beyond 6: 6; what rounds to 0 has no sign
__device__ __forceinline__ unsigned int q4_encode(const float (&x)[8], int s) {
  const float scale = q4_scale_value(s);
  unsigned int w = 0u;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], scale, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], scale, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], scale, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], scale, 3);
  const unsigned int some = (w | w >> 1 | w >> 2) & 0x11111111u;
  return s == kQ4NoNumber ? 0u : w & (some << 3 | 0x77777777u);
}
// what eight elements stand for, in bf16
__device__ __forceinline__ u32x4 q4_decode(unsigned int w, float scale) {
  return u32x4{__builtin_bit_cast(unsigned int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0)),
               __builtin_bit_cast(unsigned int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1)),
               __builtin_bit_cast(unsigned int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2)),
               __builtin_bit_cast(unsigned int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3))};
}
#endif

}  // namespace ctcspec
