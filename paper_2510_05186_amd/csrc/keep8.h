// Values kept in 8 bits: e4m3 codes, 32 consecutive values of a row under one power of two.
//
// A block's scale byte b stands for 2^(b - 127): the least power 2^k, -117 <= k <= 119, with max |x| <= 448 * 2^k over the block's finite
// values; a code is x * 2^-k rounded to e4m3 (ties to even).  448 is the largest e4m3 value, so nothing saturates but what k = 119
// leaves above it (|x| > 1.75 * 2^127, kept as that).  Scaling by a power of two is exact, so that a kept value is off by at most half an
// e4m3 step (2^-4 of the value, 2^(k - 10) below 2^(k - 6)), depends on nothing but its block, and is itself a bf16 and an fp32 number: 4
// significant bits, and at least 2^-9 * 2^-117 = 2^-126 where it is not zero, the least normal number.  A value that is not
// finite is kept as NaN (e4m3 has no infinity) and does not count for the maximum.
#pragma once
#include "common.h"

constexpr int KEEP_BLOCK = 32;
__host__ __device__ inline int keep_blocks(int cols) { return (cols + KEEP_BLOCK - 1) / KEEP_BLOCK; }

// the scale byte for the largest |x| of a block, given as fp32 bits
__device__ __forceinline__ uint32_t keep_scale_byte(uint32_t most) {
  const int b = (int)(most >> 23) - 8 + ((most & 0x7fffffu) > 0x600000u ? 1 : 0);
  return (uint32_t)min(max(b, 10), 246);
}
__device__ __forceinline__ float keep_scale(uint32_t byte) { return __uint_as_float(byte << 23); }
__device__ __forceinline__ float keep_inverse(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }

// bits of |x| where x counts for the maximum, else 0
__device__ __forceinline__ uint32_t keep_magnitude(float x) {
  const uint32_t a = __float_as_uint(x) & 0x7fffffffu;
  return a < 0x7f800000u ? a : 0u;
}
__device__ __forceinline__ uint32_t keep_encode(float x, float inverse) {
  const uint32_t bits = __float_as_uint(x);
  if ((bits & 0x7fffffffu) >= 0x7f800000u) return 0x7fu | (bits >> 31 << 7);
  const float y = fminf(fmaxf(x * inverse, -448.f), 448.f);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y, 0.f, 0, false) & 0xffu;
}
__device__ __forceinline__ float keep_decode(uint32_t code, float scale) { return __builtin_amdgcn_cvt_f32_fp8((int)code, 0) * scale; }
