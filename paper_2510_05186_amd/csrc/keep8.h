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

// 16 bytes of T and their codes; the lanes whose chunks make up a block are next to each other, their number a divisor of 16
template <typename T> struct KeepChunk;
template <> struct KeepChunk<bf16_t> {
  typedef uint2 codes_t;
  static constexpr int LANES = 4;
};
template <> struct KeepChunk<float> {
  typedef uint32_t codes_t;
  static constexpr int LANES = 8;
};
template <int CTRL> __device__ __forceinline__ uint32_t lane_swap(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true); }
// The sum over G lanes side by side (a power of two from 4 to 64), in all of them: lane swaps, no LDS
template <int G> __device__ __forceinline__ float lanes_sum(float v) {
  v += __uint_as_float(lane_swap<0xB1>(__float_as_uint(v)));          // lane ^ 1
  v += __uint_as_float(lane_swap<0x4E>(__float_as_uint(v)));          // lane ^ 2
  if (G >= 8) v += __uint_as_float(lane_swap<0x141>(__float_as_uint(v)));    // 7 - lane of eight
  if (G >= 16) v += __uint_as_float(lane_swap<0x140>(__float_as_uint(v)));   // 15 - lane of sixteen
  if (G >= 32) {
    const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(p[0]) + __uint_as_float(p[1]);
  }
  if (G >= 64) {
    const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(p[0]) + __uint_as_float(p[1]);
  }
  return v;
}
template <typename T> __device__ __forceinline__ uint32_t keep_block_max(uint32_t v) {
  v = max(v, lane_swap<0xB1>(v));                                     // lane ^ 1
  v = max(v, lane_swap<0x4E>(v));                                     // lane ^ 2
  if (KeepChunk<T>::LANES == 8) v = max(v, lane_swap<0x141>(v));      // 7 - lane of eight
  return v;
}
// largest |x| of a chunk as fp32 bits, what is not finite included
__device__ __forceinline__ uint32_t keep_most(const Vec16<bf16_t>& v) {
  typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
  typedef unsigned short u16x2_t __attribute__((ext_vector_type(2)));
  const u32x4_t w = __builtin_bit_cast(u32x4_t, v.v) & 0x7fff7fffu;
  const uint32_t w0 = w[0], w1 = w[1], w2 = w[2], w3 = w[3];           // bit_cast of an element itself takes element 0 whichever is named
  const u16x2_t m = __builtin_elementwise_max(__builtin_elementwise_max(__builtin_bit_cast(u16x2_t, w0), __builtin_bit_cast(u16x2_t, w1)),
                                              __builtin_elementwise_max(__builtin_bit_cast(u16x2_t, w2), __builtin_bit_cast(u16x2_t, w3)));
  return (uint32_t)max(m[0], m[1]) << 16;
}
__device__ __forceinline__ uint32_t keep_most(const Vec16<float>& v) {
  uint32_t m = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) m = max(m, __float_as_uint(v.v[e]) & 0x7fffffffu);
  return m;
}
// the conversion with a power of two, two values at a time (what it gives for NaN, infinities and values beyond 448 is not used)
__device__ __forceinline__ uint2 keep_encode(const Vec16<bf16_t>& v, float scale) {
  typedef short s16x2_t __attribute__((ext_vector_type(2)));
  typedef bf16_t bf16x2_t __attribute__((ext_vector_type(2)));
  s16x2_t lo = {0, 0}, hi = {0, 0};
  lo = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(lo, (bf16x2_t){v.v[0], v.v[1]}, scale, false);
  lo = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(lo, (bf16x2_t){v.v[2], v.v[3]}, scale, true);
  hi = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(hi, (bf16x2_t){v.v[4], v.v[5]}, scale, false);
  hi = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(hi, (bf16x2_t){v.v[6], v.v[7]}, scale, true);
  return make_uint2(__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi));
}
__device__ __forceinline__ uint32_t keep_encode(const Vec16<float>& v, float scale) {
  typedef short s16x2_t __attribute__((ext_vector_type(2)));
  s16x2_t c = {0, 0};
  c = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(c, v.v[0], v.v[1], scale, false);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(c, v.v[2], v.v[3], scale, true);
  return __builtin_bit_cast(uint32_t, c);
}
__device__ __forceinline__ void keep_put(uint2& c, int e, uint32_t code) { (e < 4 ? c.x : c.y) |= code << 8 * (e & 3); }
__device__ __forceinline__ void keep_put(uint32_t& c, int e, uint32_t code) { c |= code << 8 * e; }

// A chunk's codes and its block's scale byte.  Every lane of the block calls this, those behind the row's end with zeros.
template <typename T> __device__ __forceinline__ typename KeepChunk<T>::codes_t keep_chunk(const Vec16<T>& v, uint32_t& byte) {
  uint32_t most = keep_block_max<T>(keep_most(v));
  if (__builtin_expect(!__any(most > 0x7f600000u), 1)) {              // all finite, at most 448 * 2^119
    byte = keep_scale_byte(most);
    return keep_encode(v, keep_scale(byte));
  }
  most = 0;
#pragma unroll
  for (int e = 0; e < Vec16<T>::N; ++e) most = max(most, keep_magnitude(v.get(e)));
  byte = keep_scale_byte(keep_block_max<T>(most));
  const float inverse = keep_inverse(byte);
  typename KeepChunk<T>::codes_t c = {};
#pragma unroll
  for (int e = 0; e < Vec16<T>::N; ++e) keep_put(c, e, keep_encode(v.get(e), inverse));
  return c;
}

// the values that a chunk's codes stand for
__device__ __forceinline__ void keep_values(uint2 c, float scale, float* v) {
  typedef float f32x2_t __attribute__((ext_vector_type(2)));
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t w = i < 2 ? c.x : c.y;
    const f32x2_t p = (i & 1) ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, scale, true) : __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, scale, false);
    v[2 * i] = p[0];
    v[2 * i + 1] = p[1];
  }
}
__device__ __forceinline__ void keep_values(uint32_t c, float scale, float* v) {
  typedef float f32x2_t __attribute__((ext_vector_type(2)));
  const f32x2_t lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c, scale, false), hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c, scale, true);
  v[0] = lo[0];
  v[1] = lo[1];
  v[2] = hi[0];
  v[3] = hi[1];
}
__device__ __forceinline__ Vec16<bf16_t> keep_stored(uint2 c, float scale, Vec16<bf16_t>) {
  typedef bf16_t bf16x2_t __attribute__((ext_vector_type(2)));
  Vec16<bf16_t> v;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t w = i < 2 ? c.x : c.y;
    const bf16x2_t p = (i & 1) ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, false);
    v.v[2 * i] = p[0];
    v.v[2 * i + 1] = p[1];
  }
  return v;
}
__device__ __forceinline__ Vec16<float> keep_stored(uint32_t c, float scale, Vec16<float>) {
  float f[4];
  keep_values(c, scale, f);
  Vec16<float> v;
#pragma unroll
  for (int e = 0; e < 4; ++e) v.v[e] = f[e];
  return v;
}
