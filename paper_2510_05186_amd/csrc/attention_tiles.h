// What the matrix-unit attention kernels share: the geometry of a tile of rows in LDS by head size, fragments of probabilities, sums that two groups of
// waves hold.  The register and LDS scheme itself stands in attention_mfma.hip.
#pragma once
#include "common.h"

namespace {

constexpr float LOG2E = 1.4426950408889634f;

typedef int i32x4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) void lds_void_t;
typedef __attribute__((address_space(3))) bf16x8_t lds_bf16x8_t;
typedef __attribute__((address_space(3))) f32x4_t lds_f32x4_t;

// What depends on the head size: rows of ROWB bytes = CH 16-byte chunks in the LDS tiles of 64 rows, NKS k-steps of an MFMA over
// a row, NDT 32-wide pieces of it, NLD loads of 1 KB (RPL rows) by which a wave fills its quarter of a tile.
// SPLIT: the probabilities and dS, fp32 numbers, enter the second product as the sum of two bf16 numbers (16 significant bits
// between them, a rounding of 2^-17 at most) and not as one.  The general kernels multiply them in fp32; the error against 64
// bits is no larger here (o 1.6e-3, dqkv 1.8e-3: the rounding of the results), where one bf16 number would raise it by a quarter.
// The exponentials themselves are v_exp_f32 (1 ulp) of x = c s - c m rounded once, |x| 2^-24: p is off by at most 2^-23 +
// 0.7 |x| 2^-24 of itself, as expf of a rounded difference is.
// Measured for heads of 64 at 4 x 1024 tokens, 16 heads, forward and backward: 4466 us on the general kernels (one wave per row,
// no matrix unit), 97 us here.
template <int D> struct Head {
  static constexpr int ROWB = 2 * D, TILE = 64 * ROWB, CH = D / 8, NKS = D / 16, NDT = D / 32, RPL = 64 / CH, NLD = 16 / RPL;
  static constexpr bool SPLIT = D == 64;
  // rows with a result that is not finite are redone one by one (needs all of a key's queries in one workgroup: split == 1);
  // ROW_LDS: bytes of LDS that they need behind the tiles, two rows of fp32 per wave
  static constexpr bool ROW_EXACT = D == 64;
  static constexpr int ROW_LDS = ROW_EXACT ? 4 * 2 * D * 4 : 0;
  // 16-byte chunk c of tile row r is stored at chunk c ^ swz(r).  Row reads: the 16 rows that a pass touches at one chunk fall on
  // all banks; transposing reads: the 4 rows of one differ in the 64-byte group (D = 64: so do rows two apart, which share
  // the half of the 256-byte bank window)
  __device__ __forceinline__ static constexpr int swz(int r) {
    return D == 128 ? ((r & 3) << 2) | ((r >> 2) & 3) : (((r >> 1) & 1) << 2) | (((r >> 2) & 1) << 1) | ((r >> 3) & 1);
  }
};

__device__ __forceinline__ bf16x8_t pack8(const f32x16_t& s, int u) {
  bf16x8_t r;
#pragma unroll
  for (int e = 0; e < 8; ++e) r[e] = (bf16_t)s[8 * u + e];
  return r;
}
// what pack8 has rounded away, rounded
__device__ __forceinline__ bf16x8_t pack8_rest(const f32x16_t& s, const bf16x8_t& hi, int u) {
  bf16x8_t r;
#pragma unroll
  for (int e = 0; e < 8; ++e) r[e] = (bf16_t)(s[8 * u + e] - (float)hi[e]);
  return r;
}

// Two groups of waves hold partial sums of the same rows: the second group's waves leave theirs in LDS (16 bytes per lane and access), the
// first group's add them to their own
template <int TT, int NDT> __device__ __forceinline__ void meet_give(char* lds, int wave, int lane, const f32x16_t (&x)[TT][NDT]) {
  f32x4_t* p = reinterpret_cast<f32x4_t*>(lds) + wave * (TT * NDT * 4 * 64) + lane;
#pragma unroll
  for (int i = 0; i < TT * NDT * 4; ++i) {
    const f32x16_t& y = x[i / 4 / NDT][i / 4 % NDT];
    p[i * 64] = f32x4_t{y[4 * (i & 3)], y[4 * (i & 3) + 1], y[4 * (i & 3) + 2], y[4 * (i & 3) + 3]};
  }
}
template <int TT, int NDT> __device__ __forceinline__ void meet_take(const char* lds, int wave, int lane, f32x16_t (&x)[TT][NDT]) {
  const f32x4_t* p = reinterpret_cast<const f32x4_t*>(lds) + wave * (TT * NDT * 4 * 64) + lane;
#pragma unroll
  for (int i = 0; i < TT * NDT * 4; ++i) {
    const f32x4_t o = p[i * 64];
    f32x16_t& y = x[i / 4 / NDT][i / 4 % NDT];
#pragma unroll
    for (int e = 0; e < 4; ++e) y[4 * (i & 3) + e] += o[e];
  }
}

__device__ __forceinline__ void store4(bf16_t* p, const f32x16_t& x, int v, float scale) {
  bf16x4_t r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = (bf16_t)(x[v + i] * scale);
  *reinterpret_cast<bf16x4_t*>(p) = r;
}

// max over the two lanes 32 apart (the two halves of a score row), in both of them: v_permlane32_swap exchanges
// the upper half of its first operand with the lower half of its second, so swapping x with itself gives
// (x.low, x.low) and (x.high, x.high).  A vector instruction: no trip through the LDS crossbar.
__device__ __forceinline__ float pair_max32(float x) {
  const auto q = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(q[0]), __uint_as_float(q[1]));
}

}  // namespace
