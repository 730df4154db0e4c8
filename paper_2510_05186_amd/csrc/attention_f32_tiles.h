// Tiles of 16 rows on the fp32 matrix instruction, shared by the fp32 attention kernels; the fragment layouts stand in attention_f32.hip.
#pragma once
#include "attention_rows.h"

namespace {

constexpr int ROWS = 16;

template <int D> struct F32 {
  static constexpr int S = D / 16, H = D / 64, NT = D / 16;   // k-steps of a row, 64-column groups, output tiles
  static __device__ __forceinline__ void rows(f32x4_t (&v)[S], const float* row, int g) {
#pragma unroll
    for (int s = 0; s < S; ++s) v[s] = *reinterpret_cast<const f32x4_t*>(row + 16 * s + 4 * g);
  }
  // v[e][h]: base + (row 4 g + e) * ld, rows clamped to `last`
  static __device__ __forceinline__ void columns(f32x4_t (&v)[4][H], const float* base, size_t ld, int first, int last, int g, int r) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float* p = base + (size_t)min(first + 4 * g + e, last) * ld + 4 * r;
#pragma unroll
      for (int h = 0; h < H; ++h) v[e][h] = *reinterpret_cast<const f32x4_t*>(p + 64 * h);
    }
  }
  // D[4 g + v][r] = sum over columns of a-rows times b-rows
  static __device__ __forceinline__ f32x4_t product(const f32x4_t (&a)[S], const f32x4_t (&b)[S]) {
    f32x4_t d0 = {0.f, 0.f, 0.f, 0.f}, d1 = {0.f, 0.f, 0.f, 0.f};   // two chains: consecutive MFMAs do not wait for one another
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
      for (int e = 0; e < 4; e += 2) {
        d0 = __builtin_amdgcn_mfma_f32_16x16x4f32(a[s][e], b[s][e], d0, 0, 0, 0);
        d1 = __builtin_amdgcn_mfma_f32_16x16x4f32(a[s][e + 1], b[s][e + 1], d1, 0, 0, 0);
      }
    return f32x4_t{d0[0] + d1[0], d0[1] + d1[1], d0[2] + d1[2], d0[3] + d1[3]};
  }
  static __device__ __forceinline__ void accumulate(f32x4_t (&acc)[NT], const f32x4_t (&c)[4][H], const f32x4_t& p) {
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int t = 0; t < NT; ++t) acc[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(c[e][t >> 2][t & 3], p[e], acc[t], 0, 0, 0);
  }
  // this lane's part of the 16 x D result into LDS rows of D + 4 floats
  static __device__ __forceinline__ void put(float (*dst)[D + 4], const f32x4_t (&acc)[NT], int g, int r) {
#pragma unroll
    for (int h = 0; h < H; ++h)
#pragma unroll
      for (int v = 0; v < 4; ++v)
        *reinterpret_cast<f32x4_t*>(&dst[r][64 * h + 16 * g + 4 * v]) =
            f32x4_t{acc[4 * h][v], acc[4 * h + 1][v], acc[4 * h + 2][v], acc[4 * h + 3][v]};
  }
  static __device__ __forceinline__ void clear(f32x4_t (&acc)[NT]) {
#pragma unroll
    for (int t = 0; t < NT; ++t) acc[t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }
  // columns c .. c + 3 of a result row, out of the four partial results, rotated back: the partner columns lie d / 2 away
  static __device__ __forceinline__ void turn_back(f32x4_t& v, const float (*part)[ROWS][D + 4], float scale, const float2* angle, int row, int c) {
    const int k = c % (D / 2), other = c < D / 2 ? c + D / 2 : c - D / 2;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float x = (((part[0][row][other + e] + part[1][row][other + e]) + part[2][row][other + e]) + part[3][row][other + e]) * scale;
      const float2 t = angle[k + e];
      float own = v[e];
      if (c < D / 2) rope_back(own, x, t.x, t.y);
      else rope_back(x, own, t.x, t.y);
      v[e] = own;
    }
  }
  static __device__ __forceinline__ void scaled(f32x4_t (&v)[S], float f) {
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
      for (int e = 0; e < 4; ++e) v[s][e] *= f;
  }
};

// sum or maximum over the four lanes that hold a column's rows
__device__ __forceinline__ float sum_g(float x) { x += __shfl_xor(x, 16, 64); return x + __shfl_xor(x, 32, 64); }
__device__ __forceinline__ float max_g(float x) { x = fmaxf(x, __shfl_xor(x, 16, 64)); return fmaxf(x, __shfl_xor(x, 32, 64)); }

}  // namespace
