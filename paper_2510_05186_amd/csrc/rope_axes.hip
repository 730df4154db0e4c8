// Rotary positions with several axes: pair k of a head (elements k and k + d / 2) turns by the angle of the row's position on the pair's own axis,
//   lo' = lo cos - hi sin,  hi' = hi cos + lo sin,  (cos, sin) = table[positions[axis[k]][row]][k]
// and its gradient turns back.  Bound by memory: every element in and out once.
#include "common.h"

#include <string.h>

namespace {

constexpr int NT = 256, MAX_PAIRS = 128;

struct RopeAxes {
  const void* src; void* dst; const float2* table; const int* positions;
  size_t ld_src, ld_dst;
  int rows, n_positions, n_rot, n_heads, d;
  int rows_per_group, head_step;
  float sign;
  uint8_t axis[MAX_PAIRS];
};

template <typename T> __global__ __launch_bounds__(NT) void rope_axes_kernel(const RopeAxes p) {
  typedef Vec16<T> V;
  constexpr int N = V::N;
  const int half = p.d / 2, vph = half / N, c = (int)(threadIdx.x % vph) * N, slot = threadIdx.x / vph;
  const int r_in = slot / p.head_step, h0 = slot % p.head_step;
  const long row = (long)blockIdx.x * p.rows_per_group + r_in;
  if (r_in >= p.rows_per_group || row >= p.rows) return;
  float co[N], si[N];
#pragma unroll
  for (int e = 0; e < N; ++e) {
    co[e] = 1.f;
    si[e] = 0.f;
    const int a = p.axis[c + e];
    if (a != 255) {
      const int pos = p.positions[(size_t)a * p.rows + row];
      if ((unsigned)pos < (unsigned)p.n_positions) {
        const float2 t = p.table[(size_t)pos * half + c + e];
        co[e] = t.x;
        si[e] = t.y * p.sign;
      }
    }
  }
  const T* src = (const T*)p.src + row * p.ld_src + c;
  T* dst = (T*)p.dst + row * p.ld_dst + c;
  for (int h = h0; h < p.n_heads; h += p.head_step) {
    V lo = *reinterpret_cast<const V*>(src + (size_t)h * p.d), hi = *reinterpret_cast<const V*>(src + (size_t)h * p.d + half);
    if (h < p.n_rot) {
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const float x = lo.get(e), y = hi.get(e);
        lo.set(e, x * co[e] - y * si[e]);
        hi.set(e, y * co[e] + x * si[e]);
      }
    }
    *reinterpret_cast<V*>(dst + (size_t)h * p.d) = lo;
    *reinterpret_cast<V*>(dst + (size_t)h * p.d + half) = hi;
  }
}

}  // namespace

hipError_t launch_rope_axes(int dtype, const void* src, size_t ld_src, void* dst, size_t ld_dst, const float* table, int n_positions, const int* positions,
                            const uint8_t* axis, int rows, int n_rot, int n_pass, int d, int backward, hipStream_t s) {
  RopeAxes p = {src, dst, (const float2*)table, positions, ld_src, ld_dst, rows, n_positions, n_rot, src == dst ? n_rot : n_rot + n_pass, d, 0, 0, backward ? -1.f : 1.f, {}};
  memcpy(p.axis, axis, d / 2);
  const int slots = NT / (d / 2 / (dtype == DT_BF16 ? 8 : 4));
  p.rows_per_group = slots / p.n_heads < 1 ? 1 : slots / p.n_heads;
  p.head_step = slots / p.rows_per_group;
  const dim3 grid((rows + p.rows_per_group - 1) / p.rows_per_group);
  if (dtype == DT_BF16) hipLaunchKernelGGL(rope_axes_kernel<bf16_t>, grid, dim3(NT), 0, s, p);
  else hipLaunchKernelGGL(rope_axes_kernel<float>, grid, dim3(NT), 0, s, p);
  return hipGetLastError();
}
