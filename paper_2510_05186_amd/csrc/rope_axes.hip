// Rotary positions with several axes: pair k of a head (elements k and k + d / 2) turns by the angle of the row's position on the pair's own axis,
//   lo' = lo cos - hi sin,  hi' = hi cos + lo sin,  (cos, sin) = table[positions[axis[k]][row]][k]
// and its gradient turns back.
//
// Bound by memory: every element in and out once (8192 rows of 80 heads of 128, bf16, both directions: 115 us, 5.8 TB/s).  A thread has one 16-byte chunk of both
// halves of a head, so that the pairs are its own, and keeps that chunk's cos and sin for several heads of one row; the heads' loads are in flight while the positions
// lead to the angles.
#include "common.h"

#include <string.h>

namespace {

constexpr int NT = 256, MAX_PAIRS = 128, MOST_HEADS = 6;

struct RopeAxes {
  const void* src; void* dst; const float2* table; const int* positions;
  size_t ld_src, ld_dst;
  int first, rows, n_positions, n_rot, n_heads, d;                     // a launch's rows: first .. rows - 1
  int rows_per_group, head_step, n_axes;
  float sign;
  alignas(8) uint8_t axis[MAX_PAIRS];
};

// TWOS: pairs 2 i and 2 i + 1 share an axis, 16 bytes of the table at a time.  PAST: rows go past the caches in both directions.
template <typename T, int U, bool TWOS, bool PAST> __global__ __launch_bounds__(NT) void rope_axes_kernel(const RopeAxes p) {
  typedef Vec16<T> V;
  constexpr int N = V::N;
  const int half = p.d / 2, vph = half / N, c = (int)(threadIdx.x % vph) * N, slot = threadIdx.x / vph;
  const int r_in = slot / p.head_step, h0 = slot % p.head_step;
  const size_t row = p.first + (size_t)blockIdx.x * p.rows_per_group + r_in;
  if (r_in >= p.rows_per_group || row >= (size_t)p.rows) return;
  const T* src = (const T*)p.src + row * p.ld_src + c;
  T* dst = (T*)p.dst + row * p.ld_dst + c;
  V lo[U], hi[U];
  auto in = [](const T* at) {
    V v;
    if constexpr (PAST) v.v = __builtin_nontemporal_load(&reinterpret_cast<const V*>(at)->v);
    else v = *reinterpret_cast<const V*>(at);
    return v;
  };
  auto out = [](T* at, const V& v) {
    if constexpr (PAST) __builtin_nontemporal_store(v.v, &reinterpret_cast<V*>(at)->v);
    else *reinterpret_cast<V*>(at) = v;
  };
  auto load = [&](int first) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int h = first + u * p.head_step;
      if (h < p.n_heads) {
        lo[u] = in(src + (size_t)h * p.d);
        hi[u] = in(src + (size_t)h * p.d + half);
      }
    }
  };
  typedef unsigned axes_t __attribute__((ext_vector_type(N / 4)));
  const axes_t axes = *reinterpret_cast<const axes_t*>(p.axis + c);  // of this thread's pairs, a byte each
  int pos[4];                                                        // requested ahead of the heads: what is asked for first arrives first (142 -> 115 us)
#pragma unroll
  for (int a = 0; a < 4; ++a) pos[a] = p.positions[(size_t)min(a, p.n_axes - 1) * p.rows + row];
  __builtin_amdgcn_sched_barrier(0);
  load(h0);
  __builtin_amdgcn_sched_barrier(0);
  float co[N], si[N];
  unsigned still = 0;                                                // pairs that do not turn stay as they are, whatever they hold
#pragma unroll
  for (int e = 0; e < N; e += TWOS ? 2 : 1) {
    const unsigned a = axes[e / 4] >> 8 * (e % 4) & 255u;
    int at_a = pos[0];
    at_a = a == 1 ? pos[1] : at_a;
    at_a = a == 2 ? pos[2] : at_a;
    at_a = a == 3 ? pos[3] : at_a;
    at_a = a == 255 ? -1 : at_a;
    const bool on = (unsigned)at_a < (unsigned)p.n_positions;        // outside the table, and for axis 255: not turned
    if (!on) still |= (TWOS ? 3u : 1u) << e;
    const float2* at = p.table + (size_t)(on ? at_a : 0) * half + c + e;
    if constexpr (TWOS) {
      const f32x4_t t = *reinterpret_cast<const f32x4_t*>(at);
      co[e] = on ? t[0] : 1.f;
      si[e] = on ? t[1] * p.sign : 0.f;
      co[e + 1] = on ? t[2] : 1.f;
      si[e + 1] = on ? t[3] * p.sign : 0.f;
    } else {
      const float2 t = *at;
      co[e] = on ? t.x : 1.f;
      si[e] = on ? t.y * p.sign : 0.f;
    }
  }
  if (__any(still != 0)) {                                           // a loop of its own: the other one's is 9 % slower with the choice in it
    for (int h = h0; h < p.n_heads; h += p.head_step) {
      V x = in(src + (size_t)h * p.d), y = in(src + (size_t)h * p.d + half);
      if (h < p.n_rot) {
#pragma unroll
        for (int e = 0; e < N; ++e) {
          if (still >> e & 1) continue;
          const float a = x.get(e), b = y.get(e);
          x.set(e, a * co[e] - b * si[e]);
          y.set(e, b * co[e] + a * si[e]);
        }
      }
      out(dst + (size_t)h * p.d, x);
      out(dst + (size_t)h * p.d + half, y);
    }
    return;
  }
  for (int first = h0;;) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int h = first + u * p.head_step;
      if (h >= p.n_heads) break;
      if (h < p.n_rot) {
#pragma unroll
        for (int e = 0; e < N; ++e) {
          const float x = lo[u].get(e), y = hi[u].get(e);
          lo[u].set(e, x * co[e] - y * si[e]);
          hi[u].set(e, y * co[e] + x * si[e]);
        }
      }
      out(dst + (size_t)h * p.d, lo[u]);
      out(dst + (size_t)h * p.d + half, hi[u]);
    }
    first += U * p.head_step;
    if (first >= p.n_heads) break;
    load(first);
  }
}

// Rows of 32 MB and more in all go past the caches (8192 rows of 80 heads of 128, both directions: 135 -> 115 us; 4096 of 96 89 -> 70; 16384 of 12 47 -> 39), fewer do
// not: 1000 rows of 48 heads 15.2 -> 15.7, and whoever reads them next finds them there.
constexpr double PAST_BYTES = 32e6;
constexpr int MOST_GROUPS = 1 << 23;                    // 2^31 threads a launch
template <typename T, int U> void run(RopeAxes p, bool twos, hipStream_t s) {
  const bool past = (double)p.rows * p.n_heads * p.d * sizeof(T) >= PAST_BYTES;
  auto* kern = past ? (twos ? rope_axes_kernel<T, U, true, true> : rope_axes_kernel<T, U, false, true>)
                    : (twos ? rope_axes_kernel<T, U, true, false> : rope_axes_kernel<T, U, false, false>);
  for (long first = 0; first < p.rows; first += (long)MOST_GROUPS * p.rows_per_group) {
    const long groups = (p.rows - first + p.rows_per_group - 1) / p.rows_per_group;
    p.first = (int)first;
    hipLaunchKernelGGL(kern, dim3((unsigned)(groups < MOST_GROUPS ? groups : MOST_GROUPS)), dim3(NT), 0, s, p);
  }
}
template <typename T> hipError_t run_any(RopeAxes p, bool twos, hipStream_t s) {
  // Heads of a thread, `turns`: the more, the fewer angles are fetched; fewer where the chip would not be full.  Of those, the number that leaves the fewest
  // slots of a workgroup empty.
  const int slots = NT / (p.d / 2 / Vec16<T>::N);
  const long heads = (long)p.rows * p.n_heads;
  int most = (int)(heads / (2048l * slots));
  most = most < 1 ? 1 : most > MOST_HEADS ? MOST_HEADS : most;
  double best = 0.0;
  for (int turns = most; turns >= (most > 3 ? 3 : most); --turns) {
    const int step = (p.n_heads + turns - 1) / turns < slots ? (p.n_heads + turns - 1) / turns : slots, rows = slots / step;
    const int need = (p.n_heads + step - 1) / step;
    const double used = (double)p.n_heads * rows / ((double)need * slots);
    if (used > best * 1.05) {
      best = used;
      p.head_step = step;
      p.rows_per_group = rows;
    }
  }
  const int need = (p.n_heads + p.head_step - 1) / p.head_step;
  switch (need) {
    case 1: run<T, 1>(p, twos, s); break;
    case 2: run<T, 2>(p, twos, s); break;
    case 3: run<T, 3>(p, twos, s); break;
    case 4: run<T, 4>(p, twos, s); break;
    case 5: run<T, 5>(p, twos, s); break;
    default: run<T, MOST_HEADS>(p, twos, s);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rope_axes(int dtype, const void* src, size_t ld_src, void* dst, size_t ld_dst, const float* table, int n_positions, const int* positions,
                            int n_axes, const uint8_t* axis, int rows, int n_rot, int n_pass, int d, int backward, hipStream_t s) {
  RopeAxes p = {src, dst, (const float2*)table, positions, ld_src, ld_dst, 0, rows, n_positions, n_rot, src == dst ? n_rot : n_rot + n_pass, d, 0, 0, n_axes, backward ? -1.f : 1.f, {}};
  memcpy(p.axis, axis, d / 2);
  bool twos = true;
  for (int k = 0; k < d / 2; k += 2) twos = twos && axis[k] == axis[k + 1];
  return dtype == DT_BF16 ? run_any<bf16_t>(p, twos, s) : run_any<float>(p, twos, s);
}
