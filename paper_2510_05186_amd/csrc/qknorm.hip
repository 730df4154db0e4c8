// Norms of queries and keys with the position rotation, in one pass over packed qkv rows: every q and k head x becomes
// R(position) (x * r * gamma), r = 1 / sqrt(mean(x^2) + eps), and its gradient goes back the same way:
// dn = R^T dy, g = dn * gamma, dx = r (g - xh mean(g xh)) with xh = x r, dgamma = sum of dn * xh over rows and heads.
//
// Bound by memory.  A head belongs to G lanes, each with the same chunk of both halves, so that the rotation's pairs are a lane's own and a
// head's sum is a few lane swaps.  Heads are numbered through all rows, a workgroup takes 256 / G of them at a time whatever the
// number of heads; cos and sin (fp32, 512 bytes a row at d = 128) come out of the caches again for every head.
#include "keep8.h"

#include <type_traits>

namespace {

constexpr int NT = 256;
// Workgroups (8192 rows of 80 heads of 128, bf16): forward and rebuilt together 136 us with 2048, 134 with 4096, 130 with 8192, 142 with one turn each;
// backward as many as the compute units hold at once, four on each (512: 118 us, 768: 100, 1024: 94).
// Heads that one workgroup has done in three turns are left to one, which saves the launch that adds the sums (5 rows of 12 heads of 128, forward and
// backward: 10.8 us a pass among others, 13.5 with it; eight turns 16.1).
constexpr int FWD_GROUPS = 8192, BWD_GROUPS = 1024, BWD_TURNS = 3;

// item = row * heads + head
struct Items {
  size_t total;
  unsigned heads, n_q, n_rot, seq;
};
struct Head {
  unsigned row, head, pos;
  bool on;
};
// The workgroup's items base .. base + S - 1 of every turn.  All of it is the same for the whole workgroup and advances without a division; a lane's address is
// a pointer to the workgroup's first head plus an offset that never changes (these and the divisions were a third of the gradient kernel's instructions).
template <int S> struct Cursor {
  size_t base;
  unsigned row, head, pos;
  size_t step;
  unsigned step_row, step_head, step_pos;
  __device__ __forceinline__ explicit Cursor(const Items& k) {
    base = (size_t)blockIdx.x * S;
    step = (size_t)gridDim.x * S;                                      // < 2^32
    row = (unsigned)(base / k.heads);
    head = (unsigned)(base - (size_t)row * k.heads);
    pos = row % k.seq;
    step_row = (unsigned)step / k.heads;
    step_head = (unsigned)step - step_row * k.heads;
    step_pos = step_row % k.seq;
  }
  __device__ __forceinline__ void advance(const Items& k) {
    base += step;
    head += step_head;
    const unsigned carry = head >= k.heads;
    head -= carry ? k.heads : 0u;
    row += step_row + carry;
    pos += step_pos + carry;
    pos -= pos >= k.seq ? k.seq : 0u;
  }
  __device__ __forceinline__ Head lane(unsigned slot, const Items& k) const {
    const unsigned n = head + slot, r = k.heads >= S ? (n >= k.heads ? 1u : 0u) : n / k.heads;
    unsigned at = pos + r;                                              // r <= S
    if (k.seq >= S) at -= at >= k.seq ? k.seq : 0u;
    else at %= k.seq;
    return {row + r, n - r * k.heads, at, base + slot < k.total};
  }
};

// the chunk's cos and sin
template <typename T> struct Angles {
  float c[Vec16<T>::N], s[Vec16<T>::N];
  __device__ __forceinline__ void load(const float2* __restrict__ table) {
#pragma unroll
    for (int e = 0; e < Vec16<T>::N; e += 2) {
      const f32x4_t v = *reinterpret_cast<const f32x4_t*>(table + e);
      c[e] = v[0]; s[e] = v[1]; c[e + 1] = v[2]; s[e + 1] = v[3];
    }
  }
};

struct QkNorm {
  const void* src; const uint8_t* codes_in; const uint8_t* scales_in;   // the projection's output, or its kept form
  void* dst; const void* gamma_q; const void* gamma_k; const float2* table; float* stats;
  uint8_t* codes; uint8_t* scales;                                      // where src is kept (KEEP)
  Items items;
  int d; float eps;
};

template <typename T, int G, bool FROM8, bool KEEP>
__global__ __launch_bounds__(NT) void qknorm_kernel(const QkNorm p) {
  typedef Vec16<T> V;
  typedef typename KeepChunk<T>::codes_t codes_t;
  constexpr int S = NT / G;
  const int half = p.d / 2, col = (threadIdx.x % G) * V::N;
  const unsigned slot = threadIdx.x / G, n_rot = p.items.n_rot;
  const bool mine = col < half;                                        // d = 192: lanes of a head that hold nothing
  const unsigned off[2] = {slot * p.d + col, slot * p.d + col + half};
  V gain[2][2];                                                        // q, k; lower, upper half
  if (mine)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      gain[0][i] = *reinterpret_cast<const V*>((const T*)p.gamma_q + i * half + col);
      gain[1][i] = *reinterpret_cast<const V*>((const T*)p.gamma_k + i * half + col);
    }
  for (Cursor<S> cur(p.items); cur.base < p.items.total; cur.advance(p.items)) {
    const Head k = cur.lane(slot, p.items);
    const bool on = k.on && mine, turn = k.head < n_rot;
    const size_t first = cur.base * p.d;
    V x[2] = {};
    float v[2][V::N];
    Angles<T> a;
    float r = 0.f;
    if (on) {
      if constexpr (FROM8) {
        codes_t c[2];
        uint32_t b[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          c[i] = *reinterpret_cast<const codes_t*>(p.codes_in + first + off[i]);
          b[i] = p.scales_in[first / KEEP_BLOCK + off[i] / KEEP_BLOCK];
        }
        if (turn) {
          a.load(p.table + (size_t)k.pos * half + col);
          r = p.stats[(size_t)k.row * n_rot + k.head];
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          if (turn) keep_values(c[i], keep_scale(b[i]), v[i]);
          else x[i] = keep_stored(c[i], keep_scale(b[i]), V());
        }
      } else {
#pragma unroll
        for (int i = 0; i < 2; ++i) x[i] = *reinterpret_cast<const V*>((const T*)p.src + first + off[i]);
        if (turn) a.load(p.table + (size_t)k.pos * half + col);
      }
    }
    if constexpr (!FROM8) {
      float s = 0.f;
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int e = 0; e < V::N; ++e) {
          v[i][e] = x[i].get(e);
          s += v[i][e] * v[i][e];
        }
      r = rsqrtf(lanes_sum<G>(s) / p.d + p.eps);
      if (on && turn && col == 0) p.stats[(size_t)k.row * n_rot + k.head] = r;
      if constexpr (KEEP) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          uint32_t byte;
          const codes_t c = keep_chunk<T>(x[i], byte);
          if (on) {
            *reinterpret_cast<codes_t*>(p.codes + first + off[i]) = c;
            if (col % KEEP_BLOCK == 0) p.scales[first / KEEP_BLOCK + off[i] / KEEP_BLOCK] = (uint8_t)byte;
          }
        }
      }
    }
    if (!on) continue;
    T* out = (T*)p.dst + first;
    if (turn) {
      const bool is_k = k.head >= p.items.n_q;
      V o[2];
#pragma unroll
      for (int e = 0; e < V::N; ++e) {
        const float lo = v[0][e] * r * (is_k ? gain[1][0] : gain[0][0]).get(e), hi = v[1][e] * r * (is_k ? gain[1][1] : gain[0][1]).get(e);
        o[0].set(e, lo * a.c[e] - hi * a.s[e]);
        o[1].set(e, hi * a.c[e] + lo * a.s[e]);
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) *reinterpret_cast<V*>(out + off[i]) = o[i];
    } else if (FROM8 || p.dst != p.src) {
#pragma unroll
      for (int i = 0; i < 2; ++i) *reinterpret_cast<V*>(out + off[i]) = x[i];
    }
  }
}

struct QkNormBwd {
  const void* dy; const void* x; const uint8_t* codes; const uint8_t* scales; const float* stats;
  const void* gamma_q; const void* gamma_k; const float2* table; void* dx; float* partial; float* dgamma_q; float* dgamma_k;
  Items items;
  int d;
};

// dx may be dy or x: a lane has read its chunks before it writes there.  The gains' gradients of a
// workgroup's heads stay in registers, 2 N of q and of k a lane, and end in partial[blockIdx.x] (q) and partial[gridDim.x + blockIdx.x] (k), added up in a
// fixed order; a workgroup alone adds them to the accumulators itself.
template <typename T, int G, bool FROM8>
__global__ __launch_bounds__(NT) void qknorm_bwd_kernel(const QkNormBwd p) {
  typedef Vec16<T> V;
  typedef typename KeepChunk<T>::codes_t codes_t;
  constexpr int S = NT / G, N = V::N, W = G * N;
  __shared__ float sums[S][2][2][W];
  const int half = p.d / 2, col = (threadIdx.x % G) * N;
  const unsigned slot = threadIdx.x / G, n_rot = p.items.n_rot;
  const bool mine = col < half;
  V gain[2][2];
  if (mine)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      gain[0][i] = *reinterpret_cast<const V*>((const T*)p.gamma_q + i * half + col);
      gain[1][i] = *reinterpret_cast<const V*>((const T*)p.gamma_k + i * half + col);
    }
  float dg[2][2][N] = {};
  const unsigned off[2] = {slot * p.d + col, slot * p.d + col + half};
  for (Cursor<S> cur(p.items); cur.base < p.items.total; cur.advance(p.items)) {
    const Head k = cur.lane(slot, p.items);
    const bool on = k.on && mine, turn = k.head < n_rot, is_k = k.head >= p.items.n_q;
    const size_t first = cur.base * p.d;
    V dy[2] = {};
    float xh[2][N] = {}, g[2][N] = {}, r = 0.f, s = 0.f;
    if (on) {
#pragma unroll
      for (int i = 0; i < 2; ++i) dy[i].v = __builtin_nontemporal_load(&reinterpret_cast<const V*>((const T*)p.dy + first + off[i])->v);   // 94 -> 83 us, the next call 4 more
      if (turn) {
        codes_t c[2];
        uint32_t b[2];
        V x[2];
        Angles<T> a;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          if constexpr (FROM8) {
            c[i] = *reinterpret_cast<const codes_t*>(p.codes + first + off[i]);
            b[i] = p.scales[first / KEEP_BLOCK + off[i] / KEEP_BLOCK];
          } else {
            x[i] = *reinterpret_cast<const V*>((const T*)p.x + first + off[i]);
          }
        }
        a.load(p.table + (size_t)k.pos * half + col);
        r = p.stats[(size_t)k.row * n_rot + k.head];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          if constexpr (FROM8) {
            keep_values(c[i], keep_scale(b[i]), xh[i]);
          } else {
#pragma unroll
            for (int e = 0; e < N; ++e) xh[i][e] = x[i].get(e);
          }
        }
        float n[2][N];
#pragma unroll
        for (int e = 0; e < N; ++e) {
          const float lo = dy[0].get(e), hi = dy[1].get(e);
          n[0][e] = lo * a.c[e] + hi * a.s[e];
          n[1][e] = hi * a.c[e] - lo * a.s[e];
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            xh[i][e] *= r;
            g[i][e] = n[i][e] * (is_k ? gain[1][i] : gain[0][i]).get(e);
            s += g[i][e] * xh[i][e];
          }
        }
        // one of two branches for nearly every wave
#pragma unroll
        for (int q = 0; q < 2; ++q)
          if (is_k == (q == 1))
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
              for (int e = 0; e < N; ++e) dg[q][i][e] = fmaf(n[i][e], xh[i][e], dg[q][i][e]);
      }
    }
    const float m = lanes_sum<G>(s) / p.d;
    if (!on) continue;
    T* out = (T*)p.dx + first;
    if (turn) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        V o;
#pragma unroll
        for (int e = 0; e < N; ++e) o.set(e, r * (g[i][e] - xh[i][e] * m));
        *reinterpret_cast<V*>(out + off[i]) = o;
      }
    } else if (p.dx != p.dy) {
#pragma unroll
      for (int i = 0; i < 2; ++i) *reinterpret_cast<V*>(out + off[i]) = dy[i];
    }
  }
#pragma unroll
  for (int q = 0; q < 2; ++q)
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int e = 0; e < N; ++e) sums[slot][q][i][col + e] = dg[q][i][e];
  __syncthreads();
  for (int j = threadIdx.x; j < 2 * p.d; j += NT) {
    const int q = j / p.d, c = j % p.d, i = c >= half, e = c - i * half;
    float t = 0.f;
#pragma unroll 8
    for (int w = 0; w < S; ++w) t += sums[w][q][i][e];
    if (gridDim.x == 1) (q ? p.dgamma_k : p.dgamma_q)[c] += t;
    else p.partial[((size_t)q * gridDim.x + blockIdx.x) * p.d + c] = t;
  }
}

// lanes of a head: half a head's chunks, the next power of two
template <typename T, typename F> hipError_t by_head(int d, F f) {
  const int lanes = d / 2 / Vec16<T>::N;
  if constexpr (Vec16<T>::N == 8) {
    if (lanes <= 4) f(std::integral_constant<int, 4>());
    else if (lanes <= 8) f(std::integral_constant<int, 8>());
    else f(std::integral_constant<int, 16>());
  } else {
    if (lanes <= 8) f(std::integral_constant<int, 8>());
    else if (lanes <= 16) f(std::integral_constant<int, 16>());
    else f(std::integral_constant<int, 32>());
  }
  return hipGetLastError();
}
unsigned groups_of(const Items& k, int slots, unsigned most) {
  const size_t n = (k.total + slots - 1) / slots;
  return (unsigned)(n > most ? most : n);
}

template <typename T> hipError_t run_qknorm(const QkNorm& p, hipStream_t s) {
  return by_head<T>(p.d, [&](auto g) {
    const dim3 grid(groups_of(p.items, NT / g, FWD_GROUPS));
    if (p.codes_in) hipLaunchKernelGGL((qknorm_kernel<T, g, true, false>), grid, dim3(NT), 0, s, p);
    else if (p.codes) hipLaunchKernelGGL((qknorm_kernel<T, g, false, true>), grid, dim3(NT), 0, s, p);
    else hipLaunchKernelGGL((qknorm_kernel<T, g, false, false>), grid, dim3(NT), 0, s, p);
  });
}
template <typename T> hipError_t run_qknorm_bwd(const QkNormBwd& p, int rows, hipStream_t s) {
  unsigned nb = 0;
  const hipError_t e = by_head<T>(p.d, [&](auto g) {
    nb = p.items.total <= (size_t)BWD_TURNS * (NT / g) ? 1u : groups_of(p.items, NT / g, (unsigned)(rows < BWD_GROUPS ? rows : BWD_GROUPS));
    if (p.codes) hipLaunchKernelGGL((qknorm_bwd_kernel<T, g, true>), dim3(nb), dim3(NT), 0, s, p);
    else hipLaunchKernelGGL((qknorm_bwd_kernel<T, g, false>), dim3(nb), dim3(NT), 0, s, p);
  });
  if (e != hipSuccess || nb == 1) return e;
  return launch_add_columns(p.partial, p.dgamma_q, p.dgamma_k, (int)nb, p.d, s);
}

}  // namespace

hipError_t launch_qknorm_rope(int dtype, const void* src, const uint8_t* codes_in, const uint8_t* scales_in, void* dst, const void* gamma_q, const void* gamma_k,
                              const float* table, float* stats, uint8_t* codes, uint8_t* scales, int rows, int seq, int n_q, int n_kv, int d, float eps, hipStream_t s) {
  const unsigned heads = n_q + 2 * n_kv;
  const QkNorm p = {src, codes_in, scales_in, dst, gamma_q, gamma_k, (const float2*)table, stats, codes, scales,
                    {(size_t)rows * heads, heads, (unsigned)n_q, (unsigned)(n_q + n_kv), (unsigned)seq}, d, eps};
  return dtype == DT_BF16 ? run_qknorm<bf16_t>(p, s) : run_qknorm<float>(p, s);
}

hipError_t launch_qknorm_rope_bwd(int dtype, const void* dy, const void* x, const uint8_t* codes, const uint8_t* scales, const float* stats, const void* gamma_q,
                                  const void* gamma_k, const float* table, void* dx, float* partial, float* dgamma_q, float* dgamma_k, int rows, int seq, int n_q, int n_kv,
                                  int d, hipStream_t s) {
  const unsigned heads = n_q + 2 * n_kv;
  const QkNormBwd p = {dy, x, codes, scales, stats, gamma_q, gamma_k, (const float2*)table, dx, partial, dgamma_q, dgamma_k,
                       {(size_t)rows * heads, heads, (unsigned)n_q, (unsigned)(n_q + n_kv), (unsigned)seq}, d};
  return dtype == DT_BF16 ? run_qknorm_bwd<bf16_t>(p, rows, s) : run_qknorm_bwd<float>(p, rows, s);
}
