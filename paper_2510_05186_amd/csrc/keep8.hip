// Activations kept in 8 bits between the forward and the backward pass (keep8.h), and the non-linear parts of a layer that keep their
// input that way and take their gradients from it.
#include "keep8.h"

#include <type_traits>

namespace {

constexpr int NT = 256;

// ---- keep and restore, 16 bytes of x per lane and access ------------------------------------------------------
// Rows may start anywhere (an odd number of columns, a column range of wider rows): the memory system takes 16-byte accesses at any address
// of an element (4096 x 9079 bf16: 53 us, 130 with one value a lane), and only a row's last chunk goes value by value.
template <typename T> struct Loose;
template <> struct Loose<bf16_t> {
  typedef bf16_t x_t __attribute__((ext_vector_type(8), aligned(2)));
  typedef uint32_t codes_t __attribute__((ext_vector_type(2), aligned(1)));
};
template <> struct Loose<float> {
  typedef float x_t __attribute__((ext_vector_type(4), aligned(4)));
  typedef uint32_t codes_t __attribute__((aligned(1)));
};
template <typename T> __device__ __forceinline__ Vec16<T> load_values(const T* x, int left) {
  Vec16<T> v = {};
  if (left >= Vec16<T>::N) v.v = __builtin_nontemporal_load(reinterpret_cast<const typename Loose<T>::x_t*>(x));   // pack and unpack 265 -> 252 us
  else
#pragma unroll
    for (int e = 0; e < Vec16<T>::N - 1; ++e)
      if (e < left) v.v[e] = x[e];
  return v;
}
template <typename T> __device__ __forceinline__ void store_values(T* x, const Vec16<T>& v, int left) {
  if (left >= Vec16<T>::N) *reinterpret_cast<typename Loose<T>::x_t*>(x) = v.v;
  else
#pragma unroll
    for (int e = 0; e < Vec16<T>::N - 1; ++e)
      if (e < left) x[e] = v.v[e];
}
__device__ __forceinline__ uint32_t code_of(uint2 c, int e) { return (e < 4 ? c.x : c.y) >> 8 * (e & 3); }
__device__ __forceinline__ uint32_t code_of(uint32_t c, int e) { return c >> 8 * e; }
template <typename T> __device__ __forceinline__ typename KeepChunk<T>::codes_t load_codes(const uint8_t* p, int left) {
  typename KeepChunk<T>::codes_t c = {};
  if (left >= Vec16<T>::N) return __builtin_bit_cast(typename KeepChunk<T>::codes_t, *reinterpret_cast<const typename Loose<T>::codes_t*>(p));
#pragma unroll
  for (int e = 0; e < Vec16<T>::N - 1; ++e)
    if (e < left) keep_put(c, e, p[e]);
  return c;
}
template <typename T> __device__ __forceinline__ void store_codes(uint8_t* p, typename KeepChunk<T>::codes_t c, int left) {
  if (left >= Vec16<T>::N) *reinterpret_cast<typename Loose<T>::codes_t*>(p) = __builtin_bit_cast(typename Loose<T>::codes_t, c);
  else
#pragma unroll
    for (int e = 0; e < Vec16<T>::N - 1; ++e)
      if (e < left) p[e] = (uint8_t)code_of(c, e);
}

// The chunks of a row, padded to whole blocks, are numbered through all rows; a workgroup takes NT * U numbers at a time and all of its
// loads are in flight before the first is used.
struct Chunks {
  size_t total;          // rows * per_row
  Divisor per_row;       // chunks of a row, padded to whole blocks: less than 2^28
};
template <typename T> Chunks chunks_of(int rows, int cols) {
  const unsigned per_row = (unsigned)keep_blocks(cols) * KeepChunk<T>::LANES;
  return {(size_t)rows * per_row, Divisor(per_row)};
}
struct At { size_t row; int col; };
// chunk base + i, for base a multiple of NT * U and i < NT * U
template <typename T> struct Walk {
  size_t row0 = 0;
  unsigned c0;
  Divisor per_row;
  __device__ __forceinline__ Walk(size_t base, const Chunks& k) : c0((unsigned)base), per_row(k.per_row) {
    if (k.total >> 31) {
      row0 = base / per_row.d;
      c0 = (unsigned)(base - row0 * per_row.d);
    }
  }
  __device__ __forceinline__ At at(unsigned i) const {
    const unsigned n = c0 + i, r = per_row.quotient(n);
    return {row0 + r, (int)((n - r * per_row.d) * Vec16<T>::N)};
  }
};

// WHOLE: every chunk of a row is whole (the test for it costs unpack 131 -> 140 us at 16384 x 15360)
template <typename T, int U, bool WHOLE>
__global__ __launch_bounds__(NT) void pack8_kernel(const T* __restrict__ x, size_t ldx, uint8_t* __restrict__ codes, uint8_t* __restrict__ scales, const Chunks k, int rows,
                                                   int cols) {
  const int nb = keep_blocks(cols);
  for (size_t base = blockIdx.x * (size_t)(NT * U); base < k.total; base += (size_t)gridDim.x * (NT * U)) {
    const Walk<T> walk(base, k);
    Vec16<T> v[U] = {};
    At at[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      at[u] = walk.at(u * NT + threadIdx.x);
      if (at[u].row < (size_t)rows && at[u].col < cols) v[u] = load_values(x + at[u].row * ldx + at[u].col, WHOLE ? Vec16<T>::N : cols - at[u].col);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      uint32_t byte;
      const auto c = keep_chunk<T>(v[u], byte);
      if (at[u].row < (size_t)rows) {
        if (at[u].col < cols) store_codes<T>(codes + at[u].row * cols + at[u].col, c, WHOLE ? Vec16<T>::N : cols - at[u].col);
        if (at[u].col % KEEP_BLOCK == 0) scales[at[u].row * nb + at[u].col / KEEP_BLOCK] = (uint8_t)byte;
      }
    }
  }
}

template <typename T, int U, bool WHOLE>
__global__ __launch_bounds__(NT) void unpack8_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, T* __restrict__ x, size_t ldx, const Chunks k,
                                                     int rows, int cols) {
  const int nb = keep_blocks(cols);
  for (size_t base = blockIdx.x * (size_t)(NT * U); base < k.total; base += (size_t)gridDim.x * (NT * U)) {
    const Walk<T> walk(base, k);
    typename KeepChunk<T>::codes_t c[U];
    uint32_t b[U];
    At at[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      at[u] = walk.at(u * NT + threadIdx.x);
      if (at[u].row < (size_t)rows && at[u].col < cols) {
        c[u] = load_codes<T>(codes + at[u].row * cols + at[u].col, WHOLE ? Vec16<T>::N : cols - at[u].col);
        b[u] = scales[at[u].row * nb + at[u].col / KEEP_BLOCK];
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (at[u].row < (size_t)rows && at[u].col < cols)
        store_values(x + at[u].row * ldx + at[u].col, keep_stored(c[u], keep_scale(b[u]), Vec16<T>()), WHOLE ? Vec16<T>::N : cols - at[u].col);
  }
}

// ---- norms ------------------------------------------------------------------------------------------------
// A row belongs to W waves, R rows to a workgroup; a lane holds C chunks of its row, W * 64 chunks apart.  The W waves of a row add up their sums
// through LDS (`red`, of its own for every use).
template <int W> __device__ __forceinline__ float row_sum(float v, float* red /* [R * W] */, int slot, int wave) {
  v = lanes_sum<64>(v);
  if (W == 1) return v;
  if ((threadIdx.x & 63) == 0) red[slot * W + wave] = v;
  __syncthreads();
  float t = 0.f;
#pragma unroll
  for (int w = 0; w < W; ++w) t += red[slot * W + w];
  return t;
}

template <typename T, bool LN, int W, int C, int R>
__global__ __launch_bounds__(W * R * 64) void norm_fwd_pack8_kernel(const T* __restrict__ x, const T* __restrict__ gamma, const T* __restrict__ beta, T* __restrict__ out,
                                                                    float* __restrict__ stats, uint8_t* __restrict__ codes, uint8_t* __restrict__ scales, int rows, int h,
                                                                    float eps) {
  typedef Vec16<T> V;
  typedef typename KeepChunk<T>::codes_t codes_t;
  __shared__ float red[2][2][R * W];
  const int slot = threadIdx.x / (W * 64), l = threadIdx.x % (W * 64), wave = l >> 6, nb = keep_blocks(h);
  int turn = 0;                                                        // what the last rows' sums stand in is not written again before the next barrier
  for (size_t first = (size_t)blockIdx.x * R; first < (size_t)rows; first += (size_t)gridDim.x * R, turn ^= 1) {
    const size_t row = first + slot;
    const bool on = row < (size_t)rows;
    V v[C] = {};
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int col = (l + c * W * 64) * V::N;
      if (on && col < h) v[c] = *reinterpret_cast<const V*>(x + row * h + col);
    }
    float mean = 0.f, s = 0.f;
    if (LN) {
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int e = 0; e < V::N; ++e) s += v[c].get(e);
      mean = row_sum<W>(s, red[turn][0], slot, wave) / h;
      s = 0.f;
    }
#pragma unroll
    for (int c = 0; c < C; ++c) {
      if ((l + c * W * 64) * V::N < h)
#pragma unroll
        for (int e = 0; e < V::N; ++e) { const float d = v[c].get(e) - mean; s += d * d; }
    }
    const float r = rsqrtf(row_sum<W>(s, red[turn][1], slot, wave) / h + eps);
    if (on && l == 0) {
      if (LN) { stats[2 * row] = mean; stats[2 * row + 1] = r; } else stats[row] = r;
    }
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int col = (l + c * W * 64) * V::N;
      uint32_t byte;
      const codes_t code = keep_chunk<T>(v[c], byte);
      if (on && col < h) {
        *reinterpret_cast<codes_t*>(codes + row * h + col) = code;
        if (col % KEEP_BLOCK == 0) scales[row * nb + col / KEEP_BLOCK] = (uint8_t)byte;
        const V g = *reinterpret_cast<const V*>(gamma + col);
        V o, b;
        if (LN) b = *reinterpret_cast<const V*>(beta + col);
#pragma unroll
        for (int e = 0; e < V::N; ++e) {
          float f = (v[c].get(e) - mean) * r * g.get(e);
          if (LN) f += b.get(e);
          o.set(e, f);
        }
        *reinterpret_cast<V*>(out + row * h + col) = o;
      }
    }
  }
}

// Workgroup b takes the rows b R .. b R + R - 1, (b + gridDim.x) R .., the loads of the next ones in flight while the present ones are reduced and written.
// Its sums of the gains' and biases' gradients stay in registers and end in its rows of `partial`, those of its R rows added in order; a workgroup alone adds
// them to the accumulators itself.  dx may be dn or dres: rows in flight are other rows, and a lane has read its chunks of the present one.
template <typename T, bool LN, int W, int C, int R>
__global__ __launch_bounds__(W * R * 64) void norm_bwd8_kernel(const T* dn, const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales,
                                                               const float* __restrict__ stats, const T* __restrict__ gamma, const T* __restrict__ beta, const T* dres, T* dx,
                                                               T* __restrict__ out, float* __restrict__ partial, float* dgamma, float* dbeta, int rows, int h) {
  typedef Vec16<T> V;
  typedef typename KeepChunk<T>::codes_t codes_t;
  __shared__ float red[2][2][R * W];
  __shared__ f32x4_t sums[R > 1 ? R : 1][R > 1 ? C * V::N / 4 : 1][W * 64];      // 32 KB
  const int slot = threadIdx.x / (W * 64), l = threadIdx.x % (W * 64), wave = l >> 6, nb = keep_blocks(h);
  float pg[C][V::N] = {}, pb[LN ? C : 1][V::N] = {};
  V gv[C], bv[LN ? C : 1];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int col = (l + c * W * 64) * V::N;
    if (col < h) {
      gv[c] = *reinterpret_cast<const V*>(gamma + col);
      if constexpr (LN)
        if (out) bv[c] = *reinterpret_cast<const V*>(beta + col);
    }
  }
  struct Row { V d[C], res[C]; codes_t q[C]; uint32_t b[C]; float mean, r; } buf[2];
  auto load = [&](Row& k, size_t row) {
    if (row >= (size_t)rows) return;
    k.mean = LN ? stats[2 * row] : 0.f;
    k.r = LN ? stats[2 * row + 1] : stats[row];
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int col = (l + c * W * 64) * V::N;
      if (col < h) {
        k.d[c] = *reinterpret_cast<const V*>(dn + row * h + col);
        k.q[c] = *reinterpret_cast<const codes_t*>(codes + row * h + col);
        k.b[c] = scales[row * nb + col / KEEP_BLOCK];
        if (dres) k.res[c] = *reinterpret_cast<const V*>(dres + row * h + col);
      }
    }
  };
  auto process = [&](const Row& k, size_t row, int turn) {
    const bool on = row < (size_t)rows;
    float xh[C][V::N], sg = 0.f, sgx = 0.f;
    if (on) {
#pragma unroll
      for (int c = 0; c < C; ++c) {
        if ((l + c * W * 64) * V::N < h) {
          keep_values(k.q[c], keep_scale(k.b[c]), xh[c]);
#pragma unroll
          for (int e = 0; e < V::N; ++e) {
            xh[c][e] = (xh[c][e] - k.mean) * k.r;
            const float d = k.d[c].get(e), g = d * gv[c].get(e);
            if (LN) sg += g;
            sgx += g * xh[c][e];
            pg[c][e] += d * xh[c][e];
            if (LN) pb[c][e] += d;
          }
        }
      }
    }
    // both sums behind one barrier; the next row's take the other half of red
    sgx = lanes_sum<64>(sgx);
    if (LN) sg = lanes_sum<64>(sg);
    if (W > 1) {
      if ((threadIdx.x & 63) == 0) {
        red[turn][0][slot * W + wave] = sgx;
        if (LN) red[turn][1][slot * W + wave] = sg;
      }
      __syncthreads();
      sgx = sg = 0.f;
#pragma unroll
      for (int w = 0; w < W; ++w) {
        sgx += red[turn][0][slot * W + w];
        if (LN) sg += red[turn][1][slot * W + w];
      }
    }
    const float mgx = sgx / h, mg = LN ? sg / h : 0.f;
    if (!on) return;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int col = (l + c * W * 64) * V::N;
      if (col < h) {
        V o, n;
#pragma unroll
        for (int e = 0; e < V::N; ++e) {
          float v = k.r * (k.d[c].get(e) * gv[c].get(e) - mg - xh[c][e] * mgx);
          if (dres) v += k.res[c].get(e);
          o.set(e, v);
          float y = xh[c][e] * gv[c].get(e);
          if constexpr (LN) y += bv[c].get(e);
          n.set(e, y);
        }
        *reinterpret_cast<V*>(dx + row * h + col) = o;
        if (out) *reinterpret_cast<V*>(out + row * h + col) = n;
      }
    }
  };
  const size_t step = (size_t)gridDim.x * R;
  size_t row = (size_t)blockIdx.x * R + slot;
  load(buf[0], row);
  for (size_t first = (size_t)blockIdx.x * R; first < (size_t)rows; first += 2 * step, row += 2 * step) {
    load(buf[1], row + step);
    process(buf[0], row, 0);
    load(buf[0], row + 2 * step);
    process(buf[1], row + step, 1);
  }
#pragma unroll
  for (int part = 0; part < (LN ? 2 : 1); ++part) {
    float (&p)[C][V::N] = part ? reinterpret_cast<float (&)[C][V::N]>(pb) : pg;
    const bool alone = gridDim.x == 1;
    float* to = alone ? (part ? dbeta : dgamma) : partial + ((size_t)part * gridDim.x + blockIdx.x) * h;
    const auto put = [&](int at, f32x4_t v) {
      if (at >= h) return;
      if (alone) v += *reinterpret_cast<const f32x4_t*>(to + at);
      *reinterpret_cast<f32x4_t*>(to + at) = v;
    };
    if (R > 1) {
      if (part) __syncthreads();
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int e = 0; e < V::N; e += 4) sums[slot][(c * V::N + e) / 4][l] = (f32x4_t){p[c][e], p[c][e + 1], p[c][e + 2], p[c][e + 3]};
      __syncthreads();
      for (int i = threadIdx.x; i < C * V::N / 4 * W * 64; i += W * R * 64) {
        const int q = i / (W * 64), lane = i % (W * 64), at = (lane + q / (V::N / 4) * W * 64) * V::N + q % (V::N / 4) * 4;
        f32x4_t t = sums[0][q][lane];
#pragma unroll
        for (int k = 1; k < R; ++k) t += sums[k][q][lane];
        put(at, t);
      }
    } else {
#pragma unroll
      for (int c = 0; c < C; ++c) {
#pragma unroll
        for (int e = 0; e < V::N; e += 4) put((l + c * W * 64) * V::N + e, (f32x4_t){p[c][e], p[c][e + 1], p[c][e + 2], p[c][e + 3]});
      }
    }
  }
}

// Workgroups' sums, one row each, into the accumulators: 32 columns x 32 groups of rows, eight loads of a lane in flight, a fixed order (the
// lane's rows one after the other, then the 32 groups).  Bound by the latency of its few loads and of the launch.
__global__ __launch_bounds__(1024) void add_columns_kernel(const float* __restrict__ partial, float* dst0, float* dst1, int rows, int cols) {
  __shared__ float red[32][33];
  const int cx = threadIdx.x & 31, g = threadIdx.x >> 5, col = blockIdx.x * 32 + cx;
  const float* p = partial + (size_t)blockIdx.y * rows * cols + col;
  float s = 0.f;
  if (col < cols)
    for (int b0 = g; b0 < rows; b0 += 256) {
      float v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = b0 + 32 * i < rows ? p[(size_t)(b0 + 32 * i) * cols] : 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) s += v[i];
    }
  red[g][cx] = s;
  __syncthreads();
  // a wave adds up two columns, 32 lanes each
  float t = red[threadIdx.x & 31][threadIdx.x >> 5];
  t = lanes_sum<32>(t);
  const int out = blockIdx.x * 32 + (threadIdx.x >> 5);
  if ((threadIdx.x & 31) == 0 && out < cols) (blockIdx.y ? dst1 : dst0)[out] += t;
}

// ---- the MLP activation -----------------------------------------------------------------------------------
// Bound by memory, in bf16 only without the functions of common.h: those cost some 50 instructions a value (a division, expf, erff) where results keep 8
// bits of them.  There the sigmoid comes from the hardware's exp2 and reciprocal (relative error of a few 2^-23).
//
// GELU in both types: the tail of the normal distribution is exp(-x^2 / 2) F(u), u = |x| / sqrt(2), and the gradient needs the exponential anyway.  F is a polynomial in
// t = 1 / (1 + p u) or in w = 1 - t = p u t.  Its coefficients are a linear program's, over u <= 9.6: the least worst ratio of the error to the lesser of a share of
// F and an amount outright.  fp32: 2^-22 and 5e-9 by nine terms in w, of which the first is 1 / 2, so that little is rounded where x is small; with the
// roundings, of the exponent's argument above all, less than (2 x^2 + 40) 2^-24 of the tail down to 2^-126.  0.5 (1 + erf) would lose it (4 % off at -5, 0
// from -6 on), and 0.5 erfc costs issue (4096 x 11008: 95 and 113 us, forward and backward, instead of 69 and 101).  bf16: 2^-12 and 5e-8 by six terms in t
// (eight: forward 41 us instead of 37; the form in w 38).
template <typename T> struct Math;
template <> struct Math<float> {
  static __device__ __forceinline__ float sigmoid(float x) { return sigmoidf_(x); }
  static __device__ __forceinline__ float tail_factor(float x) {
    const float q = fminf(fabsf(x), 64.f) * (0.42f * 0.70710678118654752f);       // finite; the exponential is 0 long before
    const float w = q * __builtin_amdgcn_rcpf(1.f + q);
    float s = fmaf(w, 0.0361065609f, -0.125003526f);
    s = fmaf(w, s, 0.0899473243f);
    s = fmaf(w, s, 0.132865721f);
    s = fmaf(w, s, -0.0299308343f);
    s = fmaf(w, s, -0.75188043f);
    s = fmaf(w, s, 1.49120338f);
    s = fmaf(w, s, -1.34330943f);
    return fmaf(w, s, 0.5f);
  }
};
template <> struct Math<bf16_t> {
  static __device__ __forceinline__ float sigmoid(float x) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(x * -1.44269504088896341f)); }
  static __device__ __forceinline__ float tail_factor(float x) {
    const float t = __builtin_amdgcn_rcpf(fmaf(fabsf(x), 0.41f * 0.70710678118654752f, 1.f));
    float s = fmaf(t, -0.089376044f, 0.28699966f);
    s = fmaf(t, s, -0.0956544678f);
    s = fmaf(t, s, 0.180688379f);
    s = fmaf(t, s, 0.100530932f);
    s = fmaf(t, s, 0.116811496f);
    return t * s;
  }
};
template <typename T> __device__ __forceinline__ void normal(float x, float& cdf, float& density) {
  const float e = __builtin_amdgcn_exp2f(x * x * -0.72134752044448170f), tail = Math<T>::tail_factor(x) * e;       // e = exp(-x^2 / 2)
  cdf = x < 0.f ? tail : 1.f - tail;
  density = 0.39894228040143268f * e;
}
template <typename T, bool SWIGLU> __device__ __forceinline__ float activation(float x, float up) {
  if (SWIGLU) return x * Math<T>::sigmoid(x) * up;
  float cdf, density;
  normal<T>(x, cdf, density);
  return x * cdf;
}

template <typename T, bool SWIGLU, int U>
__global__ __launch_bounds__(NT) void act_fwd_pack8_kernel(const T* __restrict__ gu, T* __restrict__ a, uint8_t* __restrict__ codes, uint8_t* __restrict__ scales,
                                                           const Chunks k, int rows, int f) {
  typedef Vec16<T> V;
  typedef typename KeepChunk<T>::codes_t codes_t;
  constexpr int P = SWIGLU ? 2 : 1;
  const int nb = keep_blocks(f);
  for (size_t base = blockIdx.x * (size_t)(NT * U); base < k.total; base += (size_t)gridDim.x * (NT * U)) {
    const Walk<T> walk(base, k);
    V v[U][P] = {};
    At at[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      at[u] = walk.at(u * NT + threadIdx.x);
      if (at[u].row < (size_t)rows && at[u].col < f)
#pragma unroll
        for (int p = 0; p < P; ++p) v[u][p] = *reinterpret_cast<const V*>(gu + (at[u].row * P + p) * f + at[u].col);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
      for (int p = 0; p < P; ++p) {
        uint32_t byte;
        const codes_t c = keep_chunk<T>(v[u][p], byte);
        const size_t row = at[u].row * P + p;
        if (at[u].row < (size_t)rows) {
          if (at[u].col < f) *reinterpret_cast<codes_t*>(codes + row * f + at[u].col) = c;
          if (at[u].col % KEEP_BLOCK == 0) scales[row * nb + at[u].col / KEEP_BLOCK] = (uint8_t)byte;
        }
      }
      V o;
#pragma unroll
      for (int e = 0; e < V::N; ++e) o.set(e, activation<T, SWIGLU>(v[u][0].get(e), v[u][P - 1].get(e)));
      if (at[u].row < (size_t)rows && at[u].col < f) *reinterpret_cast<V*>(a + at[u].row * f + at[u].col) = o;
    }
  }
}

// a and dgu may be da: a thread reads its chunk of da before it writes there
template <typename T, bool SWIGLU, int U>
__global__ __launch_bounds__(NT) void act_bwd8_kernel(const T* da, const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, T* dgu, T* a, const Chunks k,
                                                      int rows, int f) {
  typedef Vec16<T> V;
  typedef typename KeepChunk<T>::codes_t codes_t;
  constexpr int P = SWIGLU ? 2 : 1;
  const int nb = keep_blocks(f);
  for (size_t base = blockIdx.x * (size_t)(NT * U); base < k.total; base += (size_t)gridDim.x * (NT * U)) {
    const Walk<T> walk(base, k);
    V d[U];
    codes_t c[U][P];
    uint32_t b[U][P];
    At at[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      at[u] = walk.at(u * NT + threadIdx.x);
      if (at[u].row < (size_t)rows && at[u].col < f) {
        d[u] = *reinterpret_cast<const V*>(da + at[u].row * f + at[u].col);
#pragma unroll
        for (int p = 0; p < P; ++p) {
          c[u][p] = *reinterpret_cast<const codes_t*>(codes + (at[u].row * P + p) * f + at[u].col);
          b[u][p] = scales[(at[u].row * P + p) * nb + at[u].col / KEEP_BLOCK];
        }
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (!(at[u].row < (size_t)rows && at[u].col < f)) continue;
      float x[P][V::N];
#pragma unroll
      for (int p = 0; p < P; ++p) keep_values(c[u][p], keep_scale(b[u][p]), x[p]);
      V o[P], act;
#pragma unroll
      for (int e = 0; e < V::N; ++e) {
        const float v = x[0][e], g = d[u].get(e);
        if constexpr (SWIGLU) {
          const float s = Math<T>::sigmoid(v), silu = v * s;
          o[0].set(e, g * x[1][e] * s * fmaf(v, 1.f - s, 1.f));
          o[1].set(e, g * silu);
          act.set(e, silu * x[1][e]);
        } else {
          float cdf, density;
          normal<T>(v, cdf, density);
          o[0].set(e, g * fmaf(v, density, cdf));
          act.set(e, v * cdf);
        }
      }
#pragma unroll
      for (int p = 0; p < P; ++p) *reinterpret_cast<V*>(dgu + (at[u].row * P + p) * f + at[u].col) = o[p];
      if (a) *reinterpret_cast<V*>(a + at[u].row * f + at[u].col) = act;
    }
  }
}


// Chunks in flight per thread.  16384 x 15360 bf16, pack and unpack: 285 us with 1, 269 with 2, 277 with 4, 296 with 8; the activation holds two or three
// operands of each: SwiGLU 4096 x 11008, forward and backward, 155 us with 1 or 2, 164 with 4; GELU 4999 x 4088 53 us with 1, 58 with 2.
constexpr int U = 2, UA = 1;
// Workgroups of norm_bwd8_kernel, one row of sums each: one per compute unit (4096 x 8192: 512 of them 65 us instead of 60, 384 74).  Rows that one workgroup has
// done in two turns are left to one, which saves the second launch (16 rows of 1024, forward and backward: 11.0 us a pass among others, 13.7 with it; four
// turns, 8 rows of 4096: 14.6 against 13.9).
constexpr int NORM_GROUPS = 256, NORM_TURNS = 2;
unsigned groups_of(const Chunks& k, int u) {
  const size_t groups = (k.total + (size_t)NT * u - 1) / ((size_t)NT * u);
  return (unsigned)(groups > (1u << 20) ? 1u << 20 : groups);
}

template <typename T> hipError_t run_pack8(const void* x, size_t ldx, uint8_t* codes, uint8_t* scales, int rows, int cols, hipStream_t s) {
  const Chunks k = chunks_of<T>(rows, cols);
  if (cols % Vec16<T>::N == 0) hipLaunchKernelGGL((pack8_kernel<T, U, true>), dim3(groups_of(k, U)), dim3(NT), 0, s, (const T*)x, ldx, codes, scales, k, rows, cols);
  else hipLaunchKernelGGL((pack8_kernel<T, U, false>), dim3(groups_of(k, U)), dim3(NT), 0, s, (const T*)x, ldx, codes, scales, k, rows, cols);
  return hipGetLastError();
}
template <typename T> hipError_t run_unpack8(const uint8_t* codes, const uint8_t* scales, void* x, size_t ldx, int rows, int cols, hipStream_t s) {
  const Chunks k = chunks_of<T>(rows, cols);
  if (cols % Vec16<T>::N == 0) hipLaunchKernelGGL((unpack8_kernel<T, U, true>), dim3(groups_of(k, U)), dim3(NT), 0, s, codes, scales, (T*)x, ldx, k, rows, cols);
  else hipLaunchKernelGGL((unpack8_kernel<T, U, false>), dim3(groups_of(k, U)), dim3(NT), 0, s, codes, scales, (T*)x, ldx, k, rows, cols);
  return hipGetLastError();
}
// f(W, C, R) for rows of h: the fewest waves that hold a row with at most two chunks a lane
template <typename T, typename F> auto norm_division(int h, F f) {
  const int chunks = h / Vec16<T>::N;
#define NORM_DIVISION(W, C, R) f(std::integral_constant<int, W>(), std::integral_constant<int, C>(), std::integral_constant<int, R>())
  if (chunks <= 64) return NORM_DIVISION(1, 1, 8);
  if (chunks <= 128) return NORM_DIVISION(1, 2, 8);
  if (chunks <= 256) return NORM_DIVISION(2, 2, 4);
  if (chunks <= 512) return NORM_DIVISION(4, 2, 2);
  if constexpr (Vec16<T>::N == 4)
    if (chunks > 1024) return NORM_DIVISION(16, 2, 1);                 // fp32 rows of more than 4096; bf16 rows of 8192, the widest, have 1024 chunks
  return NORM_DIVISION(8, 2, 1);
#undef NORM_DIVISION
}

template <typename T, bool LN>
hipError_t run_norm_fwd_pack8(const void* x, const void* gamma, const void* beta, void* out, float* stats, uint8_t* codes, uint8_t* scales, int rows, int h, float eps,
                              hipStream_t s) {
  norm_division<T>(h, [&](auto w, auto c, auto r) {
    hipLaunchKernelGGL((norm_fwd_pack8_kernel<T, LN, w, c, r>), dim3(min((rows + r - 1) / r, 1 << 20)), dim3(w * r * 64), 0, s, (const T*)x, (const T*)gamma, (const T*)beta, (T*)out, stats,
                       codes, scales, rows, h, eps);
  });
  return hipGetLastError();
}
template <typename T, bool LN>
hipError_t run_norm_bwd8(const void* dn, const uint8_t* codes, const uint8_t* scales, const float* stats, const void* gamma, const void* beta, const void* dres, void* dx,
                         void* out, float* partial, float* dgamma, float* dbeta, int rows, int h, hipStream_t s) {
  int nb = 0;
  norm_division<T>(h, [&](auto w, auto c, auto r) {
    nb = rows <= NORM_TURNS * r ? 1 : min((rows + r - 1) / r, NORM_GROUPS);
    hipLaunchKernelGGL((norm_bwd8_kernel<T, LN, w, c, r>), dim3(nb), dim3(w * r * 64), 0, s, (const T*)dn, codes, scales, stats, (const T*)gamma, (const T*)beta, (const T*)dres,
                       (T*)dx, (T*)out, partial, dgamma, dbeta, rows, h);
  });
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || nb == 1) return e;
  return launch_add_columns(partial, dgamma, LN ? dbeta : nullptr, nb, h, s);
}
template <typename T, bool SWIGLU>
hipError_t run_act_fwd_pack8(const void* gu, void* a, uint8_t* codes, uint8_t* scales, int rows, int f, hipStream_t s) {
  const Chunks k = chunks_of<T>(rows, f);
  hipLaunchKernelGGL((act_fwd_pack8_kernel<T, SWIGLU, UA>), dim3(groups_of(k, UA)), dim3(NT), 0, s, (const T*)gu, (T*)a, codes, scales, k, rows, f);
  return hipGetLastError();
}
template <typename T, bool SWIGLU>
hipError_t run_act_bwd8(const void* da, const uint8_t* codes, const uint8_t* scales, void* dgu, void* a, int rows, int f, hipStream_t s) {
  const Chunks k = chunks_of<T>(rows, f);
  hipLaunchKernelGGL((act_bwd8_kernel<T, SWIGLU, UA>), dim3(groups_of(k, UA)), dim3(NT), 0, s, (const T*)da, codes, scales, (T*)dgu, (T*)a, k, rows, f);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_add_columns(const float* partial, float* dst0, float* dst1, int rows, int cols, hipStream_t s) {
  hipLaunchKernelGGL(add_columns_kernel, dim3((cols + 31) / 32, dst1 ? 2 : 1), dim3(1024), 0, s, partial, dst0, dst1, rows, cols);
  return hipGetLastError();
}

// f<T, true / false>(...) by type and family
#define KEEP_BY_TYPE(f, ...) (dtype == DT_BF16 ? f<bf16_t>(__VA_ARGS__) : f<float>(__VA_ARGS__))
#define KEEP_BY_BOTH(f, flag, ...)                                                       \
  (dtype == DT_BF16 ? ((flag) ? f<bf16_t, true>(__VA_ARGS__) : f<bf16_t, false>(__VA_ARGS__)) \
                    : ((flag) ? f<float, true>(__VA_ARGS__) : f<float, false>(__VA_ARGS__)))

hipError_t launch_pack8(int dtype, const void* x, size_t ldx, uint8_t* codes, uint8_t* scales, int rows, int cols, hipStream_t s) {
  return KEEP_BY_TYPE(run_pack8, x, ldx, codes, scales, rows, cols, s);
}
hipError_t launch_unpack8(int dtype, const uint8_t* codes, const uint8_t* scales, void* x, size_t ldx, int rows, int cols, hipStream_t s) {
  return KEEP_BY_TYPE(run_unpack8, codes, scales, x, ldx, rows, cols, s);
}
bool norm8_shape_ok(int dtype, int h) { return h > 0 && h <= 8192 && h % (dtype == DT_BF16 ? 8 : 4) == 0; }
hipError_t launch_norm_fwd_pack8(int dtype, int family, const void* x, const void* gamma, const void* beta, void* out, float* stats, uint8_t* codes,
                                 uint8_t* scales, int rows, int h, float eps, hipStream_t s) {
  return KEEP_BY_BOTH(run_norm_fwd_pack8, family == FAM_GPT, x, gamma, beta, out, stats, codes, scales, rows, h, eps, s);
}
hipError_t launch_norm_bwd8(int dtype, int family, const void* dn, const uint8_t* codes, const uint8_t* scales, const float* stats, const void* gamma, const void* beta,
                            const void* dres, void* dx, void* out, float* partial, float* dgamma, float* dbeta, int rows, int h, hipStream_t s) {
  return KEEP_BY_BOTH(run_norm_bwd8, family == FAM_GPT, dn, codes, scales, stats, gamma, beta, dres, dx, out, partial, dgamma, dbeta, rows, h, s);
}
hipError_t launch_act_fwd_pack8(int dtype, int family, const void* gu, void* a, uint8_t* codes, uint8_t* scales, int rows, int f, hipStream_t s) {
  return KEEP_BY_BOTH(run_act_fwd_pack8, family == FAM_LLAMA, gu, a, codes, scales, rows, f, s);
}
hipError_t launch_act_bwd8(int dtype, int family, const void* da, const uint8_t* codes, const uint8_t* scales, void* dgu, void* a, int rows, int f, hipStream_t s) {
  return KEEP_BY_BOTH(run_act_bwd8, family == FAM_LLAMA, da, codes, scales, dgu, a, rows, f, s);
}
