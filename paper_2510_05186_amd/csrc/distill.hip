// Loss against a teacher's top entries.  With p = softmax(z / T) and the teacher's t_j at the words id_j,
//   loss = sum_j t_j (log t_j - log p[id_j]),   dz_v = g / T (p_v sum_j t_j - sum of t_j over id_j = v)
// for the gradient g of the row's loss.  Bound by memory: a row of logits in, a row of their gradient out; what is done with a teacher's entries (64 bits,
// one wave) runs while the row's loads are in flight.
//
// A row's maximum and sum are one pass: every thread keeps m and s = sum of exp((z - m) / T) of what it has seen, 16 bytes of the row at a time.
//  * Both directions, rows enough for the chip: a workgroup has a row in its registers from the maximum to the gradient (up to 128K words of bf16; of longer
//    ones the rest is read a second time).
//  * Rows too few for that: a row in pieces, a launch for their m and s, a second one that joins them and writes the gradient.
//  * Forward or backward alone: the pass over the row without keeping it.
// The gradient at the entries' words is written once more behind the row, whole, so that it has one rounding as every other.
#include "common.h"

namespace {

constexpr float LOG2E = 1.4426950408889634f, LOWEST = -3.402823466e38f;
constexpr int MAX_K = 1024;

// 16 bytes of a row at any address of its elements
template <typename T> struct Any16;
template <> struct Any16<bf16_t> { typedef bf16_t t __attribute__((ext_vector_type(8), aligned(2))); };
template <> struct Any16<float> { typedef float t __attribute__((ext_vector_type(4), aligned(4))); };

struct Distill {
  const void* z; const int* ids; const float* teacher; const float* dloss;
  float* loss; float* lse; void* dz;
  size_t ldz, lddz;
  int rows, vocab, k;
  float inv_t, c;                                       // 1 / T, log2(e) / T
  int log_probs;
  int pieces, piece;                                    // of a row, and elements of one (a multiple of a chunk)
  float2* stats; double2* parts;                        // [rows][pieces]: m, s; [rows]: sum of t (log t - z / T), sum of t
};

// m and s of what a thread has seen.  m starts at a finite number: minus infinity (a masked word) lies below it and adds nothing.
struct Running {
  float m = LOWEST, s = 0.f;
  template <int N> __device__ __forceinline__ void add(const float (&x)[N], float c) {
    float most = x[0];
#pragma unroll
    for (int e = 1; e < N; ++e) most = fmaxf(most, x[e]);
    const float mn = fmaxf(m, most);
    float t = 0.f;
#pragma unroll
    for (int e = 0; e < N; ++e) t += __builtin_amdgcn_exp2f((x[e] - mn) * c);
    s = fmaf(s, __builtin_amdgcn_exp2f((m - mn) * c), t);
    m = mn;
  }
  __device__ __forceinline__ void join(float m1, float s1, float c) {
    const float mn = fmaxf(m, m1);
    s = s * __builtin_amdgcn_exp2f((m - mn) * c) + s1 * __builtin_amdgcn_exp2f((m1 - mn) * c);
    m = mn;
  }
  __device__ __forceinline__ void join_wave(float c) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) join(__shfl_xor(m, o, 64), __shfl_xor(s, o, 64), c);
  }
};

// the row's entries, for the whole workgroup
struct Entries {
  int id[MAX_K];
  float t[MAX_K], z[MAX_K];
  double sum, mass;                                     // sum of t (log t - z / T), sum of t
};
struct Shared {
  Entries e;
  float m[16], s[16];
};

__device__ __forceinline__ double wave_sum64(double v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

// One wave: ids, t and z at the ids into LDS.  Read before anything of the row is written (dz may be z).
template <typename T> __device__ __forceinline__ void read_entries(const Distill& p, size_t row, Entries& e) {
  const int lane = threadIdx.x & 63;
  const int* ids = p.ids + row * p.k;
  const float* teacher = p.teacher + row * p.k;
  const T* z = (const T*)p.z + row * p.ldz;
  float most = -INFINITY;
  for (int j = lane; j < p.k; j += 64) {
    const int id = ids[j];
    const bool on = (unsigned)id < (unsigned)p.vocab;
    const float a = on ? (p.log_probs ? teacher[j] : teacher[j] * p.inv_t) : -INFINITY;
    e.id[j] = on ? id : -1;
    e.t[j] = a;
    e.z[j] = on ? (float)z[id] : 0.f;
    most = fmaxf(most, a);
  }
  most = wave_max(most);
  const double shift = p.log_probs || most == -INFINITY ? 0.0 : (double)most;
  double norm = 1.0;
  if (!p.log_probs) {
    norm = 0.0;
    for (int j = lane; j < p.k; j += 64) norm += exp((double)e.t[j] - shift);
    norm = wave_sum64(norm);
    if (norm == 0.0) norm = 1.0;                        // no entries
  }
  const double log_norm = shift + log(norm);
  double sum = 0.0, mass = 0.0;
  for (int j = lane; j < p.k; j += 64) {
    const double lt = (double)e.t[j] - log_norm, t = exp(lt);
    if (t != 0.0) sum += t * (lt - (double)e.z[j] * (double)p.inv_t);
    mass += t;
    e.t[j] = (float)t;
  }
  sum = wave_sum64(sum);
  mass = wave_sum64(mass);
  if (lane == 0) { e.sum = sum; e.mass = mass; }
}

// the gradient at entry j's word, t being all that the row's entries give it
__device__ __forceinline__ float teacher_at(const Entries& e, int k, int id) {
  float t = 0.f;
  for (int i = 0; i < k; ++i) t += e.id[i] == id ? e.t[i] : 0.f;
  return t;
}

template <typename T> __device__ __forceinline__ void load_chunk(const T* z, int at, int end, float (&x)[Vec16<T>::N]) {
  constexpr int N = Vec16<T>::N;
  if (at + N <= end) {
    const typename Any16<T>::t v = *reinterpret_cast<const typename Any16<T>::t*>(z + at);
#pragma unroll
    for (int e = 0; e < N; ++e) x[e] = (float)v[e];
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e) x[e] = at + e < end ? (float)z[at + e] : -INFINITY;
  }
}
template <typename T> __device__ __forceinline__ void store_chunk(T* dz, int at, int end, const float (&x)[Vec16<T>::N]) {
  constexpr int N = Vec16<T>::N;
  if (at + N <= end) {
    typename Any16<T>::t v;
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = (T)x[e];
    *reinterpret_cast<typename Any16<T>::t*>(dz + at) = v;
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (at + e < end) dz[at + e] = (T)x[e];
  }
}

// m and s of the whole workgroup, in all threads
template <int NT> __device__ __forceinline__ Running join_group(Running r, Shared& sh, float c) {
  r.join_wave(c);
  if ((threadIdx.x & 63) == 0) { sh.m[threadIdx.x >> 6] = r.m; sh.s[threadIdx.x >> 6] = r.s; }
  __syncthreads();
  Running all;
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) all.join(sh.m[w], sh.s[w], c);
  return all;
}
__device__ __forceinline__ double log_total(const Distill& p, const Running& r) { return (double)r.m * (double)p.inv_t + log((double)r.s); }

// ---- a row in a workgroup's registers: R chunks a thread
template <typename T, int NT, int R> __global__ __launch_bounds__(NT) void distill_row(const Distill p) {
  constexpr int N = Vec16<T>::N, STEP = NT * N, HELD = R * STEP;
  __shared__ Shared sh;
  const size_t row = blockIdx.x;
  const T* z = (const T*)p.z + row * p.ldz;
  T* dz = (T*)p.dz + row * p.lddz;
  const int first = threadIdx.x * N;
  typename Any16<T>::t held[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int at = first + r * STEP;
    if (at + N <= p.vocab) held[r] = *reinterpret_cast<const typename Any16<T>::t*>(z + at);
    else
#pragma unroll
      for (int e = 0; e < N; ++e) held[r][e] = at + e < p.vocab ? z[at + e] : (T)-INFINITY;
  }
  if (threadIdx.x < 64) read_entries<T>(p, row, sh.e);
  Running run;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    if (r * STEP >= p.vocab) break;
    float x[N];
#pragma unroll
    for (int e = 0; e < N; ++e) x[e] = (float)held[r][e];
    run.add(x, p.c);
  }
  for (int at = HELD + first; at < p.vocab; at += STEP) {
    float x[N];
    load_chunk(z, at, p.vocab, x);
    run.add(x, p.c);
  }
  const Running all = join_group<NT>(run, sh, p.c);
  const double mass = sh.e.mass;
  if (threadIdx.x == 0) {
    const double lse = log_total(p, all);
    p.lse[row] = (float)lse;
    p.loss[row] = (float)(mass == 0.0 ? 0.0 : sh.e.sum + mass * lse);
  }
  const float w = p.dloss[row] * p.inv_t;
  const bool none = w == 0.f || mass == 0.0;
  const float f = none ? 0.f : w * (float)mass / all.s;
  auto give = [&](int at, float (&x)[N]) {
#pragma unroll
    for (int e = 0; e < N; ++e) x[e] = none ? 0.f : f * __builtin_amdgcn_exp2f((x[e] - all.m) * p.c);
    store_chunk(dz, at, p.vocab, x);
  };
#pragma unroll
  for (int r = 0; r < R; ++r) {
    if (r * STEP >= p.vocab) break;
    float x[N];
#pragma unroll
    for (int e = 0; e < N; ++e) x[e] = (float)held[r][e];
    give(first + r * STEP, x);
  }
  for (int at = HELD + first; at < p.vocab; at += STEP) {
    float x[N];
    load_chunk(z, at, p.vocab, x);
    give(at, x);
  }
  if (none) return;
  __syncthreads();
  for (int j = threadIdx.x; j < p.k; j += NT) {
    const int id = sh.e.id[j];
    if (id >= 0) dz[id] = (T)(f * __builtin_amdgcn_exp2f((sh.e.z[j] - all.m) * p.c) - w * teacher_at(sh.e, p.k, id));
  }
}

// ---- m and s of a row's piece; forward alone and a whole row: loss and lse.  Grid rows x pieces.
template <typename T, int NT> __global__ __launch_bounds__(NT) void distill_stats(const Distill p) {
  constexpr int N = Vec16<T>::N, STEP = NT * N, U = 4;
  __shared__ Shared sh;
  const size_t row = blockIdx.x / p.pieces;
  const int piece = blockIdx.x % p.pieces, begin = piece * p.piece, end = min(p.vocab, begin + p.piece);
  const T* z = (const T*)p.z + row * p.ldz;
  if (piece == 0 && threadIdx.x < 64) read_entries<T>(p, row, sh.e);
  Running run;
  int at = begin + threadIdx.x * N;
  for (; at + (U - 1) * STEP + N <= end; at += U * STEP) {
    typename Any16<T>::t v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = *reinterpret_cast<const typename Any16<T>::t*>(z + at + u * STEP);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float x[N];
#pragma unroll
      for (int e = 0; e < N; ++e) x[e] = (float)v[u][e];
      run.add(x, p.c);
    }
  }
  for (; at < end; at += STEP) {
    float x[N];
    load_chunk(z, at, end, x);
    run.add(x, p.c);
  }
  const Running all = join_group<NT>(run, sh, p.c);
  if (threadIdx.x) return;
  if (p.dz || p.pieces > 1) {                            // joined by the next launch
    p.stats[blockIdx.x] = make_float2(all.m, all.s);
    if (piece == 0) p.parts[row] = make_double2(sh.e.sum, sh.e.mass);
    return;
  }
  const double lse = log_total(p, all);
  p.lse[row] = (float)lse;
  p.loss[row] = (float)(sh.e.mass == 0.0 ? 0.0 : sh.e.sum + sh.e.mass * lse);
}

// m and s of a row from its pieces, in the same order for every reader: one wave
__device__ __forceinline__ Running join_pieces(const Distill& p, size_t row) {
  Running r;
  for (int i = threadIdx.x & 63; i < p.pieces; i += 64) {
    const float2 v = p.stats[row * p.pieces + i];
    r.join(v.x, v.y, p.c);
  }
  r.join_wave(p.c);
  return r;
}
__device__ __forceinline__ void finish(const Distill& p, size_t row, const Running& r) {
  const double2 part = p.parts[row];
  const double lse = log_total(p, r);
  p.lse[row] = (float)lse;
  p.loss[row] = (float)(part.y == 0.0 ? 0.0 : part.x + part.y * lse);
}
__global__ __launch_bounds__(256) void distill_finish(const Distill p) {
  const size_t row = (size_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (row >= (size_t)p.rows) return;
  const Running r = join_pieces(p, row);
  if ((threadIdx.x & 63) == 0) finish(p, row, r);
}

// ---- the gradient of a row's piece, from lse (JOIN: from the pieces' m and s, the first piece writes loss and lse).  Grid rows x pieces.
template <typename T, int NT, bool JOIN> __global__ __launch_bounds__(NT) void distill_grad(const Distill p) {
  constexpr int N = Vec16<T>::N, STEP = NT * N, U = 4;
  __shared__ Shared sh;
  const size_t row = blockIdx.x / p.pieces;
  const int piece = blockIdx.x % p.pieces, begin = piece * p.piece, end = min(p.vocab, begin + p.piece);
  const T* z = (const T*)p.z + row * p.ldz;
  T* dz = (T*)p.dz + row * p.lddz;
  if (threadIdx.x < 64) {
    if (JOIN) {
      const Running r = join_pieces(p, row);
      if (threadIdx.x == 0) {
        sh.m[0] = r.m;
        sh.s[0] = r.s;
        if (piece == 0) finish(p, row, r);
      }
    }
    read_entries<T>(p, row, sh.e);
  }
  __syncthreads();
  const float w = p.dloss[row] * p.inv_t;
  const double mass = sh.e.mass;
  const bool none = w == 0.f || mass == 0.0;
  // p = exp((z - m) / T) / s, or exp(z / T - lse): f exp2(z c - shift)
  const float m = JOIN ? sh.m[0] : 0.f, l = JOIN ? 0.f : p.lse[row] * LOG2E;
  const float f = none ? 0.f : JOIN ? w * (float)mass / sh.s[0] : w * (float)mass;
  auto prob = [&](float x) { return f * __builtin_amdgcn_exp2f(JOIN ? (x - m) * p.c : fmaf(x, p.c, -l)); };
  int at = begin + threadIdx.x * N;
  if (none) {
    const float x[N] = {};
    for (; at < end; at += STEP) store_chunk(dz, at, end, x);
    return;
  }
  for (; at + (U - 1) * STEP + N <= end; at += U * STEP) {
    typename Any16<T>::t v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = *reinterpret_cast<const typename Any16<T>::t*>(z + at + u * STEP);
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
      for (int e = 0; e < N; ++e) v[u][e] = (T)prob((float)v[u][e]);
      *reinterpret_cast<typename Any16<T>::t*>(dz + at + u * STEP) = v[u];
    }
  }
  for (; at < end; at += STEP) {
    float x[N];
    load_chunk(z, at, end, x);
#pragma unroll
    for (int e = 0; e < N; ++e) x[e] = prob(x[e]);
    store_chunk(dz, at, end, x);
  }
  __syncthreads();
  for (int j = threadIdx.x; j < p.k; j += NT) {
    const int id = sh.e.id[j];
    if (id >= begin && id < end) dz[id] = (T)(prob(sh.e.z[j]) - w * teacher_at(sh.e, p.k, id));
  }
}

// Rows below this many leave compute units idle with a workgroup each: they go in pieces.
constexpr int FEW_ROWS = 160;
// A row's pieces: some 1024 workgroups in all, pieces of 2048 elements and more
int pieces_of(int rows, int vocab) {
  const int most = (vocab + 2047) / 2048, want = (1024 + rows - 1) / rows;
  return most < want ? most : want;
}
void divide(Distill& p, int pieces) {
  p.piece = ((p.vocab + pieces - 1) / pieces + 7) / 8 * 8;
  p.pieces = (p.vocab + p.piece - 1) / p.piece;
}

template <typename T> hipError_t run_both(const Distill& p, hipStream_t s) {
  const int chunks = (p.vocab + Vec16<T>::N - 1) / Vec16<T>::N;
  const dim3 grid(p.rows);
  if (chunks <= 256 * 2) hipLaunchKernelGGL((distill_row<T, 256, 2>), grid, dim3(256), 0, s, p);
  else if (chunks <= 256 * 8) hipLaunchKernelGGL((distill_row<T, 256, 8>), grid, dim3(256), 0, s, p);
  else if (chunks <= 512 * 8) hipLaunchKernelGGL((distill_row<T, 512, 8>), grid, dim3(512), 0, s, p);
  else if (chunks <= 1024 * 8) hipLaunchKernelGGL((distill_row<T, 1024, 8>), grid, dim3(1024), 0, s, p);
  else hipLaunchKernelGGL((distill_row<T, 1024, 16>), grid, dim3(1024), 0, s, p);
  return hipGetLastError();
}

template <typename T> hipError_t run(Distill p, hipStream_t s) {
  if (p.loss && p.dz && p.rows >= FEW_ROWS) return run_both<T>(p, s);
  if (p.loss) {
    divide(p, p.rows >= FEW_ROWS ? 1 : pieces_of(p.rows, p.vocab));
    hipLaunchKernelGGL((distill_stats<T, 256>), dim3((unsigned)p.rows * p.pieces), dim3(256), 0, s, p);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    if (p.dz) hipLaunchKernelGGL((distill_grad<T, 256, true>), dim3((unsigned)p.rows * p.pieces), dim3(256), 0, s, p);
    else if (p.pieces > 1) hipLaunchKernelGGL(distill_finish, dim3((p.rows + 3) / 4), dim3(256), 0, s, p);
    return hipGetLastError();
  }
  divide(p, p.rows >= FEW_ROWS ? 1 : pieces_of(p.rows, p.vocab));
  hipLaunchKernelGGL((distill_grad<T, 256, false>), dim3((unsigned)p.rows * p.pieces), dim3(256), 0, s, p);
  return hipGetLastError();
}

}  // namespace

uint64_t distill_ws_bytes(int rows, int vocab, int) {
  return 16 + (rows < FEW_ROWS ? 16ull * rows + 8ull * rows * pieces_of(rows, vocab) : 0);
}

hipError_t launch_distill(int dtype, const void* z, size_t ldz, const int* ids, const float* teacher, const float* dloss, float* loss, float* lse, void* dz, size_t lddz,
                          void* ws, int rows, int vocab, int k, float temperature, int log_probs, hipStream_t s) {
  Distill p = {z, ids, teacher, dloss, loss, lse, dz, ldz, lddz, rows, vocab, k, 1.f / temperature, LOG2E / temperature, log_probs, 1, vocab, nullptr, nullptr};
  p.parts = (double2*)ws;
  p.stats = (float2*)(p.parts + rows);
  return dtype == DT_BF16 ? run<bf16_t>(p, s) : run<float>(p, s);
}
