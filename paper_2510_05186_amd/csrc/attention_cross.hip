// Attention of queries to the states of another sequence, of which the first kv_len count, with its gradients: a wave per row, fp32 throughout.
#include "common.h"

namespace {

struct Cross {
  const void *q, *k, *v; const int* kv_len; const void *o_in, *dout;
  void* o; float* lse; void *dq, *dk, *dv; float* delta;
  size_t ldq, ldkv;
  int seq_q, seq_kv, batch, n_q, n_kv;
};

__device__ __forceinline__ int states(const Cross& p, int b) { return p.kv_len ? min(max(p.kv_len[b], 0), p.seq_kv) : p.seq_kv; }

template <typename T, int D, bool BWD> __global__ __launch_bounds__(256) void cross_rows(const Cross p) {
  constexpr int E = D / 64;
  const int lane = threadIdx.x & 63;
  const size_t item = (size_t)blockIdx.x * 4 + (threadIdx.x >> 6);            // (sequence, head, query)
  if (item >= (size_t)p.batch * p.n_q * p.seq_q) return;
  const int t = item % p.seq_q, a = item / p.seq_q % p.n_q, b = item / p.seq_q / p.n_q, h = a / (p.n_q / p.n_kv);
  const size_t row = (size_t)b * p.seq_q + t;
  const int n = states(p, b);
  const float scale = rsqrtf((float)D);
  const T* q = (const T*)p.q + row * p.ldq + (size_t)a * D;
  float x[E], acc[E] = {}, g[E], m = -INFINITY, l = 0.f, dd = 0.f, L = 0.f;
  for (int e = 0; e < E; ++e) x[e] = (float)q[lane + 64 * e] * scale;
  if (BWD) {
    const size_t at = row * p.n_q * D + (size_t)a * D + lane;
    for (int e = 0; e < E; ++e) {
      g[e] = (float)((const T*)p.dout)[at + 64 * e];
      dd += g[e] * (float)((const T*)p.o_in)[at + 64 * e];
    }
    dd = wave_sum(dd);
    L = p.lse[item];
    if (lane == 0) p.delta[item] = dd;
  }
  for (int j = 0; j < n; ++j) {
    const T* k = (const T*)p.k + ((size_t)b * p.seq_kv + j) * p.ldkv + (size_t)h * D + lane;
    const T* v = (const T*)p.v + ((size_t)b * p.seq_kv + j) * p.ldkv + (size_t)h * D + lane;
    float s = 0.f, dp = 0.f;
    for (int e = 0; e < E; ++e) s += x[e] * (float)k[64 * e];
    s = wave_sum(s);
    if (BWD) {
      for (int e = 0; e < E; ++e) dp += g[e] * (float)v[64 * e];
      dp = wave_sum(dp);
      const float ds = n == 1 ? 0.f : expf(s - L) * (dp - dd) * scale;
      for (int e = 0; e < E; ++e) acc[e] += ds * (float)k[64 * e];
    } else {
      const float mn = s > m || s != s ? s : m, f = expf(m - mn), w = expf(s - mn);
      l = l * f + w;
      for (int e = 0; e < E; ++e) acc[e] = acc[e] * f + w * (float)v[64 * e];
      m = mn;
    }
  }
  T* out = BWD ? (T*)p.dq + row * p.ldq + (size_t)a * D + lane : (T*)p.o + row * p.n_q * D + (size_t)a * D + lane;
  for (int e = 0; e < E; ++e) out[64 * e] = (T)(BWD || n == 0 ? acc[e] : acc[e] / l);
  if (!BWD && lane == 0) p.lse[item] = n == 0 ? -INFINITY : m + logf(l);
}

template <typename T, int D> __global__ __launch_bounds__(256) void cross_states(const Cross p) {
  constexpr int E = D / 64;
  const int lane = threadIdx.x & 63;
  const size_t item = (size_t)blockIdx.x * 4 + (threadIdx.x >> 6);            // (sequence, head, state)
  if (item >= (size_t)p.batch * p.n_kv * p.seq_kv) return;
  const int j = item % p.seq_kv, h = item / p.seq_kv % p.n_kv, b = item / p.seq_kv / p.n_kv;
  const size_t at = ((size_t)b * p.seq_kv + j) * p.ldkv + (size_t)h * D + lane;
  const int n = states(p, b);
  const float scale = rsqrtf((float)D);
  float k[E], v[E], ak[E] = {}, av[E] = {};
  if (j < n) {
    for (int e = 0; e < E; ++e) {
      k[e] = (float)((const T*)p.k)[at + 64 * e] * scale;
      v[e] = (float)((const T*)p.v)[at + 64 * e];
    }
    const int rep = p.n_q / p.n_kv;
    for (int i = 0; i < rep * p.seq_q; ++i) {
      const int a = h * rep + i / p.seq_q, t = i % p.seq_q;
      const T* q = (const T*)p.q + ((size_t)b * p.seq_q + t) * p.ldq + (size_t)a * D + lane;
      const T* g = (const T*)p.dout + (((size_t)b * p.seq_q + t) * p.n_q + a) * D + lane;
      const size_t st = ((size_t)b * p.n_q + a) * p.seq_q + t;
      float s = 0.f, dp = 0.f;
      for (int e = 0; e < E; ++e) { s += (float)q[64 * e] * k[e]; dp += (float)g[64 * e] * v[e]; }
      s = wave_sum(s);
      dp = wave_sum(dp);
      const float w = expf(s - p.lse[st]), ds = n == 1 ? 0.f : w * (dp - p.delta[st]) * scale;
      for (int e = 0; e < E; ++e) { av[e] += w * (float)g[64 * e]; ak[e] += ds * (float)q[64 * e]; }
    }
  }
  for (int e = 0; e < E; ++e) { ((T*)p.dk)[at + 64 * e] = (T)ak[e]; ((T*)p.dv)[at + 64 * e] = (T)av[e]; }
}

unsigned waves4(size_t items) { return (unsigned)((items + 3) / 4); }
template <typename T, int D> hipError_t run(const Cross& p, bool bwd, hipStream_t s) {
  const unsigned g = waves4((size_t)p.batch * p.n_q * p.seq_q);
  if (!bwd) {
    hipLaunchKernelGGL((cross_rows<T, D, false>), dim3(g), dim3(256), 0, s, p);
    return hipGetLastError();
  }
  hipLaunchKernelGGL((cross_rows<T, D, true>), dim3(g), dim3(256), 0, s, p);
  hipLaunchKernelGGL((cross_states<T, D>), dim3(waves4((size_t)p.batch * p.n_kv * p.seq_kv)), dim3(256), 0, s, p);
  return hipGetLastError();
}
hipError_t run_any(int dtype, int d, const Cross& p, bool bwd, hipStream_t s) {
  if (dtype == DT_BF16) return d == 64 ? run<bf16_t, 64>(p, bwd, s) : run<bf16_t, 128>(p, bwd, s);
  return d == 64 ? run<float, 64>(p, bwd, s) : run<float, 128>(p, bwd, s);
}

}  // namespace

uint64_t cross_attn_ws_bytes(int, int seq_q, int, int batch, int n_q, int, int) { return 4ull * batch * n_q * seq_q; }

hipError_t launch_cross_attn_fwd(int dtype, const CrossShape& c, const void* q, const void* k, const void* v, const int* kv_len, void* o, float* lse, void*, hipStream_t s) {
  Cross p = {q, k, v, kv_len, nullptr, nullptr, o, lse, nullptr, nullptr, nullptr, nullptr, c.ldq, c.ldkv, c.seq_q, c.seq_kv, c.batch, c.n_q, c.n_kv};
  return run_any(dtype, c.d, p, false, s);
}
hipError_t launch_cross_attn_bwd(int dtype, const CrossShape& c, const void* q, const void* k, const void* v, const int* kv_len, const void* o, const void* dout,
                                 const float* lse, void* dq, void* dk, void* dv, void* ws, hipStream_t s) {
  Cross p = {q, k, v, kv_len, o, dout, nullptr, const_cast<float*>(lse), dq, dk, dv, (float*)ws, c.ldq, c.ldkv, c.seq_q, c.seq_kv, c.batch, c.n_q, c.n_kv};
  return run_any(dtype, c.d, p, true, s);
}
