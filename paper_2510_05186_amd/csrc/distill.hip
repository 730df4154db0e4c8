// Loss against a teacher's top entries.  With p = softmax(z / T) and the teacher's t_j at the words id_j,
//   loss = sum_j t_j (log t_j - log p[id_j]),   dz_v = g / T (p_v sum_j t_j - sum of t_j over id_j = v)
// for the gradient g of the row's loss.  Bound by memory: a row of logits in, a row of their gradient out.
#include "common.h"

namespace {

constexpr int NT = 256;
constexpr float LOG2E = 1.4426950408889634f;

struct Distill {
  const void* z; const int* ids; const float* teacher; const float* dloss;
  float* loss; float* lse; void* dz;
  size_t ldz, lddz;
  int rows, vocab, k;
  float inv_t;
  int log_probs;
};

__device__ __forceinline__ float block_max(float v, float* lds) {
  v = wave_max(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  return fmaxf(fmaxf(lds[0], lds[1]), fmaxf(lds[2], lds[3]));
}
__device__ __forceinline__ float block_sum(float v, float* lds) {
  v = wave_sum(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  return (lds[0] + lds[1]) + (lds[2] + lds[3]);
}
__device__ __forceinline__ double block_sum(double v, double* lds) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  return (lds[0] + lds[1]) + (lds[2] + lds[3]);
}

// entry j's exponent before normalisation, minus infinity where it is not given
__device__ __forceinline__ float entry(const Distill& p, size_t row, int j, int* id) {
  *id = p.ids[row * p.k + j];
  if ((unsigned)*id >= (unsigned)p.vocab) return -INFINITY;
  const float t = p.teacher[row * p.k + j];
  return p.log_probs ? t : t * p.inv_t;
}

template <typename T> __global__ __launch_bounds__(NT) void distill_kernel(const Distill p) {
  __shared__ float red[4];
  __shared__ double redd[4];
  const size_t row = blockIdx.x;
  const T* z = (const T*)p.z + row * p.ldz;
  float m = 0.f, total = 1.f;
  double lse;
  if (p.loss) {
    m = -INFINITY;
    for (int v = threadIdx.x; v < p.vocab; v += NT) m = fmaxf(m, (float)z[v]);
    m = block_max(m, red);
    float s = 0.f;
    for (int v = threadIdx.x; v < p.vocab; v += NT) s += expf(((float)z[v] - m) * p.inv_t);
    total = block_sum(s, red);
    lse = (double)m * p.inv_t + log((double)total);
    if (threadIdx.x == 0) p.lse[row] = (float)lse;
  } else {
    lse = p.lse[row];
  }
  // the teacher's normalisation
  float tm = 0.f;
  double norm = 1.0;
  if (!p.log_probs) {
    float most = -INFINITY;
    int id;
    for (int j = threadIdx.x; j < p.k; j += NT) most = fmaxf(most, entry(p, row, j, &id));
    tm = block_max(most, red);
    if (tm == -INFINITY) tm = 0.f;
    double s = 0.0;
    for (int j = threadIdx.x; j < p.k; j += NT) s += exp((double)entry(p, row, j, &id) - tm);
    norm = block_sum(s, redd);
    if (norm == 0.0) norm = 1.0;
  }
  const double log_norm = tm + log(norm);
  double loss = 0.0, mass = 0.0;
  for (int j = threadIdx.x; j < p.k; j += NT) {
    int id;
    const double a = entry(p, row, j, &id);
    const double lt = a - log_norm, t = exp(lt);
    mass += t;
    if (t != 0.0) loss += t * (lt - (double)((float)z[id] * (double)p.inv_t) + lse);
  }
  mass = block_sum(mass, redd);
  if (p.loss) {
    loss = block_sum(loss, redd);
    if (threadIdx.x == 0) p.loss[row] = (float)loss;
  }
  if (!p.dz) return;
  T* dz = (T*)p.dz + row * p.lddz;
  const float w = p.dloss[row] * p.inv_t;
  if (w == 0.f || mass == 0.0) {
    for (int v = threadIdx.x; v < p.vocab; v += NT) dz[v] = (T)0.f;
    return;
  }
  const float wm = w * (float)mass;
  // the entries' own places are read before they may be overwritten (dz may be z)
  __syncthreads();
  extern __shared__ float own[];                                          // k values: z at the entries' words
  for (int j = threadIdx.x; j < p.k; j += NT) {
    int id;
    entry(p, row, j, &id);
    own[j] = (unsigned)id < (unsigned)p.vocab ? (float)z[id] : 0.f;
  }
  __syncthreads();
  const float lsef = (float)lse;
  auto prob = [&](float x) { return p.loss ? expf((x - m) * p.inv_t) / total : expf(x * p.inv_t - lsef); };
  for (int v = threadIdx.x; v < p.vocab; v += NT) dz[v] = (T)(wm * prob((float)z[v]));
  __syncthreads();
  for (int j = threadIdx.x; j < p.k; j += NT) {
    int id, other;
    entry(p, row, j, &id);
    if ((unsigned)id >= (unsigned)p.vocab) continue;
    double t = 0.0;
    for (int i = 0; i < p.k; ++i) {
      const double a = entry(p, row, i, &other);
      if (other == id) t += exp(a - log_norm);
    }
    dz[id] = (T)(wm * prob(own[j]) - w * (float)t);
  }
}

template <typename T> hipError_t run(const Distill& p, hipStream_t s) {
  hipLaunchKernelGGL(distill_kernel<T>, dim3(p.rows), dim3(NT), p.k * 4, s, p);
  return hipGetLastError();
}

}  // namespace

uint64_t distill_ws_bytes(int, int, int) { return 16; }

hipError_t launch_distill(int dtype, const void* z, size_t ldz, const int* ids, const float* teacher, const float* dloss, float* loss, float* lse, void* dz, size_t lddz,
                          void*, int rows, int vocab, int k, float temperature, int log_probs, hipStream_t s) {
  const Distill p = {z, ids, teacher, dloss, loss, lse, dz, ldz, lddz, rows, vocab, k, 1.f / temperature, log_probs};
  return dtype == DT_BF16 ? run<bf16_t>(p, s) : run<float>(p, s);
}
