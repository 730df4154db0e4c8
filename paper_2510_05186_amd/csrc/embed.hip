// Embedding: out[r] = scale * weight[ids[r]], and its gradient grad[t] += scale * (sum of dy[r] over the rows r with ids[r] = t).
// A row whose id is no word of the vocabulary (negative, or vocab and more: padding) is zero and has no gradient.
#include "common.h"

namespace {

constexpr int NT = 256;

template <typename T>
__global__ __launch_bounds__(NT) void embed_fwd_kernel(const int* __restrict__ ids, const T* __restrict__ weight, T* __restrict__ out, int rows, unsigned vocab, int h,
                                                       float scale) {
  typedef Vec16<T> V;
  const int nvec = h / V::N;
  const size_t total = (size_t)rows * nvec, step = (size_t)gridDim.x * NT;
  for (size_t i = blockIdx.x * (size_t)NT + threadIdx.x; i < total; i += step) {
    const size_t row = i / nvec;
    const int c = (int)(i % nvec);
    const unsigned id = (unsigned)ids[row];
    V v;
#pragma unroll
    for (int e = 0; e < V::N; ++e) v.set(e, 0.f);
    if (id < vocab) {
      v = *reinterpret_cast<const V*>(weight + (size_t)id * h + (size_t)c * V::N);
#pragma unroll
      for (int e = 0; e < V::N; ++e) v.set(e, v.get(e) * scale);
    }
    *reinterpret_cast<V*>(out + row * h + (size_t)c * V::N) = v;
  }
}

// place of every row among all rows in the order of (id, row), by counting; ids outside the vocabulary come last
__global__ __launch_bounds__(NT) void embed_rank_kernel(const int* __restrict__ ids, unsigned* __restrict__ key, unsigned* __restrict__ row_of, int rows, unsigned vocab) {
  __shared__ unsigned tile[NT];
  const int i = blockIdx.x * NT + threadIdx.x;
  unsigned mine = i < rows ? (unsigned)ids[i] : 0u;
  if (mine >= vocab) mine = 0xffffffffu;
  unsigned place = 0;
  for (int j0 = 0; j0 < rows; j0 += NT) {
    const int j = j0 + threadIdx.x;
    unsigned k = j < rows ? (unsigned)ids[j] : 0u;
    if (k >= vocab) k = 0xffffffffu;
    __syncthreads();
    tile[threadIdx.x] = k;
    __syncthreads();
    const int n = min(NT, rows - j0);
    for (int q = 0; q < n; ++q) place += tile[q] < mine || (tile[q] == mine && j0 + q < i);
  }
  if (i < rows) { key[place] = mine; row_of[place] = (unsigned)i; }
}

// one run of equal ids per workgroup (the workgroups of places where none begins end at once), its rows added in order
template <typename T>
__global__ __launch_bounds__(NT) void embed_sum_kernel(const unsigned* __restrict__ key, const unsigned* __restrict__ row_of, const T* __restrict__ dy,
                                                       float* __restrict__ grad, int rows, int h, float scale) {
  const int p = blockIdx.x;
  const unsigned id = key[p];
  if (id == 0xffffffffu || (p > 0 && key[p - 1] == id)) return;
  int end = p + 1;
  while (end < rows && key[end] == id) ++end;
  for (int c = threadIdx.x; c < h; c += NT) {
    float s = 0.f;
    for (int q = p; q < end; ++q) s += to_f32<T>(dy[(size_t)row_of[q] * h + c]);
    float* g = grad + (size_t)id * h + c;
    *g += scale * s;
  }
}

}  // namespace

uint64_t embed_bwd_ws_bytes(int rows, int h) { (void)h; return (uint64_t)rows * 8; }

hipError_t launch_embed_fwd(int dtype, const int* ids, const void* weight, void* out, int rows, unsigned vocab, int h, float scale, hipStream_t s) {
  const size_t groups = ((size_t)rows * h / (dtype == DT_BF16 ? 8 : 4) + NT - 1) / NT;
  const dim3 grid((unsigned)(groups > 8192 ? 8192 : groups));
  if (dtype == DT_BF16) hipLaunchKernelGGL(embed_fwd_kernel<bf16_t>, grid, dim3(NT), 0, s, ids, (const bf16_t*)weight, (bf16_t*)out, rows, vocab, h, scale);
  else hipLaunchKernelGGL(embed_fwd_kernel<float>, grid, dim3(NT), 0, s, ids, (const float*)weight, (float*)out, rows, vocab, h, scale);
  return hipGetLastError();
}

hipError_t launch_embed_bwd(int dtype, const int* ids, const void* dy, float* grad, void* ws, int rows, unsigned vocab, int h, float scale, hipStream_t s) {
  unsigned* key = (unsigned*)ws;
  unsigned* row_of = key + rows;
  hipLaunchKernelGGL(embed_rank_kernel, dim3((rows + NT - 1) / NT), dim3(NT), 0, s, ids, key, row_of, rows, vocab);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (dtype == DT_BF16) hipLaunchKernelGGL(embed_sum_kernel<bf16_t>, dim3(rows), dim3(NT), 0, s, key, row_of, (const bf16_t*)dy, grad, rows, h, scale);
  else hipLaunchKernelGGL(embed_sum_kernel<float>, dim3(rows), dim3(NT), 0, s, key, row_of, (const float*)dy, grad, rows, h, scale);
  return hipGetLastError();
}
