// Norms of queries and keys with the position rotation, in one pass over packed qkv rows: every q and k head x becomes
// R(position) (x * r * gamma), r = 1 / sqrt(mean(x^2) + eps), and its gradient goes back the same way:
// dn = R^T dy, g = dn * gamma, dx = r (g - xh mean(g xh)) with xh = x r, dgamma = sum of dn * xh over rows and heads.
#include "keep8.h"

namespace {

constexpr int NT = 256;

__device__ __forceinline__ uint32_t half_wave_max(uint32_t v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, o, 64));
  return v;
}

struct QkNorm {
  const void* src; const uint8_t* codes_in; const uint8_t* scales_in;   // the projection's output, or its kept form
  void* dst; const void* gamma_q; const void* gamma_k; const float2* table; float* stats;
  uint8_t* codes; uint8_t* scales;                                      // where src is kept, or null
  int rows, seq, n_q, n_kv, d; float eps;
};

// one head per wave: lane l holds elements l + 64 i, i < d / 64 (at most 4); its partner in the rotation is d / 2 away
template <typename T, bool FROM8>
__global__ __launch_bounds__(NT) void qknorm_kernel(const QkNorm p) {
  __shared__ float line[NT / 64][256];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, d = p.d, half = d / 2, heads = p.n_q + 2 * p.n_kv, n_rot = p.n_q + p.n_kv;
  const size_t items = (size_t)p.rows * heads, w = (size_t)heads * d;
  for (size_t i0 = (size_t)blockIdx.x * (NT / 64); i0 < items; i0 += (size_t)gridDim.x * (NT / 64)) {
    const size_t i = i0 + wave;
    const bool on = i < items;
    const size_t row = on ? i / heads : 0;
    const int head = on ? (int)(i % heads) : 0;
    float ss = 0.f;
    for (int c = lane; c < d; c += 64) {
      const size_t at = row * w + (size_t)head * d + c;
      const float v = FROM8 ? keep_decode(p.codes_in[at], keep_scale(p.scales_in[at / KEEP_BLOCK])) : to_f32<T>(((const T*)p.src)[at]);
      if (!FROM8 && p.codes) {
        const uint32_t b = keep_scale_byte(half_wave_max(keep_magnitude(v)));
        if (on) p.codes[at] = (uint8_t)keep_encode(v, keep_inverse(b));
        if (on && (lane & 31) == 0) p.scales[at / KEEP_BLOCK] = (uint8_t)b;
      }
      line[wave][c] = v;
      ss += v * v;
    }
    __syncthreads();
    if (on && head < n_rot) {
      float r;
      if (FROM8) r = p.stats[row * n_rot + head];
      else {
        r = rsqrtf(wave_sum(ss) / d + p.eps);
        if (lane == 0) p.stats[row * n_rot + head] = r;
      }
      const T* gamma = (const T*)(head < p.n_q ? p.gamma_q : p.gamma_k);
      for (int k = lane; k < half; k += 64) {
        const float2 cs = p.table[(row % p.seq) * half + k];
        const float lo = line[wave][k] * r * to_f32<T>(gamma[k]), hi = line[wave][k + half] * r * to_f32<T>(gamma[k + half]);
        T* o = (T*)p.dst + row * w + (size_t)head * d + k;
        o[0] = from_f32<T>(lo * cs.x - hi * cs.y);
        o[half] = from_f32<T>(hi * cs.x + lo * cs.y);
      }
    } else if (on && p.dst != p.src) {
      for (int c = lane; c < d; c += 64) ((T*)p.dst)[row * w + (size_t)head * d + c] = from_f32<T>(line[wave][c]);
    }
    __syncthreads();
  }
}

struct QkNormBwd {
  const void* dy; const void* x; const uint8_t* codes; const uint8_t* scales; const float* stats;
  const void* gamma_q; const void* gamma_k; const float2* table; void* dx; float* partial;
  int rows, seq, n_q, n_kv, d;
};

// workgroup b takes rows b, b + gridDim.x, ...; its sums of the gains' gradients stand in partial[b] (q) and partial[gridDim.x + b] (k)
template <typename T, bool FROM8>
__global__ __launch_bounds__(NT) void qknorm_bwd_kernel(const QkNormBwd p) {
  __shared__ float sums[NT / 64][2][256];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, d = p.d, half = d / 2, heads = p.n_q + 2 * p.n_kv, n_rot = p.n_q + p.n_kv;
  const size_t w = (size_t)heads * d;
  for (int i = threadIdx.x; i < (NT / 64) * 512; i += NT) (&sums[0][0][0])[i] = 0.f;
  __syncthreads();
  for (size_t row = blockIdx.x; row < (size_t)p.rows; row += gridDim.x) {
    for (int head = wave; head < heads; head += NT / 64) {
      const size_t at = row * w + (size_t)head * d;
      const T* dy = (const T*)p.dy + at;
      T* dx = (T*)p.dx + at;
      if (head >= n_rot) {
        if (p.dx != p.dy)
          for (int c = lane; c < d; c += 64) dx[c] = dy[c];
        continue;
      }
      const float r = p.stats[row * n_rot + head];
      const T* gamma = (const T*)(head < p.n_q ? p.gamma_q : p.gamma_k);
      float* sum = sums[wave][head < p.n_q ? 0 : 1];
      float glo[2], ghi[2], xlo[2], xhi[2], s = 0.f;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int k = lane + 64 * i;
        if (k < half) {
          const float2 cs = p.table[(row % p.seq) * half + k];
          const float a = to_f32<T>(dy[k]), b = to_f32<T>(dy[k + half]);
          const float nlo = a * cs.x + b * cs.y, nhi = b * cs.x - a * cs.y;
          const float vlo = FROM8 ? keep_decode(p.codes[at + k], keep_scale(p.scales[(at + k) / KEEP_BLOCK])) : to_f32<T>(((const T*)p.x)[at + k]);
          const float vhi = FROM8 ? keep_decode(p.codes[at + k + half], keep_scale(p.scales[(at + k + half) / KEEP_BLOCK])) : to_f32<T>(((const T*)p.x)[at + k + half]);
          xlo[i] = vlo * r;
          xhi[i] = vhi * r;
          sum[k] += nlo * xlo[i];
          sum[k + half] += nhi * xhi[i];
          glo[i] = nlo * to_f32<T>(gamma[k]);
          ghi[i] = nhi * to_f32<T>(gamma[k + half]);
          s += glo[i] * xlo[i] + ghi[i] * xhi[i];
        }
      }
      const float m = wave_sum(s) / d;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int k = lane + 64 * i;
        if (k < half) {
          dx[k] = from_f32<T>(r * (glo[i] - xlo[i] * m));
          dx[k + half] = from_f32<T>(r * (ghi[i] - xhi[i] * m));
        }
      }
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * d; i += NT) {
    const int g = i / d, c = i % d;
    p.partial[((size_t)g * gridDim.x + blockIdx.x) * d + c] = ((sums[0][g][c] + sums[1][g][c]) + sums[2][g][c]) + sums[3][g][c];
  }
}

// adds the workgroups' sums into the accumulators: one column per workgroup, in a fixed order
__global__ __launch_bounds__(NT) void qknorm_reduce_kernel(const float* __restrict__ partial, float* dgamma_q, float* dgamma_k, int nb, int d) {
  __shared__ float red[NT / 64];
  const int c = blockIdx.x;
  const float* src = partial + (size_t)blockIdx.y * nb * d;
  float s = 0.f;
  for (int b = threadIdx.x; b < nb; b += NT) s += src[(size_t)b * d + c];
  s = wave_sum(s);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) (blockIdx.y ? dgamma_k : dgamma_q)[c] += ((red[0] + red[1]) + red[2]) + red[3];
}

}  // namespace

hipError_t launch_qknorm_rope(int dtype, const void* src, const uint8_t* codes_in, const uint8_t* scales_in, void* dst, const void* gamma_q, const void* gamma_k,
                              const float* table, float* stats, uint8_t* codes, uint8_t* scales, int rows, int seq, int n_q, int n_kv, int d, float eps, hipStream_t s) {
  const QkNorm p = {src, codes_in, scales_in, dst, gamma_q, gamma_k, (const float2*)table, stats, codes, scales, rows, seq, n_q, n_kv, d, eps};
  const size_t groups = ((size_t)rows * (n_q + 2 * n_kv) + 3) / 4;
  const dim3 grid((unsigned)(groups > 16384 ? 16384 : groups));
  if (dtype == DT_BF16) {
    if (codes_in) hipLaunchKernelGGL((qknorm_kernel<bf16_t, true>), grid, dim3(NT), 0, s, p);
    else hipLaunchKernelGGL((qknorm_kernel<bf16_t, false>), grid, dim3(NT), 0, s, p);
  } else {
    if (codes_in) hipLaunchKernelGGL((qknorm_kernel<float, true>), grid, dim3(NT), 0, s, p);
    else hipLaunchKernelGGL((qknorm_kernel<float, false>), grid, dim3(NT), 0, s, p);
  }
  return hipGetLastError();
}

hipError_t launch_qknorm_rope_bwd(int dtype, const void* dy, const void* x, const uint8_t* codes, const uint8_t* scales, const float* stats, const void* gamma_q,
                                  const void* gamma_k, const float* table, void* dx, float* partial, float* dgamma_q, float* dgamma_k, int rows, int seq, int n_q, int n_kv,
                                  int d, hipStream_t s) {
  const QkNormBwd p = {dy, x, codes, scales, stats, gamma_q, gamma_k, (const float2*)table, dx, partial, rows, seq, n_q, n_kv, d};
  const int nb = rows < 1024 ? rows : 1024;
  if (dtype == DT_BF16) {
    if (codes) hipLaunchKernelGGL((qknorm_bwd_kernel<bf16_t, true>), dim3(nb), dim3(NT), 0, s, p);
    else hipLaunchKernelGGL((qknorm_bwd_kernel<bf16_t, false>), dim3(nb), dim3(NT), 0, s, p);
  } else {
    if (codes) hipLaunchKernelGGL((qknorm_bwd_kernel<float, true>), dim3(nb), dim3(NT), 0, s, p);
    else hipLaunchKernelGGL((qknorm_bwd_kernel<float, false>), dim3(nb), dim3(NT), 0, s, p);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(qknorm_reduce_kernel, dim3(d, 2), dim3(NT), 0, s, partial, dgamma_q, dgamma_k, nb, d);
  return hipGetLastError();
}
