// Embedding: out[r] = scale * weight[ids[r]], and its gradient grad[t] += scale * (sum of dy[r] over the rows r with ids[r] = t).
// A row whose id is no word of the vocabulary (negative, or vocab and more: padding) is zero and has no gradient.
//
// The gradient puts the tokens in order, so that equal ones stand side by side and every row of the accumulator that occurs is read and written once, without
// atomics and in an order that the ids alone decide: the rows of a token in their order, up to PIECE of them by one wave.  The runs of frequent
// tokens are cut at multiples of PIECE, and their pieces' sums are added by a second launch.  Bound by memory (dy once, the accumulator's rows in and out)
// from some thousand tokens of some thousand columns on, by the latency of the launches below that.
#include "common.h"

#include <type_traits>

namespace {

constexpr int NT = 256;

// ---- lookup -----------------------------------------------------------------------------------------------
// 16 bytes a lane; chunks numbered through all rows
template <typename T, int U>
__global__ __launch_bounds__(NT) void embed_fwd_kernel(const int* __restrict__ ids, const T* __restrict__ weight, T* __restrict__ out, size_t total, const Divisor per_row,
                                                       unsigned vocab, float scale) {
  typedef Vec16<T> V;
  for (size_t base = blockIdx.x * (size_t)(NT * U); base < total; base += (size_t)gridDim.x * (NT * U)) {
    size_t row0 = 0;
    unsigned c0 = (unsigned)base;
    if (total >> 31) {
      row0 = base / per_row.d;
      c0 = (unsigned)(base - row0 * per_row.d);
    }
    V v[U];
    bool word[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const unsigned i = u * NT + threadIdx.x, n = c0 + i, r = per_row.quotient(n);
      word[u] = false;
      if (base + i < total) {
        const unsigned id = (unsigned)ids[row0 + r];
        word[u] = id < vocab;
        if (word[u]) v[u] = *reinterpret_cast<const V*>(weight + ((size_t)id * per_row.d + (n - r * per_row.d)) * V::N);
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const size_t i = base + u * NT + threadIdx.x;
#pragma unroll
      for (int e = 0; e < V::N; ++e) v[u].set(e, word[u] ? v[u].get(e) * scale : 0.f);
      if (i < total) *reinterpret_cast<V*>(out + i * V::N) = v[u];
    }
  }
}

// ---- sort ---------------------------------------------------------------------------------------------------
// A stable radix sort by up to 9 bits of the id per pass.  Up to 16384 keys a pass is one launch: every workgroup counts the digits of ALL keys (they come out
// of the L2, 64 KB at most), those ahead of its own range apart, which gives it the place of each of its digits without waiting for the others.
// Beyond that a launch ahead of it counts each range once (65536 tokens, 256 columns: 69 us with it, 76 without).  The first pass takes the ids
// themselves and leaves out those that are no words.
constexpr int RADIX = 512, COPIES = 8;                                  // counters in 8 copies by lane: equal digits of a wave meet 8 at a time at most
constexpr int SORT_T = 1024, SORT_MAX_GROUPS = 256, SORT_COUNTED = 16384;

struct Sorted {
  unsigned* count;                                                      // [0] valid tokens, [1] runs in `long_runs`
  unsigned* long_runs;
  unsigned *key[2], *row[2];                                            // pass i leaves its order in i & 1
  unsigned* table;                                                      // keys of each range by digit, beyond SORT_COUNTED
  float* partial;
};

struct Pass {
  int shift, bits, number;
  unsigned rows, vocab, per_group;
};
__device__ __forceinline__ void count_digits(unsigned (&hist)[RADIX * COPIES], unsigned digit) { atomicAdd(&hist[digit * COPIES + (threadIdx.x & (COPIES - 1))], 1u); }

// table[g][d]: keys of digit d in range g
__global__ __launch_bounds__(SORT_T) void embed_count_kernel(const unsigned* __restrict__ ids, const Sorted w, const Pass p) {
  __shared__ unsigned hist[RADIX * COPIES];
  const unsigned tid = threadIdx.x, digits = 1u << p.bits, n = p.number == 0 ? p.rows : w.count[0];
  const unsigned* key_in = p.number == 0 ? ids : w.key[(p.number - 1) & 1];
  const unsigned begin = min(n, blockIdx.x * p.per_group), end = min(n, begin + p.per_group);
  for (unsigned i = tid; i < digits * COPIES; i += SORT_T) hist[i] = 0;
  __syncthreads();
  for (unsigned i = begin + tid; i < end; i += SORT_T) {
    const unsigned k = key_in[i];
    if (k < p.vocab) count_digits(hist, k >> p.shift & (digits - 1));
  }
  __syncthreads();
  for (unsigned d = tid; d < digits; d += SORT_T) {
    unsigned s = 0;
#pragma unroll
    for (int c = 0; c < COPIES; ++c) s += hist[d * COPIES + c];
    w.table[blockIdx.x * digits + d] = s;
  }
}

__global__ __launch_bounds__(SORT_T) void embed_sort_kernel(const unsigned* __restrict__ ids, const Sorted w, const Pass p, int counted) {
  constexpr int WAVES = SORT_T / 64;
  __shared__ union {
    unsigned hist[2][RADIX * COPIES];                                   // ahead of the range, and the rest
    unsigned wave_count[WAVES][RADIX];
  } lds;
  __shared__ unsigned place[RADIX], wave_total[WAVES];
  const unsigned tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, digits = 1u << p.bits, mask = digits - 1;
  const unsigned n = p.number == 0 ? p.rows : w.count[0];
  const unsigned* key_in = p.number == 0 ? ids : w.key[(p.number - 1) & 1];
  const unsigned* row_in = w.row[(p.number - 1) & 1];
  unsigned *key_out = w.key[p.number & 1], *row_out = w.row[p.number & 1];
  const unsigned begin = min(n, blockIdx.x * p.per_group), end = min(n, begin + p.per_group);
  unsigned ahead = 0, all = 0;                                          // of digit tid: keys ahead of the range, and all
  if (counted) {
    if (tid < digits)
      for (unsigned g0 = 0; g0 < gridDim.x; g0 += 16) {
        unsigned c[16];
#pragma unroll
        for (int u = 0; u < 16; ++u) c[u] = g0 + u < gridDim.x ? w.table[(g0 + u) * digits + tid] : 0u;
#pragma unroll
        for (int u = 0; u < 16; ++u) {
          ahead += g0 + u < blockIdx.x ? c[u] : 0u;
          all += c[u];
        }
      }
  } else {
    for (unsigned i = tid; i < digits * COPIES; i += SORT_T) lds.hist[0][i] = lds.hist[1][i] = 0;
    __syncthreads();
    for (unsigned i0 = 0; i0 < n; i0 += SORT_T * 8) {
      unsigned k[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const unsigned i = i0 + u * SORT_T + tid;
        k[u] = i < n ? key_in[i] : 0xffffffffu;
      }
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const unsigned i = i0 + u * SORT_T + tid;
        if (i < n && k[u] < p.vocab) count_digits(lds.hist[i < begin ? 0 : 1], k[u] >> p.shift & mask);
      }
    }
    __syncthreads();
    if (tid < digits) {
#pragma unroll
      for (int c = 0; c < COPIES; ++c) {
        ahead += lds.hist[0][tid * COPIES + c];
        all += lds.hist[1][tid * COPIES + c];
      }
      all += ahead;
    }
  }
  // place[d]: keys of smaller digits, and those of digit d ahead of the range
  unsigned before = all;                                                // inclusive scan over the wave, then over the waves
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const unsigned t = (unsigned)__shfl_up((int)before, o, 64);
    if (lane >= (unsigned)o) before += t;
  }
  if (lane == 63) wave_total[wave] = before;
  __syncthreads();
  unsigned sum = 0;
#pragma unroll
  for (int v = 0; v < WAVES; ++v) {
    if ((unsigned)v == wave) before += sum;
    sum += wave_total[v];
  }
  if (tid < digits) place[tid] = before - all + ahead;
  if (p.number == 0 && blockIdx.x == 0 && tid == 0) { w.count[0] = sum; w.count[1] = 0; }
  // the range, SORT_T keys at a time: a lane's place is its digit's, past the waves ahead and the lanes of its own wave ahead with the same digit
  for (unsigned i0 = begin; i0 < end; i0 += SORT_T) {
    __syncthreads();
    for (unsigned i = tid; i < (unsigned)WAVES << p.bits; i += SORT_T) lds.wave_count[i >> p.bits][i & mask] = 0;
    __syncthreads();
    const unsigned i = i0 + tid;
    const unsigned key = i < end ? key_in[i] : 0xffffffffu;
    const bool on = key < p.vocab;
    const unsigned d = key >> p.shift & mask;
    unsigned long long same = __ballot(on);
#pragma unroll
    for (int b = 0; b < 9; ++b) {                                       // bits beyond the pass's are zero in all lanes
      const unsigned long long set = __ballot(d >> b & 1);
      same &= d >> b & 1 ? set : ~set;
    }
    const unsigned rank = __popcll(same & ((1ull << lane) - 1));
    if (on && rank == 0) lds.wave_count[wave][d] = __popcll(same);
    __syncthreads();
    if (tid < digits) {
      unsigned at = place[tid];
#pragma unroll
      for (int v = 0; v < WAVES; ++v) {
        const unsigned c = lds.wave_count[v][tid];
        lds.wave_count[v][tid] = at;
        at += c;
      }
      place[tid] = at;
    }
    __syncthreads();
    if (on) {
      const unsigned at = lds.wave_count[wave][d] + rank;
      key_out[at] = key;
      row_out[at] = p.number == 0 ? i : row_in[i];
    }
  }
}

// A single launch for fewer tokens, whatever the vocabulary: a token's place is the number of smaller ones and of equal ones in earlier rows.  The waves of a
// workgroup hold all keys, 64 consecutive ones in a register; for each of the workgroup's 2 K rows a register takes one comparison and one count of bits.  The work
// goes with the square of the tokens: 600 tokens 3.6 us, two passes of the sort 8.6; 4096 4.8 and 10.6, one pass 5.3; 8192 9.1 and 12.6, one pass 6.6; 16384 24
// and 16.  Twice the rows to a workgroup: 4.8 us at 600 tokens, the same from 4096 on.
template <int K> __global__ __launch_bounds__(1024) void embed_place_kernel(const int* __restrict__ ids, const Sorted w, int rows, unsigned vocab) {
  constexpr int R = 2 * K, NONE = 0x7fffffff;                           // NONE: padding, behind all words
  static_assert(64 % R == 0, "a workgroup's rows lie in one block of 64");
  __shared__ int part[16][R], words[16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, first = (int)blockIdx.x * R, own = first / 64;
  const auto load = [&](int j) {
    const int id = j < rows ? ids[j] : NONE;
    return (unsigned)id < vocab ? id : NONE;
  };
  int k[K];
#pragma unroll
  for (int i = 0; i < K; ++i) k[i] = load((wave * K + i) * 64 + lane);
  const int block = load(own * 64 + lane);
  if (blockIdx.x == 0) {
    int n = 0;
#pragma unroll
    for (int i = 0; i < K; ++i) n += __popcll(__ballot(k[i] != NONE));
    if (lane == 0) words[wave] = n;
  }
  // k - 1 < key is k <= key: equal ones of earlier blocks count; those of the own block are the first wave's
#pragma unroll
  for (int i = 0; i < K; ++i) k[i] -= wave * K + i < own ? 1 : 0;
  int ahead = 0;
#pragma unroll 8
  for (int q = 0; q < R; ++q) {
    const int at = first % 64 + q, key = __builtin_amdgcn_readlane(block, at);
    int n = 0;
#pragma unroll
    for (int i = 0; i < K; ++i) n += __popcll(__ballot(k[i] < key));
    if (wave == 0) n += __popcll(__ballot(block == key) & ((1ull << at) - 1));
    ahead = lane == q ? n : ahead;
  }
  if (lane < R) part[wave][lane] = ahead;
  __syncthreads();
  if (wave == 0) {
    const int key = __shfl(block, first % 64 + lane % R, 64);
    if (lane < R && key != NONE) {
      int place = 0;
#pragma unroll
      for (int v = 0; v < 16; ++v) place += part[v][lane];
      w.key[0][place] = (unsigned)key;
      w.row[0][place] = (unsigned)(first + lane);
    }
    if (blockIdx.x == 0 && lane == 0) {
      int n = 0;
      for (int v = 0; v < 16; ++v) n += words[v];
      w.count[0] = (unsigned)n;
      w.count[1] = 0;
    }
  }
}

// ---- sums -----------------------------------------------------------------------------------------------------
constexpr int PIECE = 32;                                               // rows that one wave adds up

// s += the lane's chunk at column col over the rows whose numbers lanes first .. end - 1 hold, in their order; FLIGHT loads in flight, those behind the end
// of its last row again
template <int FLIGHT, typename T> __device__ __forceinline__ void add_rows(const T* __restrict__ dy, unsigned row, int first, int end, size_t h, int col, float* s) {
  typedef Vec16<T> V;
  for (int i0 = first; i0 < end; i0 += FLIGHT) {
    V v[FLIGHT];
#pragma unroll
    for (int u = 0; u < FLIGHT; ++u) {
      const size_t r = (unsigned)__builtin_amdgcn_readlane((int)row, min(i0 + u, end - 1));
      v[u].v = __builtin_nontemporal_load(&reinterpret_cast<const V*>(dy + r * h + col)->v);
    }
#pragma unroll
    for (int u = 0; u < FLIGHT; ++u)
      if (i0 + u < end)
#pragma unroll
        for (int e = 0; e < V::N; ++e) s[e] += v[u].get(e);
  }
}
template <int N> __device__ __forceinline__ void add_to(float* g, const float* s, float scale) {
#pragma unroll
  for (int i = 0; i < N; i += 4) {
    f32x4_t v = *reinterpret_cast<f32x4_t*>(g + i);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] += scale * s[i + e];
    *reinterpret_cast<f32x4_t*>(g + i) = v;
  }
}

// Wave (w, slice): places w Q .. w Q + Q - 1 of the sorted tokens, 64 chunks of columns.  Its are the runs of equal tokens that begin there, to their ends, which lie up to
// PIECE places on: one stretch of places, BATCH rows of dy in flight together with the accumulator's rows of the runs that end among them (with one run
// to a wave, 4096 tokens took 41 us instead of 26: half of the waves find no run, the others wait for one row).  A run of more than PIECE places is cut at
// multiples of PIECE: partial[2 k] is the sum of the piece that begins at place k PIECE, partial[2 k + 1] that of the piece of a long run that begins
// later in that range (only one can: it goes on behind it).
constexpr int BATCH = 8;
template <typename T, int Q>
__global__ __launch_bounds__(NT) void embed_sum_kernel(const unsigned* __restrict__ key, const unsigned* __restrict__ row_of, const T* __restrict__ dy, float* __restrict__ grad,
                                                       unsigned* count, unsigned* long_runs, float* __restrict__ partial, int rows, int h, unsigned groups, float scale) {
  static_assert(PIECE == 32 && PIECE % Q == 0 && Q + PIECE <= 64, "masks of 64 places");
  typedef Vec16<T> V;
  constexpr int N = V::N;
  const int lane = threadIdx.x & 63, slice = (int)((blockIdx.x % groups) * blockDim.x + threadIdx.x) >> 6, col = (slice * 64 + lane) * N;
  if (slice * 64 * N >= h) return;
  const bool on = col < h;
  const int at = on ? col : 0;                                          // lanes behind the last column load, and store nothing
  for (long long base = (long long)(blockIdx.x / groups) * Q; base < rows; base += (long long)(gridDim.x / groups) * Q) {
    const long long m = count[0], xa = base - PIECE + lane, xb = base + PIECE + lane;
    const auto inside = [&](long long x) { return x < 0 ? 0 : x < rows ? x : (long long)rows - 1; };
    const unsigned ka = key[inside(xa)], kb = key[inside(xb)], row = row_of[inside(base + lane)];
    if (base >= m) return;
    // bit i of `starts`: a run begins at place base + i (or the tokens have ended); of `back`: at base - PIECE + i, the first of them not looked at
    const unsigned pa = (unsigned)__shfl_up((int)ka, 1, 64), pb = (unsigned)__shfl_up((int)kb, 1, 64), last_a = (unsigned)__builtin_amdgcn_readlane((int)ka, 63);
    const unsigned long long sa = __ballot(xa <= 0 || xa >= m || (lane > 0 && ka != pa)), sb = __ballot(xb >= m || kb != (lane > 0 ? pb : last_a));
    const unsigned long long starts = sa >> 32 | sb << 32;
    const unsigned back = (unsigned)sa & ~1u;
    // a piece of a long run that began earlier: it has more than PIECE places, PIECE of them before this or from its begin to its end
    bool resumed = base % PIECE == 0 && !(starts & 1);
    if (resumed && back) {
      const int ahead = __clz((int)back) + 1, here = starts ? __ffsll((long long)starts) - 1 : 64;
      resumed = ahead + here > PIECE;
    }
    const int many = m - base < Q ? (int)(m - base) : Q;
    const unsigned long long mine = starts & ((1ull << many) - 1);
    if (!resumed && !mine) continue;
    const int first = resumed ? 0 : __ffsll((long long)mine) - 1, last = mine ? 63 - __clzll((long long)mine) : 0;   // places of the first and last run or piece
    const unsigned long long behind = starts & ~((2ull << last) - 1);
    int end = behind ? __ffsll((long long)behind) - 1 : 64;
    const bool cut = !mine || end - last > PIECE;                       // the last one is a piece
    if (cut) end = min(end, (int)(PIECE - (base + last) % PIECE) + last);
    const int resumed_end = !resumed ? -1 : (mine ? __ffsll((long long)mine) - 1 : end);
    if (cut && mine && slice == 0 && lane == 0) long_runs[atomicAdd(&count[1], 1u)] = (unsigned)(base + last);
    // whole runs, and the rest of a resumed one: BATCH rows in flight together with the accumulator's rows of the runs that end among them
    const int whole = cut ? last : end;
    float s[N] = {};
    for (int i = first; i < whole; i += BATCH) {
      V v[BATCH];
      f32x4_t g[BATCH][N / 4];
      float* to[BATCH];                                                 // rows, the same for the whole wave
      const unsigned ends = (unsigned)(starts >> (i + 1));              // bit u: a run ends with place i + u
#pragma unroll
      for (int u = 0; u < BATCH; ++u) {
        const size_t r = (unsigned)__builtin_amdgcn_readlane((int)row, min(i + u, whole - 1));
        v[u].v = __builtin_nontemporal_load(&reinterpret_cast<const V*>(dy + r * h + at)->v);   // read once: 86 -> 75 us at 16384 x 5120
      }
#pragma unroll
      for (int u = 0; u < BATCH; ++u)
        if (i + u < whole && (ends >> u & 1)) {
          const int x = i + u;
          const size_t id = (unsigned)(x < PIECE ? __builtin_amdgcn_readlane((int)ka, x + PIECE) : __builtin_amdgcn_readlane((int)kb, x - PIECE));
          to[u] = x + 1 == resumed_end ? partial + (size_t)(base / PIECE * 2) * h : grad + id * h;
#pragma unroll
          for (int c = 0; c < N / 4; ++c) g[u][c] = *reinterpret_cast<const f32x4_t*>(to[u] + at + 4 * c);
        }
#pragma unroll
      for (int u = 0; u < BATCH; ++u)
        if (i + u < whole) {
#pragma unroll
          for (int e = 0; e < N; ++e) s[e] += v[u].get(e);
          if (ends >> u & 1) {
            const bool piece = i + u + 1 == resumed_end;
#pragma unroll
            for (int e = 0; e < N; ++e) {
              g[u][e / 4][e % 4] = piece ? s[e] : fmaf(scale, s[e], g[u][e / 4][e % 4]);
              s[e] = 0.f;
            }
            if (on)
#pragma unroll
              for (int c = 0; c < N / 4; ++c) *reinterpret_cast<f32x4_t*>(to[u] + at + 4 * c) = g[u][c];
          }
        }
    }
    if (cut) {
      add_rows<16>(dy, row, last, end, (size_t)h, at, s);
      const unsigned long long p = (unsigned long long)base + last;
      float* piece = partial + (size_t)(p / PIECE * 2 + (p % PIECE ? 1 : 0)) * h + at;
      if (on)
#pragma unroll
        for (int i = 0; i < N; i += 4) *reinterpret_cast<f32x4_t*>(piece + i) = (f32x4_t){s[i], s[i + 1], s[i + 2], s[i + 3]};
    }
  }
}

// The pieces of a long run, 256 columns of it per workgroup: eight waves take every eighth piece, eight loads of a lane in flight, and are added in order.  The order
// of the list does not matter: a run's pieces are found from its first place.
constexpr int JOIN_T = 512;
__global__ __launch_bounds__(JOIN_T) void embed_join_kernel(const unsigned* __restrict__ key, const unsigned* __restrict__ count, const unsigned* __restrict__ long_runs,
                                                            const float* __restrict__ partial, float* __restrict__ grad, int h, float scale) {
  constexpr int W = JOIN_T / 64;
  __shared__ f32x4_t red[W][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const unsigned m = count[0], slices = (h + 255) / 256;
  const unsigned long long items = (unsigned long long)count[1] * slices;
  for (unsigned long long item = blockIdx.x; item < items; item += gridDim.x) {
    const unsigned p = long_runs[item / slices], id = key[p];
    const int col = (int)(item % slices) * 256 + lane * 4;
    const unsigned k0 = p / PIECE + 1;
    unsigned pieces = 0;                                                 // behind the first one: places k PIECE that still hold the token
    for (unsigned long long more = ~0ull; more == ~0ull; pieces += more == ~0ull ? 64 : __ffsll((long long)~more) - 1) {
      const unsigned long long x = ((unsigned long long)k0 + pieces + lane) * PIECE;
      more = __ballot(x < m && key[x < m ? x : 0] == id);
    }
    f32x4_t s = {0.f, 0.f, 0.f, 0.f};
    if (col < h) {
      if (wave == 0) s = *reinterpret_cast<const f32x4_t*>(partial + (size_t)(p / PIECE * 2 + (p % PIECE ? 1 : 0)) * h + col);
      for (unsigned i0 = wave; i0 < pieces; i0 += W * 8) {
        f32x4_t v[8];
#pragma unroll
        for (int u = 0; u < 8; ++u)
          if (i0 + u * W < pieces) v[u] = *reinterpret_cast<const f32x4_t*>(partial + (size_t)(k0 + i0 + u * W) * 2 * h + col);
#pragma unroll
        for (int u = 0; u < 8; ++u)
          if (i0 + u * W < pieces) s += v[u];
      }
    }
    red[wave][lane] = s;
    __syncthreads();
    if (wave == 0 && col < h) {
      for (int w = 1; w < W; ++w) s += red[w][lane];
      const float t[4] = {s[0], s[1], s[2], s[3]};
      add_to<4>(grad + (size_t)id * h + col, t, scale);
    }
    __syncthreads();
  }
}

// A few tokens, in one launch: wave (r, slice) compares all ids with row r's and adds up its token's rows if r is the first of them.
// In bf16, lookup and gradient in us, and with the launches above instead: 400 tokens of 32000 words and 512 columns 9.9, 14.6; of 50 words and 4096
// columns 19.9, 18.0; 512 tokens 10.8, 15.6 and 26.9, 17.6.
constexpr int FEW = 448;
template <typename T>
__global__ __launch_bounds__(NT) void embed_few_kernel(const int* __restrict__ ids, const T* __restrict__ dy, float* __restrict__ grad, int rows, unsigned vocab, int h,
                                                       float scale) {
  constexpr int N = Vec16<T>::N;
  const int lane = threadIdx.x & 63, slice = (int)(blockIdx.y * blockDim.x + threadIdx.x) >> 6, col = (slice * 64 + lane) * N, r = blockIdx.x;
  if (slice * 64 * N >= h) return;
  const int id = ids[r];
  if ((unsigned)id >= vocab) return;
  unsigned long long same[FEW / 64];
#pragma unroll
  for (int i = 0; i < FEW / 64; ++i) same[i] = __ballot(i * 64 + lane < rows && ids[min(i * 64 + lane, rows - 1)] == id);
#pragma unroll
  for (int i = 0; i < FEW / 64; ++i)
    if (r > i * 64 && (same[i] & (r - i * 64 >= 64 ? ~0ull : (1ull << (r - i * 64)) - 1))) return;
  float s[N] = {};
#pragma unroll
  for (int i = 0; i < FEW / 64; ++i) {
    if (!same[i]) continue;
    // lane k gets the number of the k-th row of the 64
    const int n = __popcll(same[i]), k = __popcll(same[i] & ((1ull << lane) - 1));
    const unsigned row = (unsigned)__builtin_amdgcn_ds_permute((same[i] >> lane & 1 ? k : 63) * 4, i * 64 + lane);
    if (n == 1) add_rows<1>(dy, row, 0, 1, (size_t)h, col < h ? col : 0, s);
    else add_rows<8>(dy, row, 0, n, (size_t)h, col < h ? col : 0, s);
  }
  if (col < h) add_to<N>(grad + (size_t)id * h + col, s, scale);
}

unsigned sort_range(int rows) {
  const unsigned tiles = ((unsigned)rows + SORT_T - 1) / SORT_T;
  return (tiles + SORT_MAX_GROUPS - 1) / SORT_MAX_GROUPS * SORT_T;
}

Sorted layout(void* ws, int rows, int h, uint64_t* bytes) {
  uint64_t at = 0;
  auto take = [&](uint64_t n) { void* p = (char*)ws + at; at += (n + 255) / 256 * 256; return p; };
  Sorted s;
  s.count = (unsigned*)take(8);
  s.long_runs = (unsigned*)take(((uint64_t)rows / (PIECE + 1) + 1) * 4);
  for (int i = 0; i < 2; ++i) {
    s.key[i] = (unsigned*)take((uint64_t)rows * 4);
    s.row[i] = (unsigned*)take((uint64_t)rows * 4);
  }
  const unsigned range = sort_range(rows);
  s.table = (unsigned*)take(rows > SORT_COUNTED ? (uint64_t)((unsigned)rows + range - 1) / range * RADIX * 4 : 0);
  s.partial = (float*)take(((uint64_t)rows + PIECE - 1) / PIECE * 2 * h * 4);
  *bytes = at;
  return s;
}

int id_bits(unsigned vocab) {
  int bits = 1;
  while (bits < 31 && (vocab - 1) >> bits) ++bits;
  return bits;
}
// waves side by side over a row's columns, n of them to a lane
unsigned sum_waves(int h, int n) { return (unsigned)(h / n + 63) / 64; }
// Places of a wave: the more of them, the fewer waves find only the middle of a run, but there have to be waves enough, and where most runs are of one or
// two places a wave has to wait for many rows of the accumulator.  us with 8, 16, 32: 1000 x 4096 of 32000 words 13, 15, 21; 4096 x 4096 of 32000 words
// 27, 26, 27; 49000 x 200 of 10190 words 23, 16, 19; 16384 x 5120 of 131072 words 77, 79, 84; 22713 x 1352 fp32 of 821 words 73, 50, 39.
int sum_places(int rows, unsigned vocab, unsigned waves) {
  const uint64_t all = (uint64_t)rows * waves;
  if (all < 16384) return 8;
  return (unsigned)rows < vocab || all < 98304 ? 16 : 32;
}

template <typename T>
hipError_t run_embed_bwd(const int* ids, const void* dy, float* grad, void* ws, int rows, unsigned vocab, int h, float scale, hipStream_t s) {
  const unsigned waves = sum_waves(h, Vec16<T>::N), threads = 64 * min(waves, 4u), slices = (waves + 3) / 4;
  const int order = embed_bwd_order(rows, vocab);
  if (order == EMBED_FEW) {
    hipLaunchKernelGGL(embed_few_kernel<T>, dim3(rows, slices), dim3(threads), 0, s, ids, (const T*)dy, grad, rows, vocab, h, scale);
    return hipGetLastError();
  }
  uint64_t bytes;
  const Sorted w = layout(ws, rows, h, &bytes);
  const bool placed = order == EMBED_PLACED;
  if (placed) {
    const auto place = [&](auto k) { hipLaunchKernelGGL((embed_place_kernel<k>), dim3((rows + 2 * k - 1) / (2 * k)), dim3(1024), 0, s, ids, w, rows, vocab); };
    if (rows <= 4096) place(std::integral_constant<int, 4>());
    else place(std::integral_constant<int, 8>());
  } else {
    const int passes = order, bits = id_bits(vocab), per_pass = (bits + passes - 1) / passes;
    const bool counted = rows > SORT_COUNTED;
    const unsigned per_group = sort_range(rows), groups = ((unsigned)rows + per_group - 1) / per_group;
    for (int i = 0; i < passes; ++i) {
      const Pass p = {per_pass * i, min(per_pass, bits - per_pass * i), i, (unsigned)rows, vocab, per_group};
      if (counted) hipLaunchKernelGGL(embed_count_kernel, dim3(groups), dim3(SORT_T), 0, s, (const unsigned*)ids, w, p);
      hipLaunchKernelGGL(embed_sort_kernel, dim3(groups), dim3(SORT_T), 0, s, (const unsigned*)ids, w, p, counted ? 1 : 0);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
  }
  const int last = placed ? 0 : (order - 1) & 1;
  const auto sum = [&](auto q) {
    hipLaunchKernelGGL((embed_sum_kernel<T, q>), dim3(min((rows + q - 1) / q, max(1, (1 << 22) / (int)slices)) * slices), dim3(threads), 0, s, w.key[last], w.row[last],
                       (const T*)dy, grad, w.count, w.long_runs, w.partial, rows, h, slices, scale);
  };
  switch (sum_places(rows, vocab, waves)) {
    case 8: sum(std::integral_constant<int, 8>()); break;
    case 16: sum(std::integral_constant<int, 16>()); break;
    default: sum(std::integral_constant<int, 32>());
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(embed_join_kernel, dim3(512), dim3(JOIN_T), 0, s, w.key[last], w.count, w.long_runs, w.partial, grad, h, scale);
  return hipGetLastError();
}

}  // namespace

int embed_bwd_order(int rows, unsigned vocab) {
  if (rows <= FEW) return EMBED_FEW;
  const int passes = (id_bits(vocab) + 8) / 9;
  return rows <= 4096 * (passes < 2 ? 1 : 2) ? EMBED_PLACED : passes;
}
int embed_bwd_places(int dtype, int rows, unsigned vocab, int h) { return sum_places(rows, vocab, sum_waves(h, dtype == DT_BF16 ? 8 : 4)); }

uint64_t embed_bwd_ws_bytes(int rows, int h) {
  uint64_t bytes;
  layout(nullptr, rows, h, &bytes);
  return bytes;
}

hipError_t launch_embed_fwd(int dtype, const int* ids, const void* weight, void* out, int rows, unsigned vocab, int h, float scale, hipStream_t s) {
  constexpr int U = 2;
  const unsigned per_row = (unsigned)h / (dtype == DT_BF16 ? 8 : 4);
  const size_t total = (size_t)rows * per_row, groups = (total + NT * U - 1) / (NT * U);
  const dim3 grid((unsigned)(groups > (1u << 20) ? 1u << 20 : groups));
  if (dtype == DT_BF16) hipLaunchKernelGGL((embed_fwd_kernel<bf16_t, U>), grid, dim3(NT), 0, s, ids, (const bf16_t*)weight, (bf16_t*)out, total, Divisor(per_row), vocab, scale);
  else hipLaunchKernelGGL((embed_fwd_kernel<float, U>), grid, dim3(NT), 0, s, ids, (const float*)weight, (float*)out, total, Divisor(per_row), vocab, scale);
  return hipGetLastError();
}

hipError_t launch_embed_bwd(int dtype, const int* ids, const void* dy, float* grad, void* ws, int rows, unsigned vocab, int h, float scale, hipStream_t s) {
  return dtype == DT_BF16 ? run_embed_bwd<bf16_t>(ids, dy, grad, ws, rows, vocab, h, scale, s) : run_embed_bwd<float>(ids, dy, grad, ws, rows, vocab, h, scale, s);
}
