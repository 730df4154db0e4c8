// Loss against a teacher's top entries.  With p = softmax(z / T) and the teacher's t_j at the words id_j,
//   loss = sum_j t_j (log t_j - log p[id_j]),   dz_v = g / T (p_v sum_j t_j - sum of t_j over id_j = v)
// for the gradient g of the row's loss.  Bound by memory: a row of logits in, a row of their gradient out; what is done with a teacher's entries (64 bits,
// one wave) runs while the row's loads are in flight.
//
// A row's reference and sum are one pass: every wave keeps m, the largest of its first 16 bytes a lane, and s = sum of exp((z - m) / T).  Where a later logit lies so far
// above m that s reaches 2^64 (44 T), or nothing but the lowest values is left of a row, the row (its piece) is summed again with the running maximum.
// A logit costs a conversion, a multiply-add, an exponential and an addition in each direction, half of what the running maximum would: at 4096 rows of 131072 words
// the vector units are busy half of the time that memory takes.
//  * Rows of a few words: a wave has one in its registers, in every direction.
//  * Both directions, rows enough for the chip: a workgroup has a row in its registers from the maximum to the gradient (up to 128K words of bf16; of longer
//    ones the rest is read a second time).
//  * Rows too few for that: a row in pieces, a launch for their m and s, a second one that joins them and writes the gradient.
//  * Forward or backward alone: the pass over the row without keeping it.
// The gradient at the entries' words is written once more behind the row, whole, so that it has one rounding as every other.
#include "common.h"

namespace {

constexpr float LOG2E = 1.4426950408889634f, LOWEST = -3.402823466e38f;
// A row's factor, weight / sum, below which it is not formed (its reference's rest may take 2^-16 more, and 2^-126 is the least number of full precision): the row's
// probabilities come first then, and the weight last.
constexpr float LEAST_FACTOR = 0x1p-100f;

// 16 bytes of a row at any address of its elements
template <typename T> struct Any16;
template <> struct Any16<bf16_t> { typedef bf16_t t __attribute__((ext_vector_type(8), aligned(2))); };
template <> struct Any16<float> { typedef float t __attribute__((ext_vector_type(4), aligned(4))); };

// what a row's entries make of its loss: sum + mass (log of the sum of exp(z / T) - z0 / T), with sum = sum of t (log t - (z - z0) / T), mass = sum of t and z0 one of
// their own logits, so that nothing large cancels; log t = (the teacher's value - most) / T - log_norm, with T = 1 for log-probabilities; twice: a word is named twice
struct Teacher { double sum, mass, z0, log_norm; float most; int twice; };

struct Distill {
  const void* z; const int* ids; const float* teacher; const float* dloss;
  float* loss; float* lse; void* dz;
  size_t ldz, lddz;
  int rows, vocab, k;
  double teacher_inv_t;                                 // 1 / T, or 1 where the teacher gives log-probabilities
  float inv_t, c;                                       // 1 / T, log2(e) / T
  int log_probs;
  int pieces, piece;                                    // of a row, and elements of one (a multiple of a chunk)
  float2* stats; Teacher* parts;                        // [rows][pieces]: m, s; [rows]
};

// m and s of what a thread has seen, m a running maximum.  It starts at a finite number: minus infinity (a masked word) lies below it and adds nothing.
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
  // m c as one number, and what that rounding left out: exp2((x - m) c) = exp2(x c - reference) * rest
  __device__ __forceinline__ float reference(float c) const { return m * c; }
  __device__ __forceinline__ float rest(float c) const { return __builtin_amdgcn_exp2f(fmaf(-m, c, m * c)); }
  // Whether the sum holds, and rest is some 2^16 at most.  Against the maximum s is below 2^30, the number of words.  Where a later word lies far above the reference, 1 / s falls
  // towards the least numbers (a weight of 1e-6 over 2^122 has 7 bits), and sums of pieces overflow when they are joined.  Up to 2^64 neither is near, and what the exponents lose to
  // rounding, 2^-19, is about what such a row's lse loses.  A row with a word 44 T above the first ones is read once more (if every row has one, 4096 of 131072 words bf16
  // 440 -> 618 us, 4096 of 32000 fp32 218 -> 281): a bound of 2^32 would have that from 22 T on.
  __device__ __forceinline__ bool sound(float c) const { return s > 0.f && s < 0x1p64f && fabsf(m * c) < 0x1p28f; }
};
// The same against a reference that a wave has taken from its first chunks.
struct Quick {
  float m, mc, s;
  __device__ __forceinline__ Quick(float reference, float c) : m(reference), mc(reference * c), s(0.f) {}
  template <int N> __device__ __forceinline__ void add(const float (&x)[N], float c) {
    float t = 0.f;
#pragma unroll
    for (int e = 0; e < N; ++e) t += __builtin_amdgcn_exp2f(fmaf(x[e], c, -mc));
    s += t;
  }
  __device__ __forceinline__ Running end(float c) const {
    Running r;
    r.m = m;
    r.s = s * __builtin_amdgcn_exp2f(fmaf(-m, c, mc));
    return r;
  }
};
template <int N> __device__ __forceinline__ float wave_reference(const float (&x)[N]) {
  float most = x[0];
#pragma unroll
  for (int e = 1; e < N; ++e) most = fmaxf(most, x[e]);
  return wave_max(most);
}

// a row's entries in LDS (dynamic: 16 bytes an entry): word or -1, t, logit at the word, the teacher's value
struct Entries {
  int* id; float *t, *z, *value;
  __device__ __forceinline__ Entries(float* lds, int slot, int k) : id((int*)lds + 4 * k * slot), t(lds + 4 * k * slot + k), z(t + k), value(z + k) {}
};
constexpr size_t entries_bytes(int k) { return 16ull * k; }

struct Shared {
  Teacher teacher;
  float m[16], s[16];
};

__device__ __forceinline__ double wave_sum64(double v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

// exp of a 64-bit number: of its 32-bit part, times one plus the rest (two roundings of 32 bits; the 64-bit functions take a wave a microsecond)
__device__ __forceinline__ float exp_of(double x) {
  const float hi = (float)x;
  return x < -150.0 ? 0.f : expf(hi) * (1.f + (float)(x - (double)hi));   // below: less than half of the least number
}
// log of a positive 32-bit number to 2^-26: its exponent times log 2 in 64 bits, the rest near one
__device__ __forceinline__ double log_of(float x) {
  int k;
  float f = frexpf(x, &k);
  if (f < 0.70710678f) {
    f *= 2.f;
    --k;
  }
  return (double)k * 0.69314718055994531 + (double)logf(f);
}

// entry j's value of the teacher, minus infinity where it is not there
__device__ __forceinline__ float entry(const Distill& p, size_t row, int j, int& id) {
  id = p.ids[row * p.k + j];
  const float a = p.teacher[row * p.k + j];
  if ((unsigned)id < (unsigned)p.vocab) return a;
  id = -1;
  return -INFINITY;
}
// log t of a value.  In 64 bits and from the difference: a logit over T in 32 bits is off by 2^-24 of itself, which is an error of t by as much as the logits have in common
// (1e4 at T 0.7: 5e-4 of t), and past the range for small T.
__device__ __forceinline__ double log_weight(const Distill& p, float a, float most, double log_norm) { return ((double)a - (double)most) * p.teacher_inv_t - log_norm; }

// One wave: a row's entries into LDS and what they come to.  WEIGHTS: t takes the place of the teacher's values there.  GATHER: with the logits at the words, read
// before anything of the row is written (dz may be z); without them `sum` is that of t log t alone.
template <typename T, bool WEIGHTS, bool GATHER> __device__ __forceinline__ Teacher read_entries(const Distill& p, size_t row, const Entries& e) {
  const int lane = threadIdx.x & 63;
  const T* z = (const T*)p.z + row * p.ldz;
  float most = -INFINITY, z0 = -INFINITY;
#pragma unroll 1
  for (int j = lane; j < p.k; j += 64) {
    int id;
    const float a = entry(p, row, j, id);
    e.id[j] = id;
    e.t[j] = a;
    most = fmaxf(most, a);
    if (GATHER) {
      const float x = id >= 0 ? (float)z[id] : -INFINITY;
      e.z[j] = x;
      z0 = fmaxf(z0, x);
    }
  }
  most = wave_max(most);
  z0 = wave_max(z0);
  if (!(fabsf(z0) < INFINITY)) z0 = 0.f;
  if (p.log_probs || most == -INFINITY) most = 0.f;
  double norm = 1.0;
  if (!p.log_probs) {
    norm = 0.0;
#pragma unroll 1
    for (int j = lane; j < p.k; j += 64) norm += (double)exp_of(log_weight(p, e.t[j], most, 0.0));
    norm = wave_sum64(norm);
    if (norm == 0.0) norm = 1.0;                        // no entries
  }
  const double log_norm = p.log_probs ? 0.0 : log_of((float)norm);
  double sum = 0.0, mass = 0.0;
#pragma unroll 1
  for (int j = lane; j < p.k; j += 64) {
    const double lt = log_weight(p, e.t[j], most, log_norm), t = (double)exp_of(lt);
    if (t != 0.0) sum += t * (GATHER ? lt - ((double)e.z[j] - (double)z0) * (double)p.inv_t : lt);
    mass += t;
    if (WEIGHTS) e.t[j] = (float)t;
  }
  return {wave_sum64(sum), wave_sum64(mass), z0, log_norm, most, 0};
}

// all that the row's entries give a word
__device__ __forceinline__ float teacher_at(const Entries& e, int k, int id) {
  float t = 0.f;
#pragma unroll 4
  for (int i = 0; i < k; ++i) t += e.id[i] == id ? e.t[i] : 0.f;
  return t;
}

// Whether the row whose entries a wave has read names a word twice: by a table of its words in LDS, `slots` (a power of two, twice k at least) of the wave's own.
__device__ __forceinline__ bool names_twice(const Entries& e, int k, int* table, int slots) {
  const int lane = threadIdx.x & 63;
  for (int i = lane; i < slots; i += 64) table[i] = -1;
  __threadfence_block();
  bool twice = false;
#pragma unroll 1
  for (int j = lane; j < k; j += 64) {
    const int id = e.id[j];
    if (id < 0) continue;
    for (unsigned at = (unsigned)id * 2654435769u >> 8 & (slots - 1);; at = (at + 1) & (slots - 1)) {   // a free place or the word's is found: the table is half empty
      const int was = atomicCAS(table + at, -1, id);
      if (was == id) twice = true;
      if (was == -1 || was == id) break;
    }
  }
  return __any(twice);
}
int table_slots(int k) {
  int slots = 64;
  while (slots < 2 * k) slots *= 2;
  return slots;
}
// of four rows
size_t entries_and_table_bytes(int k) { return 4 * (entries_bytes(k) + sizeof(int) * table_slots(k)); }

// What the rows' entries come to, ahead of the pass over the rows: a wave a row, four to a workgroup.  In that pass one wave's 64-bit arithmetic and its two loads
// one behind the other would hold up the other fifteen (4096 rows of 131072 words with 128 entries: 120 of 583 us).
template <typename T> __global__ __launch_bounds__(256) void distill_teacher(const Distill p, int slots) {
  extern __shared__ float lds[];
  const int wave = threadIdx.x >> 6;
  const size_t row = (size_t)blockIdx.x * 4 + wave;
  if (row >= (size_t)p.rows) return;
  const Entries e(lds, wave, p.k);
  Teacher t = read_entries<T, false, false>(p, row, e);
  t.twice = names_twice(e, p.k, (int*)lds + 16 * p.k + wave * slots, slots) ? 1 : 0;
  if ((threadIdx.x & 63) == 0) p.parts[row] = t;
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
// loss and lse of a row
__device__ __forceinline__ void finish(const Distill& p, size_t row, const Running& r, const Teacher& t) {
  const double log_s = log_of(r.s);
  p.lse[row] = (float)((double)r.m * (double)p.inv_t + log_s);
  p.loss[row] = (float)(t.mass == 0.0 ? 0.0 : t.sum + t.mass * (((double)r.m - t.z0) * (double)p.inv_t + log_s));
}

// a piece of a row summed again by the running maximum
template <typename T, int NT> __device__ __forceinline__ Running sum_again(const Distill& p, const T* z, int begin, int end, Shared& sh) {
  __syncthreads();
  Running run;
#pragma unroll 1
  for (int at = begin + (int)threadIdx.x * Vec16<T>::N; at < end; at += NT * Vec16<T>::N) {
    float x[Vec16<T>::N];
    load_chunk(z, at, end, x);
    run.add(x, p.c);
  }
  return join_group<NT>(run, sh, p.c);
}

// ---- rows in a workgroup's registers, R chunks a thread, one row after the other: a chunk that has been written makes room for the next row's, so that the memory
// system has that row's loads while it takes this row's gradient (one workgroup of 16 waves fills a compute unit: nothing else would).
// (R - 2) NT chunks are less than a row: all steps but the last two are whole, and no step is behind a branch (held would be copied around it).  Chunks of those two
// that would cross the row's end start N before it: their elements below `at` are another chunk's and are masked.  vocab >= N.
template <typename T, int NT, int R> __global__ __launch_bounds__(NT) __attribute__((amdgpu_waves_per_eu(4))) void distill_rows(const Distill p) {
  constexpr int N = Vec16<T>::N, STEP = NT * N, HELD = R * STEP;
  typedef typename Any16<T>::t chunk_t;
  typedef unsigned u32x4_t __attribute__((ext_vector_type(4)));
  extern __shared__ float lds[];
  __shared__ Shared sh;
  const int first = threadIdx.x * N, last = p.vocab - N;
  auto fetch = [&](const T* z, int step) {
    const unsigned at = step < R - 2 ? (unsigned)first : (unsigned)min(first + step * STEP, last);
    return *reinterpret_cast<const chunk_t*>(z + (step < R - 2 ? step * STEP : 0) + at);
  };
  auto values = [&](const chunk_t& v, int step, float (&x)[N]) {
#pragma unroll
    for (int e = 0; e < N; ++e) x[e] = (float)v[e];
    if (step >= R - 2) {
      const int over = first + step * STEP - last;      // elements that are another chunk's
#pragma unroll
      for (int e = 0; e < N; ++e) x[e] = e < over ? -INFINITY : x[e];
    }
  };
  u32x4_t held[R];
#pragma unroll
  for (int r = 0; r < R; ++r) held[r] = __builtin_bit_cast(u32x4_t, fetch((const T*)p.z + blockIdx.x * p.ldz, r));
  int turn = 0, id_next = -1;
  float a_next = -INFINITY;
  if ((int)threadIdx.x < p.k) a_next = entry(p, blockIdx.x, threadIdx.x, id_next);
#pragma unroll 1
  for (size_t row = blockIdx.x; row < (size_t)p.rows; row += gridDim.x, turn ^= 1) {
    const T* z = (const T*)p.z + row * p.ldz;
    T* dz = (T*)p.dz + row * p.lddz;
    const size_t next = row + gridDim.x < (size_t)p.rows ? row + gridDim.x : row;
    const T* zn = (const T*)p.z + next * p.ldz;
    const Entries en(lds, turn, p.k);
    const Teacher& teacher = p.parts[row];
    const double log_norm = teacher.log_norm;
    const float most = teacher.most;
    const int id = id_next;                             // this thread's entry, requested a row ahead
    const float a = a_next, zid = id >= 0 ? (float)z[id] : -INFINITY;
    Running part;
    {
      float x[N];
      values(__builtin_bit_cast(chunk_t, held[0]), 0, x);
      const float m = wave_reference(x);
      if (m > LOWEST) {
        Quick run(m, p.c);
        run.add(x, p.c);
#pragma unroll
        for (int r = 1; r < R; ++r) {
          values(__builtin_bit_cast(chunk_t, held[r]), r, x);
          run.add(x, p.c);
        }
#pragma unroll 1
        for (int step = R; step * STEP < p.vocab; ++step) {
          values(fetch(z, step), step, x);
          run.add(x, p.c);
        }
        part = run.end(p.c);
      } else {                                          // nothing to refer to: the running maximum, over the wave's chunks
#pragma unroll 1
        for (int at = first; at < p.vocab; at += STEP) {
          load_chunk(z, at, p.vocab, x);
          part.add(x, p.c);
        }
      }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) asm volatile("" : "+v"(held[r]));   // kept as they came: their values in 32 bits would take twice the registers
    if ((int)threadIdx.x < p.k) {
      en.id[threadIdx.x] = id;
      en.t[threadIdx.x] = exp_of(log_weight(p, a, most, log_norm));
      en.z[threadIdx.x] = zid;
      en.value[threadIdx.x] = a;
#pragma unroll 1
      for (int j = threadIdx.x + NT; j < p.k; j += NT) {
        int other;
        const float v = entry(p, row, j, other);
        en.id[j] = other;
        en.t[j] = exp_of(log_weight(p, v, most, log_norm));
        en.value[j] = v;
        en.z[j] = other >= 0 ? (float)z[other] : -INFINITY;
      }
      a_next = entry(p, next, threadIdx.x, id_next);
    }
    Running all = join_group<NT>(part, sh, p.c);
    if (!all.sound(p.c)) all = sum_again<T, NT>(p, z, 0, p.vocab, sh);
    const double mass = teacher.mass;
    const bool twice = teacher.twice;
    const float w = p.dloss[row] * p.inv_t;
    const bool none = w == 0.f || mass == 0.0;
    const float f = none ? 0.f : w * (float)mass / all.s;
    const bool sound = all.sound(p.c) && (none || fabsf(f) >= LEAST_FACTOR);
    const float fr = sound ? f * all.rest(p.c) : f, mc = all.reference(p.c);
    auto prob_slow = [&](float x) { return w * (float)mass * (__builtin_amdgcn_exp2f((x - all.m) * p.c) / all.s); };
    if (!sound) {
#pragma unroll 1
      for (int at = first; at < p.vocab; at += STEP) {
        float x[N];
        load_chunk(z, at, p.vocab, x);
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = none ? 0.f : prob_slow(x[e]);
        store_chunk(dz, at, p.vocab, x);
      }
    }
    auto give = [&](chunk_t v, int step) {
#pragma unroll
      for (int e = 0; e < N; ++e) v[e] = (T)(fr * __builtin_amdgcn_exp2f(fmaf((float)v[e], p.c, -mc)));
      const int over = step < R - 2 ? 0 : first + step * STEP - last;
      if (!sound || over >= N) return;
      if (over <= 0) {
        // rows of 64 KB and more do not stay in the caches for whoever reads them next: past them (4096 rows of 131072 words 473 -> 456 us)
        if (NT == 1024) __builtin_nontemporal_store(v, reinterpret_cast<chunk_t*>(dz + step * STEP + (unsigned)first));
        else *reinterpret_cast<chunk_t*>(dz + step * STEP + (unsigned)first) = v;
      } else
#pragma unroll
        for (int e = 0; e < N; ++e)
          if (e >= over) dz[last + e] = v[e];
    };
#pragma unroll 1
    for (int step = R; step * STEP < p.vocab; ++step) give(fetch(z, step), step);
#pragma unroll
    for (int r = 0; r < R; ++r) {
      give(__builtin_bit_cast(chunk_t, held[r]), r);
      held[r] = __builtin_bit_cast(u32x4_t, fetch(zn, r));
    }
    // (stores of one workgroup's waves to a place arrive there in the order that the barrier gives them: the entries' values come to stay)
    __syncthreads();
    if (threadIdx.x >= NT - 64) {                       // the loss, by the wave that has the fewest entries to write
      double sum = 0.0;
#pragma unroll 1
      for (int j = threadIdx.x - (NT - 64); j < p.k; j += 64) {
        const double t = (double)en.t[j];
        if (t != 0.0) sum += t * (log_weight(p, en.value[j], most, log_norm) - ((double)en.z[j] - (double)all.m) * (double)p.inv_t);
      }
      sum = wave_sum64(sum);
      if (threadIdx.x == NT - 1) finish(p, row, all, {sum, mass, all.m, 0.0, 0.f, 0});
    }
    if (!none)
      for (int j = threadIdx.x; j < p.k; j += NT) {
        const int id = en.id[j];
        if (id < 0) continue;
        dz[id] = (T)((sound ? f * __builtin_amdgcn_exp2f((en.z[j] - all.m) * p.c) : prob_slow(en.z[j])) - w * (twice ? teacher_at(en, p.k, id) : en.t[j]));
      }
  }
}

// m and s of a row or a piece of it, in all threads
template <typename T, int NT> __device__ __forceinline__ Running sum_of(const Distill& p, const T* z, int begin, int end, Shared& sh) {
  constexpr int N = Vec16<T>::N, STEP = NT * N, U = 4;
  int at = begin + threadIdx.x * N;
  float x[N];
  load_chunk(z, at, end, x);
  const float m = wave_reference(x);
  Running part;
  if (m > LOWEST) {
    Quick run(m, p.c);
    for (; at + (U - 1) * STEP + N <= end; at += U * STEP) {
      typename Any16<T>::t v[U];
#pragma unroll
      for (int u = 0; u < U; ++u) v[u] = *reinterpret_cast<const typename Any16<T>::t*>(z + at + u * STEP);
#pragma unroll
      for (int u = 0; u < U; ++u) {
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = (float)v[u][e];
        run.add(x, p.c);
      }
    }
    for (; at < end; at += STEP) {
      load_chunk(z, at, end, x);
      run.add(x, p.c);
    }
    part = run.end(p.c);
  } else {
    for (; at < end; at += STEP) {
      load_chunk(z, at, end, x);
      part.add(x, p.c);
    }
  }
  Running all = join_group<NT>(part, sh, p.c);
  if (!all.sound(p.c)) all = sum_again<T, NT>(p, z, begin, end, sh);
  return all;
}

// ---- m and s of a row's piece; forward alone and a whole row: loss and lse.  Grid rows x pieces.
template <typename T, int NT> __global__ __launch_bounds__(NT) void distill_stats(const Distill p) {
  extern __shared__ float lds[];
  __shared__ Shared sh;
  const size_t row = blockIdx.x / p.pieces;
  const int piece = blockIdx.x % p.pieces, begin = piece * p.piece, end = min(p.vocab, begin + p.piece);
  const T* z = (const T*)p.z + row * p.ldz;
  if (piece == 0 && threadIdx.x < 64) {
    const Teacher mine = read_entries<T, false, true>(p, row, Entries(lds, 0, p.k));
    if (threadIdx.x == 0) sh.teacher = mine;
  }
  const Running all = sum_of<T, NT>(p, z, begin, end, sh);
  if (threadIdx.x) return;
  if (p.pieces > 1) {                                    // joined by the next launch
    p.stats[blockIdx.x] = make_float2(all.m, all.s);
    if (piece == 0) p.parts[row] = sh.teacher;
    return;
  }
  finish(p, row, all, sh.teacher);
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
__global__ __launch_bounds__(256) void distill_finish(const Distill p) {
  const size_t row = (size_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (row >= (size_t)p.rows) return;
  const Running r = join_pieces(p, row);
  if ((threadIdx.x & 63) == 0) finish(p, row, r, p.parts[row]);
}

// An lse of this size and more is a number of 32 bits whose rounding the gradient's type would show: up to 2^-20 of p for fp32 (20000 words at T 0.7: 9.7e-7 of the gradient's
// norm in all, 4.8e-7 from the row's own sum), 2^-12 for bf16.  One more read: fp32, forward and backward, 4096 rows of 32000 words 300 -> 340 us, 20 of 100000, a workgroup each, 17 -> 36.
template <typename T> constexpr float FAR_LSE = sizeof(T) == 4 ? 16.f : 4096.f;

// ---- the gradient of a row's piece, from lse (JOIN: from the pieces' m and s, the first piece writes loss and lse).  Grid rows x pieces.
// Without JOIN a row of FAR_LSE is summed again, by the workgroup of its first piece, which has the whole row then: dz may be z, so nobody else may write before.
// PAST: stores (1), loads too (2) past the caches.
template <typename T, int NT, bool JOIN, int PAST> __global__ __launch_bounds__(NT) void distill_grad(const Distill p, int slots) {
  constexpr int N = Vec16<T>::N, STEP = NT * N, U = 4;
  extern __shared__ float lds[];
  __shared__ Shared sh;
  const size_t row = blockIdx.x / p.pieces;
  const int piece = blockIdx.x % p.pieces;
  const bool again = !JOIN && fabsf(p.lse[row]) >= FAR_LSE<T>;
  if (again && piece) return;
  const int begin = piece * p.piece, end = again ? p.vocab : min(p.vocab, begin + p.piece);
  const T* z = (const T*)p.z + row * p.ldz;
  T* dz = (T*)p.dz + row * p.lddz;
  const Entries e(lds, 0, p.k);
  if (threadIdx.x < 64) {
    if (JOIN) {
      const Running r = join_pieces(p, row);
      if (threadIdx.x == 0) {
        sh.m[0] = r.m;
        sh.s[0] = r.s;
        if (piece == 0) finish(p, row, r, p.parts[row]);
      }
    }
    Teacher mine = read_entries<T, true, true>(p, row, e);
    // few entries are gone through sooner than asked about (4096 rows of 32000 words, forward and backward: 256 entries 193 -> 183 us, 1024 750 -> 290)
    mine.twice = p.k <= 64 || names_twice(e, p.k, (int*)lds + 4 * p.k, slots);
    if (threadIdx.x == 0) sh.teacher = mine;
  }
  __syncthreads();
  const float w = p.dloss[row] * p.inv_t;
  const double mass = sh.teacher.mass;
  const bool none = w == 0.f || mass == 0.0;
  // p = exp((z - m) / T) / s, or, from lse, exp(z / T - lse): f exp2(z c - shift), with what the shift's rounding leaves out in f
  Running r;
  const float wm = w * (float)mass;
  float f = wm, shift;
  bool sound = true;
  if (JOIN) {
    r.m = sh.m[0];
    r.s = sh.s[0];
  } else if (again && !none) {
    r = sum_of<T, NT>(p, z, 0, p.vocab, sh);
  }
  if (JOIN || again) {
    f /= r.s;
    sound = r.sound(p.c) && fabsf(f) >= LEAST_FACTOR;
    shift = r.reference(p.c);
    if (sound) f *= r.rest(p.c);
  } else {
    const double exact = (double)p.lse[row] / (double)p.inv_t * (double)p.c;
    shift = (float)exact;
    f *= __builtin_amdgcn_exp2f((float)((double)shift - exact));
  }
  auto prob = [&](float x) { return f * __builtin_amdgcn_exp2f(fmaf(x, p.c, -shift)); };
  auto prob_slow = [&](float x) { return wm * (__builtin_amdgcn_exp2f((x - r.m) * p.c) / r.s); };
  int at = begin + threadIdx.x * N;
  if (none) {
    const float x[N] = {};
    for (; at < end; at += STEP) store_chunk(dz, at, end, x);
    return;
  }
  if (!sound) {
    for (; at < end; at += STEP) {
      float x[N];
      load_chunk(z, at, end, x);
#pragma unroll
      for (int e = 0; e < N; ++e) x[e] = prob_slow(x[e]);
      store_chunk(dz, at, end, x);
    }
  }
  for (; at + (U - 1) * STEP + N <= end; at += U * STEP) {
    typename Any16<T>::t v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const auto* from = reinterpret_cast<const typename Any16<T>::t*>(z + at + u * STEP);
      if constexpr (PAST == 2) v[u] = __builtin_nontemporal_load(from);
      else v[u] = *from;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
      for (int e = 0; e < N; ++e) v[u][e] = (T)prob((float)v[u][e]);
      auto* to = reinterpret_cast<typename Any16<T>::t*>(dz + at + u * STEP);
      if constexpr (PAST) __builtin_nontemporal_store(v[u], to);
      else *to = v[u];
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
    const int id = e.id[j];
    if (id >= begin && id < end) dz[id] = (T)((sound ? prob(e.z[j]) : prob_slow(e.z[j])) - w * (sh.teacher.twice ? teacher_at(e, p.k, id) : e.t[j]));
  }
}

// ---- rows of a few words: a wave has one in its registers, four to a workgroup, in every direction; the gradient has the row's own sum.  R chunks a lane.
template <typename T, int R> __global__ __launch_bounds__(256) void distill_short(const Distill p, int slots) {
  constexpr int N = Vec16<T>::N;
  extern __shared__ float lds[];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const size_t row = (size_t)blockIdx.x * 4 + wave;
  if (row >= (size_t)p.rows) return;
  const T* z = (const T*)p.z + row * p.ldz;
  float x[R][N];
#pragma unroll
  for (int r = 0; r < R; ++r) load_chunk(z, (64 * r + lane) * N, p.vocab, x[r]);
  const Entries e(lds, wave, p.k);
  const Teacher teacher = read_entries<T, true, true>(p, row, e);
  const bool twice = p.dz && names_twice(e, p.k, (int*)lds + 16 * p.k + wave * slots, slots);
  Running all;
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int i = 0; i < N; ++i) all.m = fmaxf(all.m, x[r][i]);
  all.m = wave_max(all.m);
  float sum = 0.f;
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int i = 0; i < N; ++i) {
      x[r][i] = __builtin_amdgcn_exp2f((x[r][i] - all.m) * p.c);
      sum += x[r][i];
    }
  all.s = wave_sum(sum);
  if (p.loss && lane == 0) finish(p, row, all, teacher);
  if (!p.dz) return;
  T* dz = (T*)p.dz + row * p.lddz;
  const float w = p.dloss[row] * p.inv_t;
  const bool none = w == 0.f || teacher.mass == 0.0;
  const float f = none ? 0.f : w * (float)teacher.mass / all.s;
#pragma unroll
  for (int r = 0; r < R; ++r) {
#pragma unroll
    for (int i = 0; i < N; ++i) x[r][i] = none ? 0.f : f * x[r][i];
    store_chunk(dz, (64 * r + lane) * N, p.vocab, x[r]);
  }
  if (none) return;
  __threadfence_block();                                // the row ahead of its entries; their words and weights are there for all lanes
  for (int j = lane; j < p.k; j += 64) {
    const int id = e.id[j];
    if (id >= 0) dz[id] = (T)(f * __builtin_amdgcn_exp2f((e.z[j] - all.m) * p.c) - w * (twice ? teacher_at(e, p.k, id) : e.t[j]));
  }
}

// Rows below this many leave compute units idle with a workgroup each: they go in pieces.
constexpr int FEW_ROWS = 160;
// Rows of up to this many words go a wave each, of twice as many in both directions at once (against a workgroup a row or pieces, us: bf16, both, 16384 rows of 200 words 68 -> 17,
// of 1000 75 -> 23, of 4000 102 -> 88, 100 of 4000 10.6 -> 8.4; each by itself 16384 of 1000 81 -> 38, of 2048 94 -> 55, but 4096 of 3096 29.4 -> 34.5).
constexpr int SHORT = 2048;
// A row's pieces: some 1024 workgroups in all, and at most one for every 2048 elements begun (pieces of 1368 elements for 4097, of 2000 for 50000)
int pieces_of(int rows, int vocab) {
  const int most = (vocab + 2047) / 2048, want = (1024 + rows - 1) / rows;
  return most < want ? most : want;
}
void divide(Distill& p, int pieces) {
  p.piece = ((p.vocab + pieces - 1) / pieces + 7) / 8 * 8;
  p.pieces = (p.vocab + p.piece - 1) / p.piece;
}

template <typename T, int NT, int R> hipError_t run_rows(const Distill& p, int per_unit, hipStream_t s) {
  const int most = 256 * per_unit;
  hipLaunchKernelGGL((distill_rows<T, NT, R>), dim3(p.rows < most ? p.rows : most), dim3(NT), 2 * entries_bytes(p.k), s, p);
  return hipGetLastError();
}
// the fewest steps that hold a row, in twos; workgroups that fill a compute unit
template <typename T> hipError_t run_both(const Distill& p, hipStream_t s) {
  static LdsAttrOnce lds_attr;
  if (hipError_t e = lds_attr.ensure(reinterpret_cast<const void*>(distill_teacher<T>), (int)entries_and_table_bytes(1024)); e != hipSuccess) return e;
  hipLaunchKernelGGL(distill_teacher<T>, dim3((p.rows + 3) / 4), dim3(256), entries_and_table_bytes(p.k), s, p, table_slots(p.k));
  if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  const int chunks = (p.vocab + Vec16<T>::N - 1) / Vec16<T>::N;
  if constexpr (256 * 4 * Vec16<T>::N > 2 * SHORT)      // fewer words are short rows
    if (chunks <= 256 * 4) return run_rows<T, 256, 4>(p, 4, s);
  if (chunks <= 256 * 6) return run_rows<T, 256, 6>(p, 4, s);
  if (chunks <= 256 * 8) return run_rows<T, 256, 8>(p, 4, s);
  if (chunks <= 512 * 6) return run_rows<T, 512, 6>(p, 2, s);
  if (chunks <= 512 * 8) return run_rows<T, 512, 8>(p, 2, s);
  if (chunks <= 1024 * 6) return run_rows<T, 1024, 6>(p, 1, s);
  if (chunks <= 1024 * 8) return run_rows<T, 1024, 8>(p, 1, s);
  if (chunks <= 1024 * 10) return run_rows<T, 1024, 10>(p, 1, s);
  if (chunks <= 1024 * 12) return run_rows<T, 1024, 12>(p, 1, s);
  if (chunks <= 1024 * 14) return run_rows<T, 1024, 14>(p, 1, s);
  return run_rows<T, 1024, 16>(p, 1, s);
}

// rows that one launch of the pass over whole rows takes: what their entries come to is in the workspace
constexpr int ROWS_A_LAUNCH = 16384;

template <typename T> hipError_t run_parts(Distill p, bool whole, hipStream_t s) {
  divide(p, whole ? 1 : pieces_of(p.rows, p.vocab));
  p.stats = (float2*)(p.parts + p.rows);
  const dim3 grid((unsigned)p.rows * p.pieces);
  const size_t lds = entries_bytes(p.k);
  const int slots = table_slots(p.k);
  const size_t lds_grad = lds + (p.k <= 64 ? 0 : sizeof(int) * slots);
  if (p.loss) {
    hipLaunchKernelGGL((distill_stats<T, 256>), grid, dim3(256), lds, s, p);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    if (p.dz) hipLaunchKernelGGL((distill_grad<T, 256, true, 0>), grid, dim3(256), lds_grad, s, p, slots);
    else if (p.pieces > 1) hipLaunchKernelGGL(distill_finish, dim3((p.rows + 3) / 4), dim3(256), 0, s, p);
  } else {
    // what the caches do not keep anyway: 300 rows of 131072 words (79 MB) 43.7 -> 34.2 us (41.3 with the loads), 4096 rows of 32000 124 -> 115 (103), of 131072
    // 445 -> 423 (406); 4096 rows of 1000 (8 MB) 16.5 either way, and whoever reads them next finds them there
    const double bytes = (double)p.rows * p.vocab * sizeof(T);
    if (bytes >= 160e6) hipLaunchKernelGGL((distill_grad<T, 256, false, 2>), grid, dim3(256), lds_grad, s, p, slots);
    else if (bytes >= 32e6) hipLaunchKernelGGL((distill_grad<T, 256, false, 1>), grid, dim3(256), lds_grad, s, p, slots);
    else hipLaunchKernelGGL((distill_grad<T, 256, false, 0>), grid, dim3(256), lds_grad, s, p, slots);
  }
  return hipGetLastError();
}

template <typename T, int R> hipError_t run_short(const Distill& p, hipStream_t s) {
  static LdsAttrOnce lds_attr;
  if (hipError_t e = lds_attr.ensure(reinterpret_cast<const void*>(distill_short<T, R>), (int)entries_and_table_bytes(1024)); e != hipSuccess) return e;
  hipLaunchKernelGGL((distill_short<T, R>), dim3((p.rows + 3) / 4), dim3(256), entries_and_table_bytes(p.k), s, p, table_slots(p.k));
  return hipGetLastError();
}
template <typename T> hipError_t run_short(const Distill& p, hipStream_t s) {
  constexpr int R = SHORT / (64 * Vec16<T>::N);
  if (p.vocab <= SHORT / 4) return run_short<T, R / 4>(p, s);
  if (p.vocab <= SHORT / 2) return run_short<T, R / 2>(p, s);
  return p.vocab <= SHORT ? run_short<T, R>(p, s) : run_short<T, 2 * R>(p, s);
}

template <typename T> hipError_t run(const Distill& p, hipStream_t s) {
  const bool both = p.loss && p.dz, is_short = p.vocab <= (both ? 2 * SHORT : SHORT);
  if (p.rows < FEW_ROWS && !is_short) return run_parts<T>(p, false, s);
  const int most = both && !is_short ? ROWS_A_LAUNCH : 1 << 22;   // a launch's 2^30 threads
  for (int first = 0; first < p.rows; first += most) {
    Distill q = p;
    q.rows = p.rows - first < most ? p.rows - first : most;
    q.z = (const T*)p.z + first * p.ldz;
    q.ids += (size_t)first * p.k;
    q.teacher += (size_t)first * p.k;
    q.lse += first;
    if (p.dz) {
      q.dz = (T*)p.dz + first * p.lddz;
      q.dloss += first;
    }
    if (p.loss) q.loss += first;
    if (hipError_t e = is_short ? run_short<T>(q, s) : both ? run_both<T>(q, s) : run_parts<T>(q, true, s); e != hipSuccess) return e;
    if (p.rows - first <= most) break;
  }
  return hipSuccess;
}

}  // namespace

// what the entries of a launch's rows come to, m and s of rows' pieces
uint64_t distill_ws_bytes(int rows, int vocab, int) {
  if (rows < FEW_ROWS) return sizeof(Teacher) * rows + 8ull * rows * pieces_of(rows, vocab);
  return (sizeof(Teacher) + 8ull) * (rows < ROWS_A_LAUNCH ? rows : ROWS_A_LAUNCH);
}

hipError_t launch_distill(int dtype, const void* z, size_t ldz, const int* ids, const float* teacher, const float* dloss, float* loss, float* lse, void* dz, size_t lddz,
                          void* ws, int rows, int vocab, int k, float temperature, int log_probs, hipStream_t s) {
  Distill p = {z, ids, teacher, dloss, loss, lse, dz, ldz, lddz, rows, vocab, k, log_probs ? 1.0 : 1.0 / (double)temperature, 1.f / temperature, LOG2E / temperature, log_probs, 1, vocab, nullptr, nullptr};
  p.parts = (Teacher*)ws;
  return dtype == DT_BF16 ? run<bf16_t>(p, s) : run<float>(p, s);
}
