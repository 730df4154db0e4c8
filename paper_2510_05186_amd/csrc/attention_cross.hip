// Attention of queries to the states of another sequence, of which the first kv_len count, with its gradients.
//
// bf16: the register and LDS scheme of attention_mfma.hip (every product on v_mfma_f32_32x32x16_bf16 in the orientation whose result is the next one's operand, tiles
// straight from memory into LDS), without a diagonal.  What differs:
//  * A kv head's query heads are one run of rows: row R of a group is query R % seq_q of its head R / seq_q, so that states are read once for the group and a
//    single token of eight heads fills a quarter of a tile instead of eight tiles.
//  * States beyond kv_len are never read: every block of 64 states has a buffer descriptor of its own that ends with them (so a cache of any length is within 32-bit
//    offsets), loads past it are zero, and what they score is taken out of the softmax.
//  * Work is split where rows alone do not fill the chip: forward and dQ over the states, dK / dV over the queries.  Parts leave fp32 sums in the workspace that
//    a second launch joins in a fixed order.
// The probabilities and dS enter the second products as one bf16 number (2^-8 of each at most, which adds about as much to the result's error as its own
// rounding does: 0.0024 of a tensor's norm from 64 bits, where rounding the result alone leaves 0.0017); sums, softmax and D are fp32.  Two numbers, as the causal
// kernels of heads of 64 take, bring heads of 64 to 0.0018 and less for another half of the second products and their packing (forward and backward, one / two, us: 16 / 8 heads x 8
// x 1024 x 1500 264 / 365, 16 heads x 4096 x 4096 339 / 477, 16 x 700 x 700 53 / 60, one token of 16 sequences x 16384 forward 74 / 80).  A single state has no gradient of its score: dS = p (dP - D) is 0 by definition and is not computed, since D
// comes from the rounded o.
#include "attention_f32_tiles.h"
#include "attention_tiles.h"

#include <math.h>

namespace {

constexpr float LOWEST = -3.402823466e38f;

template <typename T> struct CrossArgsOf {
  const T *q, *k, *v; const int* kv_len; const T *o_in, *dout;
  T* o; float* lse; T *dq, *dk, *dv; float *delta, *part;
  size_t ldq, ldkv;
  int seq_q, seq_kv, n_q, n_kv, rep, rows, splits;     // rows = rep seq_q, the rows of a kv head; splits: parts of the states (forward, dQ) or of the rows (dK / dV)
  int block_heads, blocks_per_head, row_blocks;         // of the rows, in the dK / dV kernel
  Divisor by_seq_q;
};
typedef CrossArgsOf<bf16_t> CrossArgs;

template <typename T> __device__ __forceinline__ int cross_states(const CrossArgsOf<T>& p, int b) { return p.kv_len ? min(max(p.kv_len[b], 0), p.seq_kv) : p.seq_kv; }

// descriptor of the first `rows` rows of `width` bytes from p on, `stride` bytes apart: loads beyond read zero.  All of it is the same for the whole wave.
__device__ __forceinline__ i32x4_t rows_desc(const void* p, int rows, unsigned stride, unsigned width) {
  const unsigned long long ad = (unsigned long long)p;
  i32x4_t d;
  d[0] = __builtin_amdgcn_readfirstlane((int)(unsigned)ad);
  d[1] = __builtin_amdgcn_readfirstlane((int)(unsigned)(ad >> 32) & 0xffff);
  d[2] = __builtin_amdgcn_readfirstlane(rows > 0 ? (int)((unsigned)(rows - 1) * stride + width) : 0);
  d[3] = 0x00020000;
  return d;
}

#define OPTSTAGE_SB() __builtin_amdgcn_sched_barrier(0)
#define OPTSTAGE_TILE_LOAD(dst, voff, desc) \
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" :: "s"(dst), "v"(voff), "s"(desc) : "memory", "m0")
// this wave's loads have landed (the barrier covers the other waves') and nobody still reads what the next ones overwrite
#define OPTSTAGE_BLOCK_SYNC() asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory")

// store4, or zeros: what a state that does not count has gathered is another's
__device__ __forceinline__ void store4_if(bf16_t* at, const f32x16_t& x, int v, float scale, bool on) {
  bf16x4_t r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = on ? (bf16_t)(x[v + i] * scale) : (bf16_t)0.f;
  *reinterpret_cast<bf16x4_t*>(at) = r;
}

typedef short i16x4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) i16x4_t lds_i16x4_t;
__device__ __forceinline__ bf16x8_t transposed8(int lo_at, int hi_at) {
  const i16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4_t*)(unsigned)lo_at);
  const i16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4_t*)(unsigned)hi_at);
  return __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}

// the blocks of 64 states of part `part` of `splits`: [first, end)
struct Blocks { int first, end; };
__device__ __forceinline__ Blocks blocks_of(int n, int part, int splits) {
  const int all = (n + 63) / 64, per = (all + splits - 1) / splits;
  return {min(all, part * per), min(all, part * per + per)};
}

// ---- forward: grid (n_kv x splits x tiles of 32 NW rows, batch), NW waves of 32 rows ----------------------------------------------------
// LDS: two stages of K, two of V, 64 states each.  Steps of consecutive tiles of 32 states are interleaved by hand as in attention_mfma.hip: the exponentials of a
// tile run between the score MFMAs of the next, the maxima of the next between its O^T MFMAs; the softmax reference is raised only when a score lies more
// than FWD_TAU / c above it.
constexpr float FWD_TAU = 8.f;

template <int D, int NW>
__global__ __launch_bounds__(64 * NW) void cross_fwd_mfma(const CrossArgs p) {
  typedef Head<D> H;
  constexpr int ROWB = H::ROWB, TILE = H::TILE, NKS = H::NKS, NDT = H::NDT;
  constexpr int WROWS = 64 / NW, NLD = WROWS / H::RPL;
  constexpr int V_RING = 2 * TILE;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 5, c32 = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int kvh = blockIdx.x % p.n_kv, at_x = blockIdx.x / p.n_kv, tile = at_x / p.splits, part = at_x % p.splits, b = blockIdx.y;
  const int n = __builtin_amdgcn_readfirstlane(cross_states(p, b));
  const Blocks kb = blocks_of(n, part, p.splits);
  const int end = min(n, 64 * kb.end);                  // states of this part end here
  const int row = tile * 32 * NW + 32 * wave + c32;
  const bool mine = row < p.rows;
  const int rowc = mine ? row : p.rows - 1, head = p.by_seq_q.quotient(rowc), t = rowc - head * p.seq_q;
  const size_t stat = ((size_t)b * p.n_kv + kvh) * p.rows + rowc, all_rows = (size_t)gridDim.y * p.n_kv * p.rows;
  const size_t out_at = (((size_t)b * p.seq_q + t) * p.n_q + kvh * p.rep + head) * D;
  const float scale = rsqrtf((float)D), c = scale * LOG2E, thr = FWD_TAU / c;

  if (kb.first >= kb.end) {                             // no states
    if (!mine) return;
    if (p.splits > 1) {
      if (g == 0) *reinterpret_cast<float2*>(p.part + (size_t)p.splits * all_rows * D + ((size_t)part * all_rows + stat) * 2) = make_float2(-INFINITY, 0.f);
      return;
    }
    const bf16x8_t zero = {};
#pragma unroll
    for (int ks = 0; ks < NKS; ++ks) *reinterpret_cast<bf16x8_t*>(p.o + out_at + 16 * ks + 8 * g) = zero;
    if (g == 0) p.lse[stat] = -INFINITY;
    return;
  }

  bf16x8_t Qf[NKS];
  {
    const bf16_t* qp = p.q + ((size_t)b * p.seq_q + t) * p.ldq + (size_t)(kvh * p.rep + head) * D + 8 * g;
#pragma unroll
    for (int ks = 0; ks < NKS; ++ks) Qf[ks] = *reinterpret_cast<const bf16x8_t*>(qp + 16 * ks);
  }
  f32x16_t acc[NDT];                                    // O^T: lane = row, registers = d
#pragma unroll
  for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
    for (int v = 0; v < 16; ++v) acc[dt][v] = 0.f;
  float mref = LOWEST, lsum = 0.f;                      // finite: a score of minus infinity lies below it and weighs nothing

  const int lds0 = (int)(unsigned)(size_t)(lds_void_t*)smem;
  int rm_addr[NKS], tr_addr[NDT][2];
  {
    const int f = H::swz(c32);
#pragma unroll
    for (int ks = 0; ks < NKS; ++ks) rm_addr[ks] = c32 * ROWB + (((2 * ks + g) ^ f) << 4);
    const int cg = (lane >> 4) & 1, e = (lane >> 2) & 3, r = lane & 3;
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
      for (int kq = 0; kq < 2; ++kq)
        tr_addr[dt][kq] = lds0 + V_RING + (4 * g + e) * ROWB + (((4 * dt + 2 * cg + (r >> 1)) ^ H::swz(8 * kq + 4 * g + e)) << 4) + (r & 1) * 8;
  }
  const unsigned stride = (unsigned)p.ldkv * 2u;
  unsigned voff[NLD];
#pragma unroll
  for (int j = 0; j < NLD; ++j) {
    const int lr = WROWS * wave + H::RPL * j + lane / H::CH;
    voff[j] = (unsigned)lr * stride + (unsigned)((lane % H::CH) ^ H::swz(lr)) * 16u;
  }
  const size_t base = ((size_t)b * p.seq_kv) * p.ldkv + (size_t)kvh * D;
  auto issue_tile = [&](const bf16_t* x, int blk, int lds) {
    const i32x4_t rs = rows_desc(x + base + (size_t)blk * 64 * p.ldkv, min(n - 64 * blk, 64), stride, ROWB);
    const unsigned dst = (unsigned)(lds0 + lds) + (WROWS * wave) * ROWB;
#pragma unroll
    for (int j = 0; j < NLD; ++j) OPTSTAGE_TILE_LOAD(dst + j * 1024, voff[j], rs);
  };
  auto tr_frag = [&](int at, int dt, int tt, int u) {
    return transposed8(tr_addr[dt][0] + at + (32 * tt + 16 * u) * ROWB, tr_addr[dt][1] + at + (32 * tt + 16 * u + 8) * ROWB);
  };
  auto rm_frag = [&](const char* at, int tt, int ks) { return *reinterpret_cast<const bf16x8_t*>(at + tt * 32 * ROWB + rm_addr[ks]); };

  constexpr int PF = 3, PT = 3;
  bf16x8_t kf[PF], trf[PT];
  // scores of tile tt of the K stage into nxt, between them the exponentials of cur; the first operand fragments of a step are read during the step before it
  auto step_scores = [&](bool with_exp, int stage_k, int tt, f32x16_t& cur, f32x16_t& nxt, int stage_v, int tv) __attribute__((always_inline)) {
    const char* sK = smem + stage_k * TILE;
    const float mc = mref * c;
    float ls = 0.f;
#pragma unroll
    for (int ks = 0; ks < NKS; ++ks) {
      OPTSTAGE_SB();
      if (ks + PF - 1 < NKS) kf[(ks + PF - 1) % PF] = rm_frag(sK, tt, ks + PF - 1);
      if (stage_v >= 0 && ks + PT - 1 >= NKS) trf[ks + PT - 1 - NKS] = tr_frag(stage_v * TILE, (ks + PT - 1 - NKS) % NDT, tv, (ks + PT - 1 - NKS) / NDT);
      OPTSTAGE_SB();
      asm volatile("s_nop 1" :: "v"(kf[ks % PF]));      // the operand has settled before an MFMA that the compiler does not see into
      if (ks == 0)
        asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, 0" : "=&v"(nxt) : "v"(kf[0]), "a"(Qf[0]));
      else
        asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+v"(nxt) : "v"(kf[ks % PF]), "a"(Qf[ks]));
      OPTSTAGE_SB();
      if (with_exp) {
        constexpr int PV = 16 / NKS;
#pragma unroll
        for (int x = 0; x < PV; ++x) {
          const int v = ks * PV + x;
          cur[v] = __builtin_amdgcn_exp2f(fmaf(cur[v], c, -mc));
          ls += cur[v];
          asm volatile("" : "+v"(cur[v]), "+v"(ls));    // stays between the MFMAs it is written between
        }
      }
      OPTSTAGE_SB();
    }
    OPTSTAGE_SB();
    lsum += ls;
  };
  // states past the part's end (a whole tile of them behind the last block) leave the softmax
  auto mask_tile = [&](int key0, f32x16_t& sc) __attribute__((always_inline)) {
    if (key0 + 32 <= end) return;                       // the same for the whole workgroup
    asm volatile("s_nop 7" ::: "memory");               // the scores' last MFMA has written its results
#pragma unroll
    for (int v = 0; v < 16; ++v)
      if (key0 + 8 * (v >> 2) + 4 * g + (v & 3) >= end) sc[v] = -INFINITY;
  };
  auto max_part = [&](int i, const f32x16_t& sc, float& mx) __attribute__((always_inline)) {
#pragma unroll
    for (int x = 0; x < 4 / NDT; ++x) {
      const int v = 2 * (i * (4 / NDT) + x);
      mx = fmaxf(mx, fmaxf(sc[v], sc[v + 1]));
    }
    asm volatile("" : "+v"(mx));
  };
  auto raise_reference = [&](float mx) __attribute__((always_inline)) {
    mx = pair_max32(mx);
    if (__any(mx > mref + thr)) {
      asm volatile("s_nop 15\n\ts_nop 7" ::: "memory"); // the last O^T MFMAs have left the matrix unit
      const float mn = fmaxf(mref, mx);
      const float alpha = mn == mref ? 1.f : __builtin_amdgcn_exp2f((mref - mn) * c);
      mref = mn;
      lsum *= alpha;
#pragma unroll
      for (int dt = 0; dt < NDT; ++dt) {
        OPTSTAGE_SB();
#pragma unroll
        for (int v = 0; v < 16; ++v) acc[dt][v] *= alpha;
      }
      OPTSTAGE_SB();
    }
  };
  // O^T += V^T P^T of the tile in cur, between the MFMAs the maxima of the next tile (scores in nxt, states from key1 on)
  auto step_output = [&](bool fill, int stage_v, int tt, int key1, f32x16_t& cur, f32x16_t& nxt, int stage_k, int tk) __attribute__((always_inline)) {
    if (fill) {
#pragma unroll
      for (int i = 0; i < PT - 1; ++i) trf[i] = tr_frag(stage_v * TILE, i % NDT, tt, i / NDT);
    }
    mask_tile(key1, nxt);
    float mx = -INFINITY;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const bf16x8_t pr = pack8(cur, u);
#pragma unroll
      for (int dt = 0; dt < NDT; ++dt) {
        const int i = u * NDT + dt, n2 = i + PT - 1, k2 = i + PF - 1 - 2 * NDT;
        OPTSTAGE_SB();
        if (n2 < 2 * NDT) trf[n2 % PT] = tr_frag(stage_v * TILE, n2 % NDT, tt, n2 / NDT);
        if (stage_k >= 0 && k2 >= 0) kf[k2] = rm_frag(smem + stage_k * TILE, tk, k2);
        if (dt == 0) asm volatile("s_nop 1" :: "v"(pr) : "memory");
        OPTSTAGE_SB();
        asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+a"(acc[dt]) : "v"(trf[i % PT]), "v"(pr));
        OPTSTAGE_SB();
        max_part(i, nxt, mx);
      }
    }
    OPTSTAGE_SB();
    raise_reference(mx);
  };
  auto fill_k = [&](int stage, int tt) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < PF - 1; ++i) kf[i] = rm_frag(smem + stage * TILE, tt, i);
  };
  f32x16_t sA, sB;
  issue_tile(p.k, kb.first, 0);
  OPTSTAGE_BLOCK_SYNC();
  if (kb.first + 1 < kb.end) issue_tile(p.k, kb.first + 1, TILE);
  issue_tile(p.v, kb.first, V_RING);
  fill_k(0, 0);
  step_scores(false, 0, 0, sB, sA, -1, 0);
  {
    asm volatile("s_nop 15\n\ts_nop 7" ::: "memory");
    mask_tile(64 * kb.first, sA);
    float mx = -INFINITY;
#pragma unroll
    for (int i = 0; i < 2 * NDT; ++i) max_part(i, sA, mx);
    raise_reference(mx);
    fill_k(0, 1);
  }
  auto block = [&](int blk, int st) __attribute__((always_inline)) {
    step_scores(true, st, 1, sA, sB, -1, 0);
    OPTSTAGE_BLOCK_SYNC();                              // K of the next block and V of this one, requested a block ago
    if (blk + 2 < kb.end) issue_tile(p.k, blk + 2, st * TILE);
    if (blk + 1 < kb.end) issue_tile(p.v, blk + 1, V_RING + (st ^ 1) * TILE);
    step_output(true, st, 0, 64 * blk + 32, sA, sB, st ^ 1, 0);
    // behind the last block these scores are of a stage that holds none of the part's states: masked, never used
    step_scores(true, st ^ 1, 0, sB, sA, st, 1);
    step_output(false, st, 1, 64 * blk + 64, sB, sA, st ^ 1, 1);
  };
  for (int blk = kb.first; blk < kb.end; blk += 2) {
    block(blk, 0);
    if (blk + 1 < kb.end) block(blk + 1, 1);
  }
  asm volatile("s_nop 15\n\ts_nop 7" ::: "memory");
  const float lt = lsum + __shfl_xor(lsum, 32, 64);
  if (!mine) return;
  if (p.splits > 1) {
    float* out = p.part + ((size_t)part * all_rows + stat) * D;
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        OPTSTAGE_SB();
        *reinterpret_cast<f32x4_t*>(out + 32 * dt + 8 * j + 4 * g) = f32x4_t{acc[dt][4 * j], acc[dt][4 * j + 1], acc[dt][4 * j + 2], acc[dt][4 * j + 3]};
      }
    if (g == 0) *reinterpret_cast<float2*>(p.part + (size_t)p.splits * all_rows * D + ((size_t)part * all_rows + stat) * 2) = make_float2(mref, lt);
    return;
  }
  const float inv = 1.f / lt;
  bf16_t* orow = p.o + out_at;
#pragma unroll
  for (int dt = 0; dt < NDT; ++dt) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      OPTSTAGE_SB();
      store4(orow + 32 * dt + 8 * j + 4 * g, acc[dt], 4 * j, inv);
    }
  }
  if (g == 0) p.lse[stat] = mref * scale + logf(lt);
}

template <typename T> __device__ __forceinline__ void store8(T* at, const float (&x)[8], float scale) {
  Vec16<T> v;
#pragma unroll
  for (int h = 0; h < 8; h += Vec16<T>::N) {
#pragma unroll
    for (int e = 0; e < Vec16<T>::N; ++e) v.set(e, x[h + e] * scale);
    *reinterpret_cast<Vec16<T>*>(at + h) = v;
  }
}

// o and lse of a row from its parts' sums, whose references are in units of `unit`: a wave a row, a lane a part for its weight, then D / 64 columns
template <typename T, int D> __global__ __launch_bounds__(256) void cross_fwd_join(const CrossArgsOf<T> p, size_t all_rows, float unit) {
  constexpr int E = D / 64, U = 8;
  typedef float sums_t __attribute__((ext_vector_type(E)));
  const size_t stat = (size_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (stat >= all_rows) return;
  const int lane = threadIdx.x & 63;
  const float c = unit * LOG2E;
  const float2* ml = reinterpret_cast<const float2*>(p.part + (size_t)p.splits * all_rows * D) + stat;
  const float2 mine = lane < p.splits ? ml[lane * all_rows] : make_float2(-INFINITY, 0.f);
  const float m = wave_max(mine.x);
  const float f = mine.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((mine.x - m) * c), l = wave_sum(mine.y * f);
  float x[E] = {};
  const float* sums = p.part + stat * D + lane * E;
  for (int s0 = 0; s0 < p.splits; s0 += U) {
    sums_t v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      // a part without states has left no sums; they come last
      const bool on = s0 + u < p.splits && __shfl(mine.x, s0 + u, 64) != -INFINITY;
      v[u] = sums_t(0.f);
      if (on) v[u] = *reinterpret_cast<const sums_t*>(sums + (size_t)(s0 + u) * all_rows * D);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const float w = __shfl(f, (s0 + u) & 63, 64);
#pragma unroll
      for (int e = 0; e < E; ++e) x[e] = fmaf(v[u][e], w, x[e]);
    }
  }
  const size_t t = stat % p.seq_q, a = stat / p.seq_q % p.n_q, b = stat / p.seq_q / p.n_q;
  const bool none = m == -INFINITY;
  const float inv = none ? 0.f : 1.f / l;
  T* o = p.o + ((b * p.seq_q + t) * p.n_q + a) * D + lane * E;
#pragma unroll
  for (int e = 0; e < E; ++e) o[e] = (T)(x[e] * inv);
  if (lane == 0) p.lse[stat] = none ? -INFINITY : m * unit + logf(l);
}

// ---- backward, dQ: grid as forward ---------------------------------------------------------------------------------------------------
// The rows' Q and dO fragments and dQ^T stay in registers; blocks of 64 states (K and V rows) stream through two stages.  Stores -D = -<dO, o> of its rows for the
// dK / dV kernel, which runs after it.
template <int D, int NW>
__global__ __launch_bounds__(64 * NW) void cross_dq_mfma(const CrossArgs p) {
  typedef Head<D> H;
  constexpr int ROWB = H::ROWB, TILE = H::TILE, NKS = H::NKS, NDT = H::NDT;
  constexpr int WROWS = 64 / NW, NLD = WROWS / H::RPL;
  constexpr int STAGE = 2 * TILE;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 5, c32 = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int kvh = blockIdx.x % p.n_kv, at_x = blockIdx.x / p.n_kv, tile = at_x / p.splits, part = at_x % p.splits, b = blockIdx.y;
  const int n = __builtin_amdgcn_readfirstlane(cross_states(p, b));
  const Blocks kb = blocks_of(n == 1 ? 0 : n, part, p.splits);   // one state: no gradient of its score
  const int row = tile * 32 * NW + 32 * wave + c32;
  const bool mine = row < p.rows;
  const int rowc = mine ? row : p.rows - 1, head = p.by_seq_q.quotient(rowc), t = rowc - head * p.seq_q;
  const size_t stat = ((size_t)b * p.n_kv + kvh) * p.rows + rowc;
  const float scale = rsqrtf((float)D), c = scale * LOG2E;
  bf16x8_t Qf[NKS], dOf[NKS];
  float Lc, Dq;
  {
    const size_t at = (size_t)(kvh * p.rep + head) * D + 8 * g, tok = (size_t)b * p.seq_q + t;
    const bf16_t *qp = p.q + tok * p.ldq + at, *dop = p.dout + tok * p.n_q * D + at, *op = p.o_in + tok * p.n_q * D + at;
    float dsum = 0.f;
#pragma unroll
    for (int ks = 0; ks < NKS; ++ks) {
      Qf[ks] = *reinterpret_cast<const bf16x8_t*>(qp + 16 * ks);
      dOf[ks] = *reinterpret_cast<const bf16x8_t*>(dop + 16 * ks);
      const bf16x8_t of = *reinterpret_cast<const bf16x8_t*>(op + 16 * ks);
#pragma unroll
      for (int e = 0; e < 8; ++e) dsum = fmaf((float)dOf[ks][e], (float)of[e], dsum);
    }
    Lc = -p.lse[stat] * LOG2E;
    Dq = dsum + __shfl_xor(dsum, 32, 64);
  }
  f32x16_t negD;                                        // the initial value of the dP^T MFMAs, which then deliver dP^T - D
#pragma unroll
  for (int ks = 0; ks < NKS; ++ks) asm volatile("" : "+a"(Qf[ks]), "+a"(dOf[ks]));
  f32x16_t acc[NDT];
#pragma unroll
  for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
    for (int v = 0; v < 16; ++v) acc[dt][v] = 0.f;
  const int lds0 = (int)(unsigned)(size_t)(lds_void_t*)smem;
  int rm_addr[NKS], tr_addr[NDT][2];
  {
    const int f = H::swz(c32);
#pragma unroll
    for (int ks = 0; ks < NKS; ++ks) {
      rm_addr[ks] = lds0 + c32 * ROWB + (((2 * ks + g) ^ f) << 4);
      asm volatile("" : "+v"(rm_addr[ks]));             // one number per read, not the terms of a sum
    }
    const int cg = (lane >> 4) & 1, e = (lane >> 2) & 3, r = lane & 3;
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
      for (int kq = 0; kq < 2; ++kq) {
        tr_addr[dt][kq] = lds0 + (4 * g + e) * ROWB + (((4 * dt + 2 * cg + (r >> 1)) ^ H::swz(8 * kq + 4 * g + e)) << 4) + (r & 1) * 8;
        asm volatile("" : "+v"(tr_addr[dt][kq]));
      }
  }
  const unsigned stride = (unsigned)p.ldkv * 2u;
  unsigned voff[NLD];
#pragma unroll
  for (int j = 0; j < NLD; ++j) {
    const int lr = WROWS * wave + H::RPL * j + lane / H::CH;
    voff[j] = (unsigned)lr * stride + (unsigned)((lane % H::CH) ^ H::swz(lr)) * 16u;
  }
  const size_t base = ((size_t)b * p.seq_kv) * p.ldkv + (size_t)kvh * D;
  auto issue_block = [&](int blk, int stage) {
    const int rows = min(n - 64 * blk, 64);
    const size_t at = base + (size_t)blk * 64 * p.ldkv;
    const i32x4_t rk = rows_desc(p.k + at, rows, stride, ROWB), rv = rows_desc(p.v + at, rows, stride, ROWB);
    const unsigned dst = (unsigned)lds0 + stage * STAGE + (WROWS * wave) * ROWB;
#pragma unroll
    for (int j = 0; j < NLD; ++j) {
      OPTSTAGE_TILE_LOAD(dst + j * 1024, voff[j], rk);
      OPTSTAGE_TILE_LOAD(dst + TILE + j * 1024, voff[j], rv);
    }
  };
  auto tr_frag = [&](int at, int dt, int tt, int u) {
    return transposed8(tr_addr[dt][0] + at + (32 * tt + 16 * u) * ROWB, tr_addr[dt][1] + at + (32 * tt + 16 * u + 8) * ROWB);
  };
  auto rm_frag = [&](int at, int tt, int ks) { return *(const lds_bf16x8_t*)(unsigned)(rm_addr[ks] + at + tt * 32 * ROWB); };
#define OPTSTAGE_MFMA_V(acc, a, b) asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+v"(acc) : "v"(a), "a"(b))
#define OPTSTAGE_MFMA_0(acc, a, b) asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, 0" : "=&v"(acc) : "v"(a), "a"(b))
  // P^T and dP^T - D of the tile of 32 states from key0 on, half tt of a stage; P is 0 behind the last state
  auto weights = [&](int sK, int tt, int key0, f32x16_t& s, f32x16_t& dp) __attribute__((always_inline)) {
    const int sV = sK + TILE;
    bf16x8_t kf[2], vf[2];
    kf[0] = rm_frag(sK, tt, 0);
#pragma unroll
    for (int ks = 0; ks < NKS; ++ks) {                  // S^T = K Q^T
      OPTSTAGE_SB();
      if (ks < NKS - 1) kf[(ks + 1) & 1] = rm_frag(sK, tt, ks + 1);
      else vf[0] = rm_frag(sV, tt, 0);
      OPTSTAGE_SB();
      if (ks == 0) OPTSTAGE_MFMA_0(s, kf[0], Qf[0]);
      else OPTSTAGE_MFMA_V(s, kf[ks & 1], Qf[ks]);
    }
#pragma unroll
    for (int ks = 0; ks < NKS; ++ks) {                  // dP^T = V dO^T, the exponentials of S^T under its MFMAs
      OPTSTAGE_SB();
      if (ks < NKS - 1) vf[(ks + 1) & 1] = rm_frag(sV, tt, ks + 1);
      OPTSTAGE_SB();
      if (ks == 0) {
        asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %3" : "=&v"(dp) : "v"(vf[0]), "a"(dOf[0]), "v"(negD));
        asm volatile("s_nop 7" ::: "memory");           // the exponentials read S^T a few cycles after the matrix unit has written it
      } else {
        OPTSTAGE_MFMA_V(dp, vf[ks & 1], dOf[ks]);
      }
      OPTSTAGE_SB();
#pragma unroll
      for (int e = 0; e < 16 / NKS; ++e) {
        const int v = (16 / NKS) * ks + e;
        s[v] = __builtin_amdgcn_exp2f(fmaf(s[v], c, Lc));
      }
    }
    OPTSTAGE_SB();
    if (key0 + 32 > n) {
      asm volatile("" ::: "memory");                    // a real branch: only the last tile pays for the mask
#pragma unroll
      for (int v = 0; v < 16; ++v)
        if (key0 + 8 * (v >> 2) + 4 * g + (v & 3) >= n) s[v] = 0.f;
    }
    asm volatile("s_nop 15\n\ts_nop 7" ::: "memory");   // dP^T has left the matrix unit
    OPTSTAGE_SB();
  };
  auto block = [&](int blk, int stage) __attribute__((always_inline)) {
    const int sK = stage * STAGE;
#pragma unroll
    for (int tt = 0; tt < 2; ++tt) {
      const int key0 = 64 * blk + 32 * tt;
      if (key0 >= n) continue;                          // the same for the whole workgroup
      f32x16_t s, dp;                                   // lane = row, registers = states key0 + 8 (v / 4) + 4 g + v % 4
      weights(sK, tt, key0, s, dp);
      bf16x8_t trf[2];                                  // dQ^T += K^T dS^T; dS^T of the second half under the MFMAs of the first
      trf[0] = tr_frag(sK, 0, tt, 0);
#pragma unroll
      for (int v = 0; v < 8; ++v) dp[v] = s[v] * dp[v];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const bf16x8_t d = pack8(dp, u);
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt) {
          const int i = u * NDT + dt;
          OPTSTAGE_SB();
          if (i < 2 * NDT - 1) trf[(i + 1) & 1] = tr_frag(sK, (dt + 1) % NDT, tt, dt == NDT - 1 ? 1 : u);
          OPTSTAGE_SB();
          acc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(trf[i & 1], d, acc[dt], 0, 0, 0);
          OPTSTAGE_SB();
          if (u == 0) {
#pragma unroll
            for (int e = 0; e < 8 / NDT; ++e) {
              const int v = 8 + (8 / NDT) * dt + e;
              dp[v] = s[v] * dp[v];
            }
          }
        }
      }
      OPTSTAGE_SB();
    }
  };
  if (kb.first < kb.end) issue_block(kb.first, 0);
#pragma unroll
  for (int v = 0; v < 16; ++v) negD[v] = -Dq;
  if (n <= 64 && kb.first < kb.end) {
    // Few states: what o's rounding leaves in D is large against dP - D (2 states: dq 2.2 times as far from 64 bits as one rounding, 16 states 1.5; from some 64 on
    // 1.45, dS's own rounding).  All of them are in this block: D is corrected by the sum of P (dP - D), which has to be 0.
    OPTSTAGE_BLOCK_SYNC();
    float sum = 0.f;
#pragma unroll
    for (int tt = 0; tt < 2; ++tt) {
      if (32 * tt >= n) continue;
      f32x16_t s, dp;
      weights(0, tt, 32 * tt, s, dp);
#pragma unroll
      for (int v = 0; v < 16; ++v) sum = fmaf(s[v], dp[v], sum);
    }
    Dq += sum + __shfl_xor(sum, 32, 64);
#pragma unroll
    for (int v = 0; v < 16; ++v) negD[v] = -Dq;
  }
  if (part == 0 && g == 0 && mine) p.delta[stat] = -Dq;
  for (int blk = kb.first; blk < kb.end; blk += 2) {
    OPTSTAGE_BLOCK_SYNC();
    if (blk + 1 < kb.end) issue_block(blk + 1, 1);
    block(blk, 0);
    if (blk + 1 < kb.end) {
      OPTSTAGE_BLOCK_SYNC();
      if (blk + 2 < kb.end) issue_block(blk + 2, 0);
      block(blk + 1, 1);
    }
  }
#undef OPTSTAGE_MFMA_V
#undef OPTSTAGE_MFMA_0
  if (!mine) return;
  if (p.splits > 1) {
    if (kb.first >= kb.end) return;                     // the join counts the parts that have states
    float* out = p.part + ((size_t)part * gridDim.y * p.n_kv * p.rows + stat) * D;
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        OPTSTAGE_SB();
        *reinterpret_cast<f32x4_t*>(out + 32 * dt + 8 * j + 4 * g) = f32x4_t{acc[dt][4 * j], acc[dt][4 * j + 1], acc[dt][4 * j + 2], acc[dt][4 * j + 3]};
      }
    return;
  }
  bf16_t* dq = p.dq + ((size_t)b * p.seq_q + t) * p.ldq + (size_t)(kvh * p.rep + head) * D;
#pragma unroll
  for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      OPTSTAGE_SB();
      store4(dq + 32 * dt + 8 * j + 4 * g, acc[dt], 4 * j, scale);
    }
}

// BLOCK: states to a block of the division into parts
template <typename T, int D, int BLOCK> __global__ __launch_bounds__(256) void cross_dq_join(const CrossArgsOf<T> p, size_t all_rows) {
  constexpr int Q = D / 8;
  const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x, stat = i / Q;
  if (stat >= all_rows) return;
  const int col = (int)(i % Q) * 8;
  const size_t t = stat % p.seq_q, a = stat / p.seq_q % p.n_q, b = stat / p.seq_q / p.n_q;
  const int n = cross_states(p, (int)b), all = n == 1 ? 0 : (n + BLOCK - 1) / BLOCK, per = (all + p.splits - 1) / p.splits;
  float x[8] = {};
  for (int s = 0; s * per < all; ++s) {
    const f32x4_t* f = reinterpret_cast<const f32x4_t*>(p.part + (s * all_rows + stat) * D + col);
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int e = 0; e < 4; ++e) x[4 * h + e] += f[h][e];
  }
  store8(p.dq + (b * p.seq_q + t) * p.ldq + a * D + col, x, rsqrtf((float)D));
}

// Blocks of up to 64 rows of a kv head: 64 queries of one head, or, of shorter sequences, as many whole heads (a divisor of theirs) as fit: then a
// block's lanes differ from the next one's by one distance, and no block holds rows of a third kind.
struct RowBlocks { int heads, per_head, all; };
__host__ __device__ __forceinline__ RowBlocks row_blocks(int seq_q, int rep) {
  if (seq_q >= 64) return {1, (seq_q + 63) / 64, rep * ((seq_q + 63) / 64)};
  int heads = 64 / seq_q < rep ? 64 / seq_q : rep;
  while (rep % heads) --heads;
  return {heads, 1, rep / heads};
}
__device__ __forceinline__ RowBlocks row_blocks(const CrossArgs& p) { return {p.block_heads, p.blocks_per_head, p.row_blocks}; }
// an offset past every descriptor's end, whatever is added to it for a block: rows span less than 15 * 2^28 bytes
constexpr unsigned PAST = 0xF0000000u;

// ---- backward, dK / dV: grid (n_kv x splits x tiles of 128 states, batch), 8 waves --------------------------------------------------
// A wave owns 32 states: K fragments, dK^T and dV^T in registers, the V rows of the workgroup's states in LDS.  Blocks of 64 rows (Q and dO, lse and -D) stream through
// two stages; rows past the last one read as zeros and add nothing.  Two groups of four waves have the same states and 32 rows of every block each; the first
// adds the second's sums at the end.  (64 states to a wave, one wave to a SIMD: 1629 us against 1650 for 64 / 8 heads x 4096 queries and states, forward's
// dQ included, but 582 / 561 for 32 heads x 4096 x 2305 and 70 / 55 for 16 heads x 2 x 1024 x 577, by its fewer workgroups.)
template <int D>
__global__ __launch_bounds__(512) void cross_dkv_mfma(const CrossArgs p) {
  typedef Head<D> H;
  constexpr int ROWB = H::ROWB, TILE = H::TILE, NKS = H::NKS, NDT = H::NDT;
  constexpr int WROWS = 8, NLD = WROWS / H::RPL;
  constexpr int STAGE = 2 * TILE + 512;                 // Q tile, dO tile, 64 lse, 64 -D
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 5, c32 = lane & 31;
  const int id = __builtin_amdgcn_readfirstlane(tid >> 6), wave = id & 3, grp = id >> 2;
  constexpr int WK = 32, GK = 4 * WK;
  const int kvh = blockIdx.x % p.n_kv, at_x = blockIdx.x / p.n_kv, k0 = at_x / p.splits * GK, part = at_x % p.splits, b = blockIdx.y;
  const int n = __builtin_amdgcn_readfirstlane(cross_states(p, b));
  const int first_k = k0 + WK * wave;
  const float scale = rsqrtf((float)D), c = scale * LOG2E;
  const size_t base = ((size_t)b * p.seq_kv) * p.ldkv + (size_t)kvh * D;
  if (k0 >= n) {                                        // states that do not count have no gradient
    if (p.splits > 1) return;                           // the join writes their zeros
    const bf16x8_t zero = {};
    for (int i = tid; i < GK * (D / 8); i += 512) {
      const int s = k0 + i / (D / 8), col = i % (D / 8) * 8;
      if (s >= p.seq_kv) break;
      *reinterpret_cast<bf16x8_t*>(p.dk + base + (size_t)s * p.ldkv + col) = zero;
      *reinterpret_cast<bf16x8_t*>(p.dv + base + (size_t)s * p.ldkv + col) = zero;
    }
    return;
  }
  bf16x8_t Kf[NKS];
  {
    const bf16_t* kp = p.k + base + (size_t)min(first_k + c32, n - 1) * p.ldkv + 8 * g;
#pragma unroll
    for (int ks = 0; ks < NKS; ++ks) Kf[ks] = *reinterpret_cast<const bf16x8_t*>(kp + 16 * ks);
  }
  f32x16_t accK[1][NDT], accV[1][NDT];                  // lane = state, registers = d
#pragma unroll
  for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
    for (int v = 0; v < 16; ++v) { accK[0][dt][v] = 0.f; accV[0][dt][v] = 0.f; }
  const int lds0 = (int)(unsigned)(size_t)(lds_void_t*)smem;
  const int half = grp * 32, row4 = lds0 + 16 * g + half * 4;
  int rm_addr[NKS], tr_addr[NDT][2];
  {
    const int f = H::swz(c32);
#pragma unroll
    for (int ks = 0; ks < NKS; ++ks) {
      rm_addr[ks] = lds0 + half * ROWB + c32 * ROWB + (((2 * ks + g) ^ f) << 4);
      asm volatile("" : "+v"(rm_addr[ks]));
    }
    const int cg = (lane >> 4) & 1, e = (lane >> 2) & 3, r = lane & 3;
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
      for (int kq = 0; kq < 2; ++kq) {
        tr_addr[dt][kq] = lds0 + half * ROWB + (4 * g + e) * ROWB + (((4 * dt + 2 * cg + (r >> 1)) ^ H::swz(8 * kq + 4 * g + e)) << 4) + (r & 1) * 8;
        asm volatile("" : "+v"(tr_addr[dt][kq]));
      }
  }
  const size_t head0 = (size_t)kvh * p.rep * D;
  const i32x4_t rs_q = rows_desc(p.q + (size_t)b * p.seq_q * p.ldq + head0, p.seq_q, (unsigned)p.ldq * 2u, (unsigned)p.rep * ROWB);
  const i32x4_t rs_do = rows_desc(p.dout + (size_t)b * p.seq_q * p.n_q * D + head0, p.seq_q, (unsigned)p.n_q * ROWB, (unsigned)p.rep * ROWB);
  const size_t stat0 = ((size_t)b * p.n_kv + kvh) * p.rows;
  const i32x4_t rs_l = rows_desc(p.lse + stat0, p.rows, 4u, 4u), rs_d = rows_desc(p.delta + stat0, p.rows, 4u, 4u);
  const int sV = 2 * STAGE + wave * WK * ROWB - half * ROWB;
  {
    const i32x4_t rs_v = rows_desc(p.v + base + (size_t)first_k * p.ldkv, min(n - first_k, WK), (unsigned)p.ldkv * 2u, ROWB);
#pragma unroll
    for (int j0 = 0; j0 < 2 * NLD; ++j0) {              // both groups read them: each loads its share
      const int j = j0 + grp * 2 * NLD, lr = H::RPL * j + lane / H::CH;
      OPTSTAGE_TILE_LOAD((unsigned)(lds0 + 2 * STAGE + wave * WK * ROWB + j * 1024), (unsigned)lr * (unsigned)p.ldkv * 2u + (unsigned)((lane % H::CH) ^ H::swz(lr)) * 16u, rs_v);
    }
  }
  // what a lane loads of a block lies where it lay in the block before, but for the same distance for all
  const RowBlocks rb = row_blocks(p);
  unsigned voff_q[NLD], voff_do[NLD];
#pragma unroll
  for (int j = 0; j < NLD; ++j) {
    const int lr = WROWS * id + H::RPL * j + lane / H::CH, hl = p.seq_q < 64 ? lr / p.seq_q : 0, t = lr - hl * p.seq_q;
    const unsigned at = (unsigned)hl * ROWB + (unsigned)((lane % H::CH) ^ H::swz(lr)) * 16u;
    voff_q[j] = hl < rb.heads ? (unsigned)t * (unsigned)p.ldq * 2u + at : PAST;
    voff_do[j] = hl < rb.heads ? (unsigned)t * (unsigned)p.n_q * ROWB + at : PAST;
  }
  const int per = (rb.all + p.splits - 1) / p.splits, it0 = min(rb.all, part * per), it1 = min(rb.all, it0 + per);
  auto issue_block = [&](int it, int stage) {
    const int head = p.seq_q < 64 ? it * rb.heads : it / rb.per_head, r0 = p.seq_q < 64 ? 0 : 64 * (it - head * rb.per_head);
    const unsigned oq = (unsigned)r0 * (unsigned)p.ldq * 2u + (unsigned)head * ROWB, od = ((unsigned)r0 * (unsigned)p.n_q + (unsigned)head) * ROWB;
    const unsigned dst = (unsigned)lds0 + stage * STAGE + (WROWS * id) * ROWB;
#pragma unroll
    for (int j = 0; j < NLD; ++j) {
      OPTSTAGE_TILE_LOAD(dst + j * 1024, voff_q[j] + oq, rs_q);
      OPTSTAGE_TILE_LOAD(dst + TILE + j * 1024, voff_do[j] + od, rs_do);
    }
    if (id < 2) {                                       // wave 0: lse of the block's rows, wave 1: -D; 0 where there is no row
      const bool on = p.seq_q < 64 ? lane < rb.heads * p.seq_q : r0 + lane < p.seq_q;
      const unsigned vo = on ? ((unsigned)head * (unsigned)p.seq_q + (unsigned)(r0 + lane)) * 4u : 0xFFFFFFF0u;
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds"
                   :: "s"((unsigned)lds0 + stage * STAGE + 2 * TILE + id * 256), "v"(vo), "s"(id == 0 ? rs_l : rs_d) : "memory", "m0");
    }
  };
  auto tr_frag = [&](int at, int dt, int u) { return transposed8(tr_addr[dt][0] + at + 16 * u * ROWB, tr_addr[dt][1] + at + (16 * u + 8) * ROWB); };
  auto rm_frag = [&](int at, int ks) { return *(const lds_bf16x8_t*)(unsigned)(rm_addr[ks] + at); };
#define OPTSTAGE_MFMA_V(acc, a, b) asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+v"(acc) : "v"(a), "v"(b))
#define OPTSTAGE_MFMA_0(acc, a, b) asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, 0" : "=&v"(acc) : "v"(a), "v"(b))
  auto block = [&](int it, int stage) __attribute__((always_inline)) {
    const int rows = p.seq_q < 64 ? rb.heads * p.seq_q : p.seq_q - 64 * (it % rb.per_head);
    if (half >= rows) return;                           // the same for the whole wave: no rows in this half of the block
    const int sQ = stage * STAGE, sDO = sQ + TILE, sL = sQ + 2 * TILE, sD = sL + 256;
    f32x16_t s, dp;                                     // lane = state, registers = rows half + 8 (v / 4) + 4 g + v % 4 of the block
    f32x4_t nL[4];
    bf16x8_t qf[2], df[2], vf[2];
    qf[0] = rm_frag(sQ, 0);
#pragma unroll
    for (int ks = 0; ks < NKS; ++ks) {                  // S = Q K^T
      OPTSTAGE_SB();
      if (ks < NKS - 1) {
        qf[(ks + 1) & 1] = rm_frag(sQ, ks + 1);
      } else {
        df[0] = rm_frag(sDO, 0);
        vf[0] = rm_frag(sV, 0);
        nL[0] = *(const lds_f32x4_t*)(unsigned)(row4 + sL);
      }
      if (ks >= NKS - 4) {                              // -D: the initial value of dP's accumulator
        const f32x4_t d4 = *(const lds_f32x4_t*)(unsigned)(row4 + sD + 8 * (ks - (NKS - 4)) * 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) dp[4 * (ks - (NKS - 4)) + i] = d4[i];
      }
      OPTSTAGE_SB();
      if (ks == 0) OPTSTAGE_MFMA_0(s, qf[0], Kf[0]);
      else OPTSTAGE_MFMA_V(s, qf[ks & 1], Kf[ks]);
      OPTSTAGE_SB();
    }
#pragma unroll
    for (int ks = 0; ks < NKS; ++ks) {                  // dP - D = dO V^T - D, the exponentials of S under its MFMAs
      OPTSTAGE_SB();
      if (ks < NKS - 1) {
        df[(ks + 1) & 1] = rm_frag(sDO, ks + 1);
        vf[(ks + 1) & 1] = rm_frag(sV, ks + 1);
      }
      constexpr int KL = NKS / 4;                       // lse of the next four rows one step ahead of its exponentials
      if (ks % KL == KL - 1 && ks / KL < 3) nL[ks / KL + 1] = *(const lds_f32x4_t*)(unsigned)(row4 + sL + 8 * (ks / KL + 1) * 4);
      OPTSTAGE_SB();
      OPTSTAGE_MFMA_V(dp, df[ks & 1], vf[ks & 1]);
      if (ks == 0) asm volatile("s_nop 7" ::: "memory"); // the exponentials read S a few cycles after the matrix unit has written it
      OPTSTAGE_SB();
#pragma unroll
      for (int e = 0; e < 16 / NKS; ++e) {
        const int v = (16 / NKS) * ks + e;
        s[v] = __builtin_amdgcn_exp2f(fmaf(s[v], c, nL[v >> 2][v & 3] * -LOG2E));
      }
    }
    OPTSTAGE_SB();
    bf16x8_t trf[2];                                    // dV^T += dO^T P, dS = P (dP - D) under its MFMAs
    trf[0] = tr_frag(sDO, 0, 0);
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const bf16x8_t pr = pack8(s, u);
#pragma unroll
      for (int dt = 0; dt < NDT; ++dt) {
        const int i = u * NDT + dt;
        OPTSTAGE_SB();
        if (i < 2 * NDT - 1) trf[(i + 1) & 1] = tr_frag(sDO, (dt + 1) % NDT, dt == NDT - 1 ? 1 : u);
        else trf[0] = tr_frag(sQ, 0, 0);
        OPTSTAGE_SB();
        accV[0][dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(trf[i & 1], pr, accV[0][dt], 0, 0, 0);
        OPTSTAGE_SB();
        if (i == 0) asm volatile("s_nop 15" ::: "memory");   // dP has left the matrix unit
#pragma unroll
        for (int e = 0; e < 8 / NDT; ++e) {
          const int v = (8 / NDT) * i + e;
          dp[v] = s[v] * dp[v];
        }
      }
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {                       // dK^T += Q^T dS
      const bf16x8_t d = pack8(dp, u);
#pragma unroll
      for (int dt = 0; dt < NDT; ++dt) {
        const int i = u * NDT + dt;
        OPTSTAGE_SB();
        if (i < 2 * NDT - 1) trf[(i + 1) & 1] = tr_frag(sQ, (dt + 1) % NDT, dt == NDT - 1 ? 1 : u);
        OPTSTAGE_SB();
        accK[0][dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(trf[i & 1], d, accK[0][dt], 0, 0, 0);
      }
    }
    OPTSTAGE_SB();
  };
#undef OPTSTAGE_MFMA_V
#undef OPTSTAGE_MFMA_0
  if (it0 < it1) issue_block(it0, 0);
  for (int it = it0; it < it1; it += 2) {
    OPTSTAGE_BLOCK_SYNC();
    if (it + 1 < it1) issue_block(it + 1, 1);
    block(it, 0);
    if (it + 1 < it1) {
      OPTSTAGE_BLOCK_SYNC();
      if (it + 2 < it1) issue_block(it + 2, 0);
      block(it + 1, 1);
    }
  }
  __syncthreads();
  if (grp == 1) meet_give<1, NDT>(smem, wave, lane, accV);
  __syncthreads();
  if (grp == 0) meet_take<1, NDT>(smem, wave, lane, accV);
  __syncthreads();
  if (grp == 1) meet_give<1, NDT>(smem, wave, lane, accK);
  __syncthreads();
  if (grp == 1) return;
  meet_take<1, NDT>(smem, wave, lane, accK);
  if (p.splits > 1 && it0 >= it1) return;               // the join counts the parts that have rows
  const int s = first_k + c32;
  if (s >= p.seq_kv) return;
  if (p.splits > 1) {
    if (s >= n) return;
    float* out = p.part + (((size_t)part * gridDim.y + b) * p.seq_kv + s) * p.n_kv * 2 * D + (size_t)kvh * 2 * D;
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        f32x4_t rk, rv;
#pragma unroll
        for (int i = 0; i < 4; ++i) { rk[i] = accK[0][dt][4 * j + i]; rv[i] = accV[0][dt][4 * j + i]; }
        *reinterpret_cast<f32x4_t*>(out + 32 * dt + 8 * j + 4 * g) = rk;
        *reinterpret_cast<f32x4_t*>(out + D + 32 * dt + 8 * j + 4 * g) = rv;
      }
    return;
  }
  bf16_t *krow = p.dk + base + (size_t)s * p.ldkv, *vrow = p.dv + base + (size_t)s * p.ldkv;
#pragma unroll
  for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      store4_if(krow + 32 * dt + 8 * j + 4 * g, accK[0][dt], 4 * j, scale, s < n && n > 1);
      store4_if(vrow + 32 * dt + 8 * j + 4 * g, accV[0][dt], 4 * j, 1.f, s < n);
    }
}

// dk and dv of a state and kv head from the parts' sums; a thread has 8 columns of one of them
template <typename T, int D> __global__ __launch_bounds__(256) void cross_dkv_join(const CrossArgsOf<T> p, size_t batch) {
  constexpr int Q = 2 * D / 8;
  const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x, per_part = batch * p.seq_kv * p.n_kv;
  if (i / Q >= per_part) return;
  const int col = (int)(i % Q) * 8 % D, is_v = (int)(i % Q) * 8 / D;
  const int h = i / Q % p.n_kv;
  const size_t row = i / Q / p.n_kv;
  const int s = row % p.seq_kv, n = cross_states(p, (int)(row / p.seq_kv));
  const int blocks = p.row_blocks, per = (blocks + p.splits - 1) / p.splits;
  float x[8] = {};
  if (s < n && (is_v || n > 1)) {
    for (int q = 0; q * per < blocks; ++q) {
      const f32x4_t* f = reinterpret_cast<const f32x4_t*>(p.part + q * per_part * 2 * D + i * 8);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] += f[e / 4][e % 4];
    }
  }
  store8((is_v ? p.dv : p.dk) + row * p.ldkv + (size_t)h * D + col, x, is_v ? 1.f : rsqrtf((float)D));
}
#undef OPTSTAGE_SB
#undef OPTSTAGE_TILE_LOAD
#undef OPTSTAGE_BLOCK_SYNC

// ---- how a call is divided -------------------------------------------------------------------------------------------------------------
struct CrossPlan { int waves, tiles, splits; };
constexpr int MOST_SPLITS = 64;                         // the join's lanes

// Forward and dQ: 32 rows to a wave; parts of the states where the workgroups are fewer than the chip holds.
//  * Two waves to a workgroup where that many tiles of 128 rows would be few: 8 heads x 300 queries and states 9.8 us, four waves 11.1; 8 x 512 x 4096 29.6 / 27.4;
//    one token of 32 / 8 heads over 16384 states 21.0 / 21.6 (one wave 22.4, eight 24).
//  * Up to 64 rows a workgroup waits for its blocks (1.1 us each) and the join costs 5 us and some 0.2 a part: about the root of twice the blocks.  One token of 32 / 8
//    heads, 16384 states (256 blocks): 1 part 272 us, 8 42, 16 26, 32 21, 64 27; 4 sequences of 16, 16 / 4 heads, 2000 states (32): 38, 8 14.4, 16 15.5.  Many sequences
//    need fewer, but of unequal length more than two workgroups to a compute unit: 16 x 8 heads, up to 16384 states 2 parts 155, 4 103, 8 83, 16 82 us.
//  * More rows are bound by the matrix unit: one workgroup per compute unit.  8 heads x 700 queries x 2000 states (48 tiles): 1 part 40, 4 24.3, 8 26.5.
CrossPlan plan_rows(const CrossShape& c) {
  const long rows = (long)(c.n_q / c.n_kv) * c.seq_q, groups = (long)c.n_kv * c.batch;
  CrossPlan p;
  p.waves = rows <= 64 || groups * ((rows + 127) / 128) <= 24 ? 2 : 4;
  p.tiles = (int)((rows + 32 * p.waves - 1) / (32 * p.waves));
  const long wgs = groups * p.tiles, blocks = (c.seq_kv + 63) / 64;
  long splits = 1;
  if (blocks >= 8 && wgs <= (rows <= 64 ? 384 : 128)) {
    splits = (rows <= 64 ? 1024 : 256) / wgs;
    const long root = (long)ceil(sqrt(2.0 * (double)blocks));
    splits = splits < root ? splits : root;
    splits = splits < MOST_SPLITS ? splits : MOST_SPLITS;
  }
  p.splits = splits < 1 ? 1 : (int)splits;
  return p;
}
// dK / dV: 128 states to a workgroup, one to a compute unit; parts of the rows (both kernels and the joins, us: 32 / 8 heads x 4096 x 1024, 64 workgroups: 1 part 488, 2 318,
// 4 257; 16 heads x 2 x 1024 x 577, 160: 55, 2 parts 76; 8 x 512 x 4096, 256: 58 / 83), of four blocks at least (forward and backward, of eight / four / two: 4 x 8 heads of 128
// x 1024 x 64 42.4 / 37.9 / 37.9, 8 x 3085 x 174 49.5 / 46.5 / 46.3, 8 x 300 x 2000 54.2 / 54.2 / 61.5, 16 of 64 x 700 x 700 51.2 / 52.8 / 52.8)
CrossPlan plan_states(const CrossShape& c) {
  const long groups = (long)c.n_kv * c.batch;
  CrossPlan p;
  p.waves = 8;
  p.tiles = (c.seq_kv + 127) / 128;
  const long wgs = groups * p.tiles, blocks = row_blocks(c.seq_q, c.n_q / c.n_kv).all;
  long splits = wgs >= 160 ? 1 : 256 / wgs;
  splits = splits < blocks / 4 ? splits : blocks / 4;
  p.splits = splits < 1 ? 1 : (int)splits;
  return p;
}

// the parts' sums stay below 256 MiB
constexpr uint64_t MOST_PARTS = 256ull << 20;
uint64_t rows_part_bytes(const CrossShape& c, int splits) { return splits > 1 ? 4ull * splits * c.batch * c.n_q * c.seq_q * (c.d + 2) : 0; }
uint64_t states_part_bytes(const CrossShape& c, int splits) { return splits > 1 ? 4ull * splits * c.batch * c.n_kv * c.seq_kv * 2 * c.d : 0; }
CrossPlan bounded(CrossPlan p, const CrossShape& c, uint64_t (*bytes)(const CrossShape&, int)) {
  while (p.splits > 1 && bytes(c, p.splits) > MOST_PARTS) --p.splits;
  return p;
}

size_t delta_floats(const CrossShape& c) { return ((size_t)c.batch * c.n_q * c.seq_q + 3) / 4 * 4; }

template <int D, int NW> hipError_t run_fwd(const CrossArgs& a, const CrossPlan& pl, int batch, hipStream_t s) {
  constexpr int smem = 4 * Head<D>::TILE;
  static LdsAttrOnce once;
  auto kern = cross_fwd_mfma<D, NW>;
  if (hipError_t e = once.ensure(reinterpret_cast<const void*>(kern), smem); e != hipSuccess) return e;
  hipLaunchKernelGGL(kern, dim3((unsigned)a.n_kv * pl.tiles * pl.splits, batch), dim3(64 * NW), smem, s, a);
  return hipGetLastError();
}
template <int D, int NW> hipError_t run_dq(const CrossArgs& a, const CrossPlan& pl, int batch, hipStream_t s) {
  constexpr int smem = 4 * Head<D>::TILE;
  static LdsAttrOnce once;
  auto kern = cross_dq_mfma<D, NW>;
  if (hipError_t e = once.ensure(reinterpret_cast<const void*>(kern), smem); e != hipSuccess) return e;
  hipLaunchKernelGGL(kern, dim3((unsigned)a.n_kv * pl.tiles * pl.splits, batch), dim3(64 * NW), smem, s, a);
  return hipGetLastError();
}
template <int D> hipError_t run_dkv(const CrossArgs& a, const CrossPlan& pl, int batch, hipStream_t s) {
  constexpr int smem = 2 * (2 * Head<D>::TILE + 512) + 2 * Head<D>::TILE;
  static LdsAttrOnce once;
  auto kern = cross_dkv_mfma<D>;
  if (hipError_t e = once.ensure(reinterpret_cast<const void*>(kern), smem); e != hipSuccess) return e;
  hipLaunchKernelGGL(kern, dim3((unsigned)a.n_kv * pl.tiles * pl.splits, batch), dim3(512), smem, s, a);
  return hipGetLastError();
}
unsigned joins(size_t items) { return (unsigned)((items + 255) / 256); }

template <int D> hipError_t cross_fwd_bf16(CrossArgs a, const CrossShape& c, hipStream_t s) {
  const CrossPlan pl = bounded(plan_rows(c), c, rows_part_bytes);
  a.splits = pl.splits;
  hipError_t e = pl.waves == 2 ? run_fwd<D, 2>(a, pl, c.batch, s) : run_fwd<D, 4>(a, pl, c.batch, s);
  if (e != hipSuccess || pl.splits == 1) return e;
  const size_t all = (size_t)c.batch * c.n_q * c.seq_q;
  hipLaunchKernelGGL((cross_fwd_join<bf16_t, D>), dim3((unsigned)((all + 3) / 4)), dim3(256), 0, s, a, all, 1.f / sqrtf((float)D));
  return hipGetLastError();
}
template <int D> hipError_t cross_bwd_bf16(CrossArgs a, const CrossShape& c, hipStream_t s) {
  CrossPlan pl = bounded(plan_rows(c), c, rows_part_bytes);
  a.splits = pl.splits;
  hipError_t e = pl.waves == 2 ? run_dq<D, 2>(a, pl, c.batch, s) : run_dq<D, 4>(a, pl, c.batch, s);
  if (e != hipSuccess) return e;
  if (pl.splits > 1) {
    const size_t all = (size_t)c.batch * c.n_q * c.seq_q;
    hipLaunchKernelGGL((cross_dq_join<bf16_t, D, 64>), dim3(joins(all * (D / 8))), dim3(256), 0, s, a, all);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  pl = bounded(plan_states(c), c, states_part_bytes);
  a.splits = pl.splits;
  e = run_dkv<D>(a, pl, c.batch, s);
  if (e != hipSuccess || pl.splits == 1) return e;
  hipLaunchKernelGGL((cross_dkv_join<bf16_t, D>), dim3(joins((size_t)c.batch * c.seq_kv * c.n_kv * (2 * D / 8))), dim3(256), 0, s, a, (size_t)c.batch);
  return hipGetLastError();
}

// ---- fp32 ------------------------------------------------------------------------------------------------------------------------------
// Scheme of attention_f32.hip: a workgroup has 16 rows (states, for dK / dV), its four waves take the other side's tiles of 16 in turn, and their sums meet
// in LDS.  Rows of a kv head and parts as above; states past the last one repeat it as keys, weigh nothing, and are zeros as values.
template <int D> struct Fp32 : F32<D> {
  typedef F32<D> F;
  // columns() of rows that end at `last`: zeros behind it
  static __device__ __forceinline__ void columns0(f32x4_t (&v)[4][F::H], const float* base, size_t ld, int first, int last, int g, int r) {
    F::columns(v, base, ld, first, last, g, r);
    if (first + 15 <= last) return;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (first + 4 * g + e > last)
#pragma unroll
        for (int h = 0; h < F::H; ++h) v[e][h] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }
};
struct RowAt { int head; size_t token; };              // of a kv head's heads; in all sequences
template <typename T> __device__ __forceinline__ RowAt row_at(const CrossArgsOf<T>& p, int b, int row) {
  const int head = p.by_seq_q.quotient(row);
  return {head, (size_t)b * p.seq_q + (row - head * p.seq_q)};
}

template <int D> __global__ __launch_bounds__(256) void cross_fwd_f32(const CrossArgsOf<float> p) {
  typedef Fp32<D> F;
  __shared__ __attribute__((aligned(16))) float part_sums[4][ROWS][D + 4];
  __shared__ float pm[4][ROWS], pl[4][ROWS];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, g = lane >> 4;
  const int kvh = blockIdx.x % p.n_kv, at_x = blockIdx.x / p.n_kv, tile = at_x / p.splits, part = at_x % p.splits, b = blockIdx.y;
  const int n = cross_states(p, b), tiles = (n + ROWS - 1) / ROWS, per = (tiles + p.splits - 1) / p.splits, t0 = min(tiles, part * per), t1 = min(tiles, t0 + per);
  const size_t all_rows = (size_t)gridDim.y * p.n_kv * p.rows, stat0 = ((size_t)b * p.n_kv + kvh) * p.rows;
  const size_t base = (size_t)b * p.seq_kv * p.ldkv + (size_t)kvh * D;
  f32x4_t q[F::S], acc[F::NT];
  {
    const RowAt at = row_at(p, b, min(tile * ROWS + r, p.rows - 1));
    F::rows(q, p.q + at.token * p.ldq + (size_t)(kvh * p.rep + at.head) * D, g);
  }
  F::scaled(q, rsqrtf((float)D));
  F::clear(acc);
  float m = LOWEST, l = 0.f;
  for (int t = t0 + wave; t < t1; t += 4) {
    f32x4_t k[F::S], v[4][F::H];
    F::rows(k, p.k + base + (size_t)min(ROWS * t + r, n - 1) * p.ldkv, g);
    F::columns0(v, p.v + base, p.ldkv, ROWS * t, n - 1, g, r);
    f32x4_t s = F::product(k, q);                       // s[e]: state 16 t + 4 g + e, row r
    if (ROWS * t + ROWS > n) {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (ROWS * t + 4 * g + e >= n) s[e] = -INFINITY;
    }
    const float mn = fmaxf(m, max_g(fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3]))));
    const float alpha = expf(m - mn);
    f32x4_t w;
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = expf(s[e] - mn);
    l = l * alpha + (w[0] + w[1]) + (w[2] + w[3]);      // this lane's states; summed over the four lanes at the end
#pragma unroll
    for (int i = 0; i < F::NT; ++i)
#pragma unroll
      for (int x = 0; x < 4; ++x) acc[i][x] *= alpha;
    F::accumulate(acc, v, w);
    m = mn;
  }
  l = sum_g(l);
  F::put(part_sums[wave], acc, g, r);
  if (g == 0) { pm[wave][r] = m; pl[wave][r] = l; }
  __syncthreads();
#pragma unroll
  for (int h = 0; h < F::H; ++h) {
    const int i = threadIdx.x + 256 * h, lr = i / (D / 4), c = (i % (D / 4)) * 4, row = tile * ROWS + lr;
    if (row >= p.rows) continue;
    const float M = fmaxf(fmaxf(pm[0][lr], pm[1][lr]), fmaxf(pm[2][lr], pm[3][lr]));
    float L = 0.f;
    f32x4_t v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float f = expf(pm[w][lr] - M);
      L += pl[w][lr] * f;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] += part_sums[w][lr][c + e] * f;
    }
    const size_t stat = stat0 + row;
    if (p.splits > 1) {
      if (t0 < t1) *reinterpret_cast<f32x4_t*>(p.part + ((size_t)part * all_rows + stat) * D + c) = v;
      if (c == 0) *reinterpret_cast<float2*>(p.part + (size_t)p.splits * all_rows * D + ((size_t)part * all_rows + stat) * 2) = t0 < t1 ? make_float2(M, L) : make_float2(-INFINITY, 0.f);
      continue;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = n ? v[e] / L : 0.f;
    const RowAt at = row_at(p, b, row);
    *reinterpret_cast<f32x4_t*>(p.o + (at.token * p.n_q + kvh * p.rep + at.head) * D + c) = v;
    if (c == 0) p.lse[stat] = n ? M + logf(L) : -INFINITY;
  }
}

// D of the row whose dO is in `dO`, o at `o`
template <int D> __device__ __forceinline__ float d_of_row(const f32x4_t (&dO)[Fp32<D>::S], const float* o, int g) {
  f32x4_t x[Fp32<D>::S];
  Fp32<D>::rows(x, o, g);
  float sum = 0.f;
#pragma unroll
  for (int s = 0; s < Fp32<D>::S; ++s)
#pragma unroll
    for (int e = 0; e < 4; ++e) sum = fmaf(dO[s][e], x[s][e], sum);
  return sum_g(sum);
}

template <int D> using PartSums = float[4][ROWS][D + 4];   // of a workgroup's waves
template <int D> __device__ __forceinline__ void dq_of_rows(const CrossArgsOf<float>& p, int at, PartSums<D>& part_sums) {
  typedef Fp32<D> F;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, g = lane >> 4;
  const int kvh = at % p.n_kv, at_x = at / p.n_kv, tile = at_x / p.splits, part = at_x % p.splits, b = blockIdx.y;
  const int n = cross_states(p, b), tiles = n == 1 ? 0 : (n + ROWS - 1) / ROWS, per = (tiles + p.splits - 1) / p.splits, t0 = min(tiles, part * per), t1 = min(tiles, t0 + per);
  const size_t base = (size_t)b * p.seq_kv * p.ldkv + (size_t)kvh * D, stat0 = ((size_t)b * p.n_kv + kvh) * p.rows;
  const float scale = rsqrtf((float)D);
  const int row_r = min(tile * ROWS + r, p.rows - 1);
  f32x4_t q[F::S], dO[F::S], acc[F::NT];
  float dsum = 0.f;
  {
    const RowAt at = row_at(p, b, row_r);
    const size_t col = (size_t)(kvh * p.rep + at.head) * D, o_at = at.token * p.n_q * D + col;
    F::rows(q, p.q + at.token * p.ldq + col, g);
    F::rows(dO, p.dout + o_at, g);
    dsum = d_of_row<D>(dO, p.o_in + o_at, g);
  }
  F::scaled(q, scale);
  F::clear(acc);
  const float L = p.lse[stat0 + row_r];
  if (part == 0 && wave == 0 && g == 0 && tile * ROWS + r < p.rows) p.delta[stat0 + row_r] = dsum;
  for (int t = t0 + wave; t < t1; t += 4) {
    f32x4_t k[F::S], v[F::S], kc[4][F::H];
    const size_t at = base + (size_t)min(ROWS * t + r, n - 1) * p.ldkv;
    F::rows(k, p.k + at, g);
    F::rows(v, p.v + at, g);
    F::columns0(kc, p.k + base, p.ldkv, ROWS * t, n - 1, g, r);
    const f32x4_t s = F::product(k, q), dp = F::product(v, dO);
    f32x4_t ds;
#pragma unroll
    for (int e = 0; e < 4; ++e) ds[e] = ROWS * t + 4 * g + e >= n ? 0.f : expf(s[e] - L) * (dp[e] - dsum);
    F::accumulate(acc, kc, ds);
  }
  F::put(part_sums[wave], acc, g, r);
  __syncthreads();
  if (p.splits > 1 && t0 >= t1) return;
#pragma unroll
  for (int h = 0; h < F::H; ++h) {
    const int i = threadIdx.x + 256 * h, lr = i / (D / 4), c = (i % (D / 4)) * 4, row = tile * ROWS + lr;
    if (row >= p.rows) continue;
    f32x4_t v;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = ((part_sums[0][lr][c + e] + part_sums[1][lr][c + e]) + part_sums[2][lr][c + e]) + part_sums[3][lr][c + e];
    if (p.splits > 1) {
      *reinterpret_cast<f32x4_t*>(p.part + ((size_t)part * gridDim.y * p.n_kv * p.rows + stat0 + row) * D + c) = v;
      continue;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] *= scale;
    const RowAt at = row_at(p, b, row);
    *reinterpret_cast<f32x4_t*>(p.dq + at.token * p.ldq + (size_t)(kvh * p.rep + at.head) * D + c) = v;
  }
}

// rows past the last one repeat it, weigh nothing and are zeros in the second products.  OWN_D: D of the rows is formed here, as dq_of_rows() does, instead of read
template <int D, bool OWN_D> __device__ __forceinline__ void dkv_of_states(const CrossArgsOf<float>& p, int at, PartSums<D>& part_sums) {
  typedef Fp32<D> F;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, g = lane >> 4;
  const int kvh = at % p.n_kv, at_x = at / p.n_kv, k0 = at_x / p.splits * ROWS, part = at_x % p.splits, b = blockIdx.y;
  const int n = cross_states(p, b), tiles = (p.rows + ROWS - 1) / ROWS, per = (tiles + p.splits - 1) / p.splits, t0 = min(tiles, part * per), t1 = min(tiles, t0 + per);
  const size_t base = (size_t)b * p.seq_kv * p.ldkv + (size_t)kvh * D, stat0 = ((size_t)b * p.n_kv + kvh) * p.rows;
  const float scale = rsqrtf((float)D);
  if (p.splits > 1 && (k0 >= n || t0 >= t1)) return;    // the join counts the parts that have rows, and writes zeros
  f32x4_t ak[F::NT], av[F::NT];
  F::clear(ak);
  F::clear(av);
  if (k0 < n) {
    f32x4_t k[F::S], v[F::S];
    const size_t at = base + (size_t)min(k0 + r, n - 1) * p.ldkv;
    F::rows(k, p.k + at, g);
    F::rows(v, p.v + at, g);
    F::scaled(k, scale);
    for (int t = t0 + wave; t < t1; t += 4) {
      const RowAt mine = row_at(p, b, min(ROWS * t + r, p.rows - 1));
      const size_t col = (size_t)(kvh * p.rep + mine.head) * D;
      f32x4_t q[F::S], dO[F::S], c[4][F::H], w, ds;
      F::rows(q, p.q + mine.token * p.ldq + col, g);
      F::rows(dO, p.dout + mine.token * p.n_q * D + col, g);
      float d_r = 0.f;
      if (OWN_D) d_r = d_of_row<D>(dO, p.o_in + mine.token * p.n_q * D + col, g);
      const f32x4_t s = F::product(q, k), dp = F::product(dO, v);   // [e]: row 16 t + 4 g + e, state k0 + r
      const float *qc[4], *gc[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int row = ROWS * t + 4 * g + e, rowc = min(row, p.rows - 1);
        const RowAt a = row_at(p, b, rowc);
        const size_t acol = (size_t)(kvh * p.rep + a.head) * D + 4 * r;
        qc[e] = p.q + a.token * p.ldq + acol;
        gc[e] = p.dout + a.token * p.n_q * D + acol;
        w[e] = row < p.rows ? expf(s[e] - p.lse[stat0 + rowc]) : 0.f;
        const float d = OWN_D ? __shfl(d_r, 4 * g + e, 64) : p.delta[stat0 + rowc];
        ds[e] = row < p.rows && n > 1 ? w[e] * (dp[e] - d) : 0.f;   // one state has no gradient of its score
      }
      const f32x4_t zero = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int h = 0; h < F::H; ++h) c[e][h] = ROWS * t + 4 * g + e < p.rows ? *reinterpret_cast<const f32x4_t*>(gc[e] + 64 * h) : zero;
      F::accumulate(av, c, w);
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int h = 0; h < F::H; ++h) c[e][h] = ROWS * t + 4 * g + e < p.rows ? *reinterpret_cast<const f32x4_t*>(qc[e] + 64 * h) : zero;
      F::accumulate(ak, c, ds);
    }
  }
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    if (which) __syncthreads();
    F::put(part_sums[wave], which ? av : ak, g, r);
    __syncthreads();
#pragma unroll
    for (int h = 0; h < F::H; ++h) {
      const int i = threadIdx.x + 256 * h, lr = i / (D / 4), c = (i % (D / 4)) * 4, s = k0 + lr;
      if (s >= p.seq_kv) continue;
      f32x4_t v;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = ((part_sums[0][lr][c + e] + part_sums[1][lr][c + e]) + part_sums[2][lr][c + e]) + part_sums[3][lr][c + e];
      if (p.splits > 1) {
        if (s < n) *reinterpret_cast<f32x4_t*>(p.part + ((((size_t)part * gridDim.y + b) * p.seq_kv + s) * p.n_kv + kvh) * 2 * D + which * D + c) = v;
        continue;
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = s >= n || (!which && n == 1) ? 0.f : which ? v[e] : v[e] * scale;
      *reinterpret_cast<f32x4_t*>((which ? p.dv : p.dk) + base + (size_t)s * p.ldkv + c) = v;
    }
  }
}

template <int D> __global__ __launch_bounds__(256) void cross_dq_f32(const CrossArgsOf<float> p) {
  __shared__ __attribute__((aligned(16))) PartSums<D> part_sums;
  dq_of_rows<D>(p, blockIdx.x, part_sums);
}
template <int D> __global__ __launch_bounds__(256) void cross_dkv_f32(const CrossArgsOf<float> p) {
  __shared__ __attribute__((aligned(16))) PartSums<D> part_sums;
  dkv_of_states<D, false>(p, blockIdx.x, part_sums);
}
// Both side by side in one launch, where neither is in parts: they are few workgroups then, and what a second launch costs is more than D twice (forward and backward,
// us: 4 heads of 64 x 128 x 77 20.7 -> 14.9, 8 of 128 x 200 x 200 47.5 -> 34.6, 2 x 16 of 64 x 240 x 240 46.5 -> 43.5, 4 x 8 of 64 x 100 x 250 38.5 either way)
template <int D> __global__ __launch_bounds__(256) void cross_bwd_f32(const CrossArgsOf<float> p, int dkv_groups) {
  __shared__ __attribute__((aligned(16))) PartSums<D> part_sums;
  if ((int)blockIdx.x < dkv_groups) dkv_of_states<D, true>(p, blockIdx.x, part_sums);
  else dq_of_rows<D>(p, blockIdx.x - dkv_groups, part_sums);
}

// Many rows (states): 16 to a wave, 64 to a workgroup, which read every tile of the other side from LDS, where its threads have put it (the next tile's loads
// are in flight meanwhile, two buffers); the kernels above read theirs from the caches, once per wave.  Which pays: wide_pays.
template <int D> struct Staged {
  static constexpr int LD = D + 4, H = D / 64;          // floats to a row in LDS: 16 rows' chunks fall on all banks
  f32x4_t v[H];
  // this thread's pieces of 16 rows: at(row) is where row 0 <= row < 16 starts, null for zeros
  template <typename F> __device__ __forceinline__ void load(F at) {
#pragma unroll
    for (int h = 0; h < H; ++h) {
      const int i = threadIdx.x + 256 * h, row = i / (D / 4), c = (i % (D / 4)) * 4;
      const float* p = at(row);
      v[h] = p ? *reinterpret_cast<const f32x4_t*>(p + c) : f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
  }
  __device__ __forceinline__ void put(float (*lds)[LD]) const {
#pragma unroll
    for (int h = 0; h < H; ++h) {
      const int i = threadIdx.x + 256 * h;
      *reinterpret_cast<f32x4_t*>(&lds[i / (D / 4)][(i % (D / 4)) * 4]) = v[h];
    }
  }
};
// four columns of a result row: 64 h + 16 g + 4 v
template <int NT> __device__ __forceinline__ f32x4_t result4(const f32x4_t (&acc)[NT], int h, int v) {
  return f32x4_t{acc[4 * h][v], acc[4 * h + 1][v], acc[4 * h + 2][v], acc[4 * h + 3][v]};
}

template <int D> __global__ __launch_bounds__(256) void cross_fwd_f32_wide(const CrossArgsOf<float> p) {
  typedef F32<D> F;
  constexpr int LD = Staged<D>::LD;
  __shared__ __attribute__((aligned(16))) float sK[2][ROWS][LD], sV[2][ROWS][LD];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, g = lane >> 4;
  const int kvh = blockIdx.x % p.n_kv, at_x = blockIdx.x / p.n_kv, tile = at_x / p.splits, part = at_x % p.splits, b = blockIdx.y;
  const int n = cross_states(p, b), tiles = (n + ROWS - 1) / ROWS, per = (tiles + p.splits - 1) / p.splits, t0 = min(tiles, part * per), t1 = min(tiles, t0 + per);
  const size_t all_rows = (size_t)gridDim.y * p.n_kv * p.rows, stat0 = ((size_t)b * p.n_kv + kvh) * p.rows;
  const size_t base = (size_t)b * p.seq_kv * p.ldkv + (size_t)kvh * D;
  const int row = 4 * ROWS * tile + ROWS * wave + r;
  const RowAt at = row_at(p, b, min(row, p.rows - 1));
  f32x4_t q[F::S], acc[F::NT];
  F::rows(q, p.q + at.token * p.ldq + (size_t)(kvh * p.rep + at.head) * D, g);
  F::scaled(q, rsqrtf((float)D));
  F::clear(acc);
  float m = LOWEST, l = 0.f;
  Staged<D> kn, vn;
  auto fetch = [&](int t) {
    kn.load([&](int i) { return ROWS * t + i < n ? p.k + base + (size_t)(ROWS * t + i) * p.ldkv : nullptr; });
    vn.load([&](int i) { return ROWS * t + i < n ? p.v + base + (size_t)(ROWS * t + i) * p.ldkv : nullptr; });
  };
  if (t0 < t1) {
    fetch(t0);
    kn.put(sK[0]);
    vn.put(sV[0]);
  }
  __syncthreads();
  for (int t = t0, buf = 0; t < t1; ++t, buf ^= 1) {
    if (t + 1 < t1) fetch(t + 1);
    f32x4_t k[F::S], v[4][F::H];
    F::rows(k, sK[buf][r], g);
    f32x4_t s = F::product(k, q);                       // s[e]: state 16 t + 4 g + e, row r
    F::columns(v, sV[buf][0], LD, 0, ROWS - 1, g, r);
    if (ROWS * t + ROWS > n) {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (ROWS * t + 4 * g + e >= n) s[e] = -INFINITY;
    }
    const float mn = fmaxf(m, max_g(fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3]))));
    const float alpha = expf(m - mn);
    f32x4_t w;
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = expf(s[e] - mn);
    l = l * alpha + (w[0] + w[1]) + (w[2] + w[3]);
#pragma unroll
    for (int i = 0; i < F::NT; ++i)
#pragma unroll
      for (int x = 0; x < 4; ++x) acc[i][x] *= alpha;
    F::accumulate(acc, v, w);
    m = mn;
    if (t + 1 < t1) {
      kn.put(sK[buf ^ 1]);
      vn.put(sV[buf ^ 1]);
    }
    __syncthreads();
  }
  l = sum_g(l);
  if (row >= p.rows) return;
  const size_t stat = stat0 + row;
  if (p.splits > 1) {
    if (g == 0) *reinterpret_cast<float2*>(p.part + (size_t)p.splits * all_rows * D + ((size_t)part * all_rows + stat) * 2) = t0 < t1 ? make_float2(m, l) : make_float2(-INFINITY, 0.f);
    if (t0 >= t1) return;
  }
  float* out = p.splits > 1 ? p.part + ((size_t)part * all_rows + stat) * D : p.o + (at.token * p.n_q + kvh * p.rep + at.head) * D;
  const float inv = p.splits > 1 ? 1.f : n ? 1.f / l : 0.f;
#pragma unroll
  for (int h = 0; h < F::H; ++h)
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      f32x4_t x = result4(acc, h, v);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] *= inv;
      *reinterpret_cast<f32x4_t*>(out + 64 * h + 16 * g + 4 * v) = x;
    }
  if (p.splits == 1 && g == 0) p.lse[stat] = n ? m + logf(l) : -INFINITY;
}

template <int D> __global__ __launch_bounds__(256) void cross_dq_f32_wide(const CrossArgsOf<float> p) {
  typedef F32<D> F;
  constexpr int LD = Staged<D>::LD;
  __shared__ __attribute__((aligned(16))) float sK[2][ROWS][LD], sV[2][ROWS][LD];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, g = lane >> 4;
  const int kvh = blockIdx.x % p.n_kv, at_x = blockIdx.x / p.n_kv, tile = at_x / p.splits, part = at_x % p.splits, b = blockIdx.y;
  const int n = cross_states(p, b), tiles = n == 1 ? 0 : (n + ROWS - 1) / ROWS, per = (tiles + p.splits - 1) / p.splits, t0 = min(tiles, part * per), t1 = min(tiles, t0 + per);
  const size_t base = (size_t)b * p.seq_kv * p.ldkv + (size_t)kvh * D, stat0 = ((size_t)b * p.n_kv + kvh) * p.rows;
  const float scale = rsqrtf((float)D);
  const int row = 4 * ROWS * tile + ROWS * wave + r, rowc = min(row, p.rows - 1);
  const RowAt at = row_at(p, b, rowc);
  const size_t col = (size_t)(kvh * p.rep + at.head) * D;
  f32x4_t q[F::S], dO[F::S], acc[F::NT];
  float dsum = 0.f;
  {
    f32x4_t x[F::S];
    F::rows(q, p.q + at.token * p.ldq + col, g);
    F::rows(dO, p.dout + at.token * p.n_q * D + col, g);
    F::rows(x, p.o_in + at.token * p.n_q * D + col, g);
#pragma unroll
    for (int s = 0; s < F::S; ++s)
#pragma unroll
      for (int e = 0; e < 4; ++e) dsum = fmaf(dO[s][e], x[s][e], dsum);
  }
  F::scaled(q, scale);
  F::clear(acc);
  dsum = sum_g(dsum);
  const float L = p.lse[stat0 + rowc];
  if (part == 0 && g == 0 && row < p.rows) p.delta[stat0 + row] = dsum;
  Staged<D> kn, vn;
  auto fetch = [&](int t) {
    kn.load([&](int i) { return ROWS * t + i < n ? p.k + base + (size_t)(ROWS * t + i) * p.ldkv : nullptr; });
    vn.load([&](int i) { return ROWS * t + i < n ? p.v + base + (size_t)(ROWS * t + i) * p.ldkv : nullptr; });
  };
  if (t0 < t1) {
    fetch(t0);
    kn.put(sK[0]);
    vn.put(sV[0]);
  }
  __syncthreads();
  for (int t = t0, buf = 0; t < t1; ++t, buf ^= 1) {
    if (t + 1 < t1) fetch(t + 1);
    f32x4_t x[F::S], kc[4][F::H], ds;
    F::rows(x, sK[buf][r], g);
    const f32x4_t s = F::product(x, q);
    F::rows(x, sV[buf][r], g);
    const f32x4_t dp = F::product(x, dO);
    F::columns(kc, sK[buf][0], LD, 0, ROWS - 1, g, r);
#pragma unroll
    for (int e = 0; e < 4; ++e) ds[e] = ROWS * t + 4 * g + e >= n ? 0.f : expf(s[e] - L) * (dp[e] - dsum);
    F::accumulate(acc, kc, ds);
    if (t + 1 < t1) {
      kn.put(sK[buf ^ 1]);
      vn.put(sV[buf ^ 1]);
    }
    __syncthreads();
  }
  if (row >= p.rows || (p.splits > 1 && t0 >= t1)) return;
  float* out = p.splits > 1 ? p.part + ((size_t)part * gridDim.y * p.n_kv * p.rows + stat0 + row) * D : p.dq + at.token * p.ldq + col;
  const float f = p.splits > 1 ? 1.f : scale;
#pragma unroll
  for (int h = 0; h < F::H; ++h)
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      f32x4_t x = result4(acc, h, v);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] *= f;
      *reinterpret_cast<f32x4_t*>(out + 64 * h + 16 * g + 4 * v) = x;
    }
}

// rows past the last one are zeros with lse and D zero: a weight of one times nothing
template <int D> __global__ __launch_bounds__(256) void cross_dkv_f32_wide(const CrossArgsOf<float> p) {
  typedef F32<D> F;
  constexpr int LD = Staged<D>::LD;
  __shared__ __attribute__((aligned(16))) float sQ[2][ROWS][LD], sG[2][ROWS][LD], sL[2][ROWS], sD[2][ROWS];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, g = lane >> 4;
  const int kvh = blockIdx.x % p.n_kv, at_x = blockIdx.x / p.n_kv, k0 = at_x / p.splits * 4 * ROWS, part = at_x % p.splits, b = blockIdx.y;
  const int n = cross_states(p, b), tiles = (p.rows + ROWS - 1) / ROWS, per = (tiles + p.splits - 1) / p.splits, t0 = min(tiles, part * per), t1 = min(tiles, t0 + per);
  const size_t base = (size_t)b * p.seq_kv * p.ldkv + (size_t)kvh * D, stat0 = ((size_t)b * p.n_kv + kvh) * p.rows;
  const float scale = rsqrtf((float)D);
  if (p.splits > 1 && (k0 >= n || t0 >= t1)) return;    // the join counts the parts that have rows, and writes zeros
  const int state = k0 + ROWS * wave + r;
  f32x4_t ak[F::NT], av[F::NT];
  F::clear(ak);
  F::clear(av);
  if (k0 < n) {
    f32x4_t k[F::S], v[F::S];
    const size_t at = base + (size_t)min(state, n - 1) * p.ldkv;
    F::rows(k, p.k + at, g);
    F::rows(v, p.v + at, g);
    F::scaled(k, scale);
    Staged<D> qn, gn;
    float ln = 0.f;
    auto fetch = [&](int t) {
      auto place = [&](int i, const float* x, size_t ld) {
        const int row = ROWS * t + i;
        if (row >= p.rows) return (const float*)nullptr;
        const RowAt a = row_at(p, b, row);
        return x + a.token * ld + (size_t)(kvh * p.rep + a.head) * D;
      };
      qn.load([&](int i) { return place(i, p.q, p.ldq); });
      gn.load([&](int i) { return place(i, p.dout, (size_t)p.n_q * D); });
      if (threadIdx.x < 2 * ROWS) {
        const int row = ROWS * t + (threadIdx.x & (ROWS - 1));
        ln = row < p.rows ? (threadIdx.x < ROWS ? p.lse : p.delta)[stat0 + row] : 0.f;
      }
    };
    auto put = [&](int buf) {
      qn.put(sQ[buf]);
      gn.put(sG[buf]);
      if (threadIdx.x < 2 * ROWS) (threadIdx.x < ROWS ? sL : sD)[buf][threadIdx.x & (ROWS - 1)] = ln;
    };
    if (t0 < t1) {
      fetch(t0);
      put(0);
    }
    __syncthreads();
    for (int t = t0, buf = 0; t < t1; ++t, buf ^= 1) {
      if (t + 1 < t1) fetch(t + 1);
      f32x4_t x[F::S], c[4][F::H], w, ds;
      F::rows(x, sQ[buf][r], g);
      const f32x4_t s = F::product(x, k);               // [e]: row 16 t + 4 g + e, state r
      F::rows(x, sG[buf][r], g);
      const f32x4_t dp = F::product(x, v);
      const f32x4_t L = *reinterpret_cast<const f32x4_t*>(&sL[buf][4 * g]), Dr = *reinterpret_cast<const f32x4_t*>(&sD[buf][4 * g]);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        w[e] = expf(s[e] - L[e]);
        ds[e] = n > 1 ? w[e] * (dp[e] - Dr[e]) : 0.f;   // one state has no gradient of its score
      }
      F::columns(c, sG[buf][0], LD, 0, ROWS - 1, g, r);
      F::accumulate(av, c, w);
      F::columns(c, sQ[buf][0], LD, 0, ROWS - 1, g, r);
      F::accumulate(ak, c, ds);
      if (t + 1 < t1) put(buf ^ 1);
      __syncthreads();
    }
  }
  if (state >= p.seq_kv || (p.splits > 1 && state >= n)) return;
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    float* out = p.splits > 1 ? p.part + ((((size_t)part * gridDim.y + b) * p.seq_kv + state) * p.n_kv + kvh) * 2 * D + which * D
                              : (which ? p.dv : p.dk) + base + (size_t)state * p.ldkv;
    const bool on = state < n && (which || n > 1);
    const float f = p.splits > 1 || which ? 1.f : scale;
#pragma unroll
    for (int h = 0; h < F::H; ++h)
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        f32x4_t x = which ? result4(av, h, v) : result4(ak, h, v);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = on ? x[e] * f : 0.f;
        *reinterpret_cast<f32x4_t*>(out + 64 * h + 16 * g + 4 * v) = x;
      }
  }
}

// 64 rows (states) to a workgroup (`waves` 4), or 16 whose waves divide the other side (1).  Forward and backward, us, 16 / 64: 16 heads of 64 x 512 x 512 (128 workgroups of 64)
// 84 / 97, 4 x 16 heads x 512 x 1024 508 / 411, 8 heads of 128 x 2048 x 2048 1017 / 773, 4 heads x 4096 x 4096 1984 / 1486; fewer workgroups but a long other side, 8 / 2
// heads x 2048 x 2048 (64 of states, 512 tiles of rows) 1022 / 801.
// Few rows (states) of many sequences and heads leave 64 mostly empty, while every workgroup reads the other side: up to 16 of them in the form of 16, where the other side is two
// tiles at least (less leaves its waves idle: 64 x 16 heads of 128 x 32 queries x 4 states 62 / 99), and up to 32 rows where it is eight.  Forward / backward: one token of 16 sequences, 32 / 8
// heads of 128 x 16384 states 332 / 1381 as 16, 784 / 1870 as 64; 32 rows x 4096 130 / 507, 206 / 539 (48 rows: 174 / 635, 208 / 586); 2000 queries x 16 heads x 16 sequences
// x 16 states 140 / 420, 140 / 512 (40 states: 197 / 860, 197 / 576).
bool wide_pays(long mine, long others, bool states, long groups) {
  if (mine <= 16 ? others >= 2 : !states && mine <= 32 && others >= 8) return false;
  const long wgs = groups * ((mine + 63) / 64);
  return wgs > 128 || (wgs >= 48 && others >= 128);
}
CrossPlan plan_f32(const CrossShape& c, bool states) {
  const long mine = states ? c.seq_kv : (long)(c.n_q / c.n_kv) * c.seq_q, others = ((states ? (long)(c.n_q / c.n_kv) * c.seq_q : c.seq_kv) + ROWS - 1) / ROWS;
  const long groups = (long)c.n_kv * c.batch;
  CrossPlan p;
  p.waves = wide_pays(mine, others, states, groups) ? 4 : 1;
  p.tiles = (int)((mine + ROWS * p.waves - 1) / (ROWS * p.waves));
  const long wgs = groups * p.tiles;
  long splits = p.waves == 4 ? (wgs >= 384 ? 1 : 512 / wgs) : (wgs >= 512 ? 1 : 1024 / wgs);
  splits = splits < others / 8 ? splits : others / 8;
  splits = splits < MOST_SPLITS ? splits : MOST_SPLITS;
  p.splits = splits < 1 ? 1 : (int)splits;
  return bounded(p, c, states ? states_part_bytes : rows_part_bytes);
}

template <int D> hipError_t cross_fwd_fp32(CrossArgsOf<float> a, const CrossShape& c, hipStream_t s) {
  const CrossPlan pl = plan_f32(c, false);
  a.splits = pl.splits;
  const dim3 grid((unsigned)a.n_kv * pl.tiles * pl.splits, c.batch);
  if (pl.waves == 4) hipLaunchKernelGGL(cross_fwd_f32_wide<D>, grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL(cross_fwd_f32<D>, grid, dim3(256), 0, s, a);
  if (pl.splits > 1) {
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    const size_t all = (size_t)c.batch * c.n_q * c.seq_q;
    hipLaunchKernelGGL((cross_fwd_join<float, D>), dim3((unsigned)((all + 3) / 4)), dim3(256), 0, s, a, all, 1.f);
  }
  return hipGetLastError();
}
template <int D> hipError_t cross_bwd_fp32(CrossArgsOf<float> a, const CrossShape& c, hipStream_t s) {
  CrossPlan pl = plan_f32(c, false);
  const CrossPlan of_states = plan_f32(c, true);
  a.splits = pl.splits;
  dim3 grid((unsigned)a.n_kv * pl.tiles * pl.splits, c.batch);
  if (pl.waves == 1 && of_states.waves == 1 && pl.splits == 1 && of_states.splits == 1) {
    const int dkv_groups = a.n_kv * of_states.tiles;
    grid.x += (unsigned)dkv_groups;
    hipLaunchKernelGGL(cross_bwd_f32<D>, grid, dim3(256), 0, s, a, dkv_groups);
    return hipGetLastError();
  }
  if (pl.waves == 4) hipLaunchKernelGGL(cross_dq_f32_wide<D>, grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL(cross_dq_f32<D>, grid, dim3(256), 0, s, a);
  if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  if (pl.splits > 1) {
    const size_t all = (size_t)c.batch * c.n_q * c.seq_q;
    hipLaunchKernelGGL((cross_dq_join<float, D, ROWS>), dim3(joins(all * (D / 8))), dim3(256), 0, s, a, all);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  pl = of_states;
  a.splits = pl.splits;
  a.row_blocks = (a.rows + ROWS - 1) / ROWS;
  grid.x = (unsigned)a.n_kv * pl.tiles * pl.splits;
  if (pl.waves == 4) hipLaunchKernelGGL(cross_dkv_f32_wide<D>, grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL(cross_dkv_f32<D>, grid, dim3(256), 0, s, a);
  if (pl.splits > 1) {
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    hipLaunchKernelGGL((cross_dkv_join<float, D>), dim3(joins((size_t)c.batch * c.seq_kv * c.n_kv * (2 * D / 8))), dim3(256), 0, s, a, (size_t)c.batch);
  }
  return hipGetLastError();
}

template <typename T> CrossArgsOf<T> cross_args(const CrossShape& c, const void* q, const void* k, const void* v, const int* kv_len, void* ws) {
  CrossArgsOf<T> a = {};
  a.q = (const T*)q; a.k = (const T*)k; a.v = (const T*)v; a.kv_len = kv_len;
  a.delta = (float*)ws; a.part = (float*)ws + delta_floats(c);
  a.ldq = c.ldq; a.ldkv = c.ldkv;
  a.seq_q = c.seq_q; a.seq_kv = c.seq_kv; a.n_q = c.n_q; a.n_kv = c.n_kv; a.rep = c.n_q / c.n_kv; a.rows = a.rep * c.seq_q; a.splits = 1;
  const RowBlocks rb = row_blocks(c.seq_q, a.rep);
  a.block_heads = rb.heads; a.blocks_per_head = rb.per_head; a.row_blocks = rb.all;
  a.by_seq_q = Divisor((unsigned)c.seq_q);
  return a;
}
template <typename T> CrossArgsOf<T> fwd_args(const CrossShape& c, const void* q, const void* k, const void* v, const int* kv_len, void* o, float* lse, void* ws) {
  CrossArgsOf<T> a = cross_args<T>(c, q, k, v, kv_len, ws);
  a.o = (T*)o; a.lse = lse;
  return a;
}
template <typename T> CrossArgsOf<T> bwd_args(const CrossShape& c, const void* q, const void* k, const void* v, const int* kv_len, const void* o, const void* dout,
                                              const float* lse, void* dq, void* dk, void* dv, void* ws) {
  CrossArgsOf<T> a = cross_args<T>(c, q, k, v, kv_len, ws);
  a.o_in = (const T*)o; a.dout = (const T*)dout; a.lse = const_cast<float*>(lse);
  a.dq = (T*)dq; a.dk = (T*)dk; a.dv = (T*)dv;
  return a;
}

}  // namespace

int cross_attn_form(int dtype, int states, int seq_q, int seq_kv, int batch, int n_q, int n_kv, int d) {
  const CrossShape c = {0, 0, seq_q, seq_kv, batch, n_q, n_kv, d};
  const CrossPlan p = dtype != DT_BF16 ? plan_f32(c, states != 0) : states ? bounded(plan_states(c), c, states_part_bytes) : bounded(plan_rows(c), c, rows_part_bytes);
  return 1000 * p.waves + p.splits;
}

// D of every row, and the parts' sums of whichever launch needs most
uint64_t cross_attn_ws_bytes(int dtype, int seq_q, int seq_kv, int batch, int n_q, int n_kv, int d) {
  const CrossShape c = {0, 0, seq_q, seq_kv, batch, n_q, n_kv, d};
  const CrossPlan by_rows = dtype == DT_BF16 ? bounded(plan_rows(c), c, rows_part_bytes) : plan_f32(c, false);
  const CrossPlan by_states = dtype == DT_BF16 ? bounded(plan_states(c), c, states_part_bytes) : plan_f32(c, true);
  const uint64_t r = rows_part_bytes(c, by_rows.splits), s = states_part_bytes(c, by_states.splits);
  return 4ull * delta_floats(c) + (r > s ? r : s);
}

hipError_t launch_cross_attn_fwd(int dtype, const CrossShape& c, const void* q, const void* k, const void* v, const int* kv_len, void* o, float* lse, void* ws, hipStream_t s) {
  if (dtype == DT_BF16) {
    const CrossArgs a = fwd_args<bf16_t>(c, q, k, v, kv_len, o, lse, ws);
    return c.d == 64 ? cross_fwd_bf16<64>(a, c, s) : cross_fwd_bf16<128>(a, c, s);
  }
  const CrossArgsOf<float> a = fwd_args<float>(c, q, k, v, kv_len, o, lse, ws);
  return c.d == 64 ? cross_fwd_fp32<64>(a, c, s) : cross_fwd_fp32<128>(a, c, s);
}
hipError_t launch_cross_attn_bwd(int dtype, const CrossShape& c, const void* q, const void* k, const void* v, const int* kv_len, const void* o, const void* dout,
                                 const float* lse, void* dq, void* dk, void* dv, void* ws, hipStream_t s) {
  if (dtype == DT_BF16) {
    const CrossArgs a = bwd_args<bf16_t>(c, q, k, v, kv_len, o, dout, lse, dq, dk, dv, ws);
    return c.d == 64 ? cross_bwd_bf16<64>(a, c, s) : cross_bwd_bf16<128>(a, c, s);
  }
  const CrossArgsOf<float> a = bwd_args<float>(c, q, k, v, kv_len, o, dout, lse, dq, dk, dv, ws);
  return c.d == 64 ? cross_bwd_fp32<64>(a, c, s) : cross_bwd_fp32<128>(a, c, s);
}
