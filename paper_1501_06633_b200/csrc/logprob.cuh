// Log probabilities of given tokens from a row of logits, with the row's entropy and its most likely tokens, and their
// gradient.
//
//   z = scale x,  m = max z,  S = sum exp(z - m),  T = sum exp(z - m) (z - m)
//   lse = m + ln S,  logprob = z_t - m - ln S,  entropy = ln S - T / S
//   dx_j = scale (dlp ([j = t] - p_j) - dH p_j (ln p_j + H)),  p_j = exp(z_j - lse)
//
// Forward.  A cluster of 1, 2, 4 or 8 CTAs has a row and reads it once: every thread keeps the running maximum of its
// values and the two sums relative to it (in 32 bits), which are joined by warp, CTA and cluster at the end.
// Differences to the maximum come first, so a term's error does not grow with the size of the logits.  The exponential takes
// numbers below 2^-126 for 0 (ex2.approx.ftz), forward and backward: one instruction for two, and such a term is below 2^-100 of a sum's
// last place; a gradient below that is 0 where elementary operations would leave a subnormal number.
//
// The largest values come from the same reading.  Groups of threads have 64 maxima between them; the k-th largest of
// those is a bound that at least k values reach, and hardly more than k do (a value above it is missed only by threads
// whose maximum is below it, and those have none).  The maxima of the threads' segments (up to
// 16 in each) tell where the values are that reach the bound; all threads read those few segments again and rank what they find by value
// and index.  Rows where more than
// kLpCandidates values do (many equal ones, as masks by the type's lowest value give) take the values above the bound
// and then the first equal ones in order; what still does not fit (large values at one residue of the thread's stride),
// and rows with NaN, take the largest one at a time.
//
// All loads are aligned: the values in front of the row's first multiple of 16 bytes, and behind its last, go to
// single threads.
//
// Bound by memory where there are rows for all SMs: 2048 x 131072 bf16 in 97 us without the largest values, 115 us with five
// (537 MB: 5.5 and 4.7 TB/s; the rereading and ranking at a row's end is hidden only by the other CTAs of the SM, of which
// there are six).  301 x 49999 fp32, one largest value: 18.5 us from memory, 15.2 where the second-level cache has the logits.  One
// row of 131072, eight CTAs: 5.0 us, with 20 largest values 9.7, all latency (loads, three levels of joins, a second reading).
// Backward: 2048 x 131072 bf16 168 to 177 us (1074 MB, 6.1 to 6.4 TB/s).  Packed both ways, 4096 x 32000 in 143 us, its 524 MB would
// take 80: latency (loads, barriers between the two packings) that half of an SM's warps do not hide, next to 24 instructions a
// value (IPC 0.61).
#pragma once
#include "fp8_util.cuh"
#include "umma_util.cuh"

namespace maxdnn {

constexpr int kLpThreads = 256;
constexpr int kLpBatch = 8;               // loads of 16 bytes that a thread has under way
constexpr int kLpSegments = 16;           // parts of a thread's values whose maxima are kept
constexpr int kLpBounds = 64;             // maxima that the bound is taken from
constexpr int kLpCandidates = 1024;
constexpr int kLpMaxTop = 32;
constexpr int kLpMaxCluster = 8;

struct LogprobArgs {
  const void *x, *target;
  float *logprob, *lse, *entropy, *top_logprob;
  int32_t* top_index;
  const float *dlogprob, *dentropy;      // bprop (lse and entropy are read there)
  void* dx;
  uint8_t *q_row, *s_row, *q_col, *s_col;
  int64_t ldx, ldd, ldq;
  int32_t rows, cols, top, wide_target;
  int32_t chunks;                        // bprop: CTAs of a row; packed: blocks of 128 columns
  float scale;
};

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
// A difference to the maximum in powers of two: below this its term is 0, and the product with it too.
constexpr float kLpFar = -1.0e4f;

__device__ __forceinline__ float lp_inf() { return __int_as_float(0x7F800000); }
__device__ __forceinline__ float exp2_fast(float v) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
  return r;
}

__device__ __forceinline__ int64_t lp_target(const LogprobArgs& a, int64_t row) {
  if (!a.target) return -1;
  const int64_t t = a.wide_target ? load_global(static_cast<const int64_t*>(a.target) + row)
                                  : (int64_t)load_global(static_cast<const int32_t*>(a.target) + row);
  return t >= 0 && t < a.cols ? t : -1;
}

// Running maximum (of x) with the sums relative to it; the second sum's differences in powers of two.
struct LpSums { float m, s, t; };

__device__ __forceinline__ float lp_far(float from, float to, float c) {       // from <= to
  return from == to ? 0.f : fmaxf((from - to) * c, kLpFar);
}
__device__ __forceinline__ void lp_raise(LpSums& a, float m, float c) {
  const float d = lp_far(a.m, m, c), f = exp2_fast(d);
  a.t = f * (a.t + a.s * d);
  a.s *= f;
  a.m = m;
}
__device__ __forceinline__ LpSums lp_join(LpSums a, LpSums b, float c) {
  const float m = fmaxf(a.m, b.m);
  lp_raise(a, m, c);
  lp_raise(b, m, c);
  return {m, a.s + b.s, a.t + b.t};
}

// Values as keys in rising order: equal values by falling index, NaN above all.
__device__ __forceinline__ uint64_t lp_key(float v, int64_t index) {
  const uint32_t b = __float_as_uint(v + 0.f);       // (-0 counts as 0)
  const uint32_t o = v != v ? 0xFFFFFFFFu : (b & 0x80000000u) ? ~b : b | 0x80000000u;
  return ((uint64_t)o << 32) | (0xFFFFFFFFu - (uint32_t)index);
}
__device__ __forceinline__ float lp_value(uint64_t key) {
  const uint32_t o = (uint32_t)(key >> 32);
  return __uint_as_float(o == 0xFFFFFFFFu ? 0x7FC00000u : (o & 0x80000000u) ? o & 0x7FFFFFFFu : ~o);
}
__device__ __forceinline__ uint32_t lp_index(uint64_t key) { return 0xFFFFFFFFu - (uint32_t)key; }

template <int XT>
struct LpVec {
  static constexpr int V = 16 / (int)sizeof(typename ElemOf<XT>::T);
  static __device__ __forceinline__ uint4 masked() {      // -inf throughout
    const uint32_t w = XT == MAXDNN_F32 ? 0xFF800000u : XT == MAXDNN_BF16 ? 0xFF80FF80u : 0xFC00FC00u;
    return make_uint4(w, w, w, w);
  }
  // The largest value (NaN do not count), without widening 16-bit ones.
  static __device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) {
    uint32_t r;
    if constexpr (XT == MAXDNN_BF16) asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    else if constexpr (XT == MAXDNN_F16) asm("max.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    else r = __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b)));
    return r;
  }
  static __device__ __forceinline__ float most(uint32_t w) {
    if constexpr (XT == MAXDNN_F32) {
      return fmaxf(__uint_as_float(w), -__int_as_float(0x7F800000));
    } else {
      const uint32_t both = larger(larger(w, (w >> 16) | (w << 16)), masked().x);      // (a NaN alone: -inf)
      if constexpr (XT == MAXDNN_BF16) return __uint_as_float(both << 16);
      else return __half2float(__ushort_as_half((unsigned short)both));
    }
  }
  static __device__ __forceinline__ float most(uint4 w) { return most(larger(larger(w.x, w.y), larger(w.z, w.w))); }
  template <int N>
  static __device__ __forceinline__ float most(const uint4 (&w)[N]) {
    uint32_t r = larger(larger(w[0].x, w[0].y), larger(w[0].z, w[0].w));
#pragma unroll
    for (int i = 1; i < N; ++i) r = larger(r, larger(larger(w[i].x, w[i].y), larger(w[i].z, w[i].w)));
    return most(r);
  }
  static __device__ __forceinline__ void pairs(uint4 w, F2 (&p)[V / 2]) {
    if constexpr (XT == MAXDNN_F32) {
      p[0] = ((F2)w.y << 32) | w.x;
      p[1] = ((F2)w.w << 32) | w.z;
    } else {
      Raw8<XT> r;
      r.a = w;
      to_pairs<XT>(r, p);
    }
  }
};
template <int XT>
__device__ __forceinline__ float lp_one(const typename ElemOf<XT>::T* p) {
  if constexpr (XT == MAXDNN_F32) return *p;
  else if constexpr (XT == MAXDNN_BF16) return __bfloat162float(*p);
  else return __half2float(*p);
}

template <int N> struct LpCount { static constexpr int value = N; };

// What a CTA shows the others of its cluster.
struct LpShared {
  LpSums sums;
  int32_t count;                           // of `best`
  uint64_t best[kLpMaxTop];                // falling
};

// A CTA's part of a row: single values in front and behind, and vectors of 16 bytes between them.
template <int XT>
struct LpPart {
  const typename ElemOf<XT>::T* row;
  int64_t head;                            // column of the row's first vector
  int32_t v0, v1;                          // this CTA's vectors
  int64_t c0, c1;                          // this CTA's columns
  int64_t extra;                           // this thread's single column, or -1
  int32_t segments, segment_vecs;          // a thread's vectors in so many segments of so many (whole batches)
};

template <int XT, int THREADS>
__device__ __forceinline__ LpPart<XT> lp_part(const void* x, int64_t first, int64_t cols, int rank, int parts, int t) {
  typedef typename ElemOf<XT>::T T;
  constexpr int V = LpVec<XT>::V;
  LpPart<XT> p;
  p.row = static_cast<const T*>(x) + first;
  const int64_t off = (int64_t)(((16u - ((uint32_t)reinterpret_cast<uintptr_t>(p.row) & 15u)) & 15u) / sizeof(T));
  p.head = off < cols ? off : cols;
  const int64_t nv = (cols - p.head) / V, tail = cols - p.head - nv * V;
  p.v0 = (int32_t)(nv * rank / parts);
  p.v1 = (int32_t)(nv * (rank + 1) / parts);
  p.c0 = rank == 0 ? 0 : p.head + (int64_t)p.v0 * V;
  p.c1 = rank == parts - 1 ? cols : p.head + (int64_t)p.v1 * V;
  const int batches = (p.v1 - p.v0 + THREADS * kLpBatch - 1) / (THREADS * kLpBatch);
  const int per_segment = (batches + kLpSegments - 1) / kLpSegments;
  p.segment_vecs = kLpBatch * per_segment;
  p.segments = batches == 0 ? 0 : (batches + per_segment - 1) / per_segment;
  p.extra = -1;
  if (rank == 0 && t < p.head) p.extra = t;
  if (rank == parts - 1 && t >= 32 && t - 32 < tail) p.extra = cols - tail + t - 32;
  return p;
}

__device__ __forceinline__ uint64_t lp_max_key(uint64_t k) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) {
    const uint64_t o = __shfl_xor_sync(0xFFFFFFFFu, k, d);
    k = o > k ? o : k;
  }
  return k;
}

template <int THREADS>
struct LpScratch {
  uint64_t keys[kLpCandidates];
  float segment[kLpSegments][THREADS];          // maxima of the threads' segments
  uint16_t again[kLpSegments * THREADS];        // segments that are read again
  float bounds[kLpBounds];
  float bound;
  int32_t count, n_again;
  int32_t per_warp[THREADS / 32];
  uint64_t warp_key[THREADS / 32];
};

// The part's values that reach `bound` (STRICT: exceed it), as keys in no particular order; returns how many.
template <int XT, int THREADS, bool STRICT>
__device__ __forceinline__ int lp_collect(const LpPart<XT>& p, float mine, float bound, LpScratch<THREADS>* w, int t) {
  constexpr int V = LpVec<XT>::V, U = 4;
  auto reaches = [&](float v) { return (STRICT ? v > bound : v >= bound) && v > -lp_inf(); };
  auto push = [&](float v, int64_t c) {
    const int at = atomicAdd(&w->count, 1);
    if (at < kLpCandidates) w->keys[at] = lp_key(v, c);
  };
  if (p.extra >= 0) {
    const float v = lp_one<XT>(p.row + p.extra);
    if (reaches(v)) push(v, p.extra);
  }
  // the segments of threads whose maximum reaches it
  if (reaches(mine))
    for (int s = 0; s < p.segments; ++s)
      if (reaches(w->segment[s][t])) w->again[atomicAdd(&w->n_again, 1)] = (uint16_t)(s * THREADS + t);
  __syncthreads();
  // their vectors, shared by all threads, U loads of each under way
  const int each = p.segment_vecs, all = w->n_again * each;
  for (int i0 = t; i0 < all; i0 += THREADS * U) {
    if (*reinterpret_cast<volatile int32_t*>(&w->count) > kLpCandidates) break;      // (it will be taken another way)
    uint4 raw[U];
    int64_t at[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + THREADS * u;
      at[u] = p.v1;
      if (i < all) {
        const int which = w->again[i / each];
        at[u] = (int64_t)p.v0 + which % THREADS + (int64_t)THREADS * (which / THREADS * each + i % each);
      }
      raw[u] = at[u] < p.v1 ? *reinterpret_cast<const uint4*>(p.row + p.head + at[u] * V) : LpVec<XT>::masked();
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (!reaches(LpVec<XT>::most(raw[u]))) continue;
      F2 q[V / 2];
      LpVec<XT>::pairs(raw[u], q);
      const int64_t c = p.head + at[u] * V;
#pragma unroll
      for (int k = 0; k < V / 2; ++k) {
        const float2 v = unf2(q[k]);
        if (reaches(v.x)) push(v.x, c + 2 * k);
        if (reaches(v.y)) push(v.y, c + 2 * k + 1);
      }
    }
  }
  __syncthreads();
  return w->count;
}

// The first `need` values equal to `bound` in the order of their columns, behind `have` keys; returns how many keys there are.
template <int XT, int THREADS>
__device__ __noinline__ int lp_first_equal(const LpPart<XT>& p, float bound, int have, int need, LpScratch<THREADS>* w, int t) {
  const int lane = t & 31, warp = t >> 5;
  int found = 0;
  for (int64_t c = p.c0; c < p.c1 && found < need; c += THREADS) {
    const bool hit = c + t < p.c1 && lp_one<XT>(p.row + c + t) == bound;
    const uint32_t hits = __ballot_sync(0xFFFFFFFFu, hit);
    if (lane == 0) w->per_warp[warp] = __popc(hits);
    __syncthreads();
    int at = found, all = 0;
    for (int i = 0; i < THREADS / 32; ++i) {
      at += i < warp ? w->per_warp[i] : 0;
      all += w->per_warp[i];
    }
    at += __popc(hits & ((1u << lane) - 1u));
    if (hit && at < need) w->keys[have + at] = lp_key(bound, c + t);
    found += all;
    __syncthreads();
  }
  return have + (found < need ? found : need);
}

// The `top` largest values one after the other; returns how many there are.
template <int XT, int THREADS>
__device__ __noinline__ int lp_one_by_one(const LpPart<XT>& p, int top, LpScratch<THREADS>* w, int t) {
  const int lane = t & 31, warp = t >> 5;
  uint64_t last = ~0ull;
  int n = 0;
  for (; n < top; ++n) {
    uint64_t best = 0;
    for (int64_t c = p.c0 + t; c < p.c1; c += THREADS) {
      const float v = lp_one<XT>(p.row + c);
      const uint64_t k = v == -lp_inf() ? 0 : lp_key(v, c);
      if ((n == 0 || k < last) && k > best) best = k;
    }
    best = lp_max_key(best);
    if (lane == 0) w->warp_key[warp] = best;
    __syncthreads();
    for (int i = 0; i < THREADS / 32; ++i) best = w->warp_key[i] > best ? w->warp_key[i] : best;
    __syncthreads();
    if (best == 0) break;
    if (t == 0) w->keys[n] = best;
    last = best;
  }
  __syncthreads();
  return n;
}

// The part's `top` largest values in falling order into sh->best.
template <int XT, int THREADS>
__device__ __forceinline__ void lp_largest(const LpPart<XT>& p, float mine, bool strange, int top, LpScratch<THREADS>* w, LpShared* sh, int t) {
  constexpr int kEach = THREADS / kLpBounds;
  float m = mine;
#pragma unroll
  for (int d = 1; d < kEach; d <<= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, d));
  if (t % kEach == 0) w->bounds[t / kEach] = m;
  if (t == 0) w->count = w->n_again = 0;
  const bool nan = __syncthreads_or(strange) != 0;
  int n;
  if (!nan) {
    if (t < kLpBounds) {
      const float v = w->bounds[t];
      int rank = 0;
#pragma unroll 8
      for (int i = 0; i < kLpBounds; i += 4) {
        const float4 o = *reinterpret_cast<const float4*>(&w->bounds[i]);
        rank += (o.x > v || (o.x == v && i < t)) + (o.y > v || (o.y == v && i + 1 < t)) + (o.z > v || (o.z == v && i + 2 < t)) +
                (o.w > v || (o.w == v && i + 3 < t));
      }
      if (rank == top - 1) w->bound = v;
    }
    __syncthreads();
    const float bound = w->bound;
    n = lp_collect<XT, THREADS, false>(p, mine, bound, w, t);
    if (n > kLpCandidates) {
      __syncthreads();
      if (t == 0) w->count = w->n_again = 0;
      __syncthreads();
      n = lp_collect<XT, THREADS, true>(p, mine, bound, w, t);
      if (n < top) n = lp_first_equal<XT, THREADS>(p, bound, n, top - n, w, t);
    }
    __syncthreads();
  }
  if (nan || n > kLpCandidates) n = lp_one_by_one<XT, THREADS>(p, top, w, t);
  for (int i = t; i < n; i += THREADS) {
    const uint64_t k = w->keys[i];
    int rank = 0;
#pragma unroll 8
    for (int j = 0; j < n; ++j) rank += w->keys[j] > k;
    if (rank < top) sh->best[rank] = k;
  }
  if (t == 0) sh->count = n < top ? n : top;
}

template <int XT, bool ENTROPY, int THREADS>
__global__ void __launch_bounds__(THREADS, 768 / THREADS) logprob_fprop_kernel(const __grid_constant__ LogprobArgs args) {
  let_next_start();
  wait_for_previous();
  constexpr int V = LpVec<XT>::V, U = kLpBatch;
  __shared__ LpShared shared;
  __shared__ __align__(16) LpScratch<THREADS> scratch;
  __shared__ LpSums per_warp[THREADS / 32];
  __shared__ uint64_t merged[kLpMaxTop];
  const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
  const int rank = (int)cluster_ctarank();
  uint32_t parts;
  asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(parts));
  const int64_t r = blockIdx.x / parts;
  const LpPart<XT> p = lp_part<XT, THREADS>(args.x, r * args.ldx, args.cols, rank, (int)parts, t);
  const float c = args.scale * kLog2e;
  LpSums sum = {-lp_inf(), 0.f, 0.f};
  float single = -lp_inf(), given = 0.f;
  int64_t token = -1;
  if (p.extra >= 0) single = lp_one<XT>(p.row + p.extra);
  if (t == 32 && rank == 0 && args.logprob) {
    token = lp_target(args, r);
    if (token >= 0) given = lp_one<XT>(p.row + token);
  }
  const uint4* vec = reinterpret_cast<const uint4*>(p.row + p.head);
  // Some vectors: their maximum first
  auto take = [&](auto& raw) {
    constexpr int N = sizeof(raw) / sizeof(uint4);
    const float most = LpVec<XT>::most(raw);
    if (most > sum.m) lp_raise(sum, most, c);
    if (sum.m == -lp_inf()) {      // nothing above -inf so far: a NaN still has to show
#pragma unroll
      for (int u = 0; u < N; ++u) {
        F2 x[V / 2];
        LpVec<XT>::pairs(raw[u], x);
#pragma unroll
        for (int i = 0; i < V / 2; ++i) {
          const float2 w = unf2(x[i]);
          if (w.x != w.x || w.y != w.y) sum.s = w.x + w.y;
        }
      }
      return most;
    }
    const F2 mm = f2(-sum.m), cc = f2(c);
    F2 s = 0, tt = 0;
#pragma unroll
    for (int u = 0; u < N; ++u) {
      F2 x[V / 2];
      LpVec<XT>::pairs(raw[u], x);
#pragma unroll
      for (int i = 0; i < V / 2; ++i) {
        const F2 d = mul2(add2(x[i], mm), cc);
        const float2 w = unf2(d);
        const F2 e = f2(exp2_fast(w.x), exp2_fast(w.y));
        s = add2(s, e);
        if (ENTROPY) tt = fma2(e, f2(fmaxf(w.x, kLpFar), fmaxf(w.y, kLpFar)), tt);
      }
    }
    sum.s += sum2(s);
    if (ENTROPY) sum.t += sum2(tt);
    return most;
  };
  // (a segment is several batches; its maximum is kept for the search of the largest values)
  int64_t v = (int64_t)p.v0 + t;
  for (int segment = 0; segment < p.segments; ++segment) {
    float top_here = -lp_inf();
#pragma unroll 1
    for (int i = 0; i < p.segment_vecs; i += U, v += U * THREADS) {
      const int64_t left = p.v1 - (v - t);          // vectors of the CTA
      if (left >= U * THREADS) {
        uint4 raw[U];
#pragma unroll
        for (int u = 0; u < U; ++u) raw[u] = load_global(vec + v + u * THREADS);
        top_here = fmaxf(top_here, take(raw));
        continue;
      }
      // the last ones, with no more of them masked than there are
      auto some = [&](auto count) {
        constexpr int N = decltype(count)::value;
        uint4 raw[N];
#pragma unroll
        for (int u = 0; u < N; ++u) raw[u] = v + u * THREADS < p.v1 ? load_global(vec + v + u * THREADS) : LpVec<XT>::masked();
        top_here = fmaxf(top_here, take(raw));
      };
      if (left > U / 2 * THREADS) some(LpCount<U>());
      else if (left > U / 4 * THREADS) some(LpCount<U / 2>());
      else if (left > U / 8 * THREADS) some(LpCount<U / 4>());
      else if (left > 0) some(LpCount<U / 8>());
      else break;
    }
    if (args.top) scratch.segment[segment][t] = top_here;
  }
  if (p.extra >= 0) {
    const LpSums one = {single == single ? single : -lp_inf(), single != single ? single : single == -lp_inf() ? 0.f : 1.f, 0.f};
    sum = lp_join(sum, one, c);
  }
  const float mine = sum.m;
  // (+inf shows as a NaN of the sum, except where it is a thread's single value)
  const bool strange = sum.s != sum.s || sum.m == lp_inf();
  if (strange) sum.s = __int_as_float(0x7FC00000);
  // the warp's, the CTA's
  float wm = sum.m;
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) wm = fmaxf(wm, __shfl_xor_sync(0xFFFFFFFFu, wm, d));
  lp_raise(sum, wm, c);
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) {
    sum.s += __shfl_xor_sync(0xFFFFFFFFu, sum.s, d);
    sum.t += __shfl_xor_sync(0xFFFFFFFFu, sum.t, d);
  }
  if (lane == 0) per_warp[warp] = sum;
  if (args.top) lp_largest<XT, THREADS>(p, mine, strange, args.top, &scratch, &shared, t);
  __syncthreads();
  if (warp == 0) {
    LpSums all = per_warp[lane % (THREADS / 32)];
#pragma unroll
    for (int d = THREADS / 64; d > 0; d >>= 1) {
      const LpSums other = {__shfl_xor_sync(0xFFFFFFFFu, all.m, d), __shfl_xor_sync(0xFFFFFFFFu, all.s, d), __shfl_xor_sync(0xFFFFFFFFu, all.t, d)};
      all = lp_join(all, other, c);
    }
    if (lane == 0) shared.sums = all;
  }
  if (parts > 1) {
    cluster_arrive();      // (release and acquire: the CTAs' results are visible)
    cluster_wait();
  } else {
    __syncthreads();
  }
  if (rank == 0) {
    auto peer = [&](const void* at, uint32_t who) { return parts > 1 ? map_to_cta(smem_u32(at), who) : smem_u32(at); };
    auto f32 = [](uint32_t at) { float f; asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(f) : "r"(at) : "memory"); return f; };
    LpSums all = shared.sums;
    for (uint32_t i = 1; i < parts; ++i) {
      const uint32_t at = peer(&shared.sums, i);
      const LpSums other = {f32(at), f32(at + 4), f32(at + 8)};
      all = lp_join(all, other, c);
    }
    const bool nothing = all.m == -lp_inf() && all.s == 0.f;
    const float ln_s = logf(all.s);
    auto logp = [&](float value) { return nothing ? -lp_inf() : (value - all.m) * args.scale - ln_s; };
    if (args.top) {
      // candidates of all CTAs: place i is number i % top of CTA i / top
      uint64_t* keys = scratch.keys;
      if (t < kLpMaxTop) merged[t] = parts == 1 && t < shared.count ? shared.best[t] : 0;
      if (parts > 1) __syncthreads();
      for (int i = t; parts > 1 && i < (int)parts * args.top; i += THREADS) {
        const uint32_t who = (uint32_t)(i / args.top), in = (uint32_t)(i % args.top);
        uint32_t count;
        asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(count) : "r"(peer(&shared.count, who)) : "memory");
        uint64_t k = 0;
        if (in < count) asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(k) : "r"(peer(&shared.best[in], who)) : "memory");
        keys[i] = k;
      }
      __syncthreads();
      for (int i = t; parts > 1 && i < (int)parts * args.top; i += THREADS) {
        const uint64_t k = keys[i];
        if (k == 0) continue;
        int at = 0;
#pragma unroll 8
        for (int j = 0; j < (int)parts * args.top; ++j) at += keys[j] > k;
        if (at < args.top) merged[at] = k;
      }
      __syncthreads();
      if (t < args.top) {
        const uint64_t k = merged[t];
        const float absent = all.s != all.s ? all.s : -lp_inf();
        if (args.top_logprob) args.top_logprob[r * args.top + t] = k ? logp(lp_value(k)) : absent;
        if (args.top_index) args.top_index[r * args.top + t] = k ? (int32_t)lp_index(k) : -1;
      }
    }
    if (t == 0) {
      if (args.lse) args.lse[r] = nothing ? -lp_inf() : all.m * args.scale + ln_s;
      if (ENTROPY && args.entropy) args.entropy[r] = nothing ? 0.f : ln_s - kLn2 * (all.t / all.s);
    }
    if (t == 32 && args.logprob) args.logprob[r] = token < 0 ? 0.f : logp(given);
  }
  if (parts > 1) {
    cluster_arrive();      // no CTA leaves while its results are read
    cluster_wait();
  }
}

// ---- backward ----
// What a row's values are turned into gradients with: g = p (a + d ln p); add: scale dlp.
struct __align__(16) LpRow { float minus_lse, a, d, add; };

__device__ __forceinline__ LpRow lp_row(const LogprobArgs& args, int64_t r, int32_t* target) {
  LpRow w;
  const float lse = load_global(args.lse + r);
  const int64_t at = lp_target(args, r);
  const float dlp = args.dlogprob && at >= 0 ? load_global(args.dlogprob + r) : 0.f;
  const float dh = args.dentropy ? load_global(args.dentropy + r) : 0.f;
  const float h = args.dentropy ? load_global(args.entropy + r) : 0.f;
  // a row of which nothing is left: no p at all
  const bool nothing = lse == -lp_inf();
  w.minus_lse = nothing ? -lp_inf() : -lse;
  w.a = nothing ? 0.f : -args.scale * (dlp + dh * h);
  w.d = nothing ? 0.f : -args.scale * dh;
  w.add = nothing ? 0.f : args.scale * dlp;
  *target = nothing ? -1 : (int32_t)at;
  return w;
}

// The larger of two values; NaN stay.
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
// Gradients of a pair of logits.  EXACT: what the power's rounding to 32 bits left of ln p, up to 2^-20 of p, goes to p (not to the
// other factor, which may be infinite).  In front of a rounding to 16 bits it would cost 174 -> 189 us at 2048 x 131072 for nothing;
// packed values, where it moves roundings and blocks' powers of two, and 32-bit ones have it (4096 x 32000 packed 139 -> 143 us).
template <bool EXACT>
__device__ __forceinline__ F2 lp_grad2(F2 x, F2 scale, F2 minus_lse, F2 a, F2 d) {
  const float2 l = unf2(fma2(x, scale, minus_lse));
  const F2 lnp = f2(max_nan(l.x, kLpFar), max_nan(l.y, kLpFar));
  const F2 power = mul2(lnp, f2(kLog2e));
  const float2 e = unf2(power);
  F2 p = f2(exp2_fast(e.x), exp2_fast(e.y));
  if (EXACT) p = fma2(p, fma2(power, f2(-kLn2), lnp), p);
  return mul2(p, fma2(d, lnp, a));
}
// The gradient at the target, from its logit: 1 - p as -(exp(ln p) - 1), which loses nothing where p is near 1 (the difference of
// p from 1 would have p's error, 2^-22, instead of its own).
__device__ __forceinline__ float lp_target_grad(const LogprobArgs& args, const LpRow& w, int64_t row, float x) {
  const float lnp = max_nan(fmaf(x, args.scale, w.minus_lse), kLpFar);
  const float dh = args.dentropy ? load_global(args.dentropy + row) : 0.f;
  const float h = args.dentropy ? load_global(args.entropy + row) : 0.f;
  return fmaf(-w.add, expm1f(lnp), -args.scale * dh * expf(lnp) * (lnp + h));
}
// `value` in the place of the target's gradient among eight columns from c on.
__device__ __forceinline__ void lp_set_target(F2 (&v)[4], float value, int32_t target, int32_t c) {
  const uint32_t in = (uint32_t)(target - c);
  if (in >= 8u) return;      // (no target: -1, which is below every column)
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float2 u = unf2(v[i]);
    if (in == 2u * i) u.x = value;
    if (in == 2u * i + 1u) u.y = value;
    v[i] = f2(u.x, u.y);
  }
}

constexpr int kLpBackVecs = 4;                                       // vectors of eight columns in each thread
constexpr int kLpBackCols = kLpThreads * 8 * kLpBackVecs;            // columns of a CTA

// SAME: x and dx of a row start at the same place in 16 bytes, so vectors between single values are aligned in both.
template <int XT, bool SAME>
__global__ void __launch_bounds__(kLpThreads, 4) logprob_bprop_kernel(const __grid_constant__ LogprobArgs args) {
  let_next_start();
  wait_for_previous();
  typedef typename ElemOf<XT>::T T;
  const int t = threadIdx.x;
  const int64_t r = blockIdx.x / args.chunks;
  const int chunk = (int)(blockIdx.x % args.chunks);
  const T* x = static_cast<const T*>(args.x) + r * args.ldx;
  T* dx = static_cast<T*>(args.dx) + r * args.ldd;
  const int64_t cols = args.cols;
  int64_t head = 0;
  if (SAME) {
    head = (int64_t)(((16u - ((uint32_t)reinterpret_cast<uintptr_t>(x) & 15u)) & 15u) / sizeof(T));
    head = head < cols ? head : cols;
  }
  const int64_t nv = SAME ? (cols - head) / 8 : (cols + 7) / 8;
  const int64_t first = (int64_t)chunk * (kLpThreads * kLpBackVecs) + t;
  Raw8<XT> raw[kLpBackVecs];
  int n[kLpBackVecs];
#pragma unroll
  for (int i = 0; i < kLpBackVecs; ++i) {
    const int64_t v = first + i * kLpThreads;
    n[i] = v < nv ? (SAME ? 8 : (int)(cols - 8 * v < 8 ? cols - 8 * v : 8)) : 0;
    raw[i] = load_raw8<XT, !SAME>(x + head + 8 * v, n[i]);
  }
  int32_t target;
  const LpRow w = lp_row(args, r, &target);
  const F2 scale = f2(args.scale), ml = f2(w.minus_lse), a = f2(w.a), d = f2(w.d);
  // the target's gradient: by the thread that has its vector, which reads the logit before it writes there (dx may be x)
  // and writes the entry once more behind its vectors
  const int64_t in = target - head;
  const uint64_t mine = (uint64_t)((in >> 3) - first);
  const bool own = in >= 0 && in < 8 * nv && mine < kLpThreads * kLpBackVecs && mine % kLpThreads == 0;
  const float own_x = own ? lp_one<XT>(x + target) : 0.f;
#pragma unroll
  for (int i = 0; i < kLpBackVecs; ++i) {
    const int64_t c = head + 8 * (first + i * kLpThreads);
    F2 g[4];
    to_pairs<XT>(raw[i], g);
#pragma unroll
    for (int k = 0; k < 4; ++k) g[k] = lp_grad2<XT == MAXDNN_F32>(g[k], scale, ml, a, d);
    store_pairs<XT, !SAME>(dx + c, g, n[i]);
  }
  if (own) dx[target] = from_float<XT>(lp_target_grad(args, w, r, own_x));
  if (SAME && chunk == 0) {      // single values in front and behind
    const int64_t tail = cols - head - 8 * nv;
    const int64_t c = t < head ? t : t >= 32 && t - 32 < tail ? cols - tail + t - 32 : -1;
    if (c >= 0) {
      const float v = lp_one<XT>(x + c);
      const float g = c != target ? unf2(lp_grad2<XT == MAXDNN_F32>(f2(v), scale, ml, a, d)).x : lp_target_grad(args, w, r, v);
      dx[c] = from_float<XT>(g);
    }
  }
}

// The gradient packed in 8 bits: a CTA has a tile of 128 x 128, thread t eight columns (8 (t mod 16)) of the four rows
// t / 16 + 32 k as 32-bit values, which serve both packed forms (and the wide one) after one reading.
constexpr int kLpPackThreads = 512;
constexpr int kLpPackRows = kBlock8 * (kBlock8 / 8) / kLpPackThreads, kLpPackStep = kBlock8 / kLpPackRows;
template <int XT, int QT, bool EDGE>
__global__ void __launch_bounds__(kLpPackThreads, 2) logprob_bprop_packed_kernel(const __grid_constant__ LogprobArgs args) {
  let_next_start();
  wait_for_previous();
  typedef typename ElemOf<XT>::T T;
  __shared__ LpRow rows[kBlock8];
  __shared__ int32_t targets[kBlock8];
  __shared__ float col_part[kLpPackThreads / 32][kBlock8];   // per warp: maxima of its rows
  __shared__ float col_inv[kBlock8];
  __shared__ uint8_t row_byte[kBlock8];
  const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
  const int cb = (int)(blockIdx.x % args.chunks), rb = (int)(blockIdx.x / args.chunks);
  const int r0 = rb * kBlock8, c0 = cb * kBlock8 + 8 * (t & 15), rg = t >> 4;
  const int n = vector_cols<EDGE>(args.cols, c0);
  const T* x = static_cast<const T*>(args.x);
  Raw8<XT> raw[kLpPackRows];
#pragma unroll
  for (int k = 0; k < kLpPackRows; ++k) {
    const int r = r0 + rg + kLpPackStep * k;
    raw[k] = load_raw8<XT, EDGE>(x + (int64_t)r * args.ldx + c0, r < args.rows ? n : 0);
  }
  // what is behind the last row has no p and no target
  if (t < kBlock8) {
    if (r0 + t < args.rows) {
      LpRow w = lp_row(args, r0 + t, &targets[t]);
      // the target's gradient, where this tile has it
      if ((uint32_t)(targets[t] - cb * kBlock8) < (uint32_t)kBlock8)
        w.add = lp_target_grad(args, w, r0 + t, lp_one<XT>(x + (int64_t)(r0 + t) * args.ldx + targets[t]));
      rows[t] = w;
    } else rows[t] = {-lp_inf(), 0.f, 0.f, 0.f}, targets[t] = -1;
  }
  __syncthreads();
  F2 g[kLpPackRows][4];
  float col_max[8], row_max[kLpPackRows];
#pragma unroll
  for (int i = 0; i < 8; ++i) col_max[i] = 0.f;
  const F2 scale = f2(args.scale);
#pragma unroll
  for (int k = 0; k < kLpPackRows; k += 2) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int in = rg + kLpPackStep * (k + h), r = r0 + in, have = r < args.rows ? n : 0;
      const LpRow w = rows[in];
      // (columns behind the last one: no p either, so that they take no part in the maxima)
      const F2 ml = f2(n > 0 ? w.minus_lse : -lp_inf()), a = f2(w.a), d = f2(w.d);
      F2 (&v)[4] = g[k + h];
      to_pairs<XT>(raw[k + h], v);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[i] = lp_grad2<true>(v[i], scale, ml, a, d);
        if (EDGE) {
          const float2 u = unf2(v[i]);
          v[i] = f2(2 * i < have ? u.x : 0.f, 2 * i + 1 < have ? u.y : 0.f);
        }
      }
      lp_set_target(v, w.add, targets[in], c0);
      row_max[k + h] = max8(v);
      if (args.dx) store_pairs<XT, true>(static_cast<T*>(args.dx) + (int64_t)r * args.ldd + c0, v, have);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 u = unf2(g[k][i]), w = unf2(g[k + 1][i]);
      col_max[2 * i] = max3abs(col_max[2 * i], u.x, w.x);
      col_max[2 * i + 1] = max3abs(col_max[2 * i + 1], u.y, w.y);
    }
  }
  float most = 0.f;
#pragma unroll
  for (int k = 0; k < kLpPackRows; ++k) most = fmaxf(most, row_max[k]);
  const bool fix = __syncthreads_or(isinf(most)) != 0;   // rare: a tile that holds an infinity, which enters no scale
  if (fix) {
#pragma unroll
    for (int i = 0; i < 8; ++i) col_max[i] = 0.f;
#pragma unroll
    for (int k = 0; k < kLpPackRows; ++k) {
      row_max[k] = finite_max8(g[k][0], g[k][1], g[k][2], g[k][3]);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 u = unf2(g[k][i]);
        col_max[2 * i] = fmaxf(col_max[2 * i], isinf(u.x) ? 0.f : fabsf(u.x));
        col_max[2 * i + 1] = fmaxf(col_max[2 * i + 1], isinf(u.y) ? 0.f : fabsf(u.y));
      }
    }
  }
  // (both ways apart: the test in every conversion costs a tenth of the kernel's instructions)
  auto pack = [&](auto fixes) {
    constexpr bool FIX = decltype(fixes)::value != 0;
    if (args.q_row) {
#pragma unroll
      for (int k = 0; k < kLpPackRows; k += 2) {
        uint32_t b[2];
        if (block_bytes<QT>(row_max[k], row_max[k + 1], &b[0], &b[1])) {
          b[0] = scale_byte<QT>(max_over_block_lanes(row_max[k]));
          b[1] = scale_byte<QT>(max_over_block_lanes(row_max[k + 1]));
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int r = r0 + rg + kLpPackStep * (k + i);
          if ((t & 15) == 0) row_byte[rg + kLpPackStep * (k + i)] = (uint8_t)b[i];
          store_bytes8<EDGE>(args.q_row + (int64_t)r * args.ldq + c0, pack8<QT>(g[k + i], inv_scale_of(b[i]), FIX), r < args.rows ? n : 0);
        }
      }
    }
    if (args.q_col) {
#pragma unroll
      for (int i = 0; i < 8; ++i) col_max[i] = fmaxf(col_max[i], __shfl_xor_sync(0xFFFFFFFFu, col_max[i], 16));
      if (lane < 16) {
#pragma unroll
        for (int i = 0; i < 8; i += 4)
          *reinterpret_cast<float4*>(&col_part[warp][8 * lane + i]) =
              make_float4(col_max[i], col_max[i + 1], col_max[i + 2], col_max[i + 3]);
      }
    }
    __syncthreads();
    if (args.q_row && t < kBlock8 && r0 + t < args.rows) args.s_row[(int64_t)cb * args.rows + r0 + t] = row_byte[t];
    if (!args.q_col) return;
    if (t < kBlock8) {
      float m = 0.f;
#pragma unroll
      for (int w = 0; w < kLpPackThreads / 32; ++w) m = fmaxf(m, col_part[w][t]);
      const uint32_t b = scale_byte<QT>(m);
      col_inv[t] = inv_scale_of(b);
      if (cb * kBlock8 + t < args.cols) args.s_col[(int64_t)rb * args.cols + cb * kBlock8 + t] = (uint8_t)b;
    }
    __syncthreads();
    F2 inv[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 u = *reinterpret_cast<const float2*>(&col_inv[8 * (t & 15) + 2 * i]);
      inv[i] = f2(u.x, u.y);
    }
#pragma unroll
    for (int k = 0; k < kLpPackRows; ++k) {
      const int r = r0 + rg + kLpPackStep * k;
      store_bytes8<EDGE>(args.q_col + (int64_t)r * args.ldq + c0, pack8<QT>(g[k], inv, FIX), r < args.rows ? n : 0);
    }
  };
  if (fix) pack(LpCount<1>());
  else pack(LpCount<0>());
}

}  // namespace maxdnn
