// Gated (or plain) activation of a feed-forward layer that works with packed activations.
//
//   a = f(g) u   (plain: a = f(g));   dg = da u f'(g),  du = da f(g)
//
// h holds g in columns [0, C) and u in [C, 2C).  Forward, a is packed as the next product's
// operand and g, u are packed as what the backward pass will read; backward, g and u come from
// there (or from h itself).  f: SiLU g s(g); GELU g P(g), P the normal distribution; GELU with
// the tanh approximation.
//
// A CTA takes 128 columns x 64 rows: 16 lanes cover a row block, thread t has eight columns of
// the rows t/16 + 16 k, so 4 (plain) or 8 (gated) loads of 16 bytes are in flight per thread.
//
// Measured: forward SiLU, gated, 8192 x 4096 bf16 with a and h packed 47 to 50 us (on different boards), 236 MB at
// 4.7 to 5.0 TB/s (copy: 6.5): 40 M warp instructions at 0.78 a cycle (three packings of 8 values each; three CTAs
// of an SM instead of four were 4 us slower, at the price of 16 bytes a thread spilled);
// backward GELU from packed h, 4097 x 2736, 23.3 us, 90 MB at 3.9 TB/s.
#pragma once
#include "fp8_util.cuh"

namespace maxdnn {

constexpr int kActThreads = 256;
constexpr int kActRows = 64;

struct Act8Args {
  const void* h;               // wide, or packed (bprop)
  const uint8_t* h_scale;
  void* a;                     // fprop, may be null
  uint8_t *q, *s;              // packed a, may be null
  uint8_t *c, *sc;             // packed h, may be null
  const void* da;
  void* dh;
  int64_t ldh, lda, ldq, ldc;
  int32_t rows, cols, col_blocks;
};

// Two forms of each function.  FULL, for fp32 activations: within a few units in the last place of f,
// however small f is.  Else, where results are rounded to 16 or 8 bits (2.4e-4 of a value at least): the
// hardware's exponential.
// 8192 x 4096 gated fp32, SiLU / GELU / tanh form, result alone: 61 / 72 / 67 us, with the short forms
// 59 / 66 / 62; with both packings 80 / 100 / 92 against 75 / 89 / 84; backward 99 and 81 (packed h) either way.
// (CUDA's normcdff and an IEEE quotient: 75 / 100 / 83 and 100 / 129 / 107.)

// 1 / (1 + exp(-x)).  Full: from exp(-|x|), which neither overflows nor loses s where it is small.
// Short: the exponential's relative error grows with |x| (1e-7 |x|), but enters s as s (1 - s) of it,
// which falls as exp(-|x|): the error of s stays below 2e-7.
template <bool FULL>
__device__ __forceinline__ float sigmoid(float x) {
  if constexpr (FULL) {
    const float e = expf(-fabsf(x));
    return __fdividef(x < 0.f ? e : 1.f, 1.f + e);
  }
  return __fdividef(1.f, 1.f + __expf(-x));
}

// The normal distribution function P(g), and exp(-g^2 / 2) (which f' needs too).  With z = |g|,
// P(-z) = exp(-z^2 / 2) t Q(t), t = 1 / (1 + 0.27 z), Q of degree 8, fitted for the least relative error on
// z <= 14.6 (2.4e-8; in fp32 arithmetic 4e-7 with an exact exponential); beyond that the exponential is 0.
// Full: what g^2 was rounded by is put back into the exponential (z is limited, so that this is a
// number).  Short: P is within 3e-5 of itself.
template <bool FULL>
__device__ __forceinline__ float normal_cdf(float g, float* gauss) {
  const float z = FULL ? fminf(fabsf(g), 16.f) : fabsf(g), hi = z * z;
  float e = FULL ? expf(-0.5f * hi) : __expf(-0.5f * hi);
  if constexpr (FULL) e = fmaf(-0.5f * fmaf(z, z, -hi), e, e);
  const float t = __fdividef(1.f, fmaf(0.27f, z, 1.f));
  float q = fmaf(0.028968822f, t, -0.126524672f);
  q = fmaf(q, t, 0.169869289f);
  q = fmaf(q, t, -0.069309689f);
  q = fmaf(q, t, 0.107896969f);
  q = fmaf(q, t, 0.072017767f);
  q = fmaf(q, t, 0.101819173f);
  q = fmaf(q, t, 0.107541606f);
  q = fmaf(q, t, 0.107720733f);
  const float tail = q * t * e;
  *gauss = e;
  return g < 0.f ? tail : 1.f - tail;
}

// f and, where asked for, f'.  (1 + tanh z) / 2 is the sigmoid of 2 z.
template <int ACT, bool GRAD, bool FULL>
__device__ __forceinline__ void activation(float g, float* f, float* df) {
  if constexpr (ACT == MAXDNN_ACT_SILU) {
    const float s = sigmoid<FULL>(g);
    *f = g * s;
    if (GRAD) *df = s * fmaf(g, 1.f - s, 1.f);
  } else if constexpr (ACT == MAXDNN_ACT_GELU) {
    float e;
    const float p = normal_cdf<FULL>(g, &e);
    *f = g * p;
    if (GRAD) *df = fmaf(g * 0.39894228040143268f, e, p);
  } else {
    const float k = 1.5957691216057308f;                    // 2 sqrt(2 / pi)
    const float q = fminf(g * g, 1e8f);                     // far out p (1 - p) is 0: no 0 x inf
    const float p = sigmoid<FULL>(k * g * fmaf(0.044715f, q, 1.f));
    *f = g * p;
    if (GRAD) *df = fmaf(g * p * (1.f - p), k * fmaf(0.134145f, q, 1.f), p);
  }
}

// Packs eight values each of two row blocks and keeps their scale bytes (null: nowhere).
template <int QT, bool EDGE>
__device__ __forceinline__ void pack_rows8(const F2 (&v)[4], const F2 (&w)[4], uint8_t* pv, uint8_t* pw, int n,
                                           bool live_v, bool live_w, uint8_t* sv, uint8_t* sw, bool first) {
  uint32_t bv, bw;
  bool fv = false, fw = false;
  if (block_bytes<QT>(max8(v), max8(w), &bv, &bw)) {
    bv = exact_byte<QT>(v, &fv);
    bw = exact_byte<QT>(w, &fw);
  }
  if (live_v) store_bytes8<EDGE>(pv, pack8<QT>(v, inv_scale_of(bv), fv), n);
  if (live_w) store_bytes8<EDGE>(pw, pack8<QT>(w, inv_scale_of(bw), fw), n);
  if (first) {
    *sv = (uint8_t)bv;
    *sw = (uint8_t)bw;
  }
}

template <int XT, int QT, int ACT, bool GATED, bool EDGE>
__global__ void __launch_bounds__(kActThreads, XT == MAXDNN_F32 ? 2 : 4) act8_fprop_kernel(const __grid_constant__ Act8Args args) {
  let_next_start();
  wait_for_previous();
  typedef typename ElemOf<XT>::T T;
  __shared__ uint8_t bytes[3][kActRows];
  const int t = threadIdx.x;
  const int cb = blockIdx.x % args.col_blocks;
  const int rb = blockIdx.x / args.col_blocks;
  const int r0 = rb * kActRows, c0 = cb * kBlock8 + 8 * (t & 15);
  const int n = vector_cols<EDGE>(args.cols, c0);
  const T* h = static_cast<const T*>(args.h);
  Raw8<XT> rg[4], ru[GATED ? 4 : 1];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int r = r0 + (t >> 4) + 16 * k;
    const int nr = r < args.rows ? n : 0;
    rg[k] = load_raw8<XT, EDGE>(h + (int64_t)r * args.ldh + c0, nr);
    if constexpr (GATED) ru[k] = load_raw8<XT, EDGE>(h + (int64_t)r * args.ldh + args.cols + c0, nr);
  }
  const bool first = (t & 15) == 0;
#pragma unroll
  for (int k = 0; k < 4; k += 2) {       // two rows at a time: their blocks share the shuffles
    const int row = (t >> 4) + 16 * k, r = r0 + row;
    const bool live[2] = {r < args.rows && n > 0, r + 16 < args.rows && n > 0};
    F2 v[2][4];
    float g[2][8], u[2][8];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      to_pairs<XT>(rg[k + i], v[i]);
      to_floats(v[i], g[i]);
    }
    if (args.c) {
      uint8_t* c = args.c + (int64_t)r * args.ldc + c0;
      pack_rows8<QT, EDGE>(v[0], v[1], c, c + 16 * args.ldc, n, live[0], live[1], &bytes[1][row],
                           &bytes[1][row + 16], first);
    }
    if constexpr (GATED) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        to_pairs<XT>(ru[k + i], v[i]);
        to_floats(v[i], u[i]);
      }
      if (args.c) {
        uint8_t* c = args.c + (int64_t)r * args.ldc + args.cols + c0;
        pack_rows8<QT, EDGE>(v[0], v[1], c, c + 16 * args.ldc, n, live[0], live[1],
                             &bytes[2][row], &bytes[2][row + 16], first);
      }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      float a[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float f, unused;
        activation<ACT, false, XT == MAXDNN_F32>(g[i][e], &f, &unused);
        a[e] = GATED ? f * u[i][e] : f;
      }
      if (args.a && live[i])
        store_float8<XT, EDGE>(static_cast<T*>(args.a) + (int64_t)(r + 16 * i) * args.lda + c0, a, n);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[i][e] = f2(a[2 * e], a[2 * e + 1]);
    }
    if (args.q) {
      uint8_t* q = args.q + (int64_t)r * args.ldq + c0;
      pack_rows8<QT, EDGE>(v[0], v[1], q, q + 16 * args.ldq, n, live[0], live[1], &bytes[0][row],
                           &bytes[0][row + 16], first);
    }
  }
  __syncthreads();
  // scales of this CTA's blocks: rows are next to each other
  const int row = t & (kActRows - 1), which = t / kActRows;
  if (r0 + row >= args.rows) return;
  const int64_t at = (int64_t)cb * args.rows + r0 + row;
  if (which == 0 && args.q) args.s[at] = bytes[0][row];
  if (which == 1 && args.c) args.sc[at] = bytes[1][row];
  if (GATED && which == 2 && args.c) args.sc[(int64_t)args.col_blocks * args.rows + at] = bytes[2][row];
}

// HT: the type of h (wide, or packed); XT: of da and dh.
template <int HT, int XT, int ACT, bool GATED, bool EDGE>
__global__ void __launch_bounds__(kActThreads) act8_bprop_kernel(const __grid_constant__ Act8Args args) {
  let_next_start();
  wait_for_previous();
  typedef typename ElemOf<HT>::T TH;
  typedef typename ElemOf<XT>::T T;
  const int t = threadIdx.x;
  const int cb = blockIdx.x % args.col_blocks;
  const int rb = blockIdx.x / args.col_blocks;
  const int r0 = rb * kActRows + (t >> 4), c0 = cb * kBlock8 + 8 * (t & 15);
  const int n = vector_cols<EDGE>(args.cols, c0);
  if (n == 0) return;
  const TH* h = static_cast<const TH*>(args.h);
  const int64_t ldh = is_fp8(HT) ? args.ldc : args.ldh;
  Raw8<HT> rg[4], ru[GATED ? 4 : 1];
  Raw8<XT> rd[4];
  float sg[4], su[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int r = r0 + 16 * k;
    const int nr = r < args.rows ? n : 0;
    rg[k] = load_raw8<HT, EDGE>(h + (int64_t)r * ldh + c0, nr);
    if constexpr (GATED) ru[k] = load_raw8<HT, EDGE>(h + (int64_t)r * ldh + args.cols + c0, nr);
    rd[k] = load_raw8<XT, EDGE>(static_cast<const T*>(args.da) + (int64_t)r * args.lda + c0, nr);
    sg[k] = su[k] = 1.f;
    if (is_fp8(HT) && nr > 0) {
      sg[k] = e8m0_value(args.h_scale[(int64_t)cb * args.rows + r]);
      if constexpr (GATED) su[k] = e8m0_value(args.h_scale[(int64_t)(args.col_blocks + cb) * args.rows + r]);
    }
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int r = r0 + 16 * k;
    if (r >= args.rows) break;
    float g[8], u[8], d[8], dg[8], du[8];
    to_float8<HT>(rg[k], g);
    if constexpr (GATED) to_float8<HT>(ru[k], u);
    to_float8<XT>(rd[k], d);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if constexpr (is_fp8(HT)) g[i] *= sg[k];
      if constexpr (is_fp8(HT) && GATED) u[i] *= su[k];
      float f, df;
      activation<ACT, true, XT == MAXDNN_F32>(g[i], &f, &df);
      if constexpr (GATED) {
        dg[i] = d[i] * u[i] * df;
        du[i] = d[i] * f;
      } else {
        dg[i] = d[i] * df;
      }
    }
    T* dh = static_cast<T*>(args.dh) + (int64_t)r * args.ldh + c0;
    store_float8<XT, EDGE>(dh, dg, n);
    if constexpr (GATED) store_float8<XT, EDGE>(dh + args.cols, du, n);
  }
}

}  // namespace maxdnn
