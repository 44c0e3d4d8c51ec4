// Layer norm over the last axis, forward and backward, with the packed forms that the 8-bit
// training step reads next.
//
//   mean = sum x / C,  rstd = 1 / sqrt(sum (x - mean)^2 / C + eps),  xh = (x - mean) rstd
//   y = xh g + b
//   dx = rstd (g dy - s1 - xh s2),  s1 = sum(g dy) / C,  s2 = sum(g dy xh) / C
//   dg = sum over rows of dy xh,  db = sum over rows of dy
//
// A row is read once and stays in registers: T threads (a warp, or several) hold it as
// vectors of eight columns, vector j of thread t at column 8 (t + T j).  The variance is summed from the
// differences to the mean, not from squares, so a row far from zero loses nothing.  All sums are
// in 32 bits.  Sixteen neighbouring lanes hold a block of 128 columns, so the packed forms take
// four shuffles for two blocks.
//
// Measured at 8192 x 4096 bf16 (copy: 6.5 TB/s): statistics alone 15 us (4.5 TB/s), y 27.7 us (4.9), y and x packed
// 40 us (3.4: two packings, 27 M warp instructions at 0.64 a cycle: one row after the other, no load of the next
// under way), backward from packed x 43.6 us with the sums over rows (3.9).  Widths that are no multiple of 8 take 3
// to 4 times that (4095 columns: 96, 117 and 140 us).  Tried when the packed forward pass took 45 us, and slower: two rows at a time to share
// the weights (50 us: half the warps), the next row prefetched in registers (51 us) or in a ring in shared
// memory (72 us, the weights then fall out of the first-level cache), 48 registers and five CTAs (50 us).
#pragma once
#include "fp8_util.cuh"
#include "ptx_util.cuh"

namespace maxdnn {

struct LayerNormArgs {
  const void* x;               // fprop: wide; bprop: wide or packed rows
  const uint8_t* x_scale;
  const void *gamma, *beta;    // null: 1, 0
  void* y;
  float *mean, *rstd;
  uint8_t *q, *s, *c, *sc;     // fprop: packed y, packed x
  const void* dy;              // bprop
  void* dx;
  float* partial;              // [grid][2][norm_sums_pitch(cols)] sums of a CTA's rows: dy xh, dy
  int64_t ldx, ldy, ldq;
  int32_t rows, cols, w_type;
  int32_t whole;               // vectors of eight columns are whole and aligned (the host's choice of instance)
  int32_t q_e5m2;
  float eps, inv_cols;
};

constexpr int kNormMaxWarps = 32;

// Columns of a row of sums: whole vectors of eight, so that a thread's eight go in two 16-byte pieces
// whatever the width (one by one, 32 bytes from lane to lane, the stores of 296 CTAs took 8 us of the 50 of
// 8192 x 4096, and as much of the 18 of 128 x 8192).
__host__ __device__ inline int64_t norm_sums_pitch(int cols) { return ((int64_t)cols + 7) / 8 * 8; }
__device__ __forceinline__ void load_sums8(const float* p, float (&v)[8]) {    // (plain loads: the kernel wrote them)
  const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
  v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
  v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
__device__ __forceinline__ void store_sums8(float* p, const float (&v)[8]) {
  reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
  reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
  return v;
}

// Packs eight values each of two row blocks (16 lanes) and stores them with the blocks' scales.
template <int QT, bool EDGE>
__device__ __forceinline__ void norm_pack_as(const F2 (&v)[4], const F2 (&w)[4], uint8_t* qv, uint8_t* qw, uint8_t* sv,
                                             uint8_t* sw, int nv, int nw, int lane) {
  uint32_t bv, bw;
  bool fv = false, fw = false;
  if (block_bytes<QT>(max8(v), max8(w), &bv, &bw)) {
    bv = exact_byte<QT>(v, &fv);
    bw = exact_byte<QT>(w, &fw);
  }
  store_bytes8<EDGE>(qv, pack8<QT>(v, inv_scale_of(bv), fv), nv);
  store_bytes8<EDGE>(qw, pack8<QT>(w, inv_scale_of(bw), fw), nw);
  if ((lane & 15) == 0) {
    if (nv > 0) *sv = (uint8_t)bv;
    if (nw > 0) *sw = (uint8_t)bw;
  }
}
// QT: the 8-bit type, or kEitherFp8: `e5m2` tells.
constexpr int kEitherFp8 = 0;
template <int QT, bool EDGE>
__device__ __forceinline__ void norm_pack(const F2 (&v)[4], const F2 (&w)[4], bool e5m2, uint8_t* qv, uint8_t* qw,
                                          uint8_t* sv, uint8_t* sw, int nv, int nw, int lane) {
  if (QT == MAXDNN_E5M2 || (QT == kEitherFp8 && e5m2))
    norm_pack_as<MAXDNN_E5M2, EDGE>(v, w, qv, qw, sv, sw, nv, nw, lane);
  else
    norm_pack_as<MAXDNN_E4M3, EDGE>(v, w, qv, qw, sv, sw, nv, nw, lane);
}

// Eight neighbouring weights.
template <bool EDGE, bool FREE = false>
__device__ __forceinline__ void load_weights8(const void* p, int c, int n, int type, float none, F2 (&w)[4]) {
  if (!p || n == 0) {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = f2(none);
  } else if (type == MAXDNN_F32) {
    to_pairs<MAXDNN_F32>(load_raw8<MAXDNN_F32, EDGE, FREE>(static_cast<const float*>(p) + c, n), w);
  } else if (type == MAXDNN_BF16) {
    to_pairs<MAXDNN_BF16>(load_raw8<MAXDNN_BF16, EDGE, FREE>(static_cast<const __nv_bfloat16*>(p) + c, n), w);
  } else {
    to_pairs<MAXDNN_F16>(load_raw8<MAXDNN_F16, EDGE, FREE>(static_cast<const __half*>(p) + c, n), w);
  }
}

// y of eight columns; columns at and after n become zeros (they take part in the block's maximum).
template <bool EDGE>
__device__ __forceinline__ void normalise8(F2 (&v)[4], F2 minus_mean, F2 rstd, const F2 (&g)[4], const F2 (&b)[4], int n) {
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = fma2(mul2(add2(v[i], minus_mean), rstd), g[i], b[i]);
  if (EDGE) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 t = unf2(v[i]);
      v[i] = f2(2 * i < n ? t.x : 0.f, 2 * i + 1 < n ? t.y : 0.f);
    }
  } else if (n == 0) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = 0;
  }
}

// Sum of squares of the differences to the mean, of the first n of eight columns.
template <bool EDGE>
__device__ __forceinline__ float squares8(const F2 (&v)[4], F2 minus_mean, int n) {
  F2 part = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    F2 d = add2(v[i], minus_mean);
    if (EDGE) {
      const float2 t = unf2(d);
      d = f2(2 * i < n ? t.x : 0.f, 2 * i + 1 < n ? t.y : 0.f);
    }
    part = fma2(d, d, part);
  }
  return EDGE || n > 0 ? sum2(part) : 0.f;
}

// WR warps have a row, vector j of the row's thread t at column 8 (t + 32 WR j); a CTA of eight
// warps has 8 / WR rows at a time.  The row stays as it was loaded (4 J registers of 16-bit values) and is
// converted again for each of the three sums.  J is at most 4 up to 8192 columns: with 16 vectors to a lane the
// unrolled code no longer fits the instruction cache (8192 x 4096 with packed y and x: a third of
// the stalls were for instructions, 89 us).
constexpr int kNormThreads = 256;
__host__ __device__ constexpr bool norm_shared_weights(int j, int wr) {
  return (j == 4 && wr <= 4) || (j == 2 && wr == 1);
}
template <int XT, int QT, int J, int WR, bool EDGE>
__global__ void __launch_bounds__(kNormThreads, J > 4 ? 2 : XT == MAXDNN_F32 || EDGE ? 3 : 4)
layer_norm_fprop_kernel(const __grid_constant__ LayerNormArgs args) {
  let_next_start();
  wait_for_previous();
  typedef typename ElemOf<XT>::T T;
  __shared__ float slots[8 / WR][2][WR];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int group = warp / WR, in_row = warp % WR, t = in_row * 32 + lane;
  const T* x = static_cast<const T*>(args.x);
  T* y = static_cast<T*>(args.y);
  // The weights as fp32 in shared memory, for every row of the CTA: whatever their type, and where
  // there are none (up to 4096 columns, 32 KB; 16384 x 1024 with packed results: 25.8 us with the
  // weights from the first-level cache, 19.9 from here.  With 64 KB for 8192 columns fewer CTAs fit an SM:
  // 92 us became 125; now 100 without).
  constexpr bool kShared = norm_shared_weights(J, WR) && !EDGE;
  extern __shared__ __align__(16) float weights[];
  const int padded = 256 * WR * J;
  if constexpr (kShared) {
    if (args.y || args.q) {
      // four planes of four columns of each vector: gamma's first and last, beta's first and last
      // (neighbouring lanes then read neighbouring 16 bytes)
      for (int c = 8 * (int)threadIdx.x; c < padded; c += 8 * kNormThreads) {
        const int n = vector_cols<EDGE>(args.cols, c);
#pragma unroll
        for (int which = 0; which < 2; ++which) {
          F2 w[4];
          load_weights8<EDGE>(which ? args.beta : args.gamma, c, n, args.w_type, which ? 0.f : 1.f, w);
#pragma unroll
          for (int i = 0; i < 4; i += 2) {
            ulonglong2 two;
            two.x = w[i];
            two.y = w[i + 1];
            *reinterpret_cast<ulonglong2*>(&weights[which * padded + (i / 2) * (padded / 2) + c / 2]) = two;
          }
        }
      }
    }
    __syncthreads();
  }
  // sum over the row's threads
  auto total = [&](float v, int slot) {
    v = warp_sum(v);
    if constexpr (WR > 1) {
      if (lane == 0) slots[group][slot][in_row] = v;
      asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "n"(WR * 32) : "memory");
      v = 0.f;
#pragma unroll
      for (int w = 0; w < WR; ++w) v += slots[group][slot][w];
    }
    return v;
  };
  for (int64_t r = (int64_t)blockIdx.x * (8 / WR) + group; r < args.rows; r += (int64_t)gridDim.x * (8 / WR)) {
    Raw8<XT> raw[J];
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const int c = 8 * (t + 32 * WR * j);
      raw[j] = load_raw8<XT, EDGE>(x + r * args.ldx + c, vector_cols<EDGE>(args.cols, c));
    }
    F2 sum = 0;
#pragma unroll
    for (int j = 0; j < J; ++j) {
      F2 v[4];
      to_pairs<XT>(raw[j], v);
      sum = add2(sum, add2(add2(v[0], v[1]), add2(v[2], v[3])));
    }
    const float mean = total(sum2(sum), 0) * args.inv_cols;
    const F2 minus_mean = f2(-mean);
    float sq = 0.f;
#pragma unroll
    for (int j = 0; j < J; ++j) {
      F2 v[4];
      convert_again(raw[j]);
      to_pairs<XT>(raw[j], v);
      sq += squares8<EDGE>(v, minus_mean, vector_cols<EDGE>(args.cols, 8 * (t + 32 * WR * j)));
    }
    const float rstd = 1.f / sqrtf(total(sq, 1) * args.inv_cols + args.eps);
    if (t == 0) {
      if (args.mean) args.mean[r] = mean;
      if (args.rstd) args.rstd[r] = rstd;
    }
    // two vectors at a time (J = 1: one, with zeros for the other)
    constexpr int kPair = J > 1 ? 2 : 1, kStep = 256 * WR;
    const int c0 = 8 * t;
    const int64_t scale_step = (int64_t)(kStep / kBlock8) * args.rows;
    uint8_t* cp = args.c ? args.c + r * args.ldq + c0 : nullptr;
    uint8_t* qp = args.q ? args.q + r * args.ldq + c0 : nullptr;
    uint8_t* scp = args.sc + (int64_t)(c0 >> 7) * args.rows + r;
    uint8_t* sqp = args.s + (int64_t)(c0 >> 7) * args.rows + r;
    T* yp = y ? y + r * args.ldy + c0 : nullptr;
#pragma unroll
    for (int j = 0; j < J; j += kPair) {
      F2 v[2][4] = {};
      int n[2] = {0, 0};
#pragma unroll
      for (int i = 0; i < kPair; ++i) {
        n[i] = vector_cols<EDGE>(args.cols, c0 + kStep * (j + i));
        convert_again(raw[j + i]);
        to_pairs<XT>(raw[j + i], v[i]);
      }
      if (args.c)
        norm_pack<QT, EDGE>(v[0], v[1], args.q_e5m2, cp + kStep * j, cp + kStep * (j + 1), scp + scale_step * j,
                            scp + scale_step * (j + 1), n[0], n[1], lane);
      if (!args.y && !args.q) continue;
#pragma unroll
      for (int i = 0; i < kPair; ++i) {
        const int c = c0 + kStep * (j + i);
        F2 g[4], b[4];
        if constexpr (kShared) {
#pragma unroll
          for (int e = 0; e < 4; e += 2) {
            const float* at = &weights[(e / 2) * (padded / 2) + c / 2];
            const ulonglong2 gg = *reinterpret_cast<const ulonglong2*>(at);
            const ulonglong2 bb = *reinterpret_cast<const ulonglong2*>(at + padded);
            g[e] = gg.x; g[e + 1] = gg.y;
            b[e] = bb.x; b[e + 1] = bb.y;
          }
        } else {
          load_weights8<EDGE, true>(args.gamma, c, n[i], args.w_type, 1.f, g);
          load_weights8<EDGE, true>(args.beta, c, n[i], args.w_type, 0.f, b);
        }
        normalise8<EDGE>(v[i], minus_mean, f2(rstd), g, b, n[i]);
        if (args.y) store_pairs<XT, EDGE>(yp + kStep * (j + i), v[i], n[i]);
      }
      if (args.q)
        norm_pack<QT, EDGE>(v[0], v[1], args.q_e5m2, qp + kStep * j, qp + kStep * (j + 1), sqp + scale_step * j,
                            sqp + scale_step * (j + 1), n[0], n[1], lane);
    }
    // no barrier here: a thread reaches the next row's first write of a slot only after the
    // second sum's barrier, which follows every read of the first slot (and the other way round)
  }
}

// Sum over the 1024 threads of a CTA.  `slot` alternates between two calls.
__device__ __forceinline__ float cta_sum(float v, float* slot, int lane, int warp) {
  v = warp_sum(v);
  if (lane == 0) slot[warp] = v;
  __syncthreads();
  float s = 0.f;
  for (int w = 0; w < kNormMaxWarps; ++w) s += slot[w];
  return s;
}

// Eight columns of the backward pass as they come from memory: xh and gamma dy, with this row's
// part of dg and db added up.
template <int XT, int YT, bool EDGE>
__device__ __forceinline__ void norm_back8(const Raw8<XT>& rx, const Raw8<YT>& rdy, float scale, float mean, float rstd,
                                           const F2 (&g)[4], int n, F2 (&xh)[4], F2 (&e)[4], F2 (&dg)[4], F2 (&db)[4],
                                           F2* s1, F2* s2) {
  to_pairs<XT>(rx, xh);
  to_pairs<YT>(rdy, e);
  // The difference first: one multiply-add with -mean rstd would round that product, 2e-5 of xh
  // for rows at 1000 with a spread of 1, and leaves the range where mean rstd does.
  // (Vectors past the row's end: zeros, so that they stay out of the sums.)
  const F2 mm = f2(EDGE || n > 0 ? -mean : 0.f), rs = f2(rstd), sc = f2(scale);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    xh[i] = mul2(is_fp8(XT) ? fma2(xh[i], sc, mm) : add2(xh[i], mm), rs);
    if (EDGE) {
      const float2 t = unf2(xh[i]);
      xh[i] = f2(2 * i < n ? t.x : 0.f, 2 * i + 1 < n ? t.y : 0.f);
    }
    dg[i] = fma2(e[i], xh[i], dg[i]);
    db[i] = add2(db[i], e[i]);
    e[i] = mul2(e[i], g[i]);
    *s1 = add2(*s1, e[i]);
    *s2 = fma2(e[i], xh[i], *s2);
  }
}

// rstd (e - s1 - xh s2) of eight columns.
__device__ __forceinline__ void norm_dx8(const F2 (&xh)[4], const F2 (&e)[4], float rstd, float s1, float s2, F2 (&o)[4]) {
  const F2 m1 = f2(-s1 * rstd), m2 = f2(-s2 * rstd), rs = f2(rstd);
#pragma unroll
  for (int i = 0; i < 4; ++i) o[i] = fma2(xh[i], m2, fma2(e[i], rs, m1));
}

// XT: the type of x (wide, or packed rows); YT: of dy and dx.  WARP_ROW: each warp of the CTA has
// a row of its own; else the CTA has one.  (Rows of up to 1024 columns, and rows whose vectors are not whole.)
template <int XT, int YT, int J, bool WARP_ROW, bool EDGE>
__global__ void __launch_bounds__(WARP_ROW ? 128 : 512)
layer_norm_bprop_kernel(const __grid_constant__ LayerNormArgs args) {
  let_next_start();
  wait_for_previous();
  typedef typename ElemOf<XT>::T TX;
  typedef typename ElemOf<YT>::T TY;
  __shared__ float slots[2][2][kNormMaxWarps];
  __shared__ float fold[WARP_ROW ? 8 * 32 * J : 1];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  const int t = WARP_ROW ? lane : (int)threadIdx.x;
  const int threads = WARP_ROW ? 32 : (int)blockDim.x;
  const int per_cta = WARP_ROW ? warps : 1;
  const TX* x = static_cast<const TX*>(args.x);
  const TY* dy = static_cast<const TY*>(args.dy);
  TY* dx = static_cast<TY*>(args.dx);
  F2 g[J][4], dg[J][4], db[J][4];
#pragma unroll
  for (int j = 0; j < J; ++j) {
    const int c = 8 * (t + threads * j);
    load_weights8<true>(args.gamma, c, min(max(args.cols - c, 0), 8), args.w_type, 1.f, g[j]);
#pragma unroll
    for (int i = 0; i < 4; ++i) dg[j][i] = db[j][i] = 0;
  }
  int flip = 0;
  for (int64_t r = (int64_t)blockIdx.x * per_cta + (WARP_ROW ? warp : 0); r < args.rows;
       r += (int64_t)gridDim.x * per_cta, flip ^= 1) {
    const float mean = args.mean[r], rstd = args.rstd[r];
    Raw8<XT> rx[J];
    Raw8<YT> rdy[J];
    float scale[J];
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const int c = 8 * (t + threads * j);
      const int n = min(max(args.cols - c, 0), 8);
      rx[j] = load_raw8<XT, EDGE>(x + r * args.ldx + c, n);
      rdy[j] = load_raw8<YT, EDGE>(dy + r * args.ldy + c, n);
      scale[j] = 1.f;
      if constexpr (is_fp8(XT)) scale[j] = n > 0 ? e8m0_value(args.x_scale[(int64_t)(c >> 7) * args.rows + r]) : 0.f;
    }
    F2 xh[J][4], e[J][4], p1 = 0, p2 = 0;
#pragma unroll
    for (int j = 0; j < J; ++j)
      norm_back8<XT, YT, EDGE>(rx[j], rdy[j], scale[j], mean, rstd, g[j], min(max(args.cols - 8 * (t + threads * j), 0), 8),
                               xh[j], e[j], dg[j], db[j], &p1, &p2);
    float s1 = warp_sum(sum2(p1)), s2 = warp_sum(sum2(p2));
    if constexpr (!WARP_ROW) {
      if (lane == 0) {
        slots[flip][0][warp] = s1;
        slots[flip][1][warp] = s2;
      }
      __syncthreads();
      s1 = s2 = 0.f;
      for (int w = 0; w < warps; ++w) {
        s1 += slots[flip][0][w];
        s2 += slots[flip][1][w];
      }
    }
    s1 *= args.inv_cols;
    s2 *= args.inv_cols;
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const int c = 8 * (t + threads * j);
      F2 o[4];
      norm_dx8(xh[j], e[j], rstd, s1, s2, o);
      store_pairs<YT, EDGE>(dx + r * args.ldy + c, o, min(max(args.cols - c, 0), 8));
    }
  }
  if (!args.partial) return;
  // this CTA's sums over its rows; a CTA of several rows adds them warp by warp
  const int64_t pitch = norm_sums_pitch(args.cols);
  float* out = args.partial + (int64_t)blockIdx.x * 2 * pitch;
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    float a[J][8];
#pragma unroll
    for (int j = 0; j < J; ++j) to_floats(which ? db[j] : dg[j], a[j]);
    if constexpr (WARP_ROW) {
      for (int w = 0; w < warps; ++w) {
        if (warp == w) {
#pragma unroll
          for (int j = 0; j < J; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              float& f = fold[(i * J + j) * 32 + lane];
              f = w == 0 ? a[j][i] : f + a[j][i];
            }
        }
        __syncthreads();
      }
      for (int c = threadIdx.x; c < args.cols; c += blockDim.x) {
        const int vecj = c >> 8, l = (c >> 3) & 31, i = c & 7;
        out[which * pitch + c] = fold[(i * J + vecj) * 32 + l];
      }
      __syncthreads();
    } else {
#pragma unroll
      for (int j = 0; j < J; ++j) {
        const int c = 8 * (t + threads * j);
        if (c < args.cols) store_sums8(out + which * pitch + c, a[j]);
      }
    }
  }
}

// The same for rows of 1025 to 8192 columns of whole vectors, with the rows to come on their way:
// a CTA has neighbouring rows, and every thread copies its own vectors of the next rows into its
// own places of a ring in shared memory (asynchronous copies of 8 or 16 bytes; nothing is exchanged
// through the ring, so it needs no barrier).  Statistics and scale bytes of kNormChunk rows are fetched
// at once.
constexpr int kNormChunk = 32;

template <int BYTES>
__device__ __forceinline__ void copy_async(uint32_t dst, const void* src) {
  if constexpr (BYTES == 8) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(dst), "l"(src) : "memory");
  } else {
#pragma unroll
    for (int i = 0; i < BYTES; i += 16)
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst + i), "l"(static_cast<const uint8_t*>(src) + i) : "memory");
  }
}

// Bytes of shared memory: the ring, then scale bytes and statistics of a chunk of rows.
__host__ __device__ constexpr int norm_ring_row(int x_bytes, int y_bytes, int threads, int j) {
  return threads * j * 8 * (x_bytes + y_bytes);
}

// J vectors in each thread of WARPS warps.  Fewer threads with more columns each take fewer
// instructions (the row's two sums are one exchange per warp), and more registers.
template <int XT, int YT, int J, int WARPS>
__global__ void __launch_bounds__(32 * WARPS, 16 / WARPS)
layer_norm_bprop_ring_kernel(const __grid_constant__ LayerNormArgs args, int depth) {
  let_next_start();
  wait_for_previous();
  typedef typename ElemOf<XT>::T TX;
  typedef typename ElemOf<YT>::T TY;
  constexpr int XB = 8 * (int)sizeof(TX), YB = 8 * (int)sizeof(TY);
  extern __shared__ __align__(16) uint8_t ring[];
  __shared__ __align__(16) float slots[2][2][WARPS];
  __shared__ float stats[2][kNormChunk];
  constexpr int threads = 32 * WARPS;
  const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
  const int row_bytes = norm_ring_row((int)sizeof(TX), (int)sizeof(TY), threads, J);
  uint8_t* scales = ring + (size_t)depth * row_bytes;      // [block][row of the chunk]
  const int blocks = (args.cols + kBlock8 - 1) / kBlock8;
  const int64_t r0 = (int64_t)args.rows * blockIdx.x / gridDim.x, r1 = (int64_t)args.rows * (blockIdx.x + 1) / gridDim.x;
  const TX* x = static_cast<const TX*>(args.x);
  const TY* dy = static_cast<const TY*>(args.dy);
  TY* dx = static_cast<TY*>(args.dx);
  // this thread's places in a ring slot: J x values, then J dy values
  auto x_at = [&](int slot, int j) { return (size_t)slot * row_bytes + (size_t)(j * threads + t) * XB; };
  auto y_at = [&](int slot, int j) {
    return (size_t)slot * row_bytes + (size_t)J * threads * XB + (size_t)(j * threads + t) * YB;
  };
  const uint32_t ring_u = smem_u32(ring);
  auto fetch = [&](int64_t r, int slot) {
    if (r < r1) {
#pragma unroll
      for (int j = 0; j < J; ++j) {
        const int c = 8 * (t + threads * j);
        if (c < args.cols) {
          copy_async<XB>(ring_u + (uint32_t)x_at(slot, j), x + r * args.ldx + c);
          copy_async<YB>(ring_u + (uint32_t)y_at(slot, j), dy + r * args.ldy + c);
        }
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  F2 g[J][4], dg[J][4], db[J][4];
#pragma unroll
  for (int j = 0; j < J; ++j) {
    const int c = 8 * (t + threads * j);
    load_weights8<true>(args.gamma, c, c < args.cols ? 8 : 0, args.w_type, 1.f, g[j]);
#pragma unroll
    for (int i = 0; i < 4; ++i) dg[j][i] = db[j][i] = 0;
  }
  for (int d = 0; d < depth - 1; ++d) fetch(r0 + d, d);
  int flip = 0, slot = 0;
  for (int64_t chunk = r0; chunk < r1; chunk += kNormChunk) {
    const int in_chunk = (int)(r1 - chunk < kNormChunk ? r1 - chunk : kNormChunk);
    __syncthreads();           // the last chunk's statistics have been read
    if (t < in_chunk) {
      stats[0][t] = args.mean[chunk + t];
      stats[1][t] = args.rstd[chunk + t];
    }
    if constexpr (is_fp8(XT)) {
      for (int i = t; i < blocks * kNormChunk; i += threads) {
        const int row = i % kNormChunk;
        if (row < in_chunk) scales[i] = args.x_scale[(int64_t)(i / kNormChunk) * args.rows + chunk + row];
      }
    }
    __syncthreads();
    for (int k = 0; k < in_chunk; ++k, flip ^= 1) {
      // the copies of the row `depth - 1` ahead go where the row before this one was
      const int64_t r = chunk + k;
      fetch(r + depth - 1, slot == 0 ? depth - 1 : slot - 1);
      if (depth == 4) asm volatile("cp.async.wait_group 3;" ::: "memory");
      else if (depth == 3) asm volatile("cp.async.wait_group 2;" ::: "memory");
      else asm volatile("cp.async.wait_group 1;" ::: "memory");
      const float mean = stats[0][k], rstd = stats[1][k];
      F2 xh[J][4], e[J][4], p1 = 0, p2 = 0;
#pragma unroll
      for (int j = 0; j < J; ++j) {
        const int c = 8 * (t + threads * j);
        Raw8<XT> rx = {};
        Raw8<YT> rdy = {};
        float scale = 0.f;
        if (c < args.cols) {
          rx = *reinterpret_cast<const Raw8<XT>*>(ring + x_at(slot, j));
          rdy = *reinterpret_cast<const Raw8<YT>*>(ring + y_at(slot, j));
          if constexpr (is_fp8(XT)) scale = e8m0_value(scales[(c >> 7) * kNormChunk + k]);
        }
        // (columns past the end: dy = 0 keeps them out of every sum)
        norm_back8<XT, YT, false>(rx, rdy, scale, mean, rstd, g[j], c < args.cols ? 8 : 0, xh[j], e[j], dg[j], db[j], &p1, &p2);
      }
      // both sums in six shuffles: the halves of the warp take one each
      float s1 = sum2(p1), s2 = sum2(p2);
      const float other = __shfl_xor_sync(0xFFFFFFFFu, lane < 16 ? s2 : s1, 16);
      float mine = (lane < 16 ? s1 : s2) + other;
#pragma unroll
      for (int d = 8; d > 0; d >>= 1) mine += __shfl_xor_sync(0xFFFFFFFFu, mine, d);
      if ((lane & 15) == 0) slots[flip][lane >> 4][warp] = mine;
      __syncthreads();
      F2 t1 = 0, t2 = 0;
#pragma unroll
      for (int w = 0; w < WARPS; w += 4) {
        const float4 a = *reinterpret_cast<const float4*>(&slots[flip][0][w]);
        const float4 b = *reinterpret_cast<const float4*>(&slots[flip][1][w]);
        t1 = add2(t1, add2(f2(a.x, a.y), f2(a.z, a.w)));
        t2 = add2(t2, add2(f2(b.x, b.y), f2(b.z, b.w)));
      }
      s1 = sum2(t1);
      s2 = sum2(t2);
      s1 *= args.inv_cols;
      s2 *= args.inv_cols;
#pragma unroll
      for (int j = 0; j < J; ++j) {
        const int c = 8 * (t + threads * j);
        F2 o[4];
        norm_dx8(xh[j], e[j], rstd, s1, s2, o);
        store_pairs<YT, false>(dx + r * args.ldy + c, o, c < args.cols ? 8 : 0);
      }
      slot = slot + 1 == depth ? 0 : slot + 1;
    }
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
  if (!args.partial) return;
  const int64_t pitch = norm_sums_pitch(args.cols);
  float* out = args.partial + (int64_t)blockIdx.x * 2 * pitch;
#pragma unroll
  for (int j = 0; j < J; ++j) {
    const int c = 8 * (t + threads * j);
    if (c >= args.cols) continue;
    float a[8], b[8];
    to_floats(dg[j], a);
    to_floats(db[j], b);
    store_sums8(out + c, a);
    store_sums8(out + pitch + c, b);
  }
}

// dg and db from the CTAs' sums, in CTA order.  A CTA takes 32 of the 2 x pitch columns; each of its
// 16 warps takes every sixteenth sum, four at a time, and the warps' results are added in warp order.
__global__ void __launch_bounds__(512) layer_norm_fold_kernel(const float* partial, int parts, int cols,
                                                              float* dgamma, float* dbeta) {
  let_next_start();
  wait_for_previous();
  __shared__ float part[16][33];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t c = (int64_t)blockIdx.x * 32 + lane, half = norm_sums_pitch(cols), pitch = 2 * half;
  float s[4] = {0.f, 0.f, 0.f, 0.f};
  if (c < pitch) {
    const float* at = partial + c;
    int p = warp;
    for (; p + 48 < parts; p += 64) {
#pragma unroll
      for (int i = 0; i < 4; ++i) s[i] += at[(int64_t)(p + 16 * i) * pitch];
    }
    for (; p < parts; p += 16) s[0] += at[(int64_t)p * pitch];
  }
  part[warp][lane] = (s[0] + s[1]) + (s[2] + s[3]);
  __syncthreads();
  if (warp != 0 || c >= pitch) return;
  float total = 0.f;
#pragma unroll
  for (int w = 0; w < 16; ++w) total += part[w][lane];
  const int64_t col = c < half ? c : c - half;
  float* to = c < half ? dgamma : dbeta;
  if (to && col < cols) to[col] = total;
}

// Rows too long for the registers of a CTA: the same sums with the row read again for each (it
// comes from the second-level cache).  One CTA of 1024 threads per row, 8192 columns at a time.
template <int XT>
__global__ void __launch_bounds__(1024) layer_norm_fprop_long_kernel(const __grid_constant__ LayerNormArgs args) {
  let_next_start();
  wait_for_previous();
  typedef typename ElemOf<XT>::T T;
  __shared__ float slots[2][kNormMaxWarps];
  const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
  const int steps = (args.cols + 8191) / 8192;
  const T* x = static_cast<const T*>(args.x);
  T* y = static_cast<T*>(args.y);
  for (int64_t r = blockIdx.x; r < args.rows; r += gridDim.x) {
    float acc = 0.f, mean = 0.f, rstd = 0.f;
    for (int pass = 0; pass < 3; ++pass) {
      for (int j = 0; j < steps; ++j) {
        const int c = 8 * t + 8192 * j;
        const int n = min(max(args.cols - c, 0), 8);
        F2 v[4], none[4] = {};
        to_pairs<XT>(load_raw8<XT, true>(x + r * args.ldx + c, n), v);
        if (pass == 0) {
          acc += sum2(add2(add2(v[0], v[1]), add2(v[2], v[3])));
        } else if (pass == 1) {
          acc += squares8<true>(v, f2(-mean), n);
        } else {
          if (args.c)
            norm_pack<kEitherFp8, true>(v, none, args.q_e5m2, args.c + r * args.ldq + c, nullptr,
                                        args.sc + (int64_t)(c >> 7) * args.rows + r, nullptr, n, 0, lane);
          F2 g[4], b[4];
          load_weights8<true, true>(args.gamma, c, n, args.w_type, 1.f, g);
          load_weights8<true, true>(args.beta, c, n, args.w_type, 0.f, b);
          normalise8<true>(v, f2(-mean), f2(rstd), g, b, n);
          if (args.y) store_pairs<XT, true>(y + r * args.ldy + c, v, n);
          if (args.q)
            norm_pack<kEitherFp8, true>(v, none, args.q_e5m2, args.q + r * args.ldq + c, nullptr,
                                        args.s + (int64_t)(c >> 7) * args.rows + r, nullptr, n, 0, lane);
        }
      }
      if (pass == 2) break;
      acc = cta_sum(acc, slots[pass], lane, warp) * args.inv_cols;
      if (pass == 0) mean = acc;
      else rstd = 1.f / sqrtf(acc + args.eps);
      acc = 0.f;
    }
    if (t == 0) {
      if (args.mean) args.mean[r] = mean;
      if (args.rstd) args.rstd[r] = rstd;
    }
  }
}

// Long rows backward: the sums of a row, then dx; dg and db go to the CTA's sums in memory
// (this CTA alone writes them, each thread always the same columns).
template <int XT, int YT>
__global__ void __launch_bounds__(1024) layer_norm_bprop_long_kernel(const __grid_constant__ LayerNormArgs args) {
  let_next_start();
  wait_for_previous();
  constexpr bool EDGE = true;
  typedef typename ElemOf<XT>::T TX;
  typedef typename ElemOf<YT>::T TY;
  __shared__ float slots[2][2][kNormMaxWarps];
  const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
  const int steps = (args.cols + 8191) / 8192;
  const TX* x = static_cast<const TX*>(args.x);
  const TY* dy = static_cast<const TY*>(args.dy);
  const int64_t pitch = norm_sums_pitch(args.cols);
  float* out = args.partial ? args.partial + (int64_t)blockIdx.x * 2 * pitch : nullptr;
  bool first = true;
  int flip = 0;
  for (int64_t r = blockIdx.x; r < args.rows; r += gridDim.x, flip ^= 1) {
    const float mean = args.mean[r], rstd = args.rstd[r];
    float s1 = 0.f, s2 = 0.f;
    for (int pass = 0; pass < 2; ++pass) {
      for (int j = 0; j < steps; ++j) {
        const int c = 8 * t + 8192 * j;
        const int n = min(max(args.cols - c, 0), 8);
        float xh[8], e[8];
        to_float8<XT>(load_raw8<XT, EDGE>(x + r * args.ldx + c, n), xh);
        to_float8<YT>(load_raw8<YT, EDGE>(dy + r * args.ldy + c, n), e);
        float scale = 1.f;
        if constexpr (is_fp8(XT)) scale = n > 0 ? e8m0_value(args.x_scale[(int64_t)(c >> 7) * args.rows + r]) : 0.f;
        F2 g2[4];
        float g8[8], o[8], pg[8] = {}, pb[8] = {};
        const bool add = pass == 0 && out && n > 0;
        if (add && !first) {
          load_sums8(out + c, pg);
          load_sums8(out + pitch + c, pb);
        }
        load_weights8<true>(args.gamma, c, n, args.w_type, 1.f, g2);
        to_floats(g2, g8);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if constexpr (is_fp8(XT)) xh[i] *= scale;
          xh[i] = i < n ? (xh[i] - mean) * rstd : 0.f;
          const float g = g8[i];
          if (pass == 0) {
            pg[i] = fmaf(e[i], xh[i], pg[i]);
            pb[i] += e[i];
            s1 = fmaf(e[i], g, s1);
            s2 = fmaf(e[i] * g, xh[i], s2);
          } else {
            o[i] = rstd * (e[i] * g - s1 - xh[i] * s2);
          }
        }
        if (add) {
          store_sums8(out + c, pg);
          store_sums8(out + pitch + c, pb);
        }
        if (pass == 1) store_float8<YT, EDGE>(static_cast<TY*>(args.dx) + r * args.ldy + c, o, n);
      }
      if (pass == 1) break;
      s1 = warp_sum(s1);
      s2 = warp_sum(s2);
      if (lane == 0) {
        slots[flip][0][warp] = s1;
        slots[flip][1][warp] = s2;
      }
      __syncthreads();
      s1 = s2 = 0.f;
      for (int w = 0; w < 32; ++w) {
        s1 += slots[flip][0][w];
        s2 += slots[flip][1][w];
      }
      s1 *= args.inv_cols;
      s2 *= args.inv_cols;
    }
    first = false;
  }
}

}  // namespace maxdnn
