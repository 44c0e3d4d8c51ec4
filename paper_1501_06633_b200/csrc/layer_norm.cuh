// Layer norm over the last axis, forward and backward, with the packed forms that the 8-bit
// training step reads next.
//
//   mean = sum x / C,  rstd = 1 / sqrt(sum (x - mean)^2 / C + eps),  xh = (x - mean) rstd
//   y = xh g + b
//   dx = rstd (g dy - s1 - xh s2),  s1 = sum(g dy) / C,  s2 = sum(g dy xh) / C
//   dg = sum over rows of dy xh,  db = sum over rows of dy
//
// A row is read once and stays in registers: T threads (a warp, or a whole CTA) hold it as
// vectors of eight columns, vector j of thread t at column 8 (t + T j).  The variance is summed from the
// differences to the mean, not from squares, so a row far from zero loses nothing.  All sums are
// in 32 bits.  Sixteen neighbouring lanes hold a block of 128 columns, so the packed forms take
// four shuffles each.
#pragma once
#include "fp8_util.cuh"

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
  float* partial;              // [grid][2][cols] sums of a CTA's rows: dy xh, dy
  int64_t ldx, ldy, ldq;
  int32_t rows, cols, w_type;
  int32_t vec_x, vec_y, vec_w; // rows (weights) allow the wide loads
  int32_t q_e5m2;
  float eps, inv_cols;
};

constexpr int kNormMaxWarps = 32;

// Sum over the T threads of a row (T = 32: a warp).  `slot` alternates between two calls.
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
  return v;
}
template <bool WARP_ROW>
__device__ __forceinline__ float row_sum(float v, float* slot, int warps, int lane, int warp) {
  v = warp_sum(v);
  if constexpr (WARP_ROW) return v;
  if (lane == 0) slot[warp] = v;
  __syncthreads();
  float s = 0.f;
  for (int w = 0; w < warps; ++w) s += slot[w];
  return s;
}

// Packs eight values of a row block (16 lanes) and stores them with the block's scale.
template <bool EDGE>
__device__ __forceinline__ void norm_pack(const float (&v)[8], bool e5m2, uint8_t* q, uint8_t* s, int n, int lane) {
  float m = max_over_block_lanes(max8(v));
  const bool fix = isinf(m);
  if (__any_sync(0xFFFFFFFFu, fix)) m = max_over_block_lanes(finite_max8(v));
  const uint32_t byte = scale_byte_of(m, e5m2);
  store_bytes8<EDGE>(q, pack8_as(v, inv_scale_of(byte), fix, e5m2), n, true);
  if ((lane & 15) == 0 && n > 0) *s = (uint8_t)byte;
}

// Eight neighbouring weights.
template <bool EDGE>
__device__ __forceinline__ void load_weights8(const void* p, int c, int n, int type, bool vec, float none, float (&w)[8]) {
  if (!p || n == 0) {
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = none;
  } else if (type == MAXDNN_F32) {
    to_float8<MAXDNN_F32>(load_raw8<MAXDNN_F32, EDGE>(static_cast<const float*>(p) + c, n, vec), w);
  } else if (type == MAXDNN_BF16) {
    to_float8<MAXDNN_BF16>(load_raw8<MAXDNN_BF16, EDGE>(static_cast<const __nv_bfloat16*>(p) + c, n, vec), w);
  } else {
    to_float8<MAXDNN_F16>(load_raw8<MAXDNN_F16, EDGE>(static_cast<const __half*>(p) + c, n, vec), w);
  }
}

// WR warps have a row, vector j of the row's thread t at column 8 (t + 32 WR j); a CTA of eight
// warps has 8 / WR rows at a time.  The row stays as it was loaded (4 J registers of 16-bit values) and is
// converted again for each of the three sums; a warp alone needs no barrier, and its J loads of
// 16 bytes a lane are all in flight.  8192 x 4096 bf16 with packed y and x: a CTA per row with the row
// as fp32 registers took 102 us.
constexpr int kNormThreads = 256;
template <int XT, int J, int WR, bool EDGE>
__global__ void __launch_bounds__(kNormThreads, J >= 16 || (J >= 8 && XT == MAXDNN_F32) ? 2 : J >= 4 ? 3 : 4)
layer_norm_fprop_kernel(const __grid_constant__ LayerNormArgs args) {
  typedef typename ElemOf<XT>::T T;
  __shared__ float slots[8 / WR][2][WR];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int group = warp / WR, in_row = warp % WR, t = in_row * 32 + lane;
  const T* x = static_cast<const T*>(args.x);
  T* y = static_cast<T*>(args.y);
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
      raw[j] = load_raw8<XT, EDGE>(x + r * args.ldx + c, min(max(args.cols - c, 0), 8), args.vec_x != 0);
    }
    float sum = 0.f;
#pragma unroll
    for (int j = 0; j < J; ++j) {
      float v[8];
      to_float8<XT>(raw[j], v);
      sum += ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
    }
    const float mean = total(sum, 0) * args.inv_cols;
    float sq = 0.f;
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const int n = args.cols - 8 * (t + 32 * WR * j);
      float v[8], part = 0.f;
      convert_again(raw[j]);
      to_float8<XT>(raw[j], v);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float d = v[i] - mean;
        if (EDGE ? i < n : n > 0) part = fmaf(d, d, part);
      }
      sq += part;
    }
    const float rstd = 1.f / sqrtf(total(sq, 1) * args.inv_cols + args.eps);
    if (t == 0) {
      if (args.mean) args.mean[r] = mean;
      if (args.rstd) args.rstd[r] = rstd;
    }
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const int c = 8 * (t + 32 * WR * j);
      const int n = min(max(args.cols - c, 0), 8);
      float v[8];
      convert_again(raw[j]);
      to_float8<XT>(raw[j], v);
      if (args.c) norm_pack<EDGE>(v, args.q_e5m2, args.c + r * args.ldq + c, args.sc + (int64_t)(c >> 7) * args.rows + r, n, lane);
      if (!args.y && !args.q) continue;
      asm volatile("" ::: "memory");      // the weights of one vector at a time: their registers are short
      float g[8], b[8];
      load_weights8<EDGE>(args.gamma, c, n, args.w_type, args.vec_w != 0, 1.f, g);
      load_weights8<EDGE>(args.beta, c, n, args.w_type, args.vec_w != 0, 0.f, b);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = (EDGE ? i < n : n > 0) ? fmaf((v[i] - mean) * rstd, g[i], b[i]) : 0.f;
      if (args.y) store_float8<XT, EDGE>(y + r * args.ldy + c, v, n, args.vec_y != 0);
      if (args.q) norm_pack<EDGE>(v, args.q_e5m2, args.q + r * args.ldq + c, args.s + (int64_t)(c >> 7) * args.rows + r, n, lane);
    }
    // no barrier here: a thread reaches the next row's first write of a slot only after the
    // second sum's barrier, which follows every read of the first slot (and the other way round)
  }
}

// XT: the type of x (wide, or packed rows); YT: of dy and dx.
template <int XT, int YT, int J, bool WARP_ROW, bool EDGE>
__global__ void __launch_bounds__(WARP_ROW ? 128 : 512)
layer_norm_bprop_kernel(const __grid_constant__ LayerNormArgs args) {
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
  float g[J][8], dg[J][8], db[J][8];
#pragma unroll
  for (int j = 0; j < J; ++j)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int c = 8 * (t + threads * j) + i;
      g[j][i] = (args.gamma && c < args.cols) ? load_weight(args.gamma, c, args.w_type) : 1.f;
      dg[j][i] = db[j][i] = 0.f;
    }
  int flip = 0;
  for (int64_t r = (int64_t)blockIdx.x * per_cta + (WARP_ROW ? warp : 0); r < args.rows;
       r += (int64_t)gridDim.x * per_cta, flip ^= 1) {
    const float mean = args.mean[r], rstd = args.rstd[r];
    float xh[J][8], e[J][8];
    float s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const int c = 8 * (t + threads * j);
      const int n = min(max(args.cols - c, 0), 8);
      to_float8<XT>(load_raw8<XT, EDGE>(x + r * args.ldx + c, n, args.vec_x != 0), xh[j]);
      to_float8<YT>(load_raw8<YT, EDGE>(dy + r * args.ldy + c, n, args.vec_y != 0), e[j]);
      float scale = 1.f;
      if constexpr (is_fp8(XT)) scale = n > 0 ? e8m0_value(args.x_scale[(int64_t)(c >> 7) * args.rows + r]) : 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if constexpr (is_fp8(XT)) xh[j][i] *= scale;
        xh[j][i] = (EDGE ? i < n : n > 0) ? (xh[j][i] - mean) * rstd : 0.f;
        dg[j][i] = fmaf(e[j][i], xh[j][i], dg[j][i]);
        db[j][i] += e[j][i];
        e[j][i] *= g[j][i];
        s1 += e[j][i];
        s2 = fmaf(e[j][i], xh[j][i], s2);
      }
    }
    s1 = warp_sum(s1);
    s2 = warp_sum(s2);
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
      const int n = min(max(args.cols - c, 0), 8);
      float o[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) o[i] = rstd * (e[j][i] - s1 - xh[j][i] * s2);
      store_float8<YT, EDGE>(dx + r * args.ldy + c, o, n, args.vec_y != 0);
    }
  }
  if (!args.partial) return;
  // this CTA's sums over its rows; a CTA of several rows adds them warp by warp
  float* out = args.partial + (int64_t)blockIdx.x * 2 * args.cols;
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    if constexpr (WARP_ROW) {
      for (int w = 0; w < warps; ++w) {
        if (warp == w) {
#pragma unroll
          for (int j = 0; j < J; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              float& f = fold[(i * J + j) * 32 + lane];
              const float a = which ? db[j][i] : dg[j][i];
              f = w == 0 ? a : f + a;
            }
        }
        __syncthreads();
      }
      for (int c = threadIdx.x; c < args.cols; c += blockDim.x) {
        const int vecj = c >> 8, l = (c >> 3) & 31, i = c & 7;
        out[(int64_t)which * args.cols + c] = fold[(i * J + vecj) * 32 + l];
      }
      __syncthreads();
    } else {
#pragma unroll
      for (int j = 0; j < J; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int c = 8 * (t + threads * j) + i;
          if (c < args.cols) out[(int64_t)which * args.cols + c] = which ? db[j][i] : dg[j][i];
        }
    }
  }
}

// dg and db from the CTAs' sums, in CTA order.  A CTA takes 32 columns; its eight warps take
// every eighth sum each and are added in warp order.
__global__ void __launch_bounds__(256) layer_norm_fold_kernel(const float* partial, int parts, int cols,
                                                              float* dgamma, float* dbeta) {
  __shared__ float part[8][33];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t c = (int64_t)blockIdx.x * 32 + lane;     // of the 2 x cols sums
  float s = 0.f;
  if (c < 2 * (int64_t)cols)
    for (int p = warp; p < parts; p += 8) s += partial[(int64_t)p * 2 * cols + c];
  part[warp][lane] = s;
  __syncthreads();
  if (warp != 0 || c >= 2 * (int64_t)cols) return;
  s = 0.f;
#pragma unroll
  for (int w = 0; w < 8; ++w) s += part[w][lane];
  if (c < cols) { if (dgamma) dgamma[c] = s; }
  else if (dbeta) dbeta[c - cols] = s;
}

// Rows too long for the registers of a CTA: the same sums with the row read again for each (it
// comes from the second-level cache).  One CTA of 1024 threads per row, 8192 columns at a time.
template <int XT>
__global__ void __launch_bounds__(1024) layer_norm_fprop_long_kernel(const __grid_constant__ LayerNormArgs args) {
  constexpr bool EDGE = true;
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
        float v[8];
        to_float8<XT>(load_raw8<XT, EDGE>(x + r * args.ldx + c, n, args.vec_x != 0), v);
        if (pass == 0) {
#pragma unroll
          for (int i = 0; i < 8; ++i) acc += v[i];
        } else if (pass == 1) {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float d = i < n ? v[i] - mean : 0.f;
            acc = fmaf(d, d, acc);
          }
        } else {
          if (args.c) norm_pack<EDGE>(v, args.q_e5m2, args.c + r * args.ldq + c, args.sc + (int64_t)(c >> 7) * args.rows + r, n, lane);
          float g[8], b[8];
          load_weights8<EDGE>(args.gamma, c, n, args.w_type, args.vec_w != 0, 1.f, g);
          load_weights8<EDGE>(args.beta, c, n, args.w_type, args.vec_w != 0, 0.f, b);
#pragma unroll
          for (int i = 0; i < 8; ++i) v[i] = (EDGE ? i < n : n > 0) ? fmaf((v[i] - mean) * rstd, g[i], b[i]) : 0.f;
          if (args.y) store_float8<XT, EDGE>(y + r * args.ldy + c, v, n, args.vec_y != 0);
          if (args.q) norm_pack<EDGE>(v, args.q_e5m2, args.q + r * args.ldq + c, args.s + (int64_t)(c >> 7) * args.rows + r, n, lane);
        }
      }
      if (pass == 2) break;
      acc = row_sum<false>(acc, slots[pass], 32, lane, warp) * args.inv_cols;
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
  constexpr bool EDGE = true;
  typedef typename ElemOf<XT>::T TX;
  typedef typename ElemOf<YT>::T TY;
  __shared__ float slots[2][2][kNormMaxWarps];
  const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
  const int steps = (args.cols + 8191) / 8192;
  const TX* x = static_cast<const TX*>(args.x);
  const TY* dy = static_cast<const TY*>(args.dy);
  float* out = args.partial ? args.partial + (int64_t)blockIdx.x * 2 * args.cols : nullptr;
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
        to_float8<XT>(load_raw8<XT, EDGE>(x + r * args.ldx + c, n, args.vec_x != 0), xh);
        to_float8<YT>(load_raw8<YT, EDGE>(dy + r * args.ldy + c, n, args.vec_y != 0), e);
        float scale = 1.f;
        if constexpr (is_fp8(XT)) scale = n > 0 ? e8m0_value(args.x_scale[(int64_t)(c >> 7) * args.rows + r]) : 0.f;
        float o[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if constexpr (is_fp8(XT)) xh[i] *= scale;
          xh[i] = i < n ? (xh[i] - mean) * rstd : 0.f;
          const float g = (args.gamma && i < n) ? load_weight(args.gamma, c + i, args.w_type) : 1.f;
          if (pass == 0) {
            if (out && i < n) {
              float* pg = out + c + i;
              float* pb = pg + args.cols;
              *pg = first ? e[i] * xh[i] : fmaf(e[i], xh[i], *pg);
              *pb = first ? e[i] : *pb + e[i];
            }
            s1 = fmaf(e[i], g, s1);
            s2 = fmaf(e[i] * g, xh[i], s2);
          } else {
            o[i] = rstd * (e[i] * g - s1 - xh[i] * s2);
          }
        }
        if (pass == 1) store_float8<YT, EDGE>(static_cast<TY*>(args.dx) + r * args.ldy + c, o, n, args.vec_y != 0);
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
