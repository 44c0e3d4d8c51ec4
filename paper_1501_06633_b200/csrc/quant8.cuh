// Packing of matrices into 8 bits with a scale for each block (rows, columns, tiles), from any
// wide type or from another packed matrix, and unpacking.
//
// One CTA takes a 128 x 128 tile of the matrix, which is whole blocks of every kind, so that one
// reading serves every packed form that is asked for.  Thread t holds eight neighbouring columns
// (8 (t mod 16)) of the eight rows t/16 + 16 k, as they lie in memory: 16 lanes cover a row
// block, and eight loads of 16 bytes are in flight in each thread.  Row maxima are shuffles over
// those 16 lanes; column maxima are a maximum over the thread's rows, a shuffle between the two
// halves of the warp and one pass through shared memory.  The values are converted again for each
// form instead of being kept as fp32 (64 registers of a thread).
//
// Measured: 8192 x 4096 bf16 to E5M2 rows and columns 31 us, 134 MB at 4.3 TB/s (copy: 6.5).  What
// takes the time: 20 M warp instructions at 0.63 a cycle with 24 warps an SM, 9.2 M of them (conversions, maxima,
// byte packing) at half rate, 16 us by themselves.  Packing 5000 x 2056 packed rows again in columns 10.2 to 11.9 us: 680
// tiles in one and a half rounds, and 96 bytes a thread spilled (the eight row scales).  Unpacking 70k x 128 to
// bf16: 27 MB in 5.7 us.
#pragma once
#include "fp8_util.cuh"

namespace maxdnn {

constexpr int kQuantThreads = 256;

struct Quant8Args {
  const void* x;
  const uint8_t* x_scale;      // packed x: its row scales
  uint8_t *q_row, *s_row, *q_col, *s_col, *q_tile, *s_tile;   // null: not asked for
  int64_t ldx, ldq;
  int32_t rows, cols;
  int32_t col_blocks;          // blocks of 128 columns
};

template <int XT, int QT, bool EDGE>
__global__ void __launch_bounds__(kQuantThreads, XT == MAXDNN_F32 ? 2 : 3) quant8_kernel(const __grid_constant__ Quant8Args args) {
  let_next_start();
  wait_for_previous();
  typedef typename ElemOf<XT>::T T;
  __shared__ float col_part[kQuantThreads / 32][kBlock8];   // per warp: maxima of its rows
  __shared__ float col_inv[kBlock8];
  __shared__ uint8_t row_byte[kBlock8];
  __shared__ float warp_max[kQuantThreads / 32];
  const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
  const int cb = blockIdx.x % args.col_blocks;
  const int rb = blockIdx.x / args.col_blocks;
  const int r0 = rb * kBlock8, c0 = cb * kBlock8 + 8 * (t & 15);
  const int n = vector_cols<EDGE>(args.cols, c0);
  const int rg = t >> 4;
  const T* x = static_cast<const T*>(args.x);
  Raw8<XT> raw[8];
  float xs[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const int r = r0 + rg + 16 * k;
    raw[k] = load_raw8<XT, EDGE, true>(x + (int64_t)r * args.ldx + c0, r < args.rows ? n : 0);
    if constexpr (is_fp8(XT))
      xs[k] = r < args.rows ? e8m0_value(args.x_scale[(int64_t)cb * args.rows + r]) : 0.f;
  }
  // the eight values of one of the thread's rows
  auto values = [&](int k, F2 (&v)[4]) {
    convert_again(raw[k]);
    to_pairs<XT>(raw[k], v);
    if constexpr (is_fp8(XT)) {
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = mul2(v[i], f2(xs[k]));
    }
  };
  const bool cols_wanted = args.q_col || args.q_tile;
  float row_max[8], col_max[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) col_max[i] = 0.f;
#pragma unroll
  for (int k = 0; k < 8; k += 2) {
    F2 v[4], w[4];
    values(k, v);
    values(k + 1, w);
    row_max[k] = max8(v);
    row_max[k + 1] = max8(w);
    if (cols_wanted) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 a = unf2(v[i]), b = unf2(w[i]);
        col_max[2 * i] = max3abs(col_max[2 * i], a.x, b.x);
        col_max[2 * i + 1] = max3abs(col_max[2 * i + 1], a.y, b.y);
      }
    }
  }
  float most = 0.f;
#pragma unroll
  for (int k = 0; k < 8; ++k) most = fmaxf(most, row_max[k]);
  const bool fix = __syncthreads_or(isinf(most)) != 0;   // rare: a tile that holds an infinity
  if (fix) {
#pragma unroll
    for (int i = 0; i < 8; ++i) col_max[i] = 0.f;
#pragma unroll 1
    for (int k = 0; k < 8; ++k) {
      // one row at a time, from memory again: registers cannot be indexed
      const int r = r0 + rg + 16 * k;
      float f[8];
      to_float8<XT>(load_raw8<XT, true>(x + (int64_t)r * args.ldx + c0, r < args.rows ? n : 0), f);
      float scale = 1.f, m = 0.f;
      if constexpr (is_fp8(XT)) scale = r < args.rows ? e8m0_value(args.x_scale[(int64_t)cb * args.rows + r]) : 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float a = is_fp8(XT) ? f[i] * scale : f[i];
        const float b = isinf(a) ? 0.f : fabsf(a);
        m = fmaxf(m, b);
        col_max[i] = fmaxf(col_max[i], b);
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) row_max[j] = j == k ? m : row_max[j];
    }
  }

  auto store = [&](uint8_t* q, int k, const F2 (&inv)[4]) {
    const int r = r0 + rg + 16 * k;
    if (r >= args.rows) return;
    F2 v[4];
    values(k, v);
    store_bytes8<EDGE>(q + (int64_t)r * args.ldq + c0, pack8<QT>(v, inv, fix), n);
  };

  if (args.q_row) {
#pragma unroll
    for (int k = 0; k < 8; k += 2) {
      uint32_t b[2];
      if (block_bytes<QT>(row_max[k], row_max[k + 1], &b[0], &b[1])) {
        b[0] = scale_byte<QT>(max_over_block_lanes(row_max[k]));
        b[1] = scale_byte<QT>(max_over_block_lanes(row_max[k + 1]));
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        if ((t & 15) == 0) row_byte[rg + 16 * (k + i)] = (uint8_t)b[i];
        const F2 inv = f2(inv_scale_of(b[i])), all[4] = {inv, inv, inv, inv};
        store(args.q_row, k + i, all);
      }
    }
  }
  if (cols_wanted) {
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
  if (args.q_row && t < kBlock8 && r0 + t < args.rows)
    args.s_row[(int64_t)cb * args.rows + r0 + t] = row_byte[t];
  if (!cols_wanted) return;
  if (t < kBlock8) {
    float m = 0.f;
#pragma unroll
    for (int w = 0; w < kQuantThreads / 32; ++w) m = fmaxf(m, col_part[w][t]);
    const uint32_t b = scale_byte<QT>(m);
    col_inv[t] = inv_scale_of(b);
    if (args.q_col && cb * kBlock8 + t < args.cols)
      args.s_col[(int64_t)rb * args.cols + cb * kBlock8 + t] = (uint8_t)b;
    m = max_over_block_lanes(m);
    m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, 16));
    if (lane == 0) warp_max[warp] = m;
  }
  __syncthreads();
  if (args.q_col) {
    F2 inv[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 c = *reinterpret_cast<const float2*>(&col_inv[8 * (t & 15) + 2 * i]);
      inv[i] = f2(c.x, c.y);
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) store(args.q_col, k, inv);
  }
  if (args.q_tile) {
    const uint32_t b = scale_byte<QT>(fmaxf(fmaxf(warp_max[0], warp_max[1]), fmaxf(warp_max[2], warp_max[3])));
    const F2 inv = f2(inv_scale_of(b)), all[4] = {inv, inv, inv, inv};
#pragma unroll
    for (int k = 0; k < 8; ++k) store(args.q_tile, k, all);
    if (t == 0) args.s_tile[(int64_t)rb * args.col_blocks + cb] = (uint8_t)b;
  }
}

struct Dequant8Args {
  const uint8_t *q, *s;
  void* x;
  int64_t ldx, ldq;
  int32_t rows, cols;
  int32_t col_blocks;
  int32_t block;               // maxdnn_block
};

// The same tile and the same eight columns x eight rows in each thread.
template <int XT, int QT, bool EDGE>
__global__ void __launch_bounds__(kQuantThreads) dequant8_kernel(const __grid_constant__ Dequant8Args args) {
  let_next_start();
  wait_for_previous();
  typedef typename ElemOf<XT>::T T;
  const int t = threadIdx.x;
  const int cb = blockIdx.x % args.col_blocks;
  const int rb = blockIdx.x / args.col_blocks;
  const int r0 = rb * kBlock8 + (t >> 4), c0 = cb * kBlock8 + 8 * (t & 15);
  const int n = vector_cols<EDGE>(args.cols, c0);
  if (n == 0) return;
  Raw8<QT> raw[8];
  uint32_t byte[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const int r = r0 + 16 * k;
    raw[k] = load_raw8<QT, EDGE>(args.q + (int64_t)r * args.ldq + c0, r < args.rows ? n : 0);
    byte[k] = 127;
    if (args.block == MAXDNN_BLOCK_ROW && r < args.rows) byte[k] = args.s[(int64_t)cb * args.rows + r];
  }
  float s[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) s[i] = 1.f;
  if (args.block == MAXDNN_BLOCK_COL) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) s[i] = e8m0_value(args.s[(int64_t)rb * args.cols + c0 + i]);
  } else if (args.block == MAXDNN_BLOCK_TILE) {
    const float one = e8m0_value(args.s[(int64_t)rb * args.col_blocks + cb]);
#pragma unroll
    for (int i = 0; i < 8; ++i) s[i] = one;
  }
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const int r = r0 + 16 * k;
    if (r >= args.rows) break;
    float v[8];
    to_float8<QT>(raw[k], v);
    const float m = e8m0_value(byte[k]);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = args.block == MAXDNN_BLOCK_ROW ? v[i] * m : v[i] * s[i];
    store_float8<XT, EDGE>(static_cast<T*>(args.x) + (int64_t)r * args.ldx + c0, v, n);
  }
}

}  // namespace maxdnn
