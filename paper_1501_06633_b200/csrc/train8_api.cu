// C ABI of the 8-bit training operators but the matrix product (see include/maxdnn.h): argument
// checks and kernel launches.
#include "act8.cuh"
#include "layer_norm.cuh"
#include "plan.h"
#include "quant8.cuh"
#include "runtime.h"

namespace maxdnn {
namespace {

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
int64_t blocks_of(int64_t n) { return (n + kBlock8 - 1) / kBlock8; }

// Whether rows of `ld` elements of type `dt` that start `off` elements in allow loads of eight values.
int vec_ok(int dt, int64_t ld, int64_t off = 0) {
  const int64_t unit = is_fp8(dt) ? 8 : 16;
  return (ld * elem_bytes(dt)) % unit == 0 && (off * elem_bytes(dt)) % unit == 0;
}

maxdnn_status launched() {
  if (cudaGetLastError() != cudaSuccess) return MAXDNN_CUDA_ERROR;
  runtime_count_launch();
  return MAXDNN_OK;
}

// ---- type dispatch: calls f with integral constants ----
template <int V> struct Const { static constexpr int value = V; };

template <class F>
maxdnn_status by_wide(int type, F f) {
  if (type == MAXDNN_F32) return f(Const<MAXDNN_F32>());
  if (type == MAXDNN_BF16) return f(Const<MAXDNN_BF16>());
  if (type == MAXDNN_F16) return f(Const<MAXDNN_F16>());
  return MAXDNN_INVALID_VALUE;
}
template <class F>
maxdnn_status by_fp8(int type, F f) {
  if (type == MAXDNN_E4M3) return f(Const<MAXDNN_E4M3>());
  if (type == MAXDNN_E5M2) return f(Const<MAXDNN_E5M2>());
  return MAXDNN_INVALID_VALUE;
}
template <class F>
maxdnn_status by_any(int type, F f) {
  return is_fp8(type) ? by_fp8(type, f) : by_wide(type, f);
}
// whole: all vectors of eight columns are whole and aligned (see load_raw8)
template <class F>
maxdnn_status by_edge(bool whole, F f) {
  return whole ? f(Const<0>()) : f(Const<1>());
}

// ------------------------------------------------------------------ packing
maxdnn_status check_quant8(const maxdnn_quant8_desc* d) {
  if (!d || d->rows < 0 || d->cols < 0) return MAXDNN_INVALID_VALUE;
  if (!is_fp8(d->q_type) || (!is_fp8(d->x_type) && !is_wide(d->x_type))) return MAXDNN_INVALID_VALUE;
  if (d->ldx < d->cols || d->ldq < d->cols) return MAXDNN_INVALID_VALUE;
  if (blocks_of(d->rows) * blocks_of(d->cols) > 0x7FFFFFFF) return MAXDNN_NOT_SUPPORTED;
  return MAXDNN_OK;
}

maxdnn_status quant8(const maxdnn_quant8_desc* d, const void* x, const void* x_scale, void* q_row, void* s_row,
                     void* q_col, void* s_col, void* q_tile, void* s_tile, cudaStream_t stream) {
  maxdnn_status st = check_quant8(d);
  if (st != MAXDNN_OK) return st;
  if (d->rows == 0 || d->cols == 0) return MAXDNN_OK;
  if (!q_row && !q_col && !q_tile) return MAXDNN_INVALID_VALUE;
  if ((q_row && !s_row) || (q_col && !s_col) || (q_tile && !s_tile)) return MAXDNN_INVALID_VALUE;
  if (is_fp8(d->x_type) && !x_scale) return MAXDNN_INVALID_VALUE;
  if (!x || !aligned16(x) || !aligned16(q_row) || !aligned16(q_col) || !aligned16(q_tile)) return MAXDNN_INVALID_VALUE;
  if (d->ldq % 16 != 0) return MAXDNN_NOT_SUPPORTED;
  RuntimeDevice dev;
  if ((st = runtime_device(&dev)) != MAXDNN_OK) return st;
  Quant8Args a = {};
  a.x = x;
  a.x_scale = static_cast<const uint8_t*>(x_scale);
  a.q_row = static_cast<uint8_t*>(q_row);
  a.s_row = static_cast<uint8_t*>(s_row);
  a.q_col = static_cast<uint8_t*>(q_col);
  a.s_col = static_cast<uint8_t*>(s_col);
  a.q_tile = static_cast<uint8_t*>(q_tile);
  a.s_tile = static_cast<uint8_t*>(s_tile);
  a.ldx = d->ldx;
  a.ldq = d->ldq;
  a.rows = d->rows;
  a.cols = d->cols;
  a.col_blocks = (int32_t)blocks_of(d->cols);
  a.vec_x = vec_ok(d->x_type, d->ldx);
  const unsigned grid = (unsigned)(blocks_of(d->rows) * blocks_of(d->cols));
  a.e5m2 = d->q_type == MAXDNN_E5M2;
  return by_any(d->x_type, [&](auto xt) {
    return by_edge(a.vec_x && d->cols % 8 == 0, [&](auto edge) {
      quant8_kernel<decltype(xt)::value, decltype(edge)::value != 0><<<grid, kQuantThreads, 0, stream>>>(a);
      return launched();
    });
  });
}

maxdnn_status dequant8(const maxdnn_quant8_desc* d, int block, const void* q, const void* s, void* x,
                       cudaStream_t stream) {
  maxdnn_status st = check_quant8(d);
  if (st != MAXDNN_OK) return st;
  if (d->rows == 0 || d->cols == 0) return MAXDNN_OK;
  if (!is_wide(d->x_type)) return MAXDNN_INVALID_VALUE;
  if (block != MAXDNN_BLOCK_ROW && block != MAXDNN_BLOCK_COL && block != MAXDNN_BLOCK_TILE) return MAXDNN_INVALID_VALUE;
  if (!q || !s || !x || !aligned16(q) || !aligned16(x)) return MAXDNN_INVALID_VALUE;
  RuntimeDevice dev;
  if ((st = runtime_device(&dev)) != MAXDNN_OK) return st;
  Dequant8Args a = {};
  a.q = static_cast<const uint8_t*>(q);
  a.s = static_cast<const uint8_t*>(s);
  a.x = x;
  a.ldx = d->ldx;
  a.ldq = d->ldq;
  a.rows = d->rows;
  a.cols = d->cols;
  a.col_blocks = (int32_t)blocks_of(d->cols);
  a.block = block;
  a.vec_x = vec_ok(d->x_type, d->ldx);
  a.vec_q = vec_ok(d->q_type, d->ldq);
  const unsigned grid = (unsigned)(blocks_of(d->rows) * blocks_of(d->cols));
  return by_wide(d->x_type, [&](auto xt) {
    return by_fp8(d->q_type, [&](auto qt) {
      return by_edge(a.vec_x && a.vec_q && d->cols % 8 == 0, [&](auto edge) {
        dequant8_kernel<decltype(xt)::value, decltype(qt)::value, decltype(edge)::value != 0>
            <<<grid, kQuantThreads, 0, stream>>>(a);
        return launched();
      });
    });
  });
}

// --------------------------------------------------------------- layer norm
// How the backward pass lays a row out over threads: `j` vectors of eight columns in each of
// `threads` (32: a warp per row, four rows per CTA); threads = 0: the kernel that reads the row again.
struct NormShape { int threads, j; };
NormShape norm_shape(int cols) {
  if (cols <= 256) return {32, 1};
  if (cols <= 512) return {32, 2};
  if (cols <= 1024) return {32, 4};
  for (int t = 128; t <= 512; t *= 2)
    if (cols <= t * 16) return {t, 2};
  return {0, 0};
}

maxdnn_status check_layer_norm(const maxdnn_layer_norm_desc* d) {
  if (!d || d->rows < 0 || d->cols <= 0) return MAXDNN_INVALID_VALUE;
  if (!is_wide(d->y_type) || !is_wide(d->w_type) || (!is_wide(d->x_type) && !is_fp8(d->x_type))) return MAXDNN_INVALID_VALUE;
  if (d->ldx < d->cols || d->ldy < d->cols) return MAXDNN_INVALID_VALUE;
  if (!(d->eps >= 0.f) || d->eps > 3.0e38f) return MAXDNN_INVALID_VALUE;
  if (is_wide(d->x_type) && d->x_type != d->y_type) return MAXDNN_NOT_SUPPORTED;
  return MAXDNN_OK;
}

// CTAs of the backward pass: each leaves one row of sums.
int norm_bprop_grid(const maxdnn_layer_norm_desc& d, int sm_count, const NormShape& s) {
  const int64_t units = s.threads == 32 ? (d.rows + 3) / 4 : d.rows;
  const int per_sm = s.threads == 0 ? 1 : s.threads >= 512 ? 1 : s.threads == 32 ? 4 : 512 / s.threads;
  const int64_t most = (int64_t)sm_count * per_sm;
  return (int)(units < most ? units : most);
}

template <int XT, int J, int WR>
maxdnn_status launch_norm_rows(const LayerNormArgs& a, int sm_count, cudaStream_t stream) {
  const int64_t units = ((int64_t)a.rows + 8 / WR - 1) / (8 / WR);
  const int64_t most = (int64_t)sm_count * 4;
  return by_edge(a.vec_x && a.vec_y && a.vec_w && a.cols % 8 == 0, [&](auto edge) {
    layer_norm_fprop_kernel<XT, J, WR, decltype(edge)::value != 0>
        <<<(unsigned)(units < most ? units : most), kNormThreads, 0, stream>>>(a);
    return launched();
  });
}

// Vectors of eight columns per thread (J) and warps per row (WR).  Few rows (fewer than the SMs
// hold warps): eight warps share a row, for the latency.  Else as few warps as hold the row in
// registers.  Rows beyond that are read again for each sum.
template <int XT>
maxdnn_status launch_norm_fprop(const LayerNormArgs& a, int sm_count, cudaStream_t stream) {
  constexpr int kMost = XT == MAXDNN_F32 ? 8 : 16;
  const int vecs = (a.cols + 7) / 8;
  if (a.rows < 4 * sm_count && vecs > 32) {
    if (vecs <= 256) return launch_norm_rows<XT, 1, 8>(a, sm_count, stream);
    if (vecs <= 512) return launch_norm_rows<XT, 2, 8>(a, sm_count, stream);
    if (vecs <= 1024) return launch_norm_rows<XT, 4, 8>(a, sm_count, stream);
  }
  if (vecs <= 32) return launch_norm_rows<XT, 1, 1>(a, sm_count, stream);
  if (vecs <= 64) return launch_norm_rows<XT, 2, 1>(a, sm_count, stream);
  if (vecs <= 128) return launch_norm_rows<XT, 4, 1>(a, sm_count, stream);
  if (vecs <= 256) return launch_norm_rows<XT, 8, 1>(a, sm_count, stream);
  if (vecs <= 32 * kMost) return launch_norm_rows<XT, kMost, 1>(a, sm_count, stream);
  if (vecs <= 64 * kMost) return launch_norm_rows<XT, kMost, 2>(a, sm_count, stream);
  if (vecs <= 128 * kMost) return launch_norm_rows<XT, kMost, 4>(a, sm_count, stream);
  if (vecs <= 256 * kMost) return launch_norm_rows<XT, kMost, 8>(a, sm_count, stream);
  const int64_t most = 2 * (int64_t)sm_count;
  layer_norm_fprop_long_kernel<XT><<<(unsigned)(a.rows < most ? a.rows : most), 1024, 0, stream>>>(a);
  return launched();
}

maxdnn_status layer_norm_fprop(const maxdnn_layer_norm_desc* d, const void* x, const void* gamma, const void* beta,
                               void* y, float* mean, float* rstd, void* q, void* s, void* c, void* sc,
                               cudaStream_t stream) {
  maxdnn_status st = check_layer_norm(d);
  if (st != MAXDNN_OK) return st;
  if (d->rows == 0) return MAXDNN_OK;
  if (!is_wide(d->x_type)) return MAXDNN_INVALID_VALUE;
  if (!x || (!y && !mean && !rstd && !q && !c)) return MAXDNN_INVALID_VALUE;
  if ((q && !s) || (c && !sc)) return MAXDNN_INVALID_VALUE;
  if (!aligned16(x) || !aligned16(y) || !aligned16(q) || !aligned16(c)) return MAXDNN_INVALID_VALUE;
  if (q || c) {
    if (!is_fp8(d->q_type) || d->ldq < d->cols) return MAXDNN_INVALID_VALUE;
    if (d->ldq % 16 != 0) return MAXDNN_NOT_SUPPORTED;
  }
  RuntimeDevice dev;
  if ((st = runtime_device(&dev)) != MAXDNN_OK) return st;
  LayerNormArgs a = {};
  a.x = x;
  a.gamma = gamma;
  a.beta = beta;
  a.y = y;
  a.mean = mean;
  a.rstd = rstd;
  a.q = static_cast<uint8_t*>(q);
  a.s = static_cast<uint8_t*>(s);
  a.c = static_cast<uint8_t*>(c);
  a.sc = static_cast<uint8_t*>(sc);
  a.ldx = d->ldx;
  a.ldy = d->ldy;
  a.ldq = d->ldq;
  a.rows = d->rows;
  a.cols = d->cols;
  a.w_type = d->w_type;
  a.vec_x = vec_ok(d->x_type, d->ldx);
  a.vec_y = vec_ok(d->y_type, d->ldy);
  a.eps = d->eps;
  a.inv_cols = 1.f / (float)d->cols;
  a.vec_w = aligned16(gamma) && aligned16(beta);
  a.q_e5m2 = (q || c) && d->q_type == MAXDNN_E5M2;
  return by_wide(d->x_type, [&](auto xt) { return launch_norm_fprop<decltype(xt)::value>(a, dev.sm_count, stream); });
}

maxdnn_status layer_norm_bprop_workspace(const maxdnn_layer_norm_desc* d, size_t* bytes) {
  maxdnn_status st = check_layer_norm(d);
  if (st != MAXDNN_OK || !bytes) return st != MAXDNN_OK ? st : MAXDNN_INVALID_VALUE;
  int sm_count = option(OPT_SM_COUNT);   // planning without a device (tests)
  if (sm_count <= 0) {
    RuntimeDevice dev;
    if ((st = runtime_device(&dev)) != MAXDNN_OK) return st;
    sm_count = dev.sm_count;
  }
  *bytes = (size_t)norm_bprop_grid(*d, sm_count, norm_shape(d->cols)) * 2 * (size_t)d->cols * 4;
  return MAXDNN_OK;
}

maxdnn_status layer_norm_bprop(const maxdnn_layer_norm_desc* d, const void* dy, const void* x, const void* x_scale,
                               const void* gamma, const float* mean, const float* rstd, void* dx, float* dgamma,
                               float* dbeta, void* workspace, size_t workspace_bytes, cudaStream_t stream) {
  maxdnn_status st = check_layer_norm(d);
  if (st != MAXDNN_OK) return st;
  if (d->rows == 0) {     // sums over no rows
    if ((dgamma && cudaMemsetAsync(dgamma, 0, (size_t)d->cols * 4, stream) != cudaSuccess) ||
        (dbeta && cudaMemsetAsync(dbeta, 0, (size_t)d->cols * 4, stream) != cudaSuccess)) {
      cudaGetLastError();
      return MAXDNN_CUDA_ERROR;
    }
    return MAXDNN_OK;
  }
  if (!dy || !x || !mean || !rstd || !dx) return MAXDNN_INVALID_VALUE;
  if (is_fp8(d->x_type) && !x_scale) return MAXDNN_INVALID_VALUE;
  if (!aligned16(dy) || !aligned16(x) || !aligned16(dx)) return MAXDNN_INVALID_VALUE;
  RuntimeDevice dev;
  if ((st = runtime_device(&dev)) != MAXDNN_OK) return st;
  const NormShape sh = norm_shape(d->cols);
  const int grid = norm_bprop_grid(*d, dev.sm_count, sh);
  const bool sums = dgamma || dbeta;
  if (sums && (!workspace || !aligned16(workspace) || workspace_bytes < (size_t)grid * 2 * (size_t)d->cols * 4))
    return MAXDNN_INVALID_VALUE;
  LayerNormArgs a = {};
  a.x = x;
  a.x_scale = static_cast<const uint8_t*>(x_scale);
  a.gamma = gamma;
  a.mean = const_cast<float*>(mean);
  a.rstd = const_cast<float*>(rstd);
  a.dy = dy;
  a.dx = dx;
  a.partial = sums ? static_cast<float*>(workspace) : nullptr;
  a.ldx = d->ldx;
  a.ldy = d->ldy;
  a.rows = d->rows;
  a.cols = d->cols;
  a.w_type = d->w_type;
  a.vec_x = vec_ok(d->x_type, d->ldx);
  a.vec_y = vec_ok(d->y_type, d->ldy);
  a.inv_cols = 1.f / (float)d->cols;
  auto run = [&](auto xt, auto yt) {
    constexpr int X = decltype(xt)::value, Y = decltype(yt)::value;
    if (sh.threads == 0) {
      layer_norm_bprop_long_kernel<X, Y><<<grid, 1024, 0, stream>>>(a);
      return launched();
    }
    return by_edge(a.vec_x && a.vec_y && d->cols % 8 == 0, [&](auto edge) {
      constexpr bool E = decltype(edge)::value != 0;
      if (sh.threads == 32 && sh.j == 1) layer_norm_bprop_kernel<X, Y, 1, true, E><<<grid, 128, 0, stream>>>(a);
      else if (sh.threads == 32 && sh.j == 2) layer_norm_bprop_kernel<X, Y, 2, true, E><<<grid, 128, 0, stream>>>(a);
      else if (sh.threads == 32) layer_norm_bprop_kernel<X, Y, 4, true, E><<<grid, 128, 0, stream>>>(a);
      else layer_norm_bprop_kernel<X, Y, 2, false, E><<<grid, sh.threads, 0, stream>>>(a);
      return launched();
    });
  };
  st = by_wide(d->y_type, [&](auto yt) {
    if (is_fp8(d->x_type)) return by_fp8(d->x_type, [&](auto xt) { return run(xt, yt); });
    return run(yt, yt);
  });
  if (st != MAXDNN_OK || !sums) return st;
  layer_norm_fold_kernel<<<(unsigned)((2 * (int64_t)d->cols + 31) / 32), 256, 0, stream>>>(a.partial, grid, d->cols,
                                                                                          dgamma, dbeta);
  return launched();
}

// --------------------------------------------------------------- activation
maxdnn_status check_act8(const maxdnn_act8_desc* d) {
  if (!d || d->rows < 0 || d->cols < 0) return MAXDNN_INVALID_VALUE;
  if (!is_wide(d->x_type)) return MAXDNN_INVALID_VALUE;
  if (d->act != MAXDNN_ACT_SILU && d->act != MAXDNN_ACT_GELU && d->act != MAXDNN_ACT_GELU_TANH) return MAXDNN_INVALID_VALUE;
  if (d->gated != 0 && d->gated != 1) return MAXDNN_INVALID_VALUE;
  if (d->cols > (1 << 30)) return MAXDNN_NOT_SUPPORTED;
  if (d->ldh < (int64_t)d->cols * (1 + d->gated)) return MAXDNN_INVALID_VALUE;
  if (((int64_t)d->rows + kActRows - 1) / kActRows * blocks_of(d->cols) > 0x7FFFFFFF) return MAXDNN_NOT_SUPPORTED;
  return MAXDNN_OK;
}

template <class F>
maxdnn_status by_act(const maxdnn_act8_desc* d, F f) {
  auto gated = [&](auto act) { return d->gated ? f(act, Const<1>()) : f(act, Const<0>()); };
  if (d->act == MAXDNN_ACT_SILU) return gated(Const<MAXDNN_ACT_SILU>());
  if (d->act == MAXDNN_ACT_GELU) return gated(Const<MAXDNN_ACT_GELU>());
  return gated(Const<MAXDNN_ACT_GELU_TANH>());
}

maxdnn_status act8_fprop(const maxdnn_act8_desc* d, const void* h, void* a_out, void* q, void* s, void* c, void* sc,
                         cudaStream_t stream) {
  maxdnn_status st = check_act8(d);
  if (st != MAXDNN_OK) return st;
  if (d->rows == 0 || d->cols == 0) return MAXDNN_OK;
  if (!h || (!a_out && !q)) return MAXDNN_INVALID_VALUE;
  if ((q && !s) || (c && !sc)) return MAXDNN_INVALID_VALUE;
  if (!aligned16(h) || !aligned16(a_out) || !aligned16(q) || !aligned16(c)) return MAXDNN_INVALID_VALUE;
  if (a_out && d->lda < d->cols) return MAXDNN_INVALID_VALUE;
  if (q || c) {
    if (!is_fp8(d->q_type)) return MAXDNN_INVALID_VALUE;
    if (q && d->ldq < d->cols) return MAXDNN_INVALID_VALUE;
    if (c && d->ldc < (int64_t)d->cols * (1 + d->gated)) return MAXDNN_INVALID_VALUE;
    if ((q && d->ldq % 16 != 0) || (c && d->ldc % 16 != 0)) return MAXDNN_NOT_SUPPORTED;
  }
  RuntimeDevice dev;
  if ((st = runtime_device(&dev)) != MAXDNN_OK) return st;
  Act8Args a = {};
  a.h = h;
  a.a = a_out;
  a.q = static_cast<uint8_t*>(q);
  a.s = static_cast<uint8_t*>(s);
  a.c = static_cast<uint8_t*>(c);
  a.sc = static_cast<uint8_t*>(sc);
  a.ldh = d->ldh;
  a.lda = d->lda;
  a.ldq = d->ldq;
  a.ldc = d->ldc;
  a.rows = d->rows;
  a.cols = d->cols;
  a.col_blocks = (int32_t)blocks_of(d->cols);
  a.vec_h = vec_ok(d->x_type, d->ldh);
  a.vec_u = vec_ok(d->x_type, d->ldh, d->cols);
  a.vec_a = vec_ok(d->x_type, d->lda);
  a.vec_cu = d->cols % 8 == 0;
  const unsigned grid = (unsigned)(((int64_t)d->rows + kActRows - 1) / kActRows * a.col_blocks);
  a.e5m2 = (q || c) && d->q_type == MAXDNN_E5M2;
  const bool whole = a.vec_h && (!d->gated || (a.vec_u && a.vec_cu)) && a.vec_a && d->cols % 8 == 0;
  return by_wide(d->x_type, [&](auto xt) {
    return by_act(d, [&](auto act, auto gated) {
      return by_edge(whole, [&](auto edge) {
        act8_fprop_kernel<decltype(xt)::value, decltype(act)::value, decltype(gated)::value != 0, decltype(edge)::value != 0>
            <<<grid, kActThreads, 0, stream>>>(a);
        return launched();
      });
    });
  });
}

maxdnn_status act8_bprop(const maxdnn_act8_desc* d, const void* da, const void* h, const void* h_scale, void* dh,
                         cudaStream_t stream) {
  maxdnn_status st = check_act8(d);
  if (st != MAXDNN_OK) return st;
  if (d->rows == 0 || d->cols == 0) return MAXDNN_OK;
  if (!da || !h || !dh || !aligned16(da) || !aligned16(h) || !aligned16(dh)) return MAXDNN_INVALID_VALUE;
  if (d->lda < d->cols) return MAXDNN_INVALID_VALUE;
  const bool packed = is_fp8(d->h_type);
  if (!packed && d->h_type != d->x_type) return is_wide(d->h_type) ? MAXDNN_NOT_SUPPORTED : MAXDNN_INVALID_VALUE;
  if (packed && (!h_scale || d->ldc < (int64_t)d->cols * (1 + d->gated))) return MAXDNN_INVALID_VALUE;
  RuntimeDevice dev;
  if ((st = runtime_device(&dev)) != MAXDNN_OK) return st;
  Act8Args a = {};
  a.h = h;
  a.h_scale = static_cast<const uint8_t*>(h_scale);
  a.da = da;
  a.dh = dh;
  a.ldh = d->ldh;
  a.lda = d->lda;
  a.ldc = d->ldc;
  a.rows = d->rows;
  a.cols = d->cols;
  a.col_blocks = (int32_t)blocks_of(d->cols);
  const int64_t ldh = packed ? d->ldc : d->ldh;
  a.vec_h = vec_ok(d->h_type, ldh);
  a.vec_u = vec_ok(d->h_type, ldh, d->cols);
  a.vec_a = vec_ok(d->x_type, d->lda);
  a.vec_dh = vec_ok(d->x_type, d->ldh);
  a.vec_du = vec_ok(d->x_type, d->ldh, d->cols);
  const unsigned grid = (unsigned)(((int64_t)d->rows + kActRows - 1) / kActRows * a.col_blocks);
  const bool whole = a.vec_h && a.vec_a && a.vec_dh && (!d->gated || (a.vec_u && a.vec_du)) && d->cols % 8 == 0;
  return by_wide(d->x_type, [&](auto xt) {
    auto run = [&](auto ht) {
      return by_act(d, [&](auto act, auto gated) {
        return by_edge(whole, [&](auto edge) {
          act8_bprop_kernel<decltype(ht)::value, decltype(xt)::value, decltype(act)::value, decltype(gated)::value != 0,
                            decltype(edge)::value != 0><<<grid, kActThreads, 0, stream>>>(a);
          return launched();
        });
      });
    };
    return packed ? by_fp8(d->h_type, run) : run(xt);
  });
}

}  // namespace
}  // namespace maxdnn

extern "C" {

maxdnn_status maxdnn_quant8(const maxdnn_quant8_desc* desc, const void* x, const void* x_scale, void* q_row,
                            void* s_row, void* q_col, void* s_col, void* q_tile, void* s_tile, void* cuda_stream) {
  return maxdnn::quant8(desc, x, x_scale, q_row, s_row, q_col, s_col, q_tile, s_tile,
                        static_cast<cudaStream_t>(cuda_stream));
}

maxdnn_status maxdnn_dequant8(const maxdnn_quant8_desc* desc, maxdnn_block block, const void* q, const void* s,
                              void* x, void* cuda_stream) {
  return maxdnn::dequant8(desc, (int)block, q, s, x, static_cast<cudaStream_t>(cuda_stream));
}

maxdnn_status maxdnn_layer_norm_fprop(const maxdnn_layer_norm_desc* desc, const void* x, const void* gamma,
                                      const void* beta, void* y, float* mean, float* rstd, void* q, void* s,
                                      void* c, void* sc, void* cuda_stream) {
  return maxdnn::layer_norm_fprop(desc, x, gamma, beta, y, mean, rstd, q, s, c, sc,
                                  static_cast<cudaStream_t>(cuda_stream));
}

maxdnn_status maxdnn_layer_norm_bprop_workspace(const maxdnn_layer_norm_desc* desc, size_t* bytes) {
  return maxdnn::layer_norm_bprop_workspace(desc, bytes);
}

maxdnn_status maxdnn_layer_norm_bprop(const maxdnn_layer_norm_desc* desc, const void* dy, const void* x,
                                      const void* x_scale, const void* gamma, const float* mean, const float* rstd,
                                      void* dx, float* dgamma, float* dbeta, void* workspace,
                                      size_t workspace_bytes, void* cuda_stream) {
  return maxdnn::layer_norm_bprop(desc, dy, x, x_scale, gamma, mean, rstd, dx, dgamma, dbeta, workspace,
                                  workspace_bytes, static_cast<cudaStream_t>(cuda_stream));
}

maxdnn_status maxdnn_act8_fprop(const maxdnn_act8_desc* desc, const void* h, void* a, void* q, void* s, void* c,
                                void* sc, void* cuda_stream) {
  return maxdnn::act8_fprop(desc, h, a, q, s, c, sc, static_cast<cudaStream_t>(cuda_stream));
}

maxdnn_status maxdnn_act8_bprop(const maxdnn_act8_desc* desc, const void* da, const void* h, const void* h_scale,
                                void* dh, void* cuda_stream) {
  return maxdnn::act8_bprop(desc, da, h, h_scale, dh, static_cast<cudaStream_t>(cuda_stream));
}

}  // extern "C"
