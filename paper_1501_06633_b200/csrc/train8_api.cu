// C ABI of the 8-bit training operators (see include/maxdnn.h): argument checks, tensor-copy
// descriptors and kernel launches.
#include <cstring>

#include "act8.cuh"
#include "gemm8.cuh"
#include "gemm8_mx.cuh"
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
  return by_any(d->x_type, [&](auto xt) {
    return by_fp8(d->q_type, [&](auto qt) {
      quant8_kernel<decltype(xt)::value, decltype(qt)::value><<<grid, kQuantThreads, 0, stream>>>(a);
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
      dequant8_kernel<decltype(xt)::value, decltype(qt)::value><<<grid, kQuantThreads, 0, stream>>>(a);
      return launched();
    });
  });
}

// --------------------------------------------------------------- layer norm
// How a row is laid out over threads: `j` vectors of eight columns in each of `threads` (32: a
// warp per row, four rows per CTA); threads = 0: the kernel that reads the row again.
struct NormShape { int threads, j; };
NormShape norm_shape(int cols, bool backward) {
  if (cols <= 256) return {32, 1};
  if (cols <= 512) return {32, 2};
  if (cols <= 1024) return {32, 4};
  for (int t = 128; t <= 512; t *= 2)
    if (cols <= t * 16) return {t, 2};
  if (!backward && cols <= 512 * 32) return {512, 4};
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
  const NormShape sh = norm_shape(d->cols, false);
  const int64_t units = sh.threads == 32 ? ((int64_t)d->rows + 3) / 4 : d->rows;
  const int per_sm = sh.threads == 0 ? 2 : sh.threads == 32 ? 16 : 2048 / sh.threads / (sh.j > 2 ? 2 : 1);
  const int64_t most = (int64_t)dev.sm_count * per_sm;
  const unsigned grid = (unsigned)(units < most ? units : most);
  const int qt_code = (q || c) ? d->q_type : MAXDNN_E4M3;
  return by_wide(d->x_type, [&](auto xt) {
    return by_fp8(qt_code, [&](auto qt) {
      constexpr int X = decltype(xt)::value, Q = decltype(qt)::value;
      if (sh.threads == 0) layer_norm_fprop_long_kernel<X, Q><<<grid, 1024, 0, stream>>>(a);
      else if (sh.threads == 32 && sh.j == 1) layer_norm_fprop_kernel<X, Q, 1, true><<<grid, 128, 0, stream>>>(a);
      else if (sh.threads == 32 && sh.j == 2) layer_norm_fprop_kernel<X, Q, 2, true><<<grid, 128, 0, stream>>>(a);
      else if (sh.threads == 32) layer_norm_fprop_kernel<X, Q, 4, true><<<grid, 128, 0, stream>>>(a);
      else if (sh.j == 2) layer_norm_fprop_kernel<X, Q, 2, false><<<grid, sh.threads, 0, stream>>>(a);
      else layer_norm_fprop_kernel<X, Q, 4, false><<<grid, sh.threads, 0, stream>>>(a);
      return launched();
    });
  });
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
  *bytes = (size_t)norm_bprop_grid(*d, sm_count, norm_shape(d->cols, true)) * 2 * (size_t)d->cols * 4;
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
  const NormShape sh = norm_shape(d->cols, true);
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
    if (sh.threads == 0) layer_norm_bprop_long_kernel<X, Y><<<grid, 1024, 0, stream>>>(a);
    else if (sh.threads == 32 && sh.j == 1) layer_norm_bprop_kernel<X, Y, 1, true><<<grid, 128, 0, stream>>>(a);
    else if (sh.threads == 32 && sh.j == 2) layer_norm_bprop_kernel<X, Y, 2, true><<<grid, 128, 0, stream>>>(a);
    else if (sh.threads == 32) layer_norm_bprop_kernel<X, Y, 4, true><<<grid, 128, 0, stream>>>(a);
    else layer_norm_bprop_kernel<X, Y, 2, false><<<grid, sh.threads, 0, stream>>>(a);
    return launched();
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
  a.vec_c = 1;
  a.vec_cu = d->cols % 8 == 0;
  const unsigned grid = (unsigned)(((int64_t)d->rows + kActRows - 1) / kActRows * a.col_blocks);
  const int qt_code = (q || c) ? d->q_type : MAXDNN_E4M3;
  return by_wide(d->x_type, [&](auto xt) {
    return by_fp8(qt_code, [&](auto qt) {
      return by_act(d, [&](auto act, auto gated) {
        act8_fprop_kernel<decltype(xt)::value, decltype(qt)::value, decltype(act)::value, decltype(gated)::value != 0>
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
  return by_wide(d->x_type, [&](auto xt) {
    auto run = [&](auto ht) {
      return by_act(d, [&](auto act, auto gated) {
        act8_bprop_kernel<decltype(ht)::value, decltype(xt)::value, decltype(act)::value, decltype(gated)::value != 0>
            <<<grid, kActThreads, 0, stream>>>(a);
        return launched();
      });
    };
    return packed ? by_fp8(d->h_type, run) : run(xt);
  });
}

// ------------------------------------------------------------ matrix product
struct Operand {
  const void *p, *s;
  int64_t ld;
  int32_t mn, type, major, block, scale_type;
};

Gemm8Scale scale_of_operand(const Operand& o, int32_t K) {
  Gemm8Scale s = {};
  s.p = o.s;
  s.is_float = o.scale_type == MAXDNN_F32;
  s.count = o.mn;
  if (o.block == MAXDNN_BLOCK_TILE) {
    s.shift = 7;
    s.step = o.major == MAXDNN_MAJOR_K ? blocks_of(K) : 1;
    s.kstep = o.major == MAXDNN_MAJOR_K ? 1 : blocks_of(o.mn);
  } else {
    s.shift = 0;
    s.step = 1;
    s.kstep = o.mn;
    s.words = (reinterpret_cast<uintptr_t>(o.s) & 3u) == 0 && o.mn % 4 == 0;
  }
  return s;
}

maxdnn_status operand_map(CUtensorMap* m, const Operand& o, int32_t K, int box_mn) {
  const bool mn = o.major == MAXDNN_MAJOR_MN;
  const uint64_t dims[2] = {(uint64_t)(mn ? o.mn : K), (uint64_t)(mn ? K : o.mn)};
  const uint64_t str[1] = {(uint64_t)o.ld};
  const uint32_t box[2] = {128u, (uint32_t)(mn ? kGemm8BlockK : box_mn)};
  return runtime_encode(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, o.p, dims, str, box, CU_TENSOR_MAP_SWIZZLE_128B);
}

// One flag per device and kernel instance: "dynamic shared memory limit raised".
template <class Kern>
maxdnn_status raise_smem(const RuntimeDevice& dev, std::atomic<bool> (&done)[64], Kern kern) {
  if (done[dev.index].load(std::memory_order_acquire)) return MAXDNN_OK;   // raising it twice does no harm
  if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024) != cudaSuccess) {
    cudaGetLastError();
    return MAXDNN_CUDA_ERROR;
  }
  done[dev.index].store(true, std::memory_order_release);
  return MAXDNN_OK;
}

template <class Kern, class... Args>
maxdnn_status launch_clusters(Kern kern, const Gemm8Plan& p, int threads, int cluster, cudaStream_t stream,
                              const Args&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)p.grid, 1, 1);
  cfg.blockDim = dim3((unsigned)threads, 1, 1);
  cfg.dynamicSmemBytes = (size_t)p.smem_bytes;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)cluster;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 1 ? 1 : 0;
  if (cudaLaunchKernelEx(&cfg, kern, args...) != cudaSuccess) {
    cudaGetLastError();
    return MAXDNN_CUDA_ERROR;
  }
  runtime_count_launch();
  return MAXDNN_OK;
}

template <int NT, bool SBV>
maxdnn_status launch_gemm8(const RuntimeDevice& dev, const Gemm8Plan& p, const CUtensorMap& ma, const CUtensorMap& mb,
                           const Gemm8Args& args, cudaStream_t stream) {
  static std::atomic<bool> done[64];
  const maxdnn_status st = raise_smem(dev, done, gemm8_kernel<NT, SBV>);
  if (st != MAXDNN_OK) return st;
  return launch_clusters(gemm8_kernel<NT, SBV>, p, gemm8_threads(NT), p.split, stream, ma, mb, args);
}

template <int NT, bool PAIR>
maxdnn_status launch_gemm8_mx(const RuntimeDevice& dev, const Gemm8Plan& p, const CUtensorMap& ma,
                              const CUtensorMap& mb, const CUtensorMap& mc, const Gemm8MxArgs& args,
                              cudaStream_t stream) {
  static std::atomic<bool> done[64];
  const maxdnn_status st = raise_smem(dev, done, gemm8_mx_kernel<NT, PAIR>);
  if (st != MAXDNN_OK) return st;
  return launch_clusters(gemm8_mx_kernel<NT, PAIR>, p, kMxThreads, PAIR ? 2 : p.split, stream, ma, mb, mc, args);
}

maxdnn_status gemm8_mx(const RuntimeDevice& dev, const maxdnn_gemm8_desc& d, const Gemm8Plan& p, const Operand& oa,
                       const Operand& ob, void* c, const CUtensorMap& ma, const CUtensorMap& mb, uint32_t idesc,
                       cudaStream_t stream) {
  Gemm8MxArgs args = {};
  args.sa = scale_of_operand(oa, d.K);
  args.sb = scale_of_operand(ob, d.K);
  args.c = c;
  args.c_row = p.swap ? 1 : d.ldc;
  args.c_col = p.swap ? d.ldc : 1;
  args.M = oa.mn;
  args.N = ob.mn;
  args.m_tiles = p.m_tiles;
  args.n_tiles = p.n_tiles;
  args.k_blocks = p.k_blocks;
  args.split = p.split;
  args.stages = p.stages;
  args.a_mn = oa.major == MAXDNN_MAJOR_MN;
  args.b_mn = ob.major == MAXDNN_MAJOR_MN;
  args.b_stage_bytes = p.b_stage_bytes;
  args.c_type = d.c_type;
  args.bulk_c = p.bulk_c;
  args.chunk = p.chunk;
  args.idesc = idesc | (1u << 23);          // scales are E8M0
  args.test_missing_arrival = (uint32_t)option(OPT_TEST_MISSING_ARRIVAL);
  args.wc = runtime_wait_ctx(dev);
  CUtensorMap mc;
  memset(&mc, 0, sizeof(mc));
  if (p.bulk_c) {
    const int cb = elem_bytes(d.c_type);
    const uint64_t dims[2] = {(uint64_t)d.N, (uint64_t)d.M}, str[1] = {(uint64_t)d.ldc * cb};
    const uint32_t box[2] = {32u, 32u};
    const maxdnn_status st = runtime_encode(
        &mc, d.c_type == MAXDNN_F32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
             : d.c_type == MAXDNN_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16,
        2, c, dims, str, box, cb == 4 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B);
    if (st != MAXDNN_OK) return st;
  }
#define MAXDNN_GEMM8_CASE(NT, PAIR) \
  if (p.tile_n == (NT) && (p.pair != 0) == (PAIR)) return launch_gemm8_mx<NT, PAIR>(dev, p, ma, mb, mc, args, stream);
  MAXDNN_GEMM8_CASE(16, false)
  MAXDNN_GEMM8_CASE(32, false)
  MAXDNN_GEMM8_CASE(64, false)
  MAXDNN_GEMM8_CASE(128, false)
  MAXDNN_GEMM8_CASE(128, true)
  MAXDNN_GEMM8_CASE(192, true)
  MAXDNN_GEMM8_CASE(224, true)
  MAXDNN_GEMM8_CASE(256, true)
#undef MAXDNN_GEMM8_CASE
  return MAXDNN_NOT_SUPPORTED;
}

maxdnn_status gemm8(const maxdnn_gemm8_desc* d, const void* a, const void* sa, const void* b, const void* sb, void* c,
                    cudaStream_t stream) {
  maxdnn_status st = check_gemm8(d);
  if (st != MAXDNN_OK) return st;
  if (d->M == 0 || d->N == 0) return MAXDNN_OK;
  if (!c || !aligned16(c)) return MAXDNN_INVALID_VALUE;
  const size_t cb = (size_t)elem_bytes(d->c_type);
  if (d->K == 0) {       // an empty sum
    if (cudaMemset2DAsync(c, (size_t)d->ldc * cb, 0, (size_t)d->N * cb, (size_t)d->M, stream) != cudaSuccess) {
      cudaGetLastError();
      return MAXDNN_CUDA_ERROR;
    }
    return MAXDNN_OK;
  }
  if (!a || !sa || !b || !sb || !aligned16(a) || !aligned16(b)) return MAXDNN_INVALID_VALUE;
  RuntimeDevice dev;
  if ((st = runtime_device(&dev)) != MAXDNN_OK) return st;
  Gemm8Plan p;
  if ((st = plan_gemm8(*d, dev.sm_count, &p)) != MAXDNN_OK) return st;
  Operand oa = {a, sa, d->lda, d->M, d->a_type, d->a_major, d->a_block, d->a_scale_type};
  Operand ob = {b, sb, d->ldb, d->N, d->b_type, d->b_major, d->b_block, d->b_scale_type};
  if (p.swap) { const Operand t = oa; oa = ob; ob = t; }
  CUtensorMap ma, mb;
  if ((st = operand_map(&ma, oa, d->K, kGemm8TileM)) != MAXDNN_OK) return st;
  if ((st = operand_map(&mb, ob, d->K, p.pair ? p.tile_n / 2 : p.tile_n)) != MAXDNN_OK) return st;
  // instruction descriptor: formats and majors of A and B, N / 8, M / 16
  const uint32_t a_mn = oa.major == MAXDNN_MAJOR_MN, b_mn = ob.major == MAXDNN_MAJOR_MN;
  const uint32_t idesc = ((oa.type == MAXDNN_E5M2 ? 1u : 0u) << 7) | ((ob.type == MAXDNN_E5M2 ? 1u : 0u) << 10) |
                         (a_mn << 15) | (b_mn << 16) | ((uint32_t)(p.tile_n >> 3) << 17) |
                         ((uint32_t)((p.pair ? 2 : 1) * kGemm8TileM >> 4) << 24);
  if (p.mx) return gemm8_mx(dev, *d, p, oa, ob, c, ma, mb, idesc, stream);
  Gemm8Args args = {};
  args.sa = scale_of_operand(oa, d->K);
  args.sb = scale_of_operand(ob, d->K);
  args.c = c;
  args.c_row = p.swap ? 1 : d->ldc;
  args.c_col = p.swap ? d->ldc : 1;
  args.M = oa.mn;
  args.N = ob.mn;
  args.m_tiles = p.m_tiles;
  args.n_tiles = p.n_tiles;
  args.k_blocks = p.k_blocks;
  args.split = p.split;
  args.stages = p.stages;
  args.a_mn = (int32_t)a_mn;
  args.b_mn = (int32_t)b_mn;
  args.b_stage_bytes = p.b_stage_bytes;
  args.c_type = d->c_type;
  args.vec_c = !p.swap && (d->ldc * (int64_t)cb) % 16 == 0;
  args.idesc = idesc | (1u << 4);           // fp32 accumulator
  args.test_missing_arrival = (uint32_t)option(OPT_TEST_MISSING_ARRIVAL);
  args.wc = runtime_wait_ctx(dev);
  const bool sbv = ob.block != MAXDNN_BLOCK_TILE;
#define MAXDNN_GEMM8_CASE(NT)                                                             \
  if (p.tile_n == (NT))                                                                   \
    return sbv ? launch_gemm8<NT, true>(dev, p, ma, mb, args, stream)                     \
               : launch_gemm8<NT, false>(dev, p, ma, mb, args, stream);
  MAXDNN_GEMM8_CASE(16)
  MAXDNN_GEMM8_CASE(32)
  MAXDNN_GEMM8_CASE(64)
  MAXDNN_GEMM8_CASE(128)
  MAXDNN_GEMM8_CASE(256)
#undef MAXDNN_GEMM8_CASE
  return MAXDNN_NOT_SUPPORTED;
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

maxdnn_status maxdnn_gemm8(const maxdnn_gemm8_desc* desc, const void* a, const void* a_scale, const void* b,
                           const void* b_scale, void* c, void* cuda_stream) {
  return maxdnn::gemm8(desc, a, a_scale, b, b_scale, c, static_cast<cudaStream_t>(cuda_stream));
}

}  // extern "C"
