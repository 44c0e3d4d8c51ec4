// C ABI of packing, unpacking and the activations that work with packed inputs (see
// include/maxdnn.h): argument checks and kernel launches.
#include "act8.cuh"
#include "api8.h"
#include "quant8.cuh"

namespace maxdnn {
namespace {

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
  const unsigned grid = (unsigned)(blocks_of(d->rows) * blocks_of(d->cols));
  return by_any(d->x_type, [&](auto xt) {
    return by_fp8(d->q_type, [&](auto qt) {
      return by_edge(vec_ok(d->x_type, d->ldx) && d->cols % 8 == 0, [&](auto edge) {
        return launch_early(quant8_kernel<decltype(xt)::value, decltype(qt)::value, decltype(edge)::value != 0>, grid, kQuantThreads, 0, 1, stream, a);
      });
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
  const unsigned grid = (unsigned)(blocks_of(d->rows) * blocks_of(d->cols));
  return by_wide(d->x_type, [&](auto xt) {
    return by_fp8(d->q_type, [&](auto qt) {
      return by_edge(vec_ok(d->x_type, d->ldx) && vec_ok(d->q_type, d->ldq) && d->cols % 8 == 0, [&](auto edge) {
        return launch_early(dequant8_kernel<decltype(xt)::value, decltype(qt)::value, decltype(edge)::value != 0>, grid, kQuantThreads, 0, 1, stream, a);
      });
    });
  });
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
  const bool vec_h = vec_ok(d->x_type, d->ldh);
  const bool vec_u = vec_ok(d->x_type, d->ldh, d->cols);
  const bool vec_a = vec_ok(d->x_type, d->lda);
  const bool vec_cu = d->cols % 8 == 0;
  const unsigned grid = (unsigned)(((int64_t)d->rows + kActRows - 1) / kActRows * a.col_blocks);
  const bool whole = vec_h && (!d->gated || (vec_u && vec_cu)) && vec_a && d->cols % 8 == 0;
  const int qt_code = (q || c) ? d->q_type : MAXDNN_E4M3;
  return by_wide(d->x_type, [&](auto xt) {
    return by_fp8(qt_code, [&](auto qt) {
      return by_act(d, [&](auto act, auto gated) {
        return by_edge(whole, [&](auto edge) {
          return launch_early(act8_fprop_kernel<decltype(xt)::value, decltype(qt)::value, decltype(act)::value, decltype(gated)::value != 0, decltype(edge)::value != 0>, grid, kActThreads, 0, 1, stream, a);
        });
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
  const bool vec_h = vec_ok(d->h_type, ldh);
  const bool vec_u = vec_ok(d->h_type, ldh, d->cols);
  const bool vec_a = vec_ok(d->x_type, d->lda);
  const bool vec_dh = vec_ok(d->x_type, d->ldh);
  const bool vec_du = vec_ok(d->x_type, d->ldh, d->cols);
  const unsigned grid = (unsigned)(((int64_t)d->rows + kActRows - 1) / kActRows * a.col_blocks);
  const bool whole = vec_h && vec_a && vec_dh && (!d->gated || (vec_u && vec_du)) && d->cols % 8 == 0;
  return by_wide(d->x_type, [&](auto xt) {
    auto run = [&](auto ht) {
      return by_act(d, [&](auto act, auto gated) {
        return by_edge(whole, [&](auto edge) {
          return launch_early(act8_bprop_kernel<decltype(ht)::value, decltype(xt)::value, decltype(act)::value, decltype(gated)::value != 0, decltype(edge)::value != 0>, grid, kActThreads, 0, 1, stream, a);
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

maxdnn_status maxdnn_act8_fprop(const maxdnn_act8_desc* desc, const void* h, void* a, void* q, void* s, void* c,
                                void* sc, void* cuda_stream) {
  return maxdnn::act8_fprop(desc, h, a, q, s, c, sc, static_cast<cudaStream_t>(cuda_stream));
}

maxdnn_status maxdnn_act8_bprop(const maxdnn_act8_desc* desc, const void* da, const void* h, const void* h_scale,
                                void* dh, void* cuda_stream) {
  return maxdnn::act8_bprop(desc, da, h, h_scale, dh, static_cast<cudaStream_t>(cuda_stream));
}

}  // extern "C"
