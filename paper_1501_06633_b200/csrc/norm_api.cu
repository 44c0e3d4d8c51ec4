// C ABI of layer norm (see include/maxdnn.h): argument checks and kernel launches.
#include "api8.h"
#include "layer_norm.cuh"

namespace maxdnn {
namespace {

// How the backward pass lays a row out over threads: `j` vectors of eight columns in each of
// `threads` (32: a warp per row, four rows per CTA); threads = 0: the kernel that reads the row
// again.  ring: rows come through the ring in shared memory, `depth` of them.
struct NormShape { int threads, j, ring, depth; };
NormShape norm_shape(const maxdnn_layer_norm_desc& d) {
  const int cols = d.cols;
  if (cols <= 256) return {32, 1, 0, 0};
  if (cols <= 512) return {32, 2, 0, 0};
  if (cols <= 1024) return {32, 4, 0, 0};
  if (cols > 8192) return {0, 0, 0, 0};
  if (cols % 8 == 0 && vec_ok(d.x_type, d.ldx) && vec_ok(d.y_type, d.ldy)) {
    const int t = cols <= 2048 ? 128 : cols <= 4096 ? 256 : 512, j = 2;
    const int row = norm_ring_row(elem_bytes(d.x_type), elem_bytes(d.y_type), t, j);
    const int room = t / 128 * 50 * 1024;    // of 227 KB: four, two or one CTA per SM
    const int depth = room / row;
    return {t, j, 1, depth < 2 ? 2 : depth > 4 ? 4 : depth};
  }
  for (int t = 128; t < 512; t *= 2)
    if (cols <= t * 16) return {t, 2, 0, 0};
  return {512, 2, 0, 0};
}

maxdnn_status check_layer_norm(const maxdnn_layer_norm_desc* d) {
  if (!d || d->rows < 0 || d->cols <= 0) return MAXDNN_INVALID_VALUE;
  if (!is_wide(d->y_type) || !is_wide(d->w_type) || (!is_wide(d->x_type) && !is_fp8(d->x_type))) return MAXDNN_INVALID_VALUE;
  if (d->ldx < d->cols || d->ldy < d->cols) return MAXDNN_INVALID_VALUE;
  if (!(d->eps >= 0.f) || d->eps > 3.0e38f) return MAXDNN_INVALID_VALUE;
  if (is_wide(d->x_type) && d->x_type != d->y_type) return MAXDNN_NOT_SUPPORTED;
  if (d->cols > (1 << 30)) return MAXDNN_NOT_SUPPORTED;    // column numbers are 32 bits
  return MAXDNN_OK;
}

// CTAs of the backward pass: each leaves one row of sums, which the fold reads again.  Where the CTAs
// of a whole device would have fewer than four rows each there are fewer of them, down to one per
// SM (packed bf16: 1024 x 4096 13.8 us with 256 CTAs, 1.4 more with 296; 512 x 4096 9.7 with 148, 1.8 more with
// 296; 300 x 2048 9.1, 0.5 less with all.  Fewer than the SMs lose: 128 x 4096 8.7 with 64, 7.5 with 128).
int norm_bprop_grid(const maxdnn_layer_norm_desc& d, int sm_count, const NormShape& s) {
  const int64_t units = s.threads == 32 ? ((int64_t)d.rows + 3) / 4 : d.rows;
  const int per_sm = s.threads == 0 ? 1 : s.threads == 32 ? 4 : s.ring ? 512 / s.threads : s.threads >= 512 ? 1 : 512 / s.threads;
  int64_t most = (int64_t)sm_count * per_sm;
  if (s.ring) {
    const int64_t few = d.rows / 4 < sm_count ? sm_count : d.rows / 4;
    if (few < most) most = few;
  }
  return (int)(units < most ? units : most);
}

template <int XT, int J, int WR>
maxdnn_status launch_norm_rows(const LayerNormArgs& a, int sm_count, cudaStream_t stream) {
  const int64_t units = ((int64_t)a.rows + 8 / WR - 1) / (8 / WR);
  const int64_t most = (int64_t)sm_count * 4;
  const unsigned grid = (unsigned)(units < most ? units : most);
  if (!a.whole) {
    return launch_early(layer_norm_fprop_kernel<XT, kEitherFp8, J, WR, true>, grid, kNormThreads, 0, 1, stream, a);
  }
  const size_t smem = norm_shared_weights(J, WR) ? 2 * 256 * WR * J * sizeof(float) : 0;     // at most 32 KB
  return launch_early(a.q_e5m2 ? layer_norm_fprop_kernel<XT, MAXDNN_E5M2, J, WR, false>
                               : layer_norm_fprop_kernel<XT, MAXDNN_E4M3, J, WR, false>,
                      grid, kNormThreads, smem, 1, stream, a);
}

// Vectors of eight columns per thread (J) and warps per row (WR).  Few rows (fewer than four for each
// SM): eight warps share a row, for the latency (three rows of 2048: 2.1 us against 2.5
// with a warp each).  Else as few warps as hold the row with J <= 4.  Rows beyond 16384 columns are read again
// for each sum.
template <int XT>
maxdnn_status launch_norm_fprop(const LayerNormArgs& a, int sm_count, cudaStream_t stream) {
  const int vecs = (a.cols + 7) / 8;
  if (a.rows < 4 * sm_count && vecs > 32 && vecs <= 512) {
    if (vecs <= 256) return launch_norm_rows<XT, 1, 8>(a, sm_count, stream);
    return launch_norm_rows<XT, 2, 8>(a, sm_count, stream);
  }
  if (vecs <= 32) return launch_norm_rows<XT, 1, 1>(a, sm_count, stream);
  if (vecs <= 64) return launch_norm_rows<XT, 2, 1>(a, sm_count, stream);
  if (vecs <= 128) return launch_norm_rows<XT, 4, 1>(a, sm_count, stream);
  if (vecs <= 256) return launch_norm_rows<XT, 4, 2>(a, sm_count, stream);
  if (vecs <= 512) return launch_norm_rows<XT, 4, 4>(a, sm_count, stream);
  if (vecs <= 1024) return launch_norm_rows<XT, 4, 8>(a, sm_count, stream);
  if (vecs <= 2048) return launch_norm_rows<XT, 8, 8>(a, sm_count, stream);
  const int64_t most = 2 * (int64_t)sm_count;
  return launch_early(layer_norm_fprop_long_kernel<XT>, (unsigned)(a.rows < most ? a.rows : most), 1024, 0, 1, stream, a);
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
  a.whole = vec_ok(d->x_type, d->ldx) && vec_ok(d->y_type, d->ldy) && aligned16(gamma) && aligned16(beta) && d->cols % 8 == 0;
  a.eps = d->eps;
  a.inv_cols = 1.f / (float)d->cols;
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
  *bytes = (size_t)norm_bprop_grid(*d, sm_count, norm_shape(*d)) * 2 * (size_t)norm_sums_pitch(d->cols) * 4;
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
  const NormShape sh = norm_shape(*d);
  const int grid = norm_bprop_grid(*d, dev.sm_count, sh);
  const bool sums = dgamma || dbeta;
  if (sums && (!workspace || !aligned16(workspace) || workspace_bytes < (size_t)grid * 2 * (size_t)norm_sums_pitch(d->cols) * 4))
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
  a.whole = vec_ok(d->x_type, d->ldx) && vec_ok(d->y_type, d->ldy) && aligned16(gamma) && d->cols % 8 == 0;
  a.inv_cols = 1.f / (float)d->cols;
  auto run = [&](auto xt, auto yt) {
    constexpr int X = decltype(xt)::value, Y = decltype(yt)::value;
    if (sh.threads == 0) {
      return launch_early(layer_norm_bprop_long_kernel<X, Y>, grid, 1024, 0, 1, stream, a);
    }
    if (sh.ring) {
      const int smem = sh.depth * norm_ring_row(elem_bytes(X), elem_bytes(Y), sh.threads, sh.j) +
                       (is_fp8(X) ? (int)blocks_of(d->cols) * kNormChunk : 0);
      auto kern = sh.threads == 128 ? layer_norm_bprop_ring_kernel<X, Y, 2, 4>
                  : sh.threads == 256 ? layer_norm_bprop_ring_kernel<X, Y, 2, 8> : layer_norm_bprop_ring_kernel<X, Y, 2, 16>;
      static std::atomic<bool> done[3][64];
      const int slot = sh.threads == 128 ? 0 : sh.threads == 256 ? 1 : 2;
      if (!done[slot][dev.index].load(std::memory_order_acquire)) {
        if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, 220 * 1024) != cudaSuccess) {
          cudaGetLastError();
          return MAXDNN_CUDA_ERROR;
        }
        done[slot][dev.index].store(true, std::memory_order_release);
      }
      return launch_early(kern, grid, sh.threads, smem, 1, stream, a, sh.depth);
    }
    return by_edge(a.whole, [&](auto edge) {
      constexpr bool E = decltype(edge)::value != 0;
      if (sh.threads != 32)      // (whole vectors: the ring)
        return launch_early(layer_norm_bprop_kernel<X, Y, 2, false, true>, grid, sh.threads, 0, 1, stream, a);
      return launch_early(sh.j == 1 ? layer_norm_bprop_kernel<X, Y, 1, true, E>
                          : sh.j == 2 ? layer_norm_bprop_kernel<X, Y, 2, true, E> : layer_norm_bprop_kernel<X, Y, 4, true, E>,
                          grid, 128, 0, 1, stream, a);
    });
  };
  st = by_wide(d->y_type, [&](auto yt) {
    if (is_fp8(d->x_type)) return by_fp8(d->x_type, [&](auto xt) { return run(xt, yt); });
    return run(yt, yt);
  });
  if (st != MAXDNN_OK || !sums) return st;
  return launch_early(layer_norm_fold_kernel, (unsigned)((2 * norm_sums_pitch(d->cols) + 31) / 32), 512, 0, 1, stream, a.partial, grid,
                      d->cols, dgamma, dbeta);
}

}  // namespace
}  // namespace maxdnn

extern "C" {

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

}  // extern "C"
