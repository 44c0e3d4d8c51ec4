// C ABI of the RMS norm (see include/maxdnn.h): argument checks and kernel launches.
#include "api8.h"
#include "rms_norm.cuh"

namespace maxdnn {
namespace {

constexpr int kRmsLong = 0;      // in place of a group's warps: the kernel that reads the row again

// Warps that hold a row of `cols` columns, sixteen to a lane.
int rms_group_warps(int cols) {
  for (int wr = 1; wr <= 32; wr *= 2)
    if (cols <= 512 * wr) return wr;
  return kRmsLong;
}

// CTAs of an SM that the ring's memory and the kernels' registers are planned for.
int rms_ctas_per_sm(int wr) { return wr <= 8 ? 3 : 1; }

// Stages of the ring that fit; 0: not even two.
int rms_depth(int wr, int64_t stage, int ctas) {
  const int64_t room = 222 * 1024 / ctas - 1024 - (wr < 8 ? 2048 * wr : 0);
  const int64_t depth = room / (rms_groups(wr) * stage);
  return depth < 2 ? 0 : depth > kRmsMaxDepth ? kRmsMaxDepth : (int)depth;
}

maxdnn_status check_rms_norm(const maxdnn_rms_norm_desc* d) {
  if (!d || d->rows < 0 || d->cols <= 0) return MAXDNN_INVALID_VALUE;
  if (!is_wide(d->y_type) || !is_wide(d->w_type) || (!is_wide(d->x_type) && !is_fp8(d->x_type))) return MAXDNN_INVALID_VALUE;
  if (d->ldx < d->cols || d->ldy < d->cols) return MAXDNN_INVALID_VALUE;
  if (!(d->eps >= 0.f) || d->eps > 3.0e38f) return MAXDNN_INVALID_VALUE;
  if (is_wide(d->x_type) && d->x_type != d->y_type) return MAXDNN_NOT_SUPPORTED;
  if (d->cols > (1 << 30)) return MAXDNN_NOT_SUPPORTED;    // column numbers are 32 bits
  return MAXDNN_OK;
}

// Rows that start at multiples of 16 bytes.
bool whole_rows(int type, int64_t ld) { return ld * elem_bytes(type) % 16 == 0; }

// The backward pass's plan: kernel, ring and CTAs (each leaves a row of sums).
struct RmsBack { int wr, depth, grid; int64_t smem; };
RmsBack rms_back(const maxdnn_rms_norm_desc& d, int sm_count) {
  RmsBack p = {rms_group_warps(d.cols), 0, 0, 0};
  if (p.wr != kRmsLong) {
    // (with and without dsum alike: the workspace is asked for before that is known)
    const int64_t stage = rms_stage_row(d.cols, elem_bytes(d.x_type)) + 2 * rms_stage_row(d.cols, elem_bytes(d.y_type));
    int ctas = p.wr > 8 ? 1 : 2;
    for (; ctas > 0 && !p.depth; --ctas) {
      p.depth = rms_depth(p.wr, stage, ctas);
      p.grid = sm_count * ctas;
    }
    p.smem = rms_groups(p.wr) * p.depth * stage;
    if (!p.depth) p.wr = kRmsLong;
  }
  if (p.wr == kRmsLong) p.grid = sm_count;
  // at least four rows to a group where the SMs all have one
  const int64_t groups = p.wr == kRmsLong ? 1 : rms_groups(p.wr);
  const int64_t few = (d.rows / 4 + groups - 1) / groups, units = (d.rows + groups - 1) / groups;
  int64_t most = few < sm_count ? sm_count : few;
  if (most < p.grid) p.grid = (int)most;
  if (units < p.grid) p.grid = (int)units;
  return p;
}

// (Up to four warps to a row at least two CTAs of an SM fit, besides what their groups' sums take.)
constexpr int rms_smem_limit(int wr) { return wr < 8 ? 112 * 1024 : 223 * 1024; }

template <int WR, class Kern>
maxdnn_status rms_raise(const RuntimeDevice& dev, std::atomic<bool> (&done)[64], Kern kern) {
  if (done[dev.index].load(std::memory_order_acquire)) return MAXDNN_OK;
  if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, rms_smem_limit(WR)) != cudaSuccess) {
    cudaGetLastError();
    return MAXDNN_CUDA_ERROR;
  }
  done[dev.index].store(true, std::memory_order_release);
  return MAXDNN_OK;
}

template <class F>
maxdnn_status by_warps(int wr, F f) {
  if (wr == 1) return f(Const<1>());
  if (wr == 2) return f(Const<2>());
  if (wr == 4) return f(Const<4>());
  if (wr == 8) return f(Const<8>());
  if (wr == 16) return f(Const<16>());
  return f(Const<32>());
}

template <int XT>
maxdnn_status launch_rms_fprop(const RuntimeDevice& dev, RmsNormArgs& a, bool whole, cudaStream_t stream) {
  const int wr = rms_group_warps(a.cols);
  const int64_t stage = rms_stage_row(a.cols, elem_bytes(XT), !whole) * (a.res ? 2 : 1);
  if (wr == kRmsLong) {
    const int64_t most = 2 * (int64_t)dev.sm_count;
    return launch_early(rms_norm_fprop_long_kernel<XT>, (unsigned)(a.rows < most ? a.rows : most), 1024, 0, 1, stream, a);
  }
  const int64_t groups = rms_groups(wr), units = (a.rows + groups - 1) / groups;
  const int ctas = rms_ctas_per_sm(wr);
  const int64_t most = (int64_t)dev.sm_count * ctas;
  a.depth = rms_depth(wr, stage, ctas);
  // a ring where some of its groups have more than one row (2000 rows of 1000: 4.3 us, 5.1 without; 900 rows of 4096: 5.5, 7.1)
  const bool ring = units > most && a.depth >= 2;
  return by_warps(wr, [&](auto w) {
    return by_edge(whole, [&](auto edge) {
      constexpr int WR = decltype(w)::value;
      constexpr bool E = decltype(edge)::value != 0;
      if (!ring)
        return launch_early(rms_norm_fprop_kernel<XT, WR, E, false>, (unsigned)(units < 2 * most ? units : 2 * most), rms_threads(WR), 0, 1,
                            stream, a);
      static std::atomic<bool> done[64];
      const maxdnn_status st = rms_raise<WR>(dev, done, rms_norm_fprop_kernel<XT, WR, E, true>);
      if (st != MAXDNN_OK) return st;
      return launch_early(rms_norm_fprop_kernel<XT, WR, E, true>, (unsigned)most, rms_threads(WR), (size_t)(groups * a.depth * stage), 1,
                          stream, a);
    });
  });
}

maxdnn_status rms_norm_fprop(const maxdnn_rms_norm_desc* d, const void* x, const void* residual, const void* gamma, void* sum,
                             void* y, float* rstd, void* q, void* s, void* c, void* sc, cudaStream_t stream) {
  maxdnn_status st = check_rms_norm(d);
  if (st != MAXDNN_OK) return st;
  if (!is_wide(d->x_type)) return MAXDNN_INVALID_VALUE;
  if ((residual || sum) && d->ldr < d->cols) return MAXDNN_INVALID_VALUE;
  if (d->rows == 0) return MAXDNN_OK;
  if (!x || (!sum && !y && !rstd && !q && !c)) return MAXDNN_INVALID_VALUE;
  if ((q && !s) || (c && !sc)) return MAXDNN_INVALID_VALUE;
  if (!aligned16(x) || !aligned16(residual) || !aligned16(sum) || !aligned16(y) || !aligned16(q) || !aligned16(c)) return MAXDNN_INVALID_VALUE;
  if (sum && ((sum == x && d->ldx != d->ldr) || sum == y)) return MAXDNN_INVALID_VALUE;
  if (q || c) {
    if (!is_fp8(d->q_type) || d->ldq < d->cols) return MAXDNN_INVALID_VALUE;
    if (d->ldq % 16 != 0) return MAXDNN_NOT_SUPPORTED;
  }
  RuntimeDevice dev;
  if ((st = runtime_device(&dev)) != MAXDNN_OK) return st;
  RmsNormArgs a = {};
  a.x = x;
  a.res = residual;
  a.gamma = gamma;
  a.sum = sum;
  a.y = y;
  a.rstd = rstd;
  a.q = static_cast<uint8_t*>(q);
  a.s = static_cast<uint8_t*>(s);
  a.c = static_cast<uint8_t*>(c);
  a.sc = static_cast<uint8_t*>(sc);
  a.ldx = d->ldx;
  a.ldr = d->ldr;
  a.ldy = d->ldy;
  a.ldq = d->ldq;
  a.rows = d->rows;
  a.cols = d->cols;
  a.w_type = d->w_type;
  a.eps = d->eps;
  a.inv_cols = 1.f / (float)d->cols;
  a.q_e5m2 = (q || c) && d->q_type == MAXDNN_E5M2;
  a.wc = runtime_wait_ctx(dev);
  const bool whole = d->cols % 8 == 0 && whole_rows(d->x_type, d->ldx) && (!(residual || sum) || whole_rows(d->x_type, d->ldr)) &&
                     (!y || whole_rows(d->y_type, d->ldy)) && aligned16(gamma);
  return by_wide(d->x_type, [&](auto xt) { return launch_rms_fprop<decltype(xt)::value>(dev, a, whole, stream); });
}

maxdnn_status rms_norm_bprop_workspace(const maxdnn_rms_norm_desc* d, size_t* bytes) {
  maxdnn_status st = check_rms_norm(d);
  if (st != MAXDNN_OK || !bytes) return st != MAXDNN_OK ? st : MAXDNN_INVALID_VALUE;
  int sm_count = option(OPT_SM_COUNT);   // planning without a device (tests)
  if (sm_count <= 0) {
    RuntimeDevice dev;
    if ((st = runtime_device(&dev)) != MAXDNN_OK) return st;
    sm_count = dev.sm_count;
  }
  *bytes = (size_t)rms_back(*d, sm_count).grid * (size_t)norm_sums_pitch(d->cols) * 4;
  return MAXDNN_OK;
}

maxdnn_status rms_norm_bprop(const maxdnn_rms_norm_desc* d, const void* dy, const void* h, const void* h_scale, const void* gamma,
                             const float* rstd, const void* dsum, void* dx, float* dgamma, void* workspace,
                             size_t workspace_bytes, cudaStream_t stream) {
  maxdnn_status st = check_rms_norm(d);
  if (st != MAXDNN_OK) return st;
  if (dsum && d->ldr < d->cols) return MAXDNN_INVALID_VALUE;
  if (d->rows == 0) {     // sums over no rows
    if (dgamma && cudaMemsetAsync(dgamma, 0, (size_t)d->cols * 4, stream) != cudaSuccess) {
      cudaGetLastError();
      return MAXDNN_CUDA_ERROR;
    }
    return MAXDNN_OK;
  }
  if (!dy || !h || !rstd || !dx) return MAXDNN_INVALID_VALUE;
  if (is_fp8(d->x_type) && !h_scale) return MAXDNN_INVALID_VALUE;
  if (!aligned16(dy) || !aligned16(h) || !aligned16(dsum) || !aligned16(dx)) return MAXDNN_INVALID_VALUE;
  if (dx == h || (dx == dsum && d->ldr != d->ldy)) return MAXDNN_INVALID_VALUE;
  RuntimeDevice dev;
  if ((st = runtime_device(&dev)) != MAXDNN_OK) return st;
  const RmsBack p = rms_back(*d, dev.sm_count);
  if (dgamma && (!workspace || !aligned16(workspace) || workspace_bytes < (size_t)p.grid * (size_t)norm_sums_pitch(d->cols) * 4))
    return MAXDNN_INVALID_VALUE;
  RmsNormArgs a = {};
  a.x = h;
  a.x_scale = static_cast<const uint8_t*>(h_scale);
  a.res = dsum;
  a.gamma = gamma;
  a.rstd = const_cast<float*>(rstd);
  a.dy = dy;
  a.dx = dx;
  a.partial = dgamma ? static_cast<float*>(workspace) : nullptr;
  a.ldx = d->ldx;
  a.ldr = d->ldr;
  a.ldy = d->ldy;
  a.rows = d->rows;
  a.cols = d->cols;
  a.w_type = d->w_type;
  a.inv_cols = 1.f / (float)d->cols;
  a.depth = p.depth;
  a.wc = runtime_wait_ctx(dev);
  const bool whole = d->cols % 8 == 0 && whole_rows(d->x_type, d->ldx) && whole_rows(d->y_type, d->ldy) &&
                     (!dsum || whole_rows(d->y_type, d->ldr)) && aligned16(gamma);
  auto run = [&](auto xt, auto yt) {
    constexpr int X = decltype(xt)::value, Y = decltype(yt)::value;
    if (p.wr == kRmsLong) return launch_early(rms_norm_bprop_long_kernel<X, Y>, p.grid, 1024, 0, 1, stream, a);
    return by_warps(p.wr, [&](auto w) {
      return by_edge(whole, [&](auto edge) {
        constexpr int WR = decltype(w)::value;
        constexpr bool E = decltype(edge)::value != 0;
        static std::atomic<bool> done[64];
        const maxdnn_status raised = rms_raise<WR>(dev, done, rms_norm_bprop_kernel<X, Y, WR, E>);
        if (raised != MAXDNN_OK) return raised;
        return launch_early(rms_norm_bprop_kernel<X, Y, WR, E>, p.grid, rms_threads(WR), (size_t)p.smem, 1, stream, a);
      });
    });
  };
  st = by_wide(d->y_type, [&](auto yt) {
    if (is_fp8(d->x_type)) return by_fp8(d->x_type, [&](auto xt) { return run(xt, yt); });
    return run(yt, yt);
  });
  if (st != MAXDNN_OK || !dgamma) return st;
  return launch_early(rms_norm_fold_kernel, (unsigned)((d->cols + 31) / 32), 512, 0, 1, stream, a.partial, p.grid, d->cols, dgamma);
}

}  // namespace
}  // namespace maxdnn

extern "C" {

maxdnn_status maxdnn_rms_norm_fprop(const maxdnn_rms_norm_desc* desc, const void* x, const void* residual, const void* gamma,
                                    void* sum, void* y, float* rstd, void* q, void* s, void* c, void* sc, void* cuda_stream) {
  return maxdnn::rms_norm_fprop(desc, x, residual, gamma, sum, y, rstd, q, s, c, sc, static_cast<cudaStream_t>(cuda_stream));
}

maxdnn_status maxdnn_rms_norm_bprop_workspace(const maxdnn_rms_norm_desc* desc, size_t* bytes) {
  return maxdnn::rms_norm_bprop_workspace(desc, bytes);
}

maxdnn_status maxdnn_rms_norm_bprop(const maxdnn_rms_norm_desc* desc, const void* dy, const void* h, const void* h_scale,
                                    const void* gamma, const float* rstd, const void* dsum, void* dx, float* dgamma,
                                    void* workspace, size_t workspace_bytes, void* cuda_stream) {
  return maxdnn::rms_norm_bprop(desc, dy, h, h_scale, gamma, rstd, dsum, dx, dgamma, workspace, workspace_bytes,
                                static_cast<cudaStream_t>(cuda_stream));
}

}  // extern "C"
