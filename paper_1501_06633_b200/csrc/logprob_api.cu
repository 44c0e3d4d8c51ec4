// C ABI of the log probabilities (see include/maxdnn.h): argument checks and kernel launches.
#include <cmath>

#include "api8.h"
#include "logprob.cuh"

namespace maxdnn {
namespace {

maxdnn_status check_logprob(const maxdnn_logprob_desc* d) {
  if (!d || d->rows < 0 || d->cols <= 0 || d->top < 0) return MAXDNN_INVALID_VALUE;
  if (!is_wide(d->x_type) || d->ldx < d->cols) return MAXDNN_INVALID_VALUE;
  if (d->target_type != MAXDNN_INDEX_I32 && d->target_type != MAXDNN_INDEX_I64) return MAXDNN_INVALID_VALUE;
  if (!(d->scale > 0.f) || std::isinf(d->scale)) return MAXDNN_INVALID_VALUE;
  if (d->scale > 0x1p127f) return MAXDNN_NOT_SUPPORTED;      // (its multiple of log2 e, which differences are taken by, may be infinite)
  if (d->top > kLpMaxTop || d->cols > (1 << 30) || d->rows > (1 << 30)) return MAXDNN_NOT_SUPPORTED;      // (numbers of rows and columns are 32 bits)
  return MAXDNN_OK;
}

bool aligned_to(const void* p, uintptr_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

// CTAs that share a row, each with 16384 columns or more (joining costs as much as reading those: 20 rows of 32000 in 7.8 us
// by one CTA each and 8.7 by four): two where that gives an SM three at most (222 rows of 131072: 17.2 us, 18.9 by one), four and
// eight where it gives two (20 rows 10.8 us, 14.1 by one; 110 rows by four, three to an SM: 19.8 us, 13.7 by two).
int logprob_cluster(const maxdnn_logprob_desc& d, int sm_count) {
  int c = 1;
  while (c < kLpMaxCluster && (int64_t)d.rows * c * 2 <= (int64_t)sm_count * (c == 1 ? 3 : 2) && d.cols / (2 * c) >= 16384) c *= 2;
  return c;
}

maxdnn_status logprob_fprop(const maxdnn_logprob_desc* d, const void* x, const void* target, float* logprob, float* lse,
                            float* entropy, float* top_logprob, int32_t* top_index, cudaStream_t stream) {
  maxdnn_status st = check_logprob(d);
  if (st != MAXDNN_OK) return st;
  if (d->rows == 0) return MAXDNN_OK;
  if (!x || !aligned16(x)) return MAXDNN_INVALID_VALUE;
  if (!logprob && !lse && !entropy && !top_logprob && !top_index) return MAXDNN_INVALID_VALUE;
  if (logprob && !target) return MAXDNN_INVALID_VALUE;
  if (!aligned_to(target, d->target_type == MAXDNN_INDEX_I64 ? 8 : 4)) return MAXDNN_INVALID_VALUE;
  if ((top_logprob || top_index) && d->top == 0) return MAXDNN_INVALID_VALUE;
  RuntimeDevice dev;
  if ((st = runtime_device(&dev)) != MAXDNN_OK) return st;
  const int parts = logprob_cluster(*d, dev.sm_count);
  if ((int64_t)d->rows * parts > 0x7FFFFFFF) return MAXDNN_NOT_SUPPORTED;
  LogprobArgs a = {};
  a.x = x;
  a.target = target;
  a.logprob = logprob;
  a.lse = lse;
  a.entropy = entropy;
  a.top_logprob = top_logprob;
  a.top_index = top_index;
  a.ldx = d->ldx;
  a.rows = d->rows;
  a.cols = d->cols;
  a.top = top_logprob || top_index ? d->top : 0;
  a.wide_target = d->target_type == MAXDNN_INDEX_I64;
  a.scale = d->scale;
  return by_wide(d->x_type, [&](auto xt) {
    constexpr int X = decltype(xt)::value;
    // many rows: smaller CTAs, so that the end of one row is under way next to the readings of more others (4000 rows of 32000: 72 us
    // instead of 89, of 131072: 199 instead of 212; 500 rows: 16.7 and 44.2 us instead of 15.9 and 41.3)
    if (parts == 1 && d->rows >= 4 * dev.sm_count)
      return launch_early(entropy ? logprob_fprop_kernel<X, true, 128> : logprob_fprop_kernel<X, false, 128>, (unsigned)d->rows, 128, 0, 1,
                          stream, a);
    return launch_early(entropy ? logprob_fprop_kernel<X, true, 256> : logprob_fprop_kernel<X, false, 256>, (unsigned)(d->rows * parts), 256, 0,
                        parts, stream, a);
  });
}

maxdnn_status logprob_bprop(const maxdnn_logprob_desc* d, const void* x, const void* target, const float* lse, const float* dlogprob,
                            const float* entropy, const float* dentropy, void* dx, void* q_row, void* s_row, void* q_col,
                            void* s_col, cudaStream_t stream) {
  maxdnn_status st = check_logprob(d);
  if (st != MAXDNN_OK) return st;
  if (d->rows == 0) return MAXDNN_OK;
  if (!x || !lse || (!dx && !q_row && !q_col)) return MAXDNN_INVALID_VALUE;
  if ((!dlogprob && !dentropy) || (dlogprob && !target) || (dentropy && !entropy)) return MAXDNN_INVALID_VALUE;
  if ((q_row && !s_row) || (q_col && !s_col)) return MAXDNN_INVALID_VALUE;
  if (!aligned16(x) || !aligned16(dx) || !aligned16(q_row) || !aligned16(q_col)) return MAXDNN_INVALID_VALUE;
  if (!aligned_to(target, d->target_type == MAXDNN_INDEX_I64 ? 8 : 4)) return MAXDNN_INVALID_VALUE;
  const bool packed = q_row || q_col;
  if (dx && d->ldd < d->cols) return MAXDNN_INVALID_VALUE;
  if (dx == x && (d->ldd != d->ldx || packed)) return MAXDNN_INVALID_VALUE;
  if (packed) {
    if (!is_fp8(d->q_type) || d->ldq < d->cols) return MAXDNN_INVALID_VALUE;
    if (d->ldq % 16 != 0) return MAXDNN_NOT_SUPPORTED;
  }
  const int64_t chunks = packed ? blocks_of(d->cols) : ((int64_t)d->cols + kLpBackCols - 1) / kLpBackCols;
  const int64_t grid = chunks * (packed ? blocks_of(d->rows) : d->rows);
  if (grid > 0x7FFFFFFF) return MAXDNN_NOT_SUPPORTED;
  RuntimeDevice dev;
  if ((st = runtime_device(&dev)) != MAXDNN_OK) return st;
  LogprobArgs a = {};
  a.x = x;
  a.target = target;
  a.lse = const_cast<float*>(lse);
  a.entropy = const_cast<float*>(entropy);
  a.dlogprob = dlogprob;
  a.dentropy = dentropy;
  a.dx = dx;
  a.q_row = static_cast<uint8_t*>(q_row);
  a.s_row = static_cast<uint8_t*>(s_row);
  a.q_col = static_cast<uint8_t*>(q_col);
  a.s_col = static_cast<uint8_t*>(s_col);
  a.ldx = d->ldx;
  a.ldd = d->ldd;
  a.ldq = d->ldq;
  a.rows = d->rows;
  a.cols = d->cols;
  a.wide_target = d->target_type == MAXDNN_INDEX_I64;
  a.chunks = (int32_t)chunks;
  a.scale = d->scale;
  return by_wide(d->x_type, [&](auto xt) {
    constexpr int X = decltype(xt)::value;
    if (packed)
      return by_fp8(d->q_type, [&](auto qt) {
        return by_edge(d->cols % 8 == 0 && vec_ok(d->x_type, d->ldx), [&](auto edge) {
          return launch_early(logprob_bprop_packed_kernel<X, decltype(qt)::value, decltype(edge)::value != 0>, (unsigned)grid, kLpPackThreads, 0, 1,
                              stream, a);
        });
      });
    // (rows of x and dx that start at the same place in 16 bytes: both bases do)
    const bool same = (d->ldx - d->ldd) * elem_bytes(d->x_type) % 16 == 0;
    return launch_early(same ? logprob_bprop_kernel<X, true> : logprob_bprop_kernel<X, false>, (unsigned)grid, kLpThreads, 0, 1, stream, a);
  });
}

}  // namespace
}  // namespace maxdnn

extern "C" {

maxdnn_status maxdnn_logprob_fprop(const maxdnn_logprob_desc* desc, const void* x, const void* target, float* logprob, float* lse,
                                   float* entropy, float* top_logprob, int32_t* top_index, void* cuda_stream) {
  return maxdnn::logprob_fprop(desc, x, target, logprob, lse, entropy, top_logprob, top_index, static_cast<cudaStream_t>(cuda_stream));
}

maxdnn_status maxdnn_logprob_bprop(const maxdnn_logprob_desc* desc, const void* x, const void* target, const float* lse,
                                   const float* dlogprob, const float* entropy, const float* dentropy, void* dx, void* q_row,
                                   void* s_row, void* q_col, void* s_col, void* cuda_stream) {
  return maxdnn::logprob_bprop(desc, x, target, lse, dlogprob, entropy, dentropy, dx, q_row, s_row, q_col, s_col,
                               static_cast<cudaStream_t>(cuda_stream));
}

}  // extern "C"
