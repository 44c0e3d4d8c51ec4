// What the entry points of the 8-bit training operators share on the host: alignment checks and
// dispatch over element types.
#pragma once
#include "fp8_util.cuh"
#include "plan.h"
#include "runtime.h"

namespace maxdnn {

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline int64_t blocks_of(int64_t n) { return (n + kBlock8 - 1) / kBlock8; }

// Whether rows of `ld` elements of type `dt` that start `off` elements in allow loads of eight values.
inline int vec_ok(int dt, int64_t ld, int64_t off = 0) {
  const int64_t unit = is_fp8(dt) ? 8 : 16;
  return (ld * elem_bytes(dt)) % unit == 0 && (off * elem_bytes(dt)) % unit == 0;
}

// A launch that may start while the kernel before it in the stream still runs (the kernels wait for
// its end themselves: wait_for_previous).  Two calls in a row of a few microseconds each overlap
// their starts: 1.5 to 2 us less for the second.
template <class... P, class... A>
maxdnn_status launch_early(void (*kern)(P...), unsigned grid, unsigned threads, size_t smem, int cluster,
                           cudaStream_t stream, A... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid, 1, 1);
  cfg.blockDim = dim3(threads, 1, 1);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)cluster;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  if (cudaLaunchKernelEx(&cfg, kern, static_cast<P>(args)...) != cudaSuccess) {
    cudaGetLastError();
    return MAXDNN_CUDA_ERROR;
  }
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

}  // namespace maxdnn
