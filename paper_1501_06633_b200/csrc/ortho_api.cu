// C ABI of the orthogonalised update (see include/maxdnn.h): tensor-copy descriptors and kernel launches.
#include <algorithm>
#include <cmath>
#include <cstring>

#include "api8.h"
#include "ortho.cuh"
#include "ortho_small.cuh"

namespace maxdnn {
namespace {

constexpr float kOrthoCoefficients[3] = {3.4445f, -4.7750f, 2.0315f};

// A batch of matrices [rows][cols] in 16-bit elements with row pitch ld.
struct Matrices {
  const void* p;
  int64_t rows, cols, ld, stride;
  CUtensorMapDataType type;
};

maxdnn_status matrix_map(CUtensorMap* m, const Matrices& x, int batch, uint32_t box_cols, uint32_t box_rows, CUtensorMapSwizzle swz) {
  const uint64_t dims[3] = {(uint64_t)x.cols, (uint64_t)x.rows, (uint64_t)batch};
  // (one matrix: any stride will do that the descriptor takes)
  const uint64_t str[2] = {(uint64_t)x.ld * 2, (uint64_t)(batch > 1 ? x.stride : x.rows * x.ld) * 2};
  const uint32_t box[3] = {box_cols, box_rows, 1u};
  return runtime_encode(m, x.type, 3, x.p, dims, str, box, swz);
}
maxdnn_status operand_map(CUtensorMap* m, const Matrices& x, int batch) { return matrix_map(m, x, batch, 64u, 64u, CU_TENSOR_MAP_SWIZZLE_128B); }
maxdnn_status part_map(CUtensorMap* m, const Matrices& x, int batch) { return matrix_map(m, x, batch, 32u, 32u, CU_TENSOR_MAP_SWIZZLE_64B); }

// Runs f with the kernel of a shape, and its PAIR.
template <class F>
maxdnn_status by_shape(int pair, int nt, F f) {
  if (pair && nt == 256) return f(ortho_chain_kernel<256, true>);
  if (pair && nt == 128) return f(ortho_chain_kernel<128, true>);
  if (!pair && nt == 128) return f(ortho_chain_kernel<128, false>);
  if (!pair && nt == 64) return f(ortho_chain_kernel<64, false>);
  return MAXDNN_NOT_SUPPORTED;
}

constexpr size_t kOrthoSmem = 227 * 1024;      // a CTA has an SM to itself

cudaLaunchConfig_t chain_config(cudaLaunchAttribute (&attr)[2], int grid, int pair, size_t smem, cudaStream_t stream) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)grid, 1, 1);
  cfg.blockDim = dim3(kOrthoThreads, 1, 1);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  attr[0].id = cudaLaunchAttributeCooperative;      // its CTAs wait for one another
  attr[0].val.cooperative = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = 2;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = pair ? 2 : 1;
  return cfg;
}

// CTAs and pairs of CTAs that a device runs at the same time, set up on its first call.
maxdnn_status chain_slots(const RuntimeDevice& dev, int (&slots)[2]) {
  static std::atomic<int> known[64];      // pairs + 1
  int pairs = known[dev.index].load(std::memory_order_acquire) - 1;
  if (pairs < 0) {
    for (int pair = 0; pair < 2; ++pair)
      for (int nt : {256, 128, 64}) {
        if (pair ? nt == 64 : nt == 256) continue;
        const maxdnn_status st = by_shape(pair, nt, [&](auto kern) {
          if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kOrthoSmem) != cudaSuccess) {
            cudaGetLastError();
            return MAXDNN_CUDA_ERROR;
          }
          return MAXDNN_OK;
        });
        if (st != MAXDNN_OK) return st;
      }
    cudaLaunchAttribute attr[2];
    const cudaLaunchConfig_t cfg = chain_config(attr, dev.sm_count / 2 * 2, 1, kOrthoSmem, nullptr);
    if (cudaOccupancyMaxActiveClusters(&pairs, ortho_chain_kernel<256, true>, &cfg) != cudaSuccess) {
      cudaGetLastError();
      pairs = 0;
    }
    pairs = std::min(pairs, dev.sm_count / 2);
    known[dev.index].store(pairs + 1, std::memory_order_release);
  }
  slots[0] = dev.sm_count;
  slots[1] = pairs;
  return MAXDNN_OK;
}

constexpr int kNominalSlots[2] = {148, 74};      // (the workspace's layout does not depend on the device)

constexpr size_t small_smem() { return (size_t)std::max(kSmallSmem, cluster_smem_floor(kSmallTmem)); }

// CTAs of the cluster that has a matrix to itself, where there is one; 0: it goes through memory.  A cluster of more than one CTA
// needs as many SMs next to one another, which a device may not have (more than eight are no part of what every device offers).
int small_cluster(const RuntimeDevice& dev, const maxdnn_ortho_desc& d) {
  const int longer = std::max(d.rows, d.cols), parts = (longer + kSmallSlice - 1) / kSmallSlice;
  if (std::min(d.rows, d.cols) > kSmallN || parts > std::min(kSmallMaxCluster, option(OPT_ORTHO_CLUSTER, kSmallMaxCluster))) return 0;
  if (parts == 1) return 1;
  static std::atomic<int> known[64][kSmallMaxCluster + 1];      // clusters that run at the same time + 1; 0: not asked for yet
  int n = known[dev.index][parts].load(std::memory_order_acquire) - 1;
  if (n < 0) {
    // (any of the kernels: all have the same threads and memory)
    auto kern = ortho_small_kernel<MAXDNN_BF16, false, false>;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)parts, 1, 1);
    cfg.blockDim = dim3(kSmallThreads, 1, 1);
    cfg.dynamicSmemBytes = small_smem();
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = (unsigned)parts;
    attr.val.clusterDim.y = 1;
    attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)small_smem()) != cudaSuccess ||
        cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess ||
        cudaOccupancyMaxActiveClusters(&n, kern, &cfg) != cudaSuccess) {
      cudaGetLastError();
      n = 0;
    }
    known[dev.index][parts].store(n + 1, std::memory_order_release);
  }
  return n > 0 ? parts : 0;
}

maxdnn_status orthogonalise_small(const RuntimeDevice& dev, const maxdnn_ortho_desc& d, int parts, const void* x, const float* coefficients,
                                  void* out, cudaStream_t stream) {
  OrthoSmallArgs a = {};
  a.x = x;
  a.out = static_cast<__nv_bfloat16*>(out);
  a.ldx = d.ldx;
  a.ldo = d.ldo;
  a.stride_x = d.stride_x;
  a.stride_o = d.stride_o;
  a.rows = d.rows;
  a.cols = d.cols;
  a.steps = d.steps;
  a.eps = d.eps;
  for (int i = 0; i < d.steps; ++i)
    for (int k = 0; k < 3; ++k) a.coefficients[i][k] = coefficients ? coefficients[3 * i + k] : kOrthoCoefficients[k];
  a.test_missing_arrival = (uint32_t)option(OPT_TEST_MISSING_ARRIVAL);
  a.wc = runtime_wait_ctx(dev);
  const size_t smem = small_smem();
  const bool whole = d.cols % 8 == 0 && vec_ok(d.x_type, d.ldx) && (d.batch == 1 || vec_ok(d.x_type, d.stride_x));
  return by_wide(d.x_type, [&](auto xt) {
    return by_edge(whole, [&](auto edge) {
      constexpr int X = decltype(xt)::value;
      constexpr bool E = decltype(edge)::value != 0;
      const bool tall = d.rows > d.cols;
      auto kern = tall ? ortho_small_kernel<X, true, E> : ortho_small_kernel<X, false, E>;
      static std::atomic<bool> done[2][64];
      if (!done[tall][dev.index].load(std::memory_order_acquire)) {
        if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess ||
            cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess) {
          cudaGetLastError();
          return MAXDNN_CUDA_ERROR;
        }
        done[tall][dev.index].store(true, std::memory_order_release);
      }
      return launch_early(kern, (unsigned)(d.batch * parts), kSmallThreads, smem, parts, stream, a);
    });
  });
}

maxdnn_status orthogonalise_workspace(const maxdnn_ortho_desc* d, size_t* bytes) {
  maxdnn_status st = check_ortho(d);
  if (st != MAXDNN_OK || !bytes) return st != MAXDNN_OK ? st : MAXDNN_INVALID_VALUE;
  OrthoPlan p;
  if ((st = plan_ortho(*d, kNominalSlots, &p)) != MAXDNN_OK) return st;
  *bytes = (size_t)p.bytes;
  return MAXDNN_OK;
}

maxdnn_status orthogonalise(const maxdnn_ortho_desc* d, const void* x, const float* coefficients, void* out, void* workspace,
                            size_t workspace_bytes, cudaStream_t stream) {
  maxdnn_status st = check_ortho(d);
  if (st != MAXDNN_OK) return st;
  if (d->batch == 0) return MAXDNN_OK;
  if (!x || !out || !aligned16(x) || !aligned16(out)) return MAXDNN_INVALID_VALUE;
  if (coefficients)
    for (int i = 0; i < 3 * d->steps; ++i)
      if (!std::isfinite(coefficients[i])) return MAXDNN_INVALID_VALUE;
  OrthoPlan p;
  if ((st = plan_ortho(*d, kNominalSlots, &p)) != MAXDNN_OK) return st;
  if (!workspace || !aligned16(workspace) || workspace_bytes < (size_t)p.bytes) return MAXDNN_INVALID_VALUE;
  RuntimeDevice dev;
  if ((st = runtime_device(&dev)) != MAXDNN_OK) return st;
  if (const int parts = small_cluster(dev, *d)) return orthogonalise_small(dev, *d, parts, x, coefficients, out, stream);
  int slots[2];
  if ((st = chain_slots(dev, slots)) != MAXDNN_OK) return st;
  if ((st = plan_ortho(*d, slots, &p)) != MAXDNN_OK) return st;
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  const int batch = d->batch;
  auto up8 = [](int64_t v) { return (v + 7) / 8 * 8; };
  // columns up to the next multiple of eight are part of the matrices: they hold zeros
  auto inside = [&](int64_t at, int64_t rows, int64_t cols, int64_t pitch) {
    return Matrices{ws + at, rows, up8(cols), pitch, rows * pitch, CU_TENSOR_MAP_DATA_TYPE_FLOAT16};
  };
  Matrices mx[2][2];
  for (int w = 0; w < 2; ++w)
    for (int part = 0; part < 2; ++part) mx[w][part] = inside(p.x[w][part], d->rows, d->cols, p.pitch_x);
  const Matrices ma = inside(p.a, p.n, p.n, p.pitch_n), mb = inside(p.b, p.n, p.n, p.pitch_n);
  const Matrices mo = {out, d->rows, d->cols, d->ldo, d->stride_o, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16};
  const bool bulk_out = d->ldo % 8 == 0 && d->cols % 8 == 0 && (batch == 1 || d->stride_o % 8 == 0);

  // ---- X
  OrthoStartArgs s = {};
  s.x = x;
  s.hi = reinterpret_cast<__half*>(ws + p.x[0][0]);
  s.lo = reinterpret_cast<__half*>(ws + p.x[0][1]);
  s.sums = reinterpret_cast<double*>(ws + p.sums);
  s.diag_a = reinterpret_cast<float*>(ws + p.diag_a);
  s.diag_b = reinterpret_cast<float*>(ws + p.diag_b);
  s.post = reinterpret_cast<float*>(ws + p.post);
  s.done = reinterpret_cast<uint32_t*>(ws + p.done);
  s.growth = 1.f;
  float grown = 1.f;
  for (int i = 0; i < d->steps; ++i) {
    grown *= std::fabs(coefficients ? coefficients[3 * i] : kOrthoCoefficients[0]);
    s.growth = std::max(s.growth, grown);
  }
  s.ldx = d->ldx;
  s.stride_x = d->stride_x;
  s.pitch = p.pitch_x;
  s.diag = p.diag;
  s.rows = d->rows;
  s.cols = d->cols;
  s.parts = p.parts;
  s.eps = d->eps;
  const int64_t most = std::max<int64_t>(1, (int64_t)dev.sm_count * 8 / batch), want = ((int64_t)d->rows + 7) / 8;
  s.row_ctas = (int32_t)std::min(want, most);
  const bool whole = d->cols % 8 == 0 && vec_ok(d->x_type, d->ldx) && (batch == 1 || vec_ok(d->x_type, d->stride_x));
  st = by_wide(d->x_type, [&](auto xt) {
    return by_edge(whole, [&](auto edge) {
      constexpr int X = decltype(xt)::value;
      constexpr bool E = decltype(edge)::value != 0;
      const maxdnn_status first = launch_early(ortho_sum_kernel<X, E>, (unsigned)(batch * p.parts), kOrthoStartThreads, 0, 1, stream, s);
      if (first != MAXDNN_OK) return first;
      return launch_early(ortho_start_kernel<X, E>, (unsigned)(batch * s.row_ctas), kOrthoStartThreads, 0, 1, stream, s);
    });
  });
  if (st != MAXDNN_OK) return st;

  // ---- all steps
  OrthoMaps maps;
  memset(&maps, 0, sizeof(maps));
  auto ok = [&](maxdnn_status r) { st = st == MAXDNN_OK ? r : st; };
  for (int w = 0; w < 2; ++w) {
    ok(operand_map(&maps.x[w], mx[w][0], batch));
    ok(part_map(&maps.x_hi[w], mx[w][0], batch));
    ok(part_map(&maps.x_lo[w], mx[w][1], batch));
  }
  ok(operand_map(&maps.a, ma, batch));
  ok(operand_map(&maps.b, mb, batch));
  ok(part_map(&maps.a_part, ma, batch));
  ok(part_map(&maps.b_part, mb, batch));
  if (bulk_out) ok(part_map(&maps.out, mo, batch));
  if (st != MAXDNN_OK) return st;
  OrthoArgs args = {};
  for (int i = 0; i < 3; ++i) args.product[i] = p.product[i];
  args.steps = d->steps;
  args.batch = batch;
  args.stages = p.stages;
  args.tall = p.tall;
  args.bulk_out = bulk_out;
  args.diag_a = s.diag_a;
  args.diag_b = s.diag_b;
  args.diag = p.diag;
  args.post = s.post;
  args.done = s.done;
  args.out = static_cast<__nv_bfloat16*>(out);
  args.ldo = d->ldo;
  args.stride_o = d->stride_o;
  args.test_missing_arrival = (uint32_t)option(OPT_TEST_MISSING_ARRIVAL);
  for (int i = 0; i < d->steps; ++i)
    for (int k = 0; k < 3; ++k) args.coefficients[i][k] = coefficients ? coefficients[3 * i + k] : kOrthoCoefficients[k];
  args.wc = runtime_wait_ctx(dev);
  return by_shape(p.pair, p.nt, [&](auto kern) {
    cudaLaunchAttribute attr[2];
    const cudaLaunchConfig_t cfg = chain_config(attr, p.grid, p.pair, (size_t)p.smem_bytes, stream);
    if (cudaLaunchKernelEx(&cfg, kern, maps, args) != cudaSuccess) {
      cudaGetLastError();
      return MAXDNN_CUDA_ERROR;
    }
    runtime_count_launch();
    return MAXDNN_OK;
  });
}

}  // namespace
}  // namespace maxdnn

extern "C" {

maxdnn_status maxdnn_orthogonalise_workspace(const maxdnn_ortho_desc* desc, size_t* bytes) {
  return maxdnn::orthogonalise_workspace(desc, bytes);
}

maxdnn_status maxdnn_orthogonalise(const maxdnn_ortho_desc* desc, const void* x, const float* coefficients, void* out, void* workspace,
                                   size_t workspace_bytes, void* cuda_stream) {
  return maxdnn::orthogonalise(desc, x, coefficients, out, workspace, workspace_bytes, static_cast<cudaStream_t>(cuda_stream));
}

}  // extern "C"
