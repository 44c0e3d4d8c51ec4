// C ABI of the orthogonalised update (see include/maxdnn.h): tensor-copy descriptors and kernel launches.
#include <algorithm>
#include <cmath>
#include <cstring>

#include "api8.h"
#include "ortho.cuh"

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
maxdnn_status operand_map(CUtensorMap* m, const Matrices& x, int batch, bool mn, int rows) {
  return matrix_map(m, x, batch, 64u, mn ? 64u : (uint32_t)rows, CU_TENSOR_MAP_SWIZZLE_128B);
}
maxdnn_status part_map(CUtensorMap* m, const Matrices& x, int batch) {
  return matrix_map(m, x, batch, 32u, 32u, CU_TENSOR_MAP_SWIZZLE_64B);
}

struct OrthoMaps { CUtensorMap a, b, in, in_lo, out, out_lo; };

template <int NT, bool PAIR, int KIND>
maxdnn_status launch_ortho(const RuntimeDevice& dev, const OrthoProduct& p, const OrthoMaps& m, const OrthoArgs& args, cudaStream_t stream) {
  static std::atomic<bool> done[64];
  if (!done[dev.index].load(std::memory_order_acquire)) {      // raising it twice does no harm
    if (cudaFuncSetAttribute(ortho_product_kernel<NT, PAIR, KIND>, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024) != cudaSuccess) {
      cudaGetLastError();
      return MAXDNN_CUDA_ERROR;
    }
    done[dev.index].store(true, std::memory_order_release);
  }
  return launch_early(ortho_product_kernel<NT, PAIR, KIND>, (unsigned)p.grid, kOrthoThreads, (size_t)p.smem_bytes, PAIR ? 2 : 1, stream, m.a,
                      m.b, m.in, m.in_lo, m.out, m.out_lo, args);
}

template <int KIND>
maxdnn_status run_product(const RuntimeDevice& dev, const OrthoProduct& p, const OrthoMaps& m, OrthoArgs args, bool a_mn, bool b_mn, int batch,
                          cudaStream_t stream) {
  args.M = p.M;
  args.N = p.N;
  args.batch = batch;
  args.m_tiles = p.m_tiles;
  args.n_tiles = p.n_tiles;
  args.tiles = p.tiles;
  args.k_steps = p.k_steps;
  args.stages = p.stages;
  args.a_mn = a_mn;
  args.b_mn = b_mn;
  args.b_rows = p.b_rows;
  args.b_stage_bytes = p.b_stage_bytes;
  // instruction descriptor: fp32 accumulator, FP16 operands, majors, N / 8, M / 16
  args.idesc = (1u << 4) | ((uint32_t)a_mn << 15) | ((uint32_t)b_mn << 16) | ((uint32_t)(p.nt >> 3) << 17) |
               ((uint32_t)((p.pair ? 2 : 1) * kOrthoTileM >> 4) << 24);
  args.test_missing_arrival = (uint32_t)option(OPT_TEST_MISSING_ARRIVAL);
  args.wc = runtime_wait_ctx(dev);
#define MAXDNN_ORTHO_CASE(NT, PAIR) \
  if (p.nt == (NT) && (p.pair != 0) == (PAIR)) return launch_ortho<NT, PAIR, KIND>(dev, p, m, args, stream);
  MAXDNN_ORTHO_CASE(256, true)
  MAXDNN_ORTHO_CASE(128, true)
  MAXDNN_ORTHO_CASE(128, false)
  MAXDNN_ORTHO_CASE(64, false)
#undef MAXDNN_ORTHO_CASE
  return MAXDNN_NOT_SUPPORTED;
}

maxdnn_status orthogonalise_workspace(const maxdnn_ortho_desc* d, size_t* bytes) {
  maxdnn_status st = check_ortho(d);
  if (st != MAXDNN_OK || !bytes) return st != MAXDNN_OK ? st : MAXDNN_INVALID_VALUE;
  OrthoPlan p;
  if ((st = plan_ortho(*d, 148, &p)) != MAXDNN_OK) return st;      // (the layout does not depend on the device)
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
  if ((st = plan_ortho(*d, 148, &p)) != MAXDNN_OK) return st;
  if (!workspace || !aligned16(workspace) || workspace_bytes < (size_t)p.bytes) return MAXDNN_INVALID_VALUE;
  RuntimeDevice dev;
  if ((st = runtime_device(&dev)) != MAXDNN_OK) return st;
  if (dev.sm_count != 148 && (st = plan_ortho(*d, dev.sm_count, &p)) != MAXDNN_OK) return st;
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

  // ---- tensor-copy descriptors: Gram and update read X [0] and X [1] in turn
  OrthoMaps gram[2], poly, update[2], last;
  memset(gram, 0, sizeof(gram));
  memset(&poly, 0, sizeof(poly));
  memset(update, 0, sizeof(update));
  auto ok = [&](maxdnn_status r) { st = st == MAXDNN_OK ? r : st; };
  const bool tall = p.tall != 0;
  for (int w = 0; w < 2; ++w) {
    // the reduction runs along the longer side: rows of X where tall
    ok(operand_map(&gram[w].a, mx[w][0], batch, tall, kOrthoTileM));
    ok(operand_map(&gram[w].b, mx[w][0], batch, tall, p.gram.b_rows));
    ok(part_map(&gram[w].out, ma, batch));
    // X from the right (its rows are the reduction), or from the left
    if (tall) {
      ok(operand_map(&update[w].a, mx[w][0], batch, false, kOrthoTileM));
      ok(operand_map(&update[w].b, mb, batch, false, p.update.b_rows));
    } else {
      ok(operand_map(&update[w].a, mb, batch, false, kOrthoTileM));
      ok(operand_map(&update[w].b, mx[w][0], batch, true, p.update.b_rows));
    }
    ok(part_map(&update[w].in, mx[w][0], batch));
    ok(part_map(&update[w].in_lo, mx[w][1], batch));
    ok(part_map(&update[w].out, mx[1 - w][0], batch));
    ok(part_map(&update[w].out_lo, mx[1 - w][1], batch));
  }
  ok(operand_map(&poly.a, ma, batch, false, kOrthoTileM));
  ok(operand_map(&poly.b, ma, batch, false, p.poly.b_rows));
  ok(part_map(&poly.in, ma, batch));
  ok(part_map(&poly.out, mb, batch));
  last = update[(d->steps - 1) & 1];
  if (bulk_out) ok(part_map(&last.out, mo, batch));
  if (st != MAXDNN_OK) return st;

  // ---- steps
  OrthoArgs args = {};
  args.diag = p.diag;
  args.diag_cols = tall;
  args.bulk_out = bulk_out;
  args.out = static_cast<__nv_bfloat16*>(out);
  args.ldo = d->ldo;
  args.stride_o = d->stride_o;
  args.post = s.post;
  float* diag_a = reinterpret_cast<float*>(ws + p.diag_a);
  float* diag_b = reinterpret_cast<float*>(ws + p.diag_b);
  for (int i = 0; i < d->steps; ++i) {
    const float* c = coefficients ? coefficients + 3 * i : kOrthoCoefficients;
    args.ca = c[0];
    args.cb = c[1];
    args.cc = c[2];
    args.scale = std::ldexp(1.f, -2 * kOrthoScaleBits);
    args.diag_in = nullptr;
    args.diag_out = diag_a;
    if ((st = run_product<kOrthoGram>(dev, p.gram, gram[i & 1], args, tall, tall, batch, stream)) != MAXDNN_OK) return st;
    args.diag_in = diag_a;
    args.diag_out = diag_b;
    if ((st = run_product<kOrthoPoly>(dev, p.poly, poly, args, false, false, batch, stream)) != MAXDNN_OK) return st;
    args.scale = std::ldexp(1.f, -kOrthoScaleBits);
    args.diag_in = diag_b;
    args.diag_out = nullptr;
    st = i + 1 < d->steps ? run_product<kOrthoUpdate>(dev, p.update, update[i & 1], args, false, !tall, batch, stream)
                          : run_product<kOrthoLast>(dev, p.update, last, args, false, !tall, batch, stream);
    if (st != MAXDNN_OK) return st;
  }
  return MAXDNN_OK;
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
