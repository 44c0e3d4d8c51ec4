// C ABI of the 8-bit matrix product (see include/maxdnn.h): tensor-copy descriptors and kernel
// launches.
#include <cstring>

#include "api8.h"
#include "gemm8.cuh"
#include "gemm8_mx.cuh"

namespace maxdnn {
namespace {

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

template <int NT, bool SBV>
maxdnn_status launch_gemm8(const RuntimeDevice& dev, const Gemm8Plan& p, const CUtensorMap& ma, const CUtensorMap& mb,
                           const Gemm8Args& args, cudaStream_t stream) {
  static std::atomic<bool> done[64];
  const maxdnn_status st = raise_smem(dev, done, gemm8_kernel<NT, SBV>);
  if (st != MAXDNN_OK) return st;
  return launch_early(gemm8_kernel<NT, SBV>, (unsigned)p.grid, gemm8_threads(NT), (size_t)p.smem_bytes, p.split, stream, ma, mb,
                      args);
}

template <int NT, bool PAIR>
maxdnn_status launch_gemm8_mx(const RuntimeDevice& dev, const Gemm8Plan& p, const CUtensorMap& ma,
                              const CUtensorMap& mb, const CUtensorMap& mc, const Gemm8MxArgs& args,
                              cudaStream_t stream) {
  static std::atomic<bool> done[64];
  const maxdnn_status st = raise_smem(dev, done, gemm8_mx_kernel<NT, PAIR>);
  if (st != MAXDNN_OK) return st;
  return launch_early(gemm8_mx_kernel<NT, PAIR>, (unsigned)p.grid, kMxThreads, (size_t)p.smem_bytes, PAIR ? 2 : p.split, stream,
                      ma, mb, mc, args);
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
  args.staged_c = p.staged_c;
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

maxdnn_status maxdnn_gemm8(const maxdnn_gemm8_desc* desc, const void* a, const void* a_scale, const void* b,
                           const void* b_scale, void* c, void* cuda_stream) {
  return maxdnn::gemm8(desc, a, a_scale, b, b_scale, c, static_cast<cudaStream_t>(cuda_stream));
}

}  // extern "C"
