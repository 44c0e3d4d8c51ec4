// Host-side planning of the 8-bit matrix product: argument checks and the choice of tile, operand
// roles and split.  Plain C++, no CUDA calls.
#pragma once
#include <stdint.h>

#include "../../include/maxdnn.h"
#include "plan.h"

namespace maxdnn {

constexpr int kGemm8TileM = 128;     // rows of a tile (TMEM lanes)
constexpr int kGemm8BlockK = 128;    // reduction steps per stage: one scale block
constexpr int kGemm8MaxSplit = 8;    // CTAs of a cluster that share one tile's reduction

// Tensor memory of a CTA.  gemm8.cuh: two accumulators of nt columns.  gemm8_mx.cuh: two where they
// fit (else one), and kMxScaleTmem groups of scale columns: four for 128 rows of A, four for each
// 128 columns of B.
constexpr int kMxScaleTmem = 4;
MAXDNN_HD constexpr int gemm8_tmem_cols(int nt) { return 2 * nt < 32 ? 32 : 2 * nt; }
MAXDNN_HD constexpr int mx_buffers(int nt) { return nt <= 224 ? 2 : 1; }
MAXDNN_HD constexpr int mx_sf_cols(int nt) { return 4 + 4 * ((nt + 127) / 128); }
MAXDNN_HD constexpr int mx_tmem_cols(int nt) {
  const int need = mx_buffers(nt) * nt + kMxScaleTmem * mx_sf_cols(nt);
  return need <= 64 ? 64 : need <= 128 ? 128 : need <= 256 ? 256 : 512;
}

struct Gemm8Plan {
  int32_t mx;          // 1: the tensor core applies the scales (both operands' are E8M0 bytes)
  int32_t pair;        // 1: tiles of 256 rows on two SMs
  int32_t swap;        // 1: the kernel's rows are the columns of C (few rows of C)
  int32_t tile_n;      // columns of a tile
  int32_t chunk;       // mx: blocks of the reduction per accumulator (a multiple of four)
  int32_t bulk_c;      // mx: C is stored by bulk tensor copies
  int32_t staged_c;    // mx: C goes through staging tiles in shared memory
  int32_t split;       // CTAs that share a tile's reduction: 1, 2, 4 or 8
  int32_t m_tiles, n_tiles, k_blocks;
  int32_t stages;
  int32_t b_stage_bytes;
  int32_t grid;
  int32_t smem_bytes;
};

maxdnn_status check_gemm8(const maxdnn_gemm8_desc* d);
maxdnn_status plan_gemm8(const maxdnn_gemm8_desc& d, int sm_count, Gemm8Plan* plan);

}  // namespace maxdnn
