// Planning of the 8-bit matrix product (see gemm8.h).
#include "gemm8.h"

#include <algorithm>

#include "plan.h"

namespace maxdnn {

namespace {

bool fp8(int t) { return t == MAXDNN_E4M3 || t == MAXDNN_E5M2; }

// 128-byte rows of packed values: what an operand's copies and scales need of its description.
maxdnn_status check_operand(int type, int major, int block, int scale_type, int64_t ld, int mn, int k) {
  if (!fp8(type)) return MAXDNN_INVALID_VALUE;
  if (major != MAXDNN_MAJOR_K && major != MAXDNN_MAJOR_MN) return MAXDNN_INVALID_VALUE;
  if (scale_type != MAXDNN_E8M0 && scale_type != MAXDNN_F32) return MAXDNN_INVALID_VALUE;
  // blocks lie along the reduction: row blocks of a K-major matrix, column blocks of the other
  const int along = major == MAXDNN_MAJOR_K ? MAXDNN_BLOCK_ROW : MAXDNN_BLOCK_COL;
  if (block != along && block != MAXDNN_BLOCK_TILE) return MAXDNN_INVALID_VALUE;
  if (ld < (major == MAXDNN_MAJOR_K ? k : mn)) return MAXDNN_INVALID_VALUE;
  if (ld % 16 != 0) return MAXDNN_NOT_SUPPORTED;
  return MAXDNN_OK;
}

}  // namespace

maxdnn_status check_gemm8(const maxdnn_gemm8_desc* d) {
  if (!d || d->M < 0 || d->N < 0 || d->K < 0) return MAXDNN_INVALID_VALUE;
  if (d->c_type != MAXDNN_F32 && d->c_type != MAXDNN_BF16 && d->c_type != MAXDNN_F16) return MAXDNN_INVALID_VALUE;
  if (d->ldc < d->N) return MAXDNN_INVALID_VALUE;
  maxdnn_status st = check_operand(d->a_type, d->a_major, d->a_block, d->a_scale_type, d->lda, d->M, d->K);
  if (st != MAXDNN_OK) return st;
  st = check_operand(d->b_type, d->b_major, d->b_block, d->b_scale_type, d->ldb, d->N, d->K);
  if (st != MAXDNN_OK) return st;
  if (d->M > (1 << 30) || d->N > (1 << 30) || d->K > (1 << 30)) return MAXDNN_NOT_SUPPORTED;
  return MAXDNN_OK;
}

maxdnn_status plan_gemm8(const maxdnn_gemm8_desc& d, int sm_count, Gemm8Plan* plan) {
  static const int kTileN[5] = {16, 32, 64, 128, 256};
  static const int kSplit[4] = {1, 2, 4, 8};
  const int k_blocks = (d.K + kGemm8BlockK - 1) / kGemm8BlockK;
  double best = 0;
  bool found = false;
  for (int swap = 0; swap < 2; ++swap) {
    if (option_is_set(OPT_GEMM8_SWAP) && option(OPT_GEMM8_SWAP) != swap) continue;
    const int64_t M = swap ? d.N : d.M, N = swap ? d.M : d.N;
    const int b_major = swap ? d.a_major : d.b_major;
    for (int nt : kTileN) {
      if (option_is_set(OPT_GEMM8_COLS) && option(OPT_GEMM8_COLS) != nt) continue;
      const int64_t m_tiles = (M + kGemm8TileM - 1) / kGemm8TileM, n_tiles = (N + nt - 1) / nt;
      const int64_t tiles = m_tiles * n_tiles;
      const int b_stage = b_major == MAXDNN_MAJOR_MN ? std::max(nt, 128) * 128 : nt * 128;
      // clocks of one block: MMAs, reading and adding the product, filling the stage
      const double mma = 2.0 * nt, add = 100.0 + 1.2 * nt, fill = (16384 + b_stage) / 48.0;
      const double per_block = std::max(mma, std::max(add, fill));
      for (int split : kSplit) {
        if (option_is_set(OPT_GEMM8_SPLIT) && option(OPT_GEMM8_SPLIT) != split) continue;
        if (split > k_blocks) continue;
        if (split > 1 && tiles * split > 2 * sm_count && !option_is_set(OPT_GEMM8_SPLIT)) continue;
        const int64_t units = split == 1 ? std::min<int64_t>(tiles, sm_count) : tiles;
        const int64_t waves = split == 1 ? (tiles + sm_count - 1) / sm_count : (tiles * split + sm_count - 1) / sm_count;
        const int64_t blocks = (k_blocks + split - 1) / split;
        const double t = (double)waves * ((double)blocks * per_block + 1500.0) + (split > 1 ? 1500.0 + 4.0 * nt : 0.0);
        if (found && t >= best) continue;
        found = true;
        best = t;
        plan->swap = swap;
        plan->tile_n = nt;
        plan->split = split;
        plan->m_tiles = (int32_t)m_tiles;
        plan->n_tiles = (int32_t)n_tiles;
        plan->k_blocks = k_blocks;
        plan->b_stage_bytes = b_stage;
        plan->grid = (int32_t)(units * split);
      }
    }
  }
  if (!found) return MAXDNN_NOT_SUPPORTED;
  if ((int64_t)plan->m_tiles * plan->n_tiles > (1 << 30)) return MAXDNN_NOT_SUPPORTED;
  const int warps = 4 * (plan->tile_n < 64 ? 1 : plan->tile_n / 64), cw = std::min(plan->tile_n, 64);
  const int fixed = 1024 + 64 + warps * 2 * cw * 4;
  const int per_stage = 16384 + plan->b_stage_bytes + 16;
  plan->stages = std::min(12, (232448 - fixed) / per_stage);
  plan->smem_bytes = fixed + plan->stages * per_stage;
  return MAXDNN_OK;
}

}  // namespace maxdnn
