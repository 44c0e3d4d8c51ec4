// Planning of the 8-bit matrix product (see gemm8.h).
#include "gemm8.h"

#include <algorithm>

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

// One tile shape of the search below, with what it measured (microseconds): a block of the
// reduction in a long run, and what a tile takes besides (ring fill, reading and storing the result).
struct Shape { int mx, pair, nt; double block, tile; };

maxdnn_status plan_gemm8(const maxdnn_gemm8_desc& d, int sm_count, Gemm8Plan* plan) {
  static const Shape kShapes[] = {
      {1, 0, 16, 0.20, 1.6}, {1, 0, 32, 0.20, 1.6}, {1, 0, 64, 0.21, 1.8}, {1, 0, 128, 0.28, 2.0},
      {1, 1, 128, 0.255, 3.1}, {1, 1, 192, 0.32, 3.6}, {1, 1, 224, 0.37, 3.8}, {1, 1, 256, 0.42, 4.0},
      {0, 0, 16, 0.35, 1.6}, {0, 0, 32, 0.38, 1.6}, {0, 0, 64, 0.45, 1.8}, {0, 0, 128, 0.65, 2.0},
      {0, 0, 256, 1.05, 3.0}};
  static const int kSplit[4] = {1, 2, 4, 8};
  const int k_blocks = (d.K + kGemm8BlockK - 1) / kGemm8BlockK;
  const int mx = d.a_scale_type == MAXDNN_E8M0 && d.b_scale_type == MAXDNN_E8M0;
  const int c_bytes = d.c_type == MAXDNN_F32 ? 4 : 2;
  // no shape is faster than reading the operands and writing the result
  const double memory = 5.0 + ((double)d.M * d.K + (double)d.N * d.K + (double)d.M * d.N * c_bytes) / 5.8e6;
  double best = 0;
  bool found = false;
  for (int swap = 0; swap < 2; ++swap) {
    if (option_is_set(OPT_GEMM8_SWAP) && option(OPT_GEMM8_SWAP) != swap) continue;
    const int64_t M = swap ? d.N : d.M, N = swap ? d.M : d.N;
    const int b_major = swap ? d.a_major : d.b_major;
    for (const Shape& s : kShapes) {
      if (s.mx != mx) continue;
      if (option_is_set(OPT_GEMM8_COLS) && option(OPT_GEMM8_COLS) != s.nt) continue;
      if (option_is_set(OPT_GEMM8_PAIR) && (option(OPT_GEMM8_PAIR) > 0) != (s.pair != 0)) continue;
      const int tile_m = s.pair ? 2 * kGemm8TileM : kGemm8TileM, rows_b = s.pair ? s.nt / 2 : s.nt;
      const int64_t m_tiles = (M + tile_m - 1) / tile_m, n_tiles = (N + s.nt - 1) / s.nt;
      const int64_t tiles = m_tiles * n_tiles;
      const int b_stage = b_major == MAXDNN_MAJOR_MN ? std::max(rows_b, 128) * 128 : rows_b * 128;
      const int slots = s.pair ? sm_count / 2 : mx && s.nt <= 32 ? 2 * sm_count : sm_count;   // tiles that run side by side
      // results are added up from accumulators of so many blocks (gemm8_mx.cuh)
      const int chunk = mx ? (d.c_type == MAXDNN_F32 ? 16 : 128) : 1;
      for (int split : kSplit) {
        if (option_is_set(OPT_GEMM8_SPLIT) && option(OPT_GEMM8_SPLIT) != split) continue;
        if (split > k_blocks || (split > 1 && s.pair)) continue;
        if (split > 1 && tiles * split > 2 * sm_count && !option_is_set(OPT_GEMM8_SPLIT)) continue;
        const int64_t units = split == 1 ? std::min<int64_t>(tiles, slots) : tiles;
        const int64_t waves = (tiles * split + slots - 1) / slots;
        const int64_t blocks = (k_blocks + split - 1) / split;
        // 3.4 us is a call with one block; sharing a tile costs an exchange of totals, and so does
        // storing C without bulk copies; two CTAs on an SM share its issue slots
        const bool bulk = mx && !swap && split == 1 && s.nt >= 32 && (d.ldc * c_bytes) % 16 == 0 &&
                          ((int64_t)d.N * c_bytes) % 16 == 0;
        const double crowd = s.nt <= 32 && mx ? std::max(1.0, 0.4 + 0.6 * (double)std::min<int64_t>(tiles * split, slots) / sm_count) : 1.0;
        const double run = 3.4 + (double)(waves * blocks) * s.block * crowd + s.tile * (1.0 + (double)(waves - 1) / 3.0) +
                           (split > 1 ? 1.0 + 0.008 * s.nt : bulk ? 0.0 : 0.8);
        // every tile reads its operands from the second-level cache
        const double fill = 5.0 + (double)tiles * k_blocks * (16384 + b_stage) * (s.pair ? 2 : 1) / 11.0e6;
        const double t = std::max(std::max(run, fill), memory) + 0.05 * run;
        if (found && t >= best) continue;
        found = true;
        best = t;
        plan->mx = mx;
        plan->pair = s.pair;
        plan->swap = swap;
        plan->tile_n = s.nt;
        plan->chunk = chunk;
        plan->split = split;
        plan->m_tiles = (int32_t)m_tiles;
        plan->n_tiles = (int32_t)n_tiles;
        plan->k_blocks = k_blocks;
        plan->b_stage_bytes = b_stage;
        plan->grid = (int32_t)(units * (s.pair ? 2 : split));
        // bulk copies of 32 rows x 32 columns: rows of C contiguous, starting and ending at
        // multiples of 16 bytes (a copy that is cut at the tensor's edge writes whole 16 bytes)
        plan->bulk_c = bulk;
        plan->staged_c = mx && !swap && split == 1;
      }
    }
  }
  if (!found) return MAXDNN_NOT_SUPPORTED;
  if ((int64_t)plan->m_tiles * plan->n_tiles > (1 << 30)) return MAXDNN_NOT_SUPPORTED;
  int fixed = 1024 + 192;
  if (plan->mx) {
    fixed += (plan->staged_c ? 8 * 32 * 32 * (plan->bulk_c ? c_bytes : 4) : 0) + 8 * 128 * (4 + 4 * ((plan->tile_n + 127) / 128));
  } else {
    const int warps = 4 * (plan->tile_n < 64 ? 1 : plan->tile_n / 64), cw = std::min(plan->tile_n, 64);
    fixed += warps * 2 * cw * 4;
  }
  const int per_stage = 16384 + plan->b_stage_bytes + 16;
  // a CTA of one tile needs no more stages than it has blocks; two CTAs of an SM share its memory
  const int blocks = (k_blocks + plan->split - 1) / plan->split;
  const int ctas_per_tile = plan->pair ? 2 : plan->split;
  const bool one_tile = (int64_t)plan->m_tiles * plan->n_tiles * ctas_per_tile <= plan->grid;
  plan->stages = std::min(12, (232448 - fixed) / per_stage);
  if (plan->mx && plan->tile_n <= 32 && plan->grid > sm_count) plan->stages = std::min(plan->stages, (115200 - fixed) / per_stage);
  if (one_tile) plan->stages = std::max(2, std::min(plan->stages, blocks));
  if (plan->split > 1) {        // the totals take the place of the ring
    const int need = (plan->tile_n + 4) * kGemm8TileM * 4, ring = per_stage - 16;
    plan->stages = std::max(plan->stages, (need + ring - 1) / ring);
  }
  plan->smem_bytes = fixed + plan->stages * per_stage;
  if (plan->pair || plan->split > 1)
    plan->smem_bytes = std::max(plan->smem_bytes,
                                cluster_smem_floor(plan->mx ? mx_tmem_cols(plan->tile_n) : gemm8_tmem_cols(plan->tile_n)));
  return MAXDNN_OK;
}

}  // namespace maxdnn
