// Planning of the orthogonalised update (see ortho.h).
#include "ortho.h"

#include <algorithm>

#include "gemm8.h"

namespace maxdnn {

namespace {

// Tile shapes with what a stage of 64 reduction steps takes in a long run and what a tile takes besides, in microseconds.
struct Shape { int pair, nt; double step, tile; };
constexpr Shape kShapes[] = {{1, 256, 0.29, 3.0}, {1, 128, 0.18, 2.2}, {0, 128, 0.17, 2.0}, {0, 64, 0.13, 1.6}};

int64_t tiles_of(int64_t M, int64_t N, int tile_m, int nt, bool symmetric) {
  const int64_t mt = (M + tile_m - 1) / tile_m, n_tiles = (N + nt - 1) / nt;
  if (!symmetric) return mt * n_tiles;
  int64_t all = 0;
  for (int64_t i = 0; i < mt; ++i) all += std::min<int64_t>(n_tiles, (i + 1) * tile_m / nt);
  return all;
}

void plan_product(OrthoProduct* p, int64_t M, int64_t N, int64_t K, bool symmetric, int batch, int sm_count) {
  double best = 0;
  for (const Shape& s : kShapes) {
    const int tile_m = s.pair ? 2 * kOrthoTileM : kOrthoTileM;
    const int64_t tiles = tiles_of(M, N, tile_m, s.nt, symmetric), slots = s.pair ? sm_count / 2 : sm_count;
    const int64_t k_steps = (K + kOrthoBlockK - 1) / kOrthoBlockK, waves = (tiles * batch + slots - 1) / slots;
    // a tile's result is stored while the next one's sums run
    const double t = waves * std::max(k_steps * s.step, s.tile) + s.tile;
    if (best > 0 && t >= best) continue;
    best = t;
    p->M = (int32_t)M;
    p->N = (int32_t)N;
    p->K = (int32_t)K;
    p->symmetric = symmetric;
    p->pair = s.pair;
    p->nt = s.nt;
    p->m_tiles = (int32_t)((M + tile_m - 1) / tile_m);
    p->n_tiles = (int32_t)((N + s.nt - 1) / s.nt);
    p->tiles = (int32_t)tiles;
    p->k_steps = (int32_t)k_steps;
    p->b_rows = s.pair ? s.nt / 2 : s.nt;
    p->b_stage_bytes = p->b_rows * 2 * kOrthoBlockK;
    p->grid = (int32_t)(std::min<int64_t>(tiles * batch, slots) * (s.pair ? 2 : 1));
  }
  const int fixed = 1024 + 512 + kOrthoStaging, per_stage = 2 * kOrthoTileM * kOrthoBlockK + p->b_stage_bytes + 16;
  p->stages = std::min(8, (232448 - fixed) / per_stage);
  p->smem_bytes = fixed + p->stages * per_stage;
  if (p->pair) p->smem_bytes = std::max(p->smem_bytes, cluster_smem_floor(2 * p->nt));
}

}  // namespace

maxdnn_status check_ortho(const maxdnn_ortho_desc* d) {
  if (!d || d->batch < 0 || d->rows <= 0 || d->cols <= 0 || d->steps <= 0) return MAXDNN_INVALID_VALUE;
  if (d->x_type != MAXDNN_F32 && d->x_type != MAXDNN_BF16 && d->x_type != MAXDNN_F16) return MAXDNN_INVALID_VALUE;
  if (d->ldx < d->cols || d->ldo < d->cols) return MAXDNN_INVALID_VALUE;
  if (!(d->eps >= 0.f) || d->eps > 3.0e38f) return MAXDNN_INVALID_VALUE;
  if (d->batch > 1 && (d->stride_x < 0 || d->stride_o < (d->rows - 1) * d->ldo + d->cols)) return MAXDNN_INVALID_VALUE;
  if (d->rows > kOrthoMaxSize || d->cols > kOrthoMaxSize || d->steps > kOrthoMaxSteps || d->batch > kOrthoMaxSize) return MAXDNN_NOT_SUPPORTED;
  return MAXDNN_OK;
}

maxdnn_status plan_ortho(const maxdnn_ortho_desc& d, int sm_count, OrthoPlan* p) {
  *p = OrthoPlan();
  p->tall = d.rows > d.cols;
  p->n = std::min(d.rows, d.cols);
  p->m = std::max(d.rows, d.cols);
  const int64_t batch = d.batch;
  auto up = [](int64_t v, int64_t to) { return (v + to - 1) / to * to; };
  p->pitch_x = up(d.cols, 64);
  p->pitch_n = up(p->n, 64);
  p->diag = up(p->n, 32);
  // a CTA takes at least 64 rows of 8 warps' vectors
  const int64_t work = (int64_t)d.rows * up(d.cols, 256) / (64 * 256);
  p->parts = (int32_t)std::max<int64_t>(1, std::min<int64_t>(kOrthoMaxParts, std::min<int64_t>(work, (d.rows + 7) / 8)));
  int64_t at = 0;
  auto take = [&](int64_t bytes) { const int64_t here = at; at += up(bytes, 1024); return here; };
  for (int w = 0; w < 2; ++w)
    for (int part = 0; part < 2; ++part) p->x[w][part] = take(batch * d.rows * p->pitch_x * 2);
  p->a = take(batch * p->n * p->pitch_n * 2);
  p->b = take(batch * p->n * p->pitch_n * 2);
  p->diag_a = take(batch * p->diag * 4);
  p->diag_b = take(batch * p->diag * 4);
  p->post = take(batch * 4);
  p->sums = take(batch * p->parts * 8);
  p->bytes = std::max<int64_t>(at, 16);
  plan_product(&p->gram, p->n, p->n, p->m, true, d.batch, sm_count);
  plan_product(&p->poly, p->n, p->n, p->n, true, d.batch, sm_count);
  plan_product(&p->update, d.rows, d.cols, p->n, false, d.batch, sm_count);
  if ((int64_t)p->update.tiles * batch > (1 << 30) || (int64_t)p->gram.tiles * batch > (1 << 30)) return MAXDNN_NOT_SUPPORTED;
  return MAXDNN_OK;
}

}  // namespace maxdnn
