// Planning of the orthogonalised update (see ortho.h).
#include "ortho.h"

#include <algorithm>

#include "gemm8.h"

namespace maxdnn {

namespace {

// Tile shapes with what the MMAs of a stage of 64 reduction steps take, what a tile's end takes and what a product takes
// besides its tiles (a first copy, the exchange between CTAs), in microseconds.
struct Shape { int pair, nt; double step, end, fixed; };
constexpr Shape kShapes[] = {{1, 256, 0.30, 3.5, 3.0}, {1, 128, 0.16, 2.0, 3.0}, {0, 128, 0.15, 2.0, 3.0}, {0, 64, 0.09, 1.2, 3.0}};
// What all SMs together read from the second-level cache (bytes in a microsecond; 4096 x 4096: 46 bytes a cycle and SM), and
// how long a copy takes from its start to its end: a ring of stages cannot be faster than that for all of its stages.
constexpr double kCacheRate = 11.0e6, kCopyTime = 1.0;
int b_stage_bytes(const Shape& s) { return (s.pair ? s.nt / 2 : s.nt) * kOrthoBlockK * 2; }
int ring_stages(int b_stage) {
  const int fixed = 1024 + 512 + 2048 + kOrthoStaging, per_stage = 2 * kOrthoTileM * kOrthoBlockK + b_stage + 16;
  return std::min(8, (232448 - fixed) / per_stage);
}

int64_t tiles_of(int64_t M, int64_t N, int tile_m, int nt, bool symmetric) {
  const int64_t mt = (M + tile_m - 1) / tile_m, n_tiles = (N + nt - 1) / nt;
  if (!symmetric) return mt * n_tiles;
  int64_t all = 0;
  for (int64_t i = 0; i < mt; ++i) all += std::min<int64_t>(n_tiles, (i + 1) * tile_m / nt);
  return all;
}

// The tiles of one product in a given shape; returns the time that it should take.
double plan_product(OrthoProduct* p, int64_t M, int64_t N, int64_t K, bool symmetric, int batch, const Shape& s, int slots) {
  const int tile_m = s.pair ? 2 * kOrthoTileM : kOrthoTileM;
  const int64_t tiles = tiles_of(M, N, tile_m, s.nt, symmetric), all = tiles * batch;
  p->M = (int32_t)M;
  p->N = (int32_t)N;
  p->symmetric = symmetric;
  p->m_tiles = (int32_t)((M + tile_m - 1) / tile_m);
  p->n_tiles = (int32_t)((N + s.nt - 1) / s.nt);
  p->tiles = (int32_t)tiles;
  p->k_steps = (int32_t)((K + kOrthoBlockK - 1) / kOrthoBlockK);
  // halves have to be boxes of 64 columns for each CTA
  const int64_t rest = all % slots;
  const bool halves = rest > 0 && 2 * rest <= slots && s.nt / 2 / (s.pair ? 2 : 1) >= 64;
  p->full = (int32_t)(halves ? all - rest : all);
  p->items = (int32_t)(p->full + (halves ? 2 * rest : 0));
  const int64_t active = std::min<int64_t>(p->items, slots) * (s.pair ? 2 : 1);
  const double fill = (double)active * (2 * kOrthoTileM * kOrthoBlockK + b_stage_bytes(s)) / kCacheRate;
  const double step = std::max(std::max(s.step, fill), kCopyTime / ring_stages(b_stage_bytes(s)));
  const double tile = std::max(p->k_steps * step, s.end), whole = (double)((all - rest) / slots);
  return s.fixed + whole * tile + (rest == 0 ? 0.0 : halves ? 0.6 * tile : tile) + s.end;
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

maxdnn_status plan_ortho(const maxdnn_ortho_desc& d, const int (&slots)[2], OrthoPlan* p) {
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
  p->diag_b = take(batch * p->diag * 8);
  p->post = take(batch * 4);
  p->done = take(4);
  p->sums = take(batch * p->parts * 8);
  p->bytes = at;
  // one shape for all products of the launch: the one that a step should take least in
  double best = 0;
  for (const Shape& s : kShapes) {
    OrthoProduct q[3] = {};
    const int n_slots = slots[s.pair];
    if (n_slots <= 0) continue;
    const int tile_m = s.pair ? 2 * kOrthoTileM : kOrthoTileM;
    // (numbers of tiles are 32 bits)
    if (tiles_of(d.rows, d.cols, tile_m, s.nt, false) * batch > (1 << 28) || tiles_of(p->n, p->n, tile_m, s.nt, true) * batch > (1 << 28)) continue;
    const double t = plan_product(&q[kOrthoGram], p->n, p->n, p->m, true, d.batch, s, n_slots) +
                     plan_product(&q[kOrthoPoly], p->n, p->n, p->n, true, d.batch, s, n_slots) +
                     plan_product(&q[kOrthoUpdate], d.rows, d.cols, p->n, false, d.batch, s, n_slots);
    if (best > 0 && t >= best) continue;
    best = t;
    p->pair = s.pair;
    p->nt = s.nt;
    int32_t most = 0;
    for (int i = 0; i < 3; ++i) {
      p->product[i] = q[i];
      most = std::max(most, q[i].items);
    }
    p->grid = std::min<int32_t>(most, n_slots) * (s.pair ? 2 : 1);
  }
  if (best == 0) return MAXDNN_NOT_SUPPORTED;
  p->product[kOrthoGram].a_mode = p->product[kOrthoGram].b_mode = p->tall ? kOrthoRowsAreK : kOrthoKAlongRows;
  p->product[kOrthoPoly].a_mode = p->product[kOrthoPoly].b_mode = kOrthoSymmetric;
  p->product[kOrthoUpdate].a_mode = p->tall ? kOrthoKAlongRows : kOrthoSymmetric;
  p->product[kOrthoUpdate].b_mode = p->tall ? kOrthoSymmetric : kOrthoRowsAreK;
  const int b_stage = (p->pair ? p->nt / 2 : p->nt) * kOrthoBlockK * 2;
  p->stages = ring_stages(b_stage);
  p->smem_bytes = 1024 + 512 + 2048 + kOrthoStaging + p->stages * (2 * kOrthoTileM * kOrthoBlockK + b_stage + 16);
  if (p->pair) p->smem_bytes = std::max(p->smem_bytes, cluster_smem_floor(2 * p->nt));
  return MAXDNN_OK;
}

}  // namespace maxdnn
