// Host-side planning of the orthogonalised update: argument checks, the workspace's layout and the choice of a tile
// shape.  Plain C++, no CUDA calls.
#pragma once
#include <stdint.h>

#include "../../include/maxdnn.h"
#include "plan.h"

namespace maxdnn {

constexpr int kOrthoTileM = 128;       // rows of a CTA's tile (TMEM lanes)
constexpr int kOrthoBlockK = 64;       // reduction steps per stage: 128 bytes of FP16
constexpr int kOrthoMaxSteps = 32;
constexpr int kOrthoMaxSize = 65536;
constexpr int kOrthoScaleBits = 10;    // X is held as 2^10 X: its entries (at most 1) then are normal FP16 numbers down to 6e-8
constexpr int kOrthoMaxParts = 128;    // CTAs that share a matrix's sum of squares
constexpr int kOrthoStaging = 8 * 2 * 4096;   // eight warps, two slots of two 32 x 32 tiles of FP16

enum OrthoKind : int { kOrthoGram = 0, kOrthoPoly = 1, kOrthoUpdate = 2, kOrthoLast = 3 };
// How an operand lies: its rows are the product's rows or columns; its rows are the reduction; symmetric, stored up to the
// end of its diagonal blocks.
enum OrthoMode : int { kOrthoKAlongRows = 0, kOrthoRowsAreK = 1, kOrthoSymmetric = 2 };

// One product C[M][N] over K.
struct OrthoProduct {
  int32_t M, N;
  int32_t symmetric;       // only tiles that reach the diagonal or below are computed
  int32_t a_mode, b_mode;
  int32_t m_tiles, n_tiles, tiles, k_steps;    // tiles: of one matrix
  int32_t full, items;     // of all matrices: whole tiles, then halves
};

struct OrthoPlan {
  int32_t tall;                    // rows > cols: products from the right
  int32_t pair, nt;                // tile: 128 (256 where pair) rows x nt columns
  int32_t stages, smem_bytes, grid;
  int32_t n, m;                    // shorter and longer side
  int32_t parts;                   // CTAs that share a sum of squares
  int64_t pitch_x, pitch_n;        // elements
  int64_t diag;                    // floats of a matrix's diagonal
  // byte offsets into the workspace
  int64_t x[2][2], a, b, diag_a, diag_b, post, done, sums, bytes;     // x: [which][hi, lo]
  OrthoProduct product[3];         // Gram, Poly, Update
};

maxdnn_status check_ortho(const maxdnn_ortho_desc* d);
// slots[0], slots[1]: CTAs, and pairs of CTAs, that the device runs at the same time.
maxdnn_status plan_ortho(const maxdnn_ortho_desc& d, const int (&slots)[2], OrthoPlan* plan);

}  // namespace maxdnn
