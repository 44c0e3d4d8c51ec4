// Newton-Schulz products of the orthogonalised update: C[m, n] = sum_k a[m, k] b[n, k] on FP16 operands with 32-bit
// sums (tcgen05 MMA, TMEM accumulators, bulk tensor copies), for a batch of matrices, with what a step does to the product:
//
//   Gram    A = X X^T                      stored in FP16; symmetric
//   Poly    B = b A + c A A                stored in FP16; symmetric
//   Update  X' = a X + B X                 (or a X + X B); stored as two FP16 numbers, hi + lo
//   Last    out = a X + B X                stored in BF16
//
// Precision.  An entry of X that is rounded to FP16 is off by 2^-12 of it, spread over all directions, and a step multiplies
// what lies in the directions of small singular values by a = 3.4: from a low-rank gradient five steps make 2 % of
// the result out of that rounding (17 % with BF16).  So X is kept as hi + lo (22 bits; lo is held 2^11 times as large, or it
// would end where hi does), which the a X term reads; the products read hi, whose rounding they only let act along the
// directions that they keep.  What is left comes from the diagonals
// of A and B, whose entries near 1 are the largest: their rounding residues are kept in 32 bits and added where the matrices are
// used, (A A)_mn += (r_m + r_n) A_mn and (B X)_mn += r_m X_mn.  Against 64 bits over several spectra: 3e-4 to 1.3e-3 of
// the result's norm; its rounding to BF16 is 1.7e-3.
//
// Symmetric products compute the tiles that reach the diagonal or below it, and store each 32 x 32 part twice, as it is and
// transposed; half of the operations.  X is read along either axis by the MMA's descriptors ("MN-major" where the reduction is
// the row number), so nothing is transposed in memory.
//
// Roles.  Warp 0 copies A, warp 3 copies B, warp 1 issues the MMAs; warps 4-11 finish the tiles.  Two accumulators alternate, so
// a tile is finished while the next one's MMAs run.  A finishing warp has 32 rows x up to 128 columns, 32 x 32 at a
// time: bulk copies bring the parts of X (A) it needs into its two slots in shared memory, one part ahead, and store the result
// from the same slot.
// PAIR.  Two CTAs share a tile of 256 rows (cta_group::2): each stages its 128 rows of A and half of the columns of B.
// Every wait on a barrier in shared memory is bounded and ends in a status code; TMEM is always freed.  (Waits for tensor
// memory and at a cluster's end: see gemm8.cuh.)
#pragma once
#include "fp8_util.cuh"
#include "ortho.h"
#include "umma_util.cuh"

namespace maxdnn {

constexpr int kOrthoThreads = 384;
constexpr int kOrthoEpiWarps = 8;
constexpr float kOrthoLo = 2048.f;      // X = (hi + lo / kOrthoLo) 2^-10

struct OrthoArgs {
  int32_t M, N, batch;
  int32_t m_tiles, n_tiles, tiles, k_steps, stages;
  int32_t a_mn, b_mn;            // operand is MN-major
  int32_t b_rows, b_stage_bytes;
  uint32_t idesc;
  float scale;                   // of the sums (Gram), of the result (Last)
  float ca, cb, cc;              // a, b, c
  const float* diag_in;          // residues of A (Poly) or B (Update, Last)
  float* diag_out;               // of A (Gram) or B (Poly)
  const float* post;             // Last: a power of two for each matrix
  int64_t diag;                  // floats of a matrix's diagonal
  int32_t diag_cols;             // Update: the residue of column n belongs to X_mn (products from the right), not of row m
  int32_t bulk_out;              // Last: out's rows allow bulk stores
  __nv_bfloat16* out;
  int64_t ldo, stride_o;
  uint32_t test_missing_arrival;
  WaitCtx wc;
};

// Coordinates (column, row, matrix).
__device__ __forceinline__ void tma_load_3d_hint(uint32_t dst, const CUtensorMap* m, uint32_t bar, int c0, int c1, int c2,
                                                 uint64_t policy) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.L2::cache_hint "
      "[%0], [%1, {%3, %4, %5}], [%2], %6;" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(m)), "r"(bar), "r"(c0), "r"(c1), "r"(c2), "l"(policy)
      : "memory");
}
__device__ __forceinline__ void tma_load_3d_pair(uint32_t dst, const CUtensorMap* m, uint32_t bar, int c0, int c1, int c2,
                                                 uint64_t policy) {
  asm volatile(
      "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
      ".L2::cache_hint [%0], [%1, {%3, %4, %5}], [%2], %6;" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(m)), "r"(bar), "r"(c0), "r"(c1), "r"(c2), "l"(policy)
      : "memory");
}
__device__ __forceinline__ void tma_store_3d(const CUtensorMap* m, uint32_t src, int c0, int c1, int c2) {
  asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%2, %3, %4}], [%1];" ::"l"(
                   reinterpret_cast<uint64_t>(m)),
               "r"(src), "r"(c0), "r"(c1), "r"(c2)
               : "memory");
}

// Tile number t of a matrix: its first row and column.  Symmetric: row by row of tiles, `ratio` (tile rows / columns) more
// in each, up to all n_tiles.  Else groups of eight rows of tiles, column by column, so that tiles at work together share operands.
__device__ __forceinline__ void ortho_tile(const OrthoArgs& args, bool symmetric, int ratio, int t, int* mt, int* nt) {
  if (!symmetric) {
    const int per_group = 8 * args.n_tiles, group = t / per_group, first = group * 8;
    const int height = min(8, args.m_tiles - first), in = t - group * per_group;
    *mt = first + in % height;
    *nt = in / height;
    return;
  }
  // tiles of the rows before row i: ratio i (i + 1) / 2 (only the last row may have fewer than its share)
  int i = (int)((sqrtf(1.f + 8.f * (float)t / (float)ratio) - 1.f) * 0.5f);
  while (ratio * i * (i + 1) / 2 > t) --i;
  while (ratio * (i + 1) * (i + 2) / 2 <= t) ++i;
  *mt = i;
  *nt = t - ratio * i * (i + 1) / 2;
}

template <int NT, bool PAIR, int KIND>
__global__ void __launch_bounds__(kOrthoThreads, 1)
ortho_product_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                     const __grid_constant__ CUtensorMap map_in, const __grid_constant__ CUtensorMap map_in_lo,
                     const __grid_constant__ CUtensorMap map_out, const __grid_constant__ CUtensorMap map_out_lo,
                     const __grid_constant__ OrthoArgs args) {
  constexpr bool kSym = KIND == kOrthoGram || KIND == kOrthoPoly;
  constexpr int kLoads = KIND == kOrthoGram ? 0 : KIND == kOrthoPoly ? 1 : 2;      // tiles of 32 x 32 that a part needs
  constexpr int kUnits = NT / 64;                   // parts of 32 columns of a finishing warp
  constexpr int kTileM = PAIR ? 2 * kOrthoTileM : kOrthoTileM;
  constexpr int kRatio = kTileM / NT > 0 ? kTileM / NT : 1;
  constexpr uint32_t kAStage = kOrthoTileM * kOrthoBlockK * 2;
  constexpr uint32_t kTmemWanted = 2 * NT;
  static_assert(kTileM % NT == 0, "a symmetric product's rows of tiles grow by whole tiles");
  extern __shared__ uint8_t smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* base_ptr = smem_raw + (base - smem_u32(smem_raw));
  const int stages = args.stages;
  const uint32_t b_off = (uint32_t)stages * kAStage;
  const uint32_t st_off = b_off + (uint32_t)stages * (uint32_t)args.b_stage_bytes;
  const uint32_t full_bar = base + st_off + kOrthoStaging;
  const uint32_t empty_bar = full_bar + 8u * stages;
  const uint32_t accf_bar = empty_bar + 8u * stages;       // 2
  const uint32_t acce_bar = accf_bar + 16u;                // 2
  const uint32_t load_bar = acce_bar + 16u;                // 2 for each finishing warp
  const uint32_t done_bar = load_bar + 16u * kOrthoEpiWarps;
  const uint32_t tmem_slot = done_bar + 8u;
  volatile uint32_t* tmem_slot_ptr = reinterpret_cast<volatile uint32_t*>(base_ptr + (tmem_slot - base));

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = PAIR ? (int)cluster_ctarank() : 0;
  const int unit = (int)blockIdx.x / (PAIR ? 2 : 1), n_units = (int)gridDim.x / (PAIR ? 2 : 1);
  const int n_tiles = args.tiles * args.batch;
  const bool leader = !PAIR || rank == 0;

  if (threadIdx.x == 0) {
    const uint32_t extra = (args.test_missing_arrival != 0 && blockIdx.x == 0) ? 1u : 0u;   // test hook
    for (int s = 0; s < stages; ++s) {
      mbar_init(full_bar + 8u * s, 2 + extra);          // the (leader's) two copy warps
      mbar_init(empty_bar + 8u * s, 1);
    }
    for (int a = 0; a < 2; ++a) {
      mbar_init(accf_bar + 8u * a, 1);
      mbar_init(acce_bar + 8u * a, kOrthoEpiWarps * (PAIR ? 2 : 1));
    }
    for (int w = 0; w < 2 * kOrthoEpiWarps; ++w) mbar_init(load_bar + 8u * w, 1);
    mbar_init(done_bar, 1);
    fence_mbar_init();
    fence_proxy_async_smem();
  }
  if (warp == 1) {
    if constexpr (PAIR) {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(tmem_slot), "r"(kTmemWanted) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
      asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(tmem_slot), "r"(kTmemWanted) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
  }
  tcgen05_fence_before();
  __syncthreads();
  if constexpr (PAIR) {
    cluster_arrive();      // both CTAs' barriers exist before anything arrives on them from the peer
    cluster_wait();
  }
  tcgen05_fence_after();
  const uint32_t tmem_base = *tmem_slot_ptr;
  // only now: the next kernel's CTA takes its tensor memory after this one has its own
  let_next_start();
  wait_for_previous();

  if (warp == 0 || warp == 3) {
    // ------------------------------------------------------------ copies
    const bool is_a = warp == 0;
    const CUtensorMap* map = is_a ? &map_a : &map_b;
    if (lane == 0) prefetch_tensormap(map);
    const uint64_t policy = l2_policy_evict_last();
    const uint32_t bytes = is_a ? kAStage : (uint32_t)args.b_stage_bytes;
    const uint32_t tx = (PAIR ? 2u : 1u) * bytes;
    const uint32_t report = PAIR ? map_to_cta(full_bar, 0) : full_bar;
    const bool mn = is_a ? args.a_mn != 0 : args.b_mn != 0;
    // MN-major tiles come in columns of 64 (128 bytes)
    const int boxes = mn ? (is_a ? kOrthoTileM : args.b_rows) / 64 : 1;
    int stage = 0;
    uint32_t phase = 0;
    bool ok = true;
    for (int tile = unit; tile < n_tiles && ok; tile += n_units) {
      const int matrix = tile / args.tiles;
      int mt, nt;
      ortho_tile(args, kSym, kRatio, tile - matrix * args.tiles, &mt, &nt);
      const int i0 = is_a ? mt * kTileM + rank * kOrthoTileM : nt * NT + rank * (NT / 2);
      for (int ks = 0; ks < args.k_steps; ++ks) {
        if (!mbar_wait(empty_bar + 8u * stage, phase ^ 1u, args.wc, kDevTimeoutEmpty)) {
          ok = false;
          break;
        }
        const uint32_t dst = base + (is_a ? (uint32_t)stage * kAStage : b_off + (uint32_t)stage * (uint32_t)args.b_stage_bytes);
        if (elect_one()) {
          if (leader) mbar_arrive_expect_tx(full_bar + 8u * stage, tx);
          const int k = ks * kOrthoBlockK;
          for (int b = 0; b < boxes; ++b) {
            const int c0 = mn ? i0 + 64 * b : k, c1 = mn ? k : i0;
            if constexpr (PAIR) tma_load_3d_pair(dst + 8192u * b, map, report + 8u * stage, c0, c1, matrix, policy);
            else tma_load_3d_hint(dst + 8192u * b, map, report + 8u * stage, c0, c1, matrix, policy);
          }
        }
        __syncwarp();
        if (++stage == stages) { stage = 0; phase ^= 1u; }
      }
    }
    if (!ok) {
      // leaving early: give copies already issued time to land (a pair's report to the leader)
      if constexpr (PAIR) {
        const uint64_t t0 = globaltimer_ns();
        while (globaltimer_ns() - t0 < 200000ull) {}
      } else {
        for (int s = 0; s < stages; ++s) mbar_wait_grace(full_bar + 8u * s, s < stage ? phase : (phase ^ 1u));
      }
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------ MMAs (the leader's, for both CTAs)
    if (leader) {
      // rows of 128 bytes with the 128-byte swizzle; groups of eight 1024 bytes apart, MN-major columns of 64 8192
      const uint64_t desc = make_smem_desc(0, 8192u, 1024u, 2u);
      const uint64_t step_a = (args.a_mn ? 2048u : 32u) >> 4, step_b = (args.b_mn ? 2048u : 32u) >> 4;
      const uint64_t desc_a = desc | (uint64_t)((base & 0x3FFFFu) >> 4);
      const uint64_t desc_b = desc | (uint64_t)(((base + b_off) & 0x3FFFFu) >> 4);
      const uint32_t b_stage = (uint32_t)args.b_stage_bytes >> 4;
      int stage = 0;
      uint32_t phase = 0, acc_n = 0;
      bool ok = true, ready = false;
      for (int tile = unit; tile < n_tiles && ok; tile += n_units, ++acc_n) {
        const uint32_t acc = acc_n & 1u, d = tmem_base + acc * NT;
        if (!mbar_wait(acce_bar + 8u * acc, ((acc_n >> 1) & 1u) ^ 1u, args.wc, kDevTimeoutAccFree)) {
          ok = false;
          break;
        }
        tcgen05_fence_after();
        for (int ks = 0; ks < args.k_steps; ++ks) {
          if (!ready && !mbar_wait(full_bar + 8u * stage, phase, args.wc, kDevTimeoutFull)) {
            ok = false;
            break;
          }
          const int next = stage + 1 == stages ? 0 : stage + 1;
          const uint32_t next_phase = stage + 1 == stages ? phase ^ 1u : phase;
          ready = mbar_test_wait(full_bar + 8u * next, next_phase);
          tcgen05_fence_after();
          if (elect_one()) {
            uint64_t a = desc_a + (uint64_t)((uint32_t)stage * (kAStage >> 4));
            uint64_t b = desc_b + (uint64_t)((uint32_t)stage * b_stage);
#pragma unroll
            for (int j = 0; j < kOrthoBlockK / 16; ++j) {
              if constexpr (PAIR) tcgen05_mma_pair<true>(d, a, b, args.idesc, ks > 0 || j > 0);
              else tcgen05_mma<true>(d, a, b, args.idesc, ks > 0 || j > 0);
              a += step_a;
              b += step_b;
            }
            if constexpr (PAIR) tcgen05_commit_pair(empty_bar + 8u * stage);
            else tcgen05_commit(empty_bar + 8u * stage);
          }
          stage = next;
          phase = next_phase;
        }
        if (ok && elect_one()) {
          if constexpr (PAIR) tcgen05_commit_pair(accf_bar + 8u * acc);
          else tcgen05_commit(accf_bar + 8u * acc);
        }
      }
      // every MMA issued so far has finished before TMEM is released
      if (elect_one()) {
        if constexpr (PAIR) tcgen05_commit_pair(done_bar, 1);
        else tcgen05_commit(done_bar);
      }
      mbar_wait(done_bar, 0, args.wc, kDevTimeoutDrain);
    }
  } else if (warp >= 4) {
    // ------------------------------------------------------------ what a step does to the product
    const int q = warp & 3;                   // TMEM lanes this warp may read
    const int ew = warp - 4;
    const int u0 = (ew >> 2) * kUnits;        // its first part of 32 columns
    const uint32_t release = PAIR ? map_to_cta(acce_bar, 0) : acce_bar;
    const uint32_t slots = base + st_off + (uint32_t)ew * 8192u, loaded = load_bar + 16u * ew;
    uint8_t* slots_ptr = base_ptr + st_off + (size_t)ew * 8192;
    const uint32_t swz = (uint32_t)((lane >> 1) & 3);
    uint32_t acc_n = 0, n_loads = 0, n_parts = 0;      // loads issued, parts finished; slot: the last bit
    bool ok = true;
    for (int tile = unit; tile < n_tiles && ok; tile += n_units, ++acc_n) {
      const int matrix = tile / args.tiles;
      int mt, nt;
      ortho_tile(args, kSym, kRatio, tile - matrix * args.tiles, &mt, &nt);
      const int m_warp = mt * kTileM + rank * kOrthoTileM + q * 32, m = m_warp + lane;
      const int n_first = nt * NT + u0 * 32;
      auto wanted = [&](int u) {
        const int n0 = n_first + 32 * u;
        return u < kUnits && m_warp < args.M && n0 < args.N && (!kSym || n0 <= m_warp);
      };
      // brings what part u needs into the next slot, once that slot's store has been read
      auto load = [&](int u) {
        if (kLoads == 0 || !wanted(u)) return;
        if (lane == 0) {
          bulk_wait_read<0>();
          const uint32_t bar = loaded + 8u * (n_loads & 1u), dst = slots + 4096u * (n_loads & 1u);
          mbar_arrive_expect_tx(bar, 2048u * kLoads);
          const uint64_t policy = l2_policy_evict_first();
          tma_load_3d_hint(dst, &map_in, bar, n_first + 32 * u, m_warp, matrix, policy);
          if (kLoads == 2) tma_load_3d_hint(dst + 2048u, &map_in_lo, bar, n_first + 32 * u, m_warp, matrix, policy);
        }
        ++n_loads;
        __syncwarp();
      };
      load(0);
      const float* r_in = KIND == kOrthoGram ? nullptr : args.diag_in + matrix * args.diag;
      const float out_scale = KIND == kOrthoLast ? args.scale * load_global(args.post + matrix) : 0.f;
      const float r_m = KIND != kOrthoGram && m < args.M && (kSym || !args.diag_cols) ? load_global(r_in + m) : 0.f;
      const uint32_t acc = acc_n & 1u;
      if (!mbar_wait(accf_bar + 8u * acc, (acc_n >> 1) & 1u, args.wc, kDevTimeoutAccum)) {
        ok = false;
        break;
      }
      tcgen05_fence_after();
      const uint32_t t_row = tmem_base + ((uint32_t)(q * 32) << 16) + acc * NT + (uint32_t)(u0 * 32);
#pragma unroll 1
      for (int u = 0; u < kUnits; ++u) {
        if (!wanted(u)) break;
        if (u + 1 < kUnits) load(u + 1);
        const int n0 = n_first + 32 * u;
        uint32_t v[32];
        tmem_ld_32x32(t_row + (uint32_t)(32 * u), v);
        tmem_wait_ld();
        const uint32_t slot = n_parts & 1u;
        uint8_t* part = slots_ptr + 4096 * slot;
        if (kLoads > 0) {
          if (!mbar_wait(loaded + 8u * slot, (n_parts >> 1) & 1u, args.wc, kDevTimeoutFull)) ok = false;
        } else {
          if (lane == 0) bulk_wait_read<1>();      // the store before last had this slot
          __syncwarp();
        }
        uint8_t* row = part + lane * 64;
        const bool diagonal = kSym && n0 == m_warp;      // the part's diagonal is the matrix's
#pragma unroll
        for (int i = 0; i < 4; ++i) {                    // eight columns
          uint4* hi_at = reinterpret_cast<uint4*>(row + ((i ^ swz) << 4));
          float x[8], y[8];
          if constexpr (kLoads > 0) {
            Raw8<MAXDNN_F16> raw;
            raw.a = *hi_at;
            to_float8<MAXDNN_F16>(raw, x);
          }
          if constexpr (KIND == kOrthoGram) {
#pragma unroll
            for (int k = 0; k < 8; ++k) y[k] = __uint_as_float(v[8 * i + k]) * args.scale;
          } else {
            float r_n[8];
            if (KIND == kOrthoPoly || args.diag_cols) {
              const float4* p = reinterpret_cast<const float4*>(r_in + n0 + 8 * i);
              const float4 a = load_global(p), b = load_global(p + 1);
              r_n[0] = a.x; r_n[1] = a.y; r_n[2] = a.z; r_n[3] = a.w;
              r_n[4] = b.x; r_n[5] = b.y; r_n[6] = b.z; r_n[7] = b.w;
            } else {
#pragma unroll
              for (int k = 0; k < 8; ++k) r_n[k] = 0.f;
            }
            if constexpr (KIND == kOrthoPoly) {
#pragma unroll
              for (int k = 0; k < 8; ++k) {
                const float r_here = diagonal && 8 * i + k == lane ? r_m : 0.f;
                const float square = fmaf(r_here, r_here, fmaf(r_m + r_n[k], x[k], __uint_as_float(v[8 * i + k])));
                y[k] = fmaf(args.cb, x[k] + r_here, args.cc * square);
              }
            } else {
              Raw8<MAXDNN_F16> raw;
              raw.a = *reinterpret_cast<const uint4*>(row + 2048 + ((i ^ swz) << 4));
              float lo[8];
              to_float8<MAXDNN_F16>(raw, lo);
#pragma unroll
              for (int k = 0; k < 8; ++k) {
                const float full = fmaf(lo[k], 1.f / kOrthoLo, x[k]);
                y[k] = fmaf(args.ca, full, fmaf(r_m + r_n[k], full, __uint_as_float(v[8 * i + k])));
              }
            }
          }
          if constexpr (KIND == kOrthoLast) {
            uint32_t w[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const __nv_bfloat162 t = __floats2bfloat162_rn(y[2 * k] * out_scale, y[2 * k + 1] * out_scale);
              w[k] = *reinterpret_cast<const uint32_t*>(&t);
            }
            *hi_at = make_uint4(w[0], w[1], w[2], w[3]);
          } else {
            uint32_t w[4], z[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const __half2 t = __floats2half2_rn(y[2 * k], y[2 * k + 1]);
              w[k] = *reinterpret_cast<const uint32_t*>(&t);
              if (!kSym || diagonal) {
                const float2 back = __half22float2(t);
                if constexpr (kSym) {
                  if (8 * i + 2 * k == lane && m < args.M) args.diag_out[matrix * args.diag + m] = y[2 * k] - back.x;
                  if (8 * i + 2 * k + 1 == lane && m < args.M) args.diag_out[matrix * args.diag + m] = y[2 * k + 1] - back.y;
                } else {
                  const __half2 rest = __floats2half2_rn((y[2 * k] - back.x) * kOrthoLo, (y[2 * k + 1] - back.y) * kOrthoLo);
                  z[k] = *reinterpret_cast<const uint32_t*>(&rest);
                }
              }
            }
            *hi_at = make_uint4(w[0], w[1], w[2], w[3]);
            if constexpr (!kSym) {
              *reinterpret_cast<uint4*>(row + 2048 + ((i ^ swz) << 4)) = make_uint4(z[0], z[1], z[2], z[3]);
            } else if (!diagonal) {
              // transposed: row n of the second tile, this thread's column
#pragma unroll
              for (int k = 0; k < 8; ++k) {
                const int n = 8 * i + k;
                *reinterpret_cast<uint16_t*>(part + 2048 + n * 64 + (((lane >> 3) ^ ((n >> 1) & 3)) << 4) + 2 * (lane & 7)) =
                    (uint16_t)(w[k >> 1] >> (16 * (k & 1)));
              }
            }
          }
        }
        const uint32_t src = slots + 4096u * slot;
        if (KIND == kOrthoLast && !args.bulk_out) {
          // rows that bulk copies cannot store: a row of 32 neighbours at a time
          __syncwarp();
          const int n = n0 + lane;
          for (int r = 0; r < 32 && m_warp + r < args.M; ++r) {
            const __nv_bfloat16 t = *reinterpret_cast<const __nv_bfloat16*>(
                part + r * 64 + (((lane >> 3) ^ ((r >> 1) & 3)) << 4) + 2 * (lane & 7));
            if (n < args.N) args.out[matrix * args.stride_o + (int64_t)(m_warp + r) * args.ldo + n] = t;
          }
          fence_proxy_async_smem();      // (the next copy into this slot follows these reads and writes)
          __syncwarp();
        } else {
          fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0) {
            tma_store_3d(&map_out, src, n0, m_warp, matrix);
            if (KIND == kOrthoUpdate) tma_store_3d(&map_out_lo, src + 2048u, n0, m_warp, matrix);
            if (kSym && !diagonal) tma_store_3d(&map_out, src + 2048u, m_warp, n0, matrix);
            bulk_commit();
          }
        }
        ++n_parts;
      }
      tcgen05_fence_before();
      __syncwarp();
      if (lane == 0) {
        if constexpr (PAIR) mbar_arrive_cluster(release + 8u * acc);
        else mbar_arrive(release + 8u * acc);
      }
    }
    if (!ok && kLoads > 0)
      for (int s = 0; s < 2; ++s) mbar_wait_grace(loaded + 8u * s, ((n_loads - 1 - (uint32_t)(((n_loads - 1) & 1u) != (uint32_t)s)) >> 1) & 1u);
    if (lane == 0) bulk_wait_all();
  }

  tcgen05_fence_before();
  __syncthreads();
  if constexpr (PAIR) {
    cluster_arrive();      // neither CTA leaves while its peer may still use its memory or barriers
    cluster_wait();
  }
  if (warp == 1) {
    tcgen05_fence_after();
    if constexpr (PAIR)
      asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(kTmemWanted) : "memory");
    else
      asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(kTmemWanted) : "memory");
  }
}

// ---- X = G / (|G| + eps) ----
struct OrthoStartArgs {
  const void* x;
  __half *hi, *lo;
  double* sums;                // [batch][parts]
  float *diag_a, *diag_b, *post;
  int64_t ldx, stride_x, pitch, diag;
  int32_t rows, cols, parts;
  int32_t row_ctas;            // CTAs of a matrix in the second kernel
  float eps, growth;           // growth: what the steps' a multiply a small X by at most
};

constexpr int kOrthoStartThreads = 256;

// A part of a matrix's sum of squares: a warp to a row.  In 64 bits: gradients' squares leave the range of 32.
template <int XT, bool EDGE>
__global__ void __launch_bounds__(kOrthoStartThreads) ortho_sum_kernel(const __grid_constant__ OrthoStartArgs args) {
  let_next_start();
  wait_for_previous();
  typedef typename ElemOf<XT>::T T;
  __shared__ double per_warp[kOrthoStartThreads / 32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int matrix = blockIdx.x / args.parts, part = blockIdx.x % args.parts;
  const T* x = static_cast<const T*>(args.x) + matrix * args.stride_x;
  double sum = 0.0;
  for (int r = part * 8 + warp; r < args.rows; r += 8 * args.parts) {
    for (int c = 8 * lane; c < args.cols; c += 256) {
      float v[8];
      to_float8<XT>(load_raw8<XT, EDGE>(x + r * args.ldx + c, vector_cols<EDGE>(args.cols, c)), v);
#pragma unroll
      for (int i = 0; i < 8; ++i) sum = fma((double)v[i], (double)v[i], sum);
    }
  }
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, d);
  if (lane == 0) per_warp[warp] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < kOrthoStartThreads / 32; ++w) sum += per_warp[w];
    args.sums[(int64_t)matrix * args.parts + part] = sum;
  }
}

// X in two FP16 numbers, zeros up to the next multiple of eight columns, and diagonals of zeros.
// Where |G| is far below eps, X is so small that every step is X' = a X to 2^-24 (b and c come with X^2): it is then
// started larger by a power of two, which takes it out of the range where FP16 ends, and the result made smaller by it.
template <int XT, bool EDGE>
__global__ void __launch_bounds__(kOrthoStartThreads) ortho_start_kernel(const __grid_constant__ OrthoStartArgs args) {
  let_next_start();
  wait_for_previous();
  typedef typename ElemOf<XT>::T T;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int matrix = blockIdx.x / args.row_ctas, part = blockIdx.x % args.row_ctas;
  double total = 0.0;
  for (int i = 0; i < args.parts; ++i) total += args.sums[(int64_t)matrix * args.parts + i];
  // (a sum that is no number, or infinite: every entry becomes NaN)
  const double norm = sqrt(total);
  double factor = norm < 1e300 ? (double)(1 << kOrthoScaleBits) / (norm + (double)args.eps) : __longlong_as_double(0x7FF8000000000000ll);
  const double largest = norm / (norm + (double)args.eps) * (double)args.growth;      // that X may become while it is small
  int larger = 0;
  if (largest > 0.0 && largest < 0x1p-13) larger = -13 - ilogb(largest) - 1;
  factor = ldexp(factor, larger);
  if (part == 0 && threadIdx.x == 0) args.post[matrix] = (float)ldexp(1.0, -larger);
  const float narrow = (float)factor;
  const bool wide = !(narrow > 1e-30f && narrow < 1e30f);      // (the factor, not the result, may be out of range)
  if (part == 0)
    for (int64_t i = threadIdx.x; i < args.diag; i += kOrthoStartThreads) args.diag_a[matrix * args.diag + i] = args.diag_b[matrix * args.diag + i] = 0.f;
  const T* x = static_cast<const T*>(args.x) + matrix * args.stride_x;
  const int64_t out = (int64_t)matrix * args.rows * args.pitch;
  for (int r = part * 8 + warp; r < args.rows; r += 8 * args.row_ctas) {
    for (int c = 8 * lane; c < args.cols; c += 256) {
      float v[8];
      to_float8<XT>(load_raw8<XT, EDGE>(x + r * args.ldx + c, vector_cols<EDGE>(args.cols, c)), v);
      uint32_t hi[4], lo[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float a = v[2 * i] * narrow, b = v[2 * i + 1] * narrow;
        if (wide) {
          a = (float)((double)v[2 * i] * factor);
          b = (float)((double)v[2 * i + 1] * factor);
        }
        const __half2 h = __floats2half2_rn(a, b);
        const float2 back = __half22float2(h);
        const __half2 l = __floats2half2_rn((a - back.x) * kOrthoLo, (b - back.y) * kOrthoLo);
        hi[i] = *reinterpret_cast<const uint32_t*>(&h);
        lo[i] = *reinterpret_cast<const uint32_t*>(&l);
      }
      const int64_t at = out + r * args.pitch + c;
      *reinterpret_cast<uint4*>(args.hi + at) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
      *reinterpret_cast<uint4*>(args.lo + at) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
    }
  }
}

}  // namespace maxdnn
