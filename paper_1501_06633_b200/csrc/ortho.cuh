// Newton-Schulz products of the orthogonalised update, for a batch of matrices: all steps in one launch, three products a step
// on FP16 operands with 32-bit sums (tcgen05 MMA, TMEM accumulators, bulk tensor copies), each with what the step does to it:
//
//   Gram    A = X X^T                      stored in FP16; symmetric
//   Poly    B = b A + c A A                stored in FP16; symmetric
//   Update  X' = a X + B X                 (or a X + X B); stored as two FP16 numbers, hi + lo; the last step's in BF16
//
// Precision.  An entry of X that is rounded to FP16 is off by 2^-12 of it, spread over all directions, and a step multiplies
// what lies in the directions of small singular values by a = 3.4: from a low-rank gradient five steps make 2 % of
// the result out of that rounding (17 % with BF16).  So X is kept as hi + lo (22 bits; lo is held 2^11 times as large, or it
// would end where hi does), which the a X term reads; the products read hi, whose rounding they only let act along the
// directions that they keep.  What is left comes from the diagonals of A and B, whose entries near 1 are the largest: they
// are kept in 32 bits (r: what FP16 left of them, d: all), and (A A)_mn += (r_m + r_n) A_mn, (B X)_mn += r_m hi_mn + d_m lo_mn.
// Against 64 bits over several spectra and sizes: 4e-4 to 1.3e-3 of the result's norm; its rounding to BF16 is 1.7e-3.
//
// Symmetric products compute the tiles that reach the diagonal or below it, half of the operations, and store no others: where a later
// product reads a part above the diagonal it reads the mirrored part instead, transposed by the MMA's descriptor
// ("MN-major").  X is read along either axis the same way, so nothing is transposed in memory.
//
// One launch.  Kernels of their own for each product would start 3 steps times, and a start (launch, barriers, tensor memory, the
// first copies) with the end of the kernel before costs about 6 us; the exchange that replaces it costs about 4.  Here the CTAs of
// a cooperative launch go from product to product: the warps that finish tiles report a CTA's end of a product to a counter in
// memory, and one warp of each CTA waits for all of them and lets the CTA's others on.
//
// Roles.  Warp 0 copies A, warp 3 copies B, warp 1 issues the MMAs, warp 2 watches the counter; warps 4-11 finish the tiles.
// Two accumulators alternate, so a tile is finished while the next one's MMAs run.  A finishing warp has 32 rows x up
// to 128 columns, 32 x 32 at a time: bulk copies bring the parts of X (A) it needs into its two slots in shared memory,
// one part ahead, and store the result from the same slot.
// PAIR.  Two CTAs share a tile of 256 rows (cta_group::2): each stages its 128 rows of A and half of the columns of B.
// Halves.  Where the last round of tiles would leave at least half of the CTAs without one, its tiles are cut in two.
//
// Bound by what SMs read from the second-level cache: a stage of 32 KB for 256 x 256 x 64 takes 628 cycles, one of
// 24 KB for 256 x 128 x 64 518, or 47 to 52 bytes a cycle and SM, where the MMAs need 512 and 256.  4096 x 4096, five
// steps: 1145 us by itself and 1320 us in a long run (power); 1.37 TFLOP are 827 us at the library's measured rate and 977 at its sustained one.  With 3, 4 and 5 stages 1541, 1424 and
// 1385 us, without the cache hint 1431, a launch for each product 1376 (long runs).  1000 x 2309: 200 us, 15 products with few tiles for each SM.
// Every wait on a barrier or the counter is bounded and ends in a status code; TMEM is always freed.  (Waits for tensor
// memory and at a cluster's end: see gemm8.cuh.)
#pragma once
#include "fp8_util.cuh"
#include "ortho.h"
#include "umma_util.cuh"

namespace maxdnn {

constexpr int kOrthoThreads = 384;
constexpr int kOrthoEpiWarps = 8;
constexpr float kOrthoLo = 2048.f;      // X = (hi + lo / kOrthoLo) 2^-10

struct OrthoMaps {
  // operands in boxes of 64 x 64; parts of 32 x 32
  CUtensorMap x[2], a, b, x_hi[2], x_lo[2], a_part, b_part, out;
};

struct OrthoArgs {
  OrthoProduct product[3];       // Gram, Poly, Update
  int32_t steps, batch, stages;
  int32_t tall;                  // products from the right: the residues of column n belong to X_mn, not those of row m
  int32_t bulk_out;              // out's rows allow bulk stores
  float *diag_a, *diag_b;        // [batch][diag] r of A; [batch][2][diag] r and d of B
  int64_t diag;
  const float* post;             // a power of two for each matrix's result
  uint32_t* done;                // CTAs that have finished a product, counted over all products
  __nv_bfloat16* out;
  int64_t ldo, stride_o;
  uint32_t test_missing_arrival;
  float coefficients[kOrthoMaxSteps][3];
  WaitCtx wc;
};

// Coordinates (column, row, matrix).
template <bool PAIR>
__device__ __forceinline__ void ortho_load(uint32_t dst, const CUtensorMap* m, uint32_t bar, int c0, int c1, int c2, uint64_t policy) {
  if constexpr (PAIR)
    asm volatile(
        "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
        ".L2::cache_hint [%0], [%1, {%3, %4, %5}], [%2], %6;" ::"r"(dst),
        "l"(reinterpret_cast<uint64_t>(m)), "r"(bar), "r"(c0), "r"(c1), "r"(c2), "l"(policy)
        : "memory");
  else
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.L2::cache_hint "
        "[%0], [%1, {%3, %4, %5}], [%2], %6;" ::"r"(dst),
        "l"(reinterpret_cast<uint64_t>(m)), "r"(bar), "r"(c0), "r"(c1), "r"(c2), "l"(policy)
        : "memory");
}
__device__ __forceinline__ void ortho_store(const CUtensorMap* m, uint32_t src, int c0, int c1, int c2) {
  asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%2, %3, %4}], [%1];" ::"l"(
                   reinterpret_cast<uint64_t>(m)),
               "r"(src), "r"(c0), "r"(c1), "r"(c2)
               : "memory");
}
// Orders copies by the copy engine on both sides of what this thread has seen or will tell.
__device__ __forceinline__ void fence_proxy_async_global() { asm volatile("fence.proxy.async.global;" ::: "memory"); }

__device__ __forceinline__ uint32_t load_acquire_gpu(const uint32_t* p) {
  uint32_t v;
  asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
  return v;
}
__device__ __forceinline__ uint32_t load_acquire_cta(uint32_t smem) {
  uint32_t v;
  asm volatile("ld.acquire.cta.shared.u32 %0, [%1];" : "=r"(v) : "r"(smem) : "memory");
  return v;
}
__device__ __forceinline__ void store_release_cta(uint32_t smem, uint32_t v) {
  asm volatile("st.release.cta.shared.u32 [%0], %1;" ::"r"(smem), "r"(v) : "memory");
}
// Waits until `seen()` is at least `want`: two seconds at most, as the waits on barriers.
template <class F>
__device__ __forceinline__ bool ortho_wait(F seen, uint32_t want, const WaitCtx& wc) {
  if (seen() >= want) return true;
  const uint64_t t0 = globaltimer_ns();
  for (;;) {
#pragma unroll 1
    for (int i = 0; i < 64; ++i)
      if (seen() >= want) return true;
    if (globaltimer_ns() - t0 > kWaitBudgetNs) break;
    if (launch_gave_up(wc)) return false;
  }
  record_give_up(wc, kDevTimeoutPeer);
  return false;
}

// Piece number `item` of a product: a tile, or behind the whole tiles half of one.
struct OrthoItem { int matrix, m0, n0, cols; };
template <int NT, int TILE_M>
__device__ __forceinline__ OrthoItem ortho_item(const OrthoProduct& p, int item) {
  OrthoItem o;
  const int past = item - p.full;
  const int tile = past < 0 ? item : p.full + (past >> 1);
  o.matrix = tile / p.tiles;
  const int t = tile - o.matrix * p.tiles;
  int mt, nt;
  if (p.symmetric) {
    // row by row of tiles; rows before row i have kRatio i (i + 1) / 2 (only the last row may have fewer than its share)
    constexpr int kRatio = TILE_M / NT;
    int i = (int)((sqrtf(1.f + 8.f * (float)t / (float)kRatio) - 1.f) * 0.5f);
    while (kRatio * i * (i + 1) / 2 > t) --i;
    while (kRatio * (i + 1) * (i + 2) / 2 <= t) ++i;
    mt = i;
    nt = t - kRatio * i * (i + 1) / 2;
  } else {
    // groups of eight rows of tiles, column by column: tiles at work together share operands
    const int per_group = 8 * p.n_tiles, group = t / per_group, first = group * 8;
    const int height = min(8, p.m_tiles - first), in = t - group * per_group;
    mt = first + in % height;
    nt = in / height;
  }
  o.m0 = mt * TILE_M;
  o.n0 = nt * NT + (past >= 0 && (past & 1) ? NT / 2 : 0);
  o.cols = past < 0 ? NT : NT / 2;
  return o;
}

// How an operand's tile lies in memory.  Symmetric matrices: stored up to the end of the diagonal block of TILE_M.
template <int TILE_M>
__device__ __forceinline__ bool ortho_mn_major(int mode, int first, int k) {
  return mode == kOrthoRowsAreK || (mode == kOrthoSymmetric && k / TILE_M > first / TILE_M);
}

template <int K> struct OrthoKindOf { static constexpr int value = K; };

// Whether any of the 256 threads that finish tiles says so.
__device__ __forceinline__ int epilogue_any(bool p) {
  int r;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %1, 0;\n\t"
      "barrier.cta.red.or.pred q, 1, 256, p;\n\tselp.b32 %0, 1, 0, q;\n\t}"
      : "=r"(r)
      : "r"((int)p)
      : "memory");
  return r;
}
template <int NT, bool PAIR>
__global__ void __launch_bounds__(kOrthoThreads, 1)
ortho_chain_kernel(const __grid_constant__ OrthoMaps maps, const __grid_constant__ OrthoArgs args) {
  constexpr int kTileM = PAIR ? 2 * kOrthoTileM : kOrthoTileM;
  constexpr uint32_t kAStage = kOrthoTileM * kOrthoBlockK * 2;
  constexpr uint32_t kBStage = (PAIR ? NT / 2 : NT) * kOrthoBlockK * 2;
  constexpr uint32_t kTmemWanted = 2 * NT;
  static_assert(kTileM % NT == 0, "a symmetric product's rows of tiles grow by whole tiles");
  extern __shared__ uint8_t smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* base_ptr = smem_raw + (base - smem_u32(smem_raw));
  const int stages = args.stages;
  const uint32_t b_off = (uint32_t)stages * kAStage;
  const uint32_t st_off = b_off + (uint32_t)stages * kBStage;
  const uint32_t full_bar = base + st_off + kOrthoStaging;
  const uint32_t empty_bar = full_bar + 8u * stages;
  const uint32_t accf_bar = empty_bar + 8u * stages;       // 2
  const uint32_t acce_bar = accf_bar + 16u;                // 2
  const uint32_t load_bar = acce_bar + 16u;                // 2 for each finishing warp
  const uint32_t done_bar = load_bar + 16u * kOrthoEpiWarps;
  const uint32_t tmem_slot = done_bar + 8u;
  const uint32_t passed = tmem_slot + 4u;                  // products that all CTAs have finished, as far as this CTA knows
  const uint32_t diag_off = (passed + 4u - base + 15u) & ~15u;      // each finishing warp: r and d of 32 columns
  volatile uint32_t* tmem_slot_ptr = reinterpret_cast<volatile uint32_t*>(base_ptr + (tmem_slot - base));

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = PAIR ? (int)cluster_ctarank() : 0;
  const int unit = (int)blockIdx.x / (PAIR ? 2 : 1), n_units = (int)gridDim.x / (PAIR ? 2 : 1);
  const bool leader = !PAIR || rank == 0;
  const int n_products = 3 * args.steps;

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
    store_release_cta(passed, 0);
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
  // product number p may read what the ones before it wrote
  auto wait_product = [&](int p) {
    const bool ok = ortho_wait([&] { return load_acquire_cta(passed); }, (uint32_t)p, args.wc);
    fence_proxy_async_global();
    return ok;
  };

  if (warp == 0 || warp == 3) {
    // ------------------------------------------------------------ copies
    const bool is_a = warp == 0;
    const uint64_t policy = l2_policy_evict_last();
    const uint32_t report = PAIR ? map_to_cta(full_bar, 0) : full_bar;
    int stage = 0;
    uint32_t phase = 0;
    bool ok = true;
    for (int pn = 0; pn < n_products && ok; ++pn) {
      const int kind = pn % 3, which = (pn / 3) & 1;
      const OrthoProduct& p = args.product[kind];
      const CUtensorMap* map = kind == kOrthoGram ? &maps.x[which] : kind == kOrthoPoly ? &maps.a
                               : is_a == (args.tall != 0) ? &maps.x[which] : &maps.b;
      const int mode = is_a ? p.a_mode : p.b_mode;
      ok = wait_product(pn);
      for (int item = unit; item < p.items && ok; item += n_units) {
        const OrthoItem o = ortho_item<NT, kTileM>(p, item);
        const int side = is_a ? o.m0 : o.n0;                         // of the (pair's) tile
        const int rows = is_a ? kOrthoTileM : PAIR ? o.cols / 2 : o.cols;
        const int first = side + rank * rows;
        const uint32_t tx = (PAIR ? 2u : 1u) * (uint32_t)rows * (2u * kOrthoBlockK);
        for (int ks = 0; ks < p.k_steps; ++ks) {
          if (!mbar_wait(empty_bar + 8u * stage, phase ^ 1u, args.wc, kDevTimeoutEmpty)) {
            ok = false;
            break;
          }
          const uint32_t dst = base + (is_a ? (uint32_t)stage * kAStage : b_off + (uint32_t)stage * kBStage);
          if (elect_one()) {
            if (leader) mbar_arrive_expect_tx(full_bar + 8u * stage, tx);
            const int k = ks * kOrthoBlockK;
            const bool mn = ortho_mn_major<kTileM>(mode, side, k);
#pragma unroll 1
            for (int r = 0; r < rows; r += 64)
              ortho_load<PAIR>(dst + 128u * r, map, report + 8u * stage, mn ? first + r : k, mn ? k : first + r, o.matrix, policy);
          }
          __syncwarp();
          if (++stage == stages) { stage = 0; phase ^= 1u; }
        }
      }
    }
    if (PAIR && ok) ok = wait_stages_free(empty_bar, stages, stage, phase, args.wc);
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
      const uint64_t desc_a = desc | (uint64_t)((base & 0x3FFFFu) >> 4);
      const uint64_t desc_b = desc | (uint64_t)(((base + b_off) & 0x3FFFFu) >> 4);
      int stage = 0;
      uint32_t phase = 0, acc_n = 0;
      bool ok = true, ready = false;
      for (int pn = 0; pn < n_products && ok; ++pn) {
        const OrthoProduct& p = args.product[pn % 3];
        for (int item = unit; item < p.items && ok; item += n_units, ++acc_n) {
          const OrthoItem o = ortho_item<NT, kTileM>(p, item);
          const uint32_t acc = acc_n & 1u, d = tmem_base + acc * NT;
          // instruction descriptor: fp32 accumulator, FP16 operands, N / 8, M / 16; the majors change along the reduction
          const uint32_t shape = (1u << 4) | ((uint32_t)(o.cols >> 3) << 17) | ((uint32_t)(kTileM >> 4) << 24);
          if (!mbar_wait(acce_bar + 8u * acc, ((acc_n >> 1) & 1u) ^ 1u, args.wc, kDevTimeoutAccFree)) {
            ok = false;
            break;
          }
          tcgen05_fence_after();
          for (int ks = 0; ks < p.k_steps; ++ks) {
            if (!ready && !mbar_wait(full_bar + 8u * stage, phase, args.wc, kDevTimeoutFull)) {
              ok = false;
              break;
            }
            const int next = stage + 1 == stages ? 0 : stage + 1;
            const uint32_t next_phase = stage + 1 == stages ? phase ^ 1u : phase;
            ready = mbar_test_wait(full_bar + 8u * next, next_phase);
            const bool a_mn = ortho_mn_major<kTileM>(p.a_mode, o.m0, ks * kOrthoBlockK);
            const bool b_mn = ortho_mn_major<kTileM>(p.b_mode, o.n0, ks * kOrthoBlockK);
            const uint32_t idesc = shape | ((uint32_t)a_mn << 15) | ((uint32_t)b_mn << 16);
            const uint64_t step_a = (a_mn ? 2048u : 32u) >> 4, step_b = (b_mn ? 2048u : 32u) >> 4;
            tcgen05_fence_after();
            if (elect_one()) {
              uint64_t a = desc_a + (uint64_t)((uint32_t)stage * (kAStage >> 4));
              uint64_t b = desc_b + (uint64_t)((uint32_t)stage * (kBStage >> 4));
#pragma unroll
              for (int j = 0; j < kOrthoBlockK / 16; ++j) {
                if constexpr (PAIR) tcgen05_mma_pair<true>(d, a, b, idesc, ks > 0 || j > 0);
                else tcgen05_mma<true>(d, a, b, idesc, ks > 0 || j > 0);
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
      }
      // every MMA issued so far has finished before TMEM is released
      if (elect_one()) {
        if constexpr (PAIR) tcgen05_commit_pair(done_bar, 1);
        else tcgen05_commit(done_bar);
      }
      mbar_wait(done_bar, 0, args.wc, kDevTimeoutDrain);
    }
  } else if (warp == 2) {
    // ------------------------------------------------------------ the other CTAs' progress
    if (lane == 0) {
      for (int pn = 1; pn < n_products; ++pn) {
        if (!ortho_wait([&] { return load_acquire_gpu(args.done); }, (uint32_t)pn * gridDim.x, args.wc)) break;
        store_release_cta(passed, (uint32_t)pn);
      }
    }
  } else {
    // ------------------------------------------------------------ what a step does to the product
    const int q = warp & 3;                   // TMEM lanes this warp may read
    const int ew = warp - 4;
    const uint32_t release = PAIR ? map_to_cta(acce_bar, 0) : acce_bar;
    const uint32_t slots = base + st_off + (uint32_t)ew * 8192u, loaded = load_bar + 16u * ew;
    uint8_t* slots_ptr = base_ptr + st_off + (size_t)ew * 8192;
    const uint32_t swz = (uint32_t)((lane >> 1) & 3);
    float* diag_here = reinterpret_cast<float*>(base_ptr + diag_off) + 64 * ew;
    uint32_t acc_n = 0, n_parts = 0, load_phase = 0;      // accumulators; parts (the slot is the last bit); a bit for each slot's loads
    bool ok = true;

    auto product = [&](auto kind_of, int pn) {
      constexpr int KIND = decltype(kind_of)::value;
      constexpr int kLoads = KIND == kOrthoGram ? 0 : KIND == kOrthoPoly ? 1 : 2;      // tiles of 32 x 32 that a part needs
      const int step = pn / 3, which = step & 1;
      const OrthoProduct& p = args.product[KIND == kOrthoLast ? kOrthoUpdate : KIND];
      const float ca = args.coefficients[step][0], cb = args.coefficients[step][1], cc = args.coefficients[step][2];
      const CUtensorMap* in = KIND == kOrthoPoly ? &maps.a_part : &maps.x_hi[which];
      const CUtensorMap* out = KIND == kOrthoGram ? &maps.a_part : KIND == kOrthoPoly ? &maps.b_part
                               : KIND == kOrthoUpdate ? &maps.x_hi[1 - which] : &maps.out;
      for (int item = unit; item < p.items && ok; item += n_units, ++acc_n) {
        const OrthoItem o = ortho_item<NT, kTileM>(p, item);
        const int units = o.cols / 64, u0 = (ew >> 2) * units;       // this warp's parts
        const int m_warp = o.m0 + rank * kOrthoTileM + q * 32, m = m_warp + lane;
        const int n_first = o.n0 + u0 * 32;
        auto wanted = [&](int u) { return u < units && m_warp < p.M && n_first + 32 * u < p.N; };
        const uint32_t first_part = n_parts;
        // brings what part u needs into the next slot, once that slot's store has been read
        auto load = [&](int u) {
          if (kLoads == 0 || !wanted(u)) return;
          if (lane == 0) {
            bulk_wait_read<0>();
            const uint32_t slot = (first_part + (uint32_t)u) & 1u, bar = loaded + 8u * slot, dst = slots + 4096u * slot;
            mbar_arrive_expect_tx(bar, 2048u * kLoads);
            const uint64_t policy = l2_policy_evict_first();
            ortho_load<false>(dst, in, bar, n_first + 32 * u, m_warp, o.matrix, policy);
            if (kLoads == 2) ortho_load<false>(dst + 2048u, &maps.x_lo[which], bar, n_first + 32 * u, m_warp, o.matrix, policy);
          }
          __syncwarp();
        };
        load(0);
        const float* r_a = args.diag_a + o.matrix * args.diag;
        const float* r_b = args.diag_b + 2 * o.matrix * args.diag;
        const float* d_b = r_b + args.diag;
        // Poly: r of this row.  Update: what hi and lo are multiplied by besides the product (products from the left)
        float r_m = 0.f, k_hi = ca, k_lo = ca;
        if (m < p.M) {
          if (KIND == kOrthoPoly) r_m = load_global(r_a + m);
          if (KIND >= kOrthoUpdate && !args.tall) {
            k_hi += load_global(r_b + m);
            k_lo += load_global(d_b + m);
          }
        }
        k_lo *= 1.f / kOrthoLo;
        // a column's r (and d) for each part, fetched before the product is there (diagonals end at multiples of 32)
        const bool by_column = KIND == kOrthoPoly || (KIND >= kOrthoUpdate && args.tall);
        float r_n[4] = {}, d_n[4] = {};
        if (by_column) {
#pragma unroll
          for (int u = 0; u < 4; ++u)
            if (wanted(u)) {
              r_n[u] = load_global((KIND == kOrthoPoly ? r_a : r_b) + n_first + 32 * u + lane);
              if (KIND != kOrthoPoly) d_n[u] = load_global(d_b + n_first + 32 * u + lane);
            }
        }
        const float gram_scale = __int_as_float((127 - 2 * kOrthoScaleBits) << 23);
        const float out_scale = KIND == kOrthoLast ? __int_as_float((127 - kOrthoScaleBits) << 23) * load_global(args.post + o.matrix) : 0.f;
        const uint32_t acc = acc_n & 1u;
        if (!mbar_wait(accf_bar + 8u * acc, (acc_n >> 1) & 1u, args.wc, kDevTimeoutAccum)) {
          ok = false;
          break;
        }
        tcgen05_fence_after();
        const uint32_t t_row = tmem_base + ((uint32_t)(q * 32) << 16) + acc * NT + (uint32_t)(u0 * 32);
#pragma unroll 1
        for (int u = 0; u < units; ++u) {
          if (!wanted(u)) break;
          if (u + 1 < units) load(u + 1);
          const int n0 = n_first + 32 * u;
          if (by_column) {
            diag_here[lane] = u == 0 ? r_n[0] : u == 1 ? r_n[1] : u == 2 ? r_n[2] : r_n[3];
            if (KIND != kOrthoPoly) diag_here[32 + lane] = u == 0 ? d_n[0] : u == 1 ? d_n[1] : u == 2 ? d_n[2] : d_n[3];
            __syncwarp();
          }
          uint32_t v[32];
          tmem_ld_32x32(t_row + (uint32_t)(32 * u), v);
          tmem_wait_ld();
          const uint32_t slot = n_parts & 1u;
          uint8_t* part = slots_ptr + 4096 * slot;
          if (kLoads > 0) {
            if (!mbar_wait(loaded + 8u * slot, (load_phase >> slot) & 1u, args.wc, kDevTimeoutFull)) ok = false;
            load_phase ^= 1u << slot;
          } else {
            if (lane == 0) bulk_wait_read<1>();      // the store before last had this slot
            __syncwarp();
          }
          uint8_t* row = part + lane * 64;
          const bool diagonal = (KIND == kOrthoGram || KIND == kOrthoPoly) && n0 == m_warp;      // the part's diagonal is the matrix's
#pragma unroll
          for (int i = 0; i < 4; ++i) {                    // eight columns, in pairs
            uint4* hi_at = reinterpret_cast<uint4*>(row + ((i ^ swz) << 4));
            uint4* lo_at = reinterpret_cast<uint4*>(row + 2048 + ((i ^ swz) << 4));
            F2 x[4], lo[4];
            if constexpr (kLoads > 0) {
              Raw8<MAXDNN_F16> raw;
              raw.a = *hi_at;
              to_pairs<MAXDNN_F16>(raw, x);
            }
            if constexpr (kLoads > 1) {
              Raw8<MAXDNN_F16> raw;
              raw.a = *lo_at;
              to_pairs<MAXDNN_F16>(raw, lo);
            }
            uint32_t w[4], z[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const F2 sum = ((F2)v[8 * i + 2 * k + 1] << 32) | v[8 * i + 2 * k];
              const bool mine = diagonal && 8 * i + 2 * k == (lane & ~1);      // one of the two is on the diagonal
              F2 y2;
              if constexpr (KIND == kOrthoGram) {
                y2 = mul2(sum, f2(gram_scale));
              } else if constexpr (KIND == kOrthoPoly) {
                const F2 r2 = *reinterpret_cast<const F2*>(diag_here + 8 * i + 2 * k);
                y2 = fma2(f2(cb), x[k], mul2(f2(cc), fma2(add2(f2(r_m), r2), x[k], sum)));
              } else if (args.tall) {
                const F2 r2 = *reinterpret_cast<const F2*>(diag_here + 8 * i + 2 * k);
                const F2 d2 = *reinterpret_cast<const F2*>(diag_here + 32 + 8 * i + 2 * k);
                y2 = fma2(add2(f2(ca), r2), x[k], fma2(mul2(add2(f2(ca), d2), f2(1.f / kOrthoLo)), lo[k], sum));
              } else {
                y2 = fma2(f2(k_hi), x[k], fma2(f2(k_lo), lo[k], sum));
              }
              float2 y = unf2(y2);
              if constexpr (KIND == kOrthoLast) {
                const __nv_bfloat162 t = __floats2bfloat162_rn(y.x * out_scale, y.y * out_scale);
                w[k] = *reinterpret_cast<const uint32_t*>(&t);
              } else {
                // (A_mm has r besides what FP16 holds of it, on both sides of its square too)
                if (KIND == kOrthoPoly && mine) (lane & 1 ? y.y : y.x) += r_m * fmaf(cc, r_m, cb);
                const __half2 t = __floats2half2_rn(y.x, y.y);
                w[k] = *reinterpret_cast<const uint32_t*>(&t);
                if constexpr (KIND == kOrthoUpdate) {
                  const float2 back = __half22float2(t);
                  const float2 left = unf2(mul2(add2(f2(y.x, y.y), f2(-back.x, -back.y)), f2(kOrthoLo)));
                  const __half2 rest = __floats2half2_rn(left.x, left.y);
                  z[k] = *reinterpret_cast<const uint32_t*>(&rest);
                } else if (mine && m < p.M) {
                  const float2 back = __half22float2(t);
                  const float all = lane & 1 ? y.y : y.x, rest = all - (lane & 1 ? back.y : back.x);
                  if (KIND == kOrthoGram) {
                    args.diag_a[o.matrix * args.diag + m] = rest;
                  } else {
                    args.diag_b[2 * o.matrix * args.diag + m] = rest;
                    args.diag_b[(2 * o.matrix + 1) * args.diag + m] = all;
                  }
                }
              }
            }
            if constexpr (KIND == kOrthoUpdate) *lo_at = make_uint4(z[0], z[1], z[2], z[3]);
            *hi_at = make_uint4(w[0], w[1], w[2], w[3]);
          }
          const uint32_t src = slots + 4096u * slot;
          if (KIND == kOrthoLast && !args.bulk_out) {
            // rows that bulk copies cannot store: a row of 32 neighbours at a time
            __syncwarp();
            const int n = n0 + lane;
            for (int r = 0; r < 32 && m_warp + r < p.M; ++r) {
              const __nv_bfloat16 t = *reinterpret_cast<const __nv_bfloat16*>(
                  part + r * 64 + (((lane >> 3) ^ ((r >> 1) & 3)) << 4) + 2 * (lane & 7));
              if (n < p.N) args.out[o.matrix * args.stride_o + (int64_t)(m_warp + r) * args.ldo + n] = t;
            }
            fence_proxy_async_smem();      // (the next copy into this slot follows these reads and writes)
            __syncwarp();
          } else {
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) {
              ortho_store(out, src, n0, m_warp, o.matrix);
              if (KIND == kOrthoUpdate) ortho_store(&maps.x_lo[1 - which], src + 2048u, n0, m_warp, o.matrix);
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
    };

    for (int pn = 0; pn < n_products; ++pn) {
      if (ok) ok = wait_product(pn);
      if (ok) {
        if (pn + 1 == n_products) product(OrthoKindOf<kOrthoLast>(), pn);
        else if (pn % 3 == kOrthoGram) product(OrthoKindOf<kOrthoGram>(), pn);
        else if (pn % 3 == kOrthoPoly) product(OrthoKindOf<kOrthoPoly>(), pn);
        else product(OrthoKindOf<kOrthoUpdate>(), pn);
      }
      // this CTA's results are written; a warp that gave up keeps the others company, but the CTA does not report
      if (lane == 0) {
        bulk_wait_all();
        fence_proxy_async_global();
      }
      __syncwarp();
      const int failed = epilogue_any(!ok);
      // (the barrier orders the other warps' writes before this thread's release)
      if (ew == 0 && lane == 0 && !failed) asm volatile("red.release.gpu.global.add.u32 [%0], 1;" ::"l"(args.done) : "memory");
    }
    if (!ok)      // leaving early: copies already issued land within microseconds
      for (int s = 0; s < 2; ++s) mbar_wait_grace(loaded + 8u * s, (load_phase >> s) & 1u);
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
  uint32_t* done;
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
    for (int64_t i = threadIdx.x; i < args.diag; i += kOrthoStartThreads)
      args.diag_a[matrix * args.diag + i] = args.diag_b[2 * matrix * args.diag + i] = args.diag_b[(2 * matrix + 1) * args.diag + i] = 0.f;
  if (blockIdx.x == 0 && threadIdx.x == 0) *args.done = 0;
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
