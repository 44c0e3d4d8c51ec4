// 8-bit matrix product with power-of-two scales, which the tensor core applies itself (tcgen05
// block-scaled MMA: one scale per row and 32 reduction steps; a block of 128 passes its scale to
// four MMAs in a row).
//
//   C[m, n] = sum_k (a[m, k] 2^ea) (b[n, k] 2^eb)
//
// Nothing is left to do between the blocks of the reduction, so an accumulator takes a whole
// chunk of it.  The tensor core truncates its fp32 accumulator at every MMA (towards zero), so terms of
// one sign lose about half a unit of the running sum each time, and the loss grows with the length.
// Chunks are added in registers with round-to-nearest.  An fp32 result takes chunks of sixteen
// blocks (64 MMAs).  Measured on a weight gradient over 16384 tokens, 8192 x 4096 (error against 64 bits, relative;
// time of a short run at a high clock / back to back): chunks of 4 blocks 1.1e-7, 674 us; 8: 1.6e-7, 512; 16:
// 3.0e-7, 462 / 540; 32: 428 / 498; one accumulator 1.5e-6, 396 / 460 (fp32 arithmetic throughout: 3.6e-7).
// A 16-bit result takes chunks of 128 blocks (512 MMAs): at most 6.2e-5 of it for terms of one sign, against 2.4e-4
// for the rounding to fp16; with one accumulator for 2^18 terms of one sign its bf16 values were off, for 2^20
// its fp16 values.
//
// Roles.  Warp 0 copies A, warp 3 copies B, warp 1 issues the MMAs, warp 2 gathers the scales:
// the bytes of four blocks and 128 rows, which lie [block][row] in memory, become 32 rows of 16
// bytes in shared memory (row r's four bytes in word r / 32 of line r mod 32); one tensor-memory
// copy of those 512 bytes replicates them to the four lane quarters, and the MMA picks the byte of
// its block.  Warps 4-11 hold the totals (32 rows x up to 128 columns each) and store C: through a swizzled
// staging tile and bulk tensor stores where C's rows allow it, else element by element.
//
// PAIR.  Two CTAs share a tile of 256 rows: each stages its 128 rows of A and half of the columns
// of B, one MMA reads both halves of B, and each CTA keeps its rows of the product.  Per SM that is 32 KB
// for 256 x 256 x 128 steps instead of 48 KB for 128 x 256 x 128.  Scales: each CTA gathers those of its rows and
// of all columns.  Both CTAs' copies report to the leader's barriers; its commits reach both.
//
// Accumulators.  Two where tensor memory holds them next to the scales (NT <= 224), so that one
// is read while the other fills; NT = 256 has one, and the MMAs wait while it is read: the tensor pipe is busy in
// 82 % of that weight gradient's cycles with a 16-bit C, 61 % with an fp32 C (either major).
//
// Few tiles (not PAIR): a cluster of 2, 4 or 8 CTAs shares a tile's reduction, as in gemm8.cuh.
//
// Measured: 8192 x 8192 x 8192 to bf16 390 to 396 us in short runs = 2.8 PFLOP/s (MMAs in 88 % of the cycles; the
// power limit holds the clock at 1.2 to 1.4 GHz, so that with the copies left out it would be 3.4), 2048 x 4096 x 4096
// 31 us in short runs, 36 back to back, one token through 4096 x 4096 7.4 us (16.8 MB: 2.3 TB/s; the start of a call, a
// memory latency and the exchange between the CTAs are 5 of them).
#pragma once
#include "gemm8.cuh"

namespace maxdnn {

constexpr int kMxThreads = 384;
constexpr int kMxEpiWarps = 8;
constexpr int kMxScaleBatch = 4;                   // scale groups (four blocks each) gathered at a time
constexpr int kMxScaleBufs = 2 * kMxScaleBatch;    // groups in shared memory

__host__ __device__ constexpr int mx_units(int nt) { return (nt + 63) / 64; }           // 32 columns each, per warp
__host__ __device__ constexpr int mx_sf_bytes(int nt) { return 128 * mx_sf_cols(nt); }

struct Gemm8MxArgs {
  Gemm8Scale sa, sb;
  void* c;
  int64_t c_row, c_col;
  int32_t M, N;
  int32_t m_tiles, n_tiles, k_blocks;
  int32_t split, stages;
  int32_t a_mn, b_mn;
  int32_t b_stage_bytes;
  int32_t c_type;
  int32_t bulk_c;              // C is stored by bulk tensor copies; 0: element by element
  int32_t staged_c;            // C goes through staging tiles (bulk copies, or rows of odd pitch)
  int32_t chunk;               // blocks per accumulator
  uint32_t idesc;
  uint32_t test_missing_arrival;
  WaitCtx wc;
};

template <bool PAIR>
__device__ __forceinline__ void tcgen05_mma_mx(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sfa,
                                               uint32_t sfb, uint32_t accumulate) {
  if constexpr (PAIR)
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate)
        : "memory");
  else
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate)
        : "memory");
}

// 32 lines of 16 bytes (8 lines = 128 bytes apart) to four columns of all four lane quarters.
template <bool PAIR>
__device__ __forceinline__ void tcgen05_copy_scales(uint32_t taddr, uint32_t smem) {
  const uint64_t desc = make_smem_desc(smem, 128u, 128u, 0u);
  if constexpr (PAIR)
    asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
  else
    asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
}

__device__ __forceinline__ void tma_load_2d_pair(uint32_t dst, const CUtensorMap* m, uint32_t bar, int c0, int c1,
                                                 uint64_t policy) {
  asm volatile(
      "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
      ".L2::cache_hint [%0], [%1, {%3, %4}], [%2], %5;" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(m)), "r"(bar), "r"(c0), "r"(c1), "l"(policy)
      : "memory");
}

__device__ __forceinline__ void tma_store_2d_hint(const CUtensorMap* m, uint32_t src, int c0, int c1, uint64_t policy) {
  asm volatile(
      "cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group.L2::cache_hint [%0, {%2, %3}], [%1], %4;" ::"l"(
          reinterpret_cast<uint64_t>(m)),
      "r"(src), "r"(c0), "r"(c1), "l"(policy)
      : "memory");
}

// The scale bytes of rows row0 + 4 lane .. + 3 in each of the blocks kb .. kb + 3 (clamped to the
// last row and block): one word per block.
__device__ __forceinline__ void mx_load_scales(const Gemm8Scale& s, int row0, int lane, int kb, int last,
                                               uint32_t (&raw)[4]) {
  const uint8_t* p = static_cast<const uint8_t*>(s.p);
  const int r = row0 + 4 * lane;
  if (s.shift) {    // row0 is a multiple of 16: the four rows have one scale
    p += (int64_t)(min(r, s.count - 1) >> s.shift) * s.step;
#pragma unroll
    for (int b = 0; b < 4; ++b) raw[b] = 0x01010101u * load_global(p + (int64_t)min(kb + b, last) * s.kstep);
  } else {
    if (s.words && r + 3 < s.count) {
#pragma unroll
      for (int b = 0; b < 4; ++b)
        raw[b] = load_global(reinterpret_cast<const uint32_t*>(p + (int64_t)min(kb + b, last) * s.kstep + r));
    } else {
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        const uint8_t* q = p + (int64_t)min(kb + b, last) * s.kstep;
        raw[b] = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) raw[b] |= (uint32_t)load_global(q + min(r + i, s.count - 1)) << (8 * i);
      }
    }
  }
}

// Those bytes as the tensor-memory copy wants them: row r's four block bytes in word r / 32 of the
// 16-byte line r mod 32.
__device__ __forceinline__ void mx_store_scales(uint8_t* dst, int lane, const uint32_t (&raw)[4]) {
  // transpose of 4 x 4 bytes
  const uint32_t a = __byte_perm(raw[0], raw[1], 0x5140), b = __byte_perm(raw[0], raw[1], 0x7362);
  const uint32_t c = __byte_perm(raw[2], raw[3], 0x5140), d = __byte_perm(raw[2], raw[3], 0x7362);
  const uint32_t w[4] = {__byte_perm(a, c, 0x5410), __byte_perm(a, c, 0x7632), __byte_perm(b, d, 0x5410),
                         __byte_perm(b, d, 0x7632)};
  uint8_t* p = dst + ((4 * lane) & 31) * 16 + (lane >> 3) * 4;
#pragma unroll
  for (int i = 0; i < 4; ++i) *reinterpret_cast<uint32_t*>(p + 16 * i) = w[i];
}

// Few columns: two CTAs share an SM, so that one's copies run while the other starts or ends.
__host__ __device__ constexpr int mx_ctas_per_sm(int nt) { return nt <= 32 ? 2 : 1; }

template <int NT, bool PAIR>
__global__ void __launch_bounds__(kMxThreads, mx_ctas_per_sm(NT))
gemm8_mx_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                const __grid_constant__ CUtensorMap map_c, const __grid_constant__ Gemm8MxArgs args) {
  constexpr int kBuf = mx_buffers(NT);
  constexpr int kUnits = mx_units(NT);
  constexpr int kUnitCols = NT < 32 ? NT : 32;
  constexpr int kAllUnits = (NT + 31) / 32;
  constexpr int kSfCols = mx_sf_cols(NT);
  constexpr uint32_t kSfBytes = mx_sf_bytes(NT);
  constexpr uint32_t kAStage = kGemm8TileM * kGemm8BlockK;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* base_ptr = smem_raw + (base - smem_u32(smem_raw));
  const int stages = args.stages;
  const uint32_t b_off = (uint32_t)stages * kAStage;
  const uint32_t st_off = b_off + (uint32_t)stages * (uint32_t)args.b_stage_bytes;
  const uint32_t stg_bytes = args.c_type == MAXDNN_F32 || !args.bulk_c ? 4096u : 2048u;   // 32 rows x 32 columns
  const uint32_t sf_off = st_off + (args.staged_c ? kMxEpiWarps * stg_bytes : 0u);
  const uint32_t bar_off = sf_off + kMxScaleBufs * kSfBytes;
  const uint32_t full_bar = base + bar_off;
  const uint32_t empty_bar = full_bar + 8u * stages;
  const uint32_t sff_bar = empty_bar + 8u * stages;    // scales of a group are in shared memory
  const uint32_t sfe_bar = sff_bar + 8u * kMxScaleBufs;    // and no longer needed
  const uint32_t accf_bar = sfe_bar + 8u * kMxScaleBufs;   // 2
  const uint32_t acce_bar = accf_bar + 16u;            // 2
  const uint32_t done_bar = acce_bar + 16u;
  const uint32_t tmem_slot = done_bar + 8u;
  volatile uint32_t* tmem_slot_ptr = reinterpret_cast<volatile uint32_t*>(base_ptr + (tmem_slot - base));

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int split = PAIR ? 1 : args.split;
  const int rank = (PAIR || split > 1) ? (int)cluster_ctarank() : 0;
  const int per_unit = PAIR ? 2 : split;               // CTAs of a tile
  const int unit = (int)blockIdx.x / per_unit, n_units = (int)gridDim.x / per_unit;
  const int n_tiles = args.m_tiles * args.n_tiles;
  const int kb0 = PAIR ? 0 : (int)((int64_t)args.k_blocks * rank / split);
  const int kb1 = PAIR ? args.k_blocks : (int)((int64_t)args.k_blocks * (rank + 1) / split);
  const bool leader = !PAIR || rank == 0;
  const int tile_m = PAIR ? 2 * kGemm8TileM : kGemm8TileM;

  if (threadIdx.x == 0) {
    const uint32_t extra = (args.test_missing_arrival != 0 && blockIdx.x == 0) ? 1u : 0u;   // test hook
    for (int s = 0; s < stages; ++s) {
      mbar_init(full_bar + 8u * s, 2 + extra);          // the (leader's) two copy warps
      mbar_init(empty_bar + 8u * s, 1);
    }
    for (int a = 0; a < kMxScaleBufs; ++a) {
      mbar_init(sff_bar + 8u * a, PAIR ? 2 : 1);
      mbar_init(sfe_bar + 8u * a, 1);
    }
    for (int a = 0; a < 2; ++a) {
      mbar_init(accf_bar + 8u * a, 1);
      mbar_init(acce_bar + 8u * a, kMxEpiWarps * (PAIR ? 2 : 1));
    }
    mbar_init(done_bar, 1);
    fence_mbar_init();
    fence_proxy_async_smem();
  }
  if (warp == 1) {
    if constexpr (PAIR) {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(tmem_slot),
                   "r"((uint32_t)mx_tmem_cols(NT)) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
      asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(tmem_slot),
                   "r"((uint32_t)mx_tmem_cols(NT)) : "memory");
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
  // Only now: a CTA of the next kernel that shares this SM takes its tensor memory after this one has
  // its own (it holds it while it waits for this kernel's end).
  let_next_start();
  wait_for_previous();

  if (warp == 0 || warp == 3) {
    // ------------------------------------------------------------ copies
    const bool is_a = warp == 0;
    if (lane == 0) prefetch_tensormap(is_a ? &map_a : &map_b);
    const uint64_t policy = l2_policy_evict_last();
    const uint32_t tx = (PAIR ? 2u : 1u) * (is_a ? kAStage : (uint32_t)args.b_stage_bytes);
    const uint32_t report = PAIR ? map_to_cta(full_bar, 0) : full_bar;
    int stage = 0;
    uint32_t phase = 0;
    bool ok = true;
    for (int tile = unit; tile < n_tiles && ok; tile += n_units) {
      int mt, nt;
      gemm8_tile(args.m_tiles, args.n_tiles, tile, &mt, &nt);
      const int i0 = is_a ? mt * tile_m + (PAIR ? rank * kGemm8TileM : 0) : nt * NT + (PAIR ? rank * (NT / 2) : 0);
      const bool mn = is_a ? args.a_mn != 0 : args.b_mn != 0;
      for (int kb = kb0; kb < kb1; ++kb) {
        if (!mbar_wait(empty_bar + 8u * stage, phase ^ 1u, args.wc, kDevTimeoutEmpty)) {
          ok = false;
          break;
        }
        const uint32_t dst = base + (is_a ? (uint32_t)stage * kAStage : b_off + (uint32_t)stage * (uint32_t)args.b_stage_bytes);
        if (elect_one()) {
          if (leader) mbar_arrive_expect_tx(full_bar + 8u * stage, tx);
          const int k = kb * kGemm8BlockK;
          const CUtensorMap* map = is_a ? &map_a : &map_b;
          if constexpr (PAIR) tma_load_2d_pair(dst, map, report + 8u * stage, mn ? i0 : k, mn ? k : i0, policy);
          else tma_load_2d_hint(dst, map, report + 8u * stage, mn ? i0 : k, mn ? k : i0, policy);
        }
        __syncwarp();
        if (++stage == stages) { stage = 0; phase ^= 1u; }
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
  } else if (warp == 2) {
    // ------------------------------------------------------------ scales
    // The fence that hands the bytes to the tensor-memory copy also waits for loads on their way,
    // so loads and fences alternate, four groups at a time: one load latency per sixteen blocks, while
    // the MMAs work on the four groups before.
    constexpr int kSides = kSfCols / 4;          // 128 rows of A, then of B's columns
    const uint32_t report = PAIR ? map_to_cta(sff_bar, 0) : sff_bar;
    uint32_t raw[kMxScaleBatch][kSides][4];
    int tile = unit, kb = kb0, m0 = 0, n0 = 0;   // the next group to load
    const int my_tiles = unit < n_tiles ? (n_tiles - unit + n_units - 1) / n_units : 0;
    const uint32_t groups = (uint32_t)my_tiles * (uint32_t)((kb1 - kb0 + 3) / 4);
    bool ok = true;
    for (uint32_t g0 = 0; g0 < groups && ok; g0 += kMxScaleBatch) {
#pragma unroll
      for (int b = 0; b < kMxScaleBatch; ++b) {
        if (g0 + b >= groups) break;
        if (kb == kb0) {
          int mt, nt;
          gemm8_tile(args.m_tiles, args.n_tiles, tile, &mt, &nt);
          m0 = mt * tile_m + (PAIR ? rank * kGemm8TileM : 0);
          n0 = nt * NT;
        }
        mx_load_scales(args.sa, m0, lane, kb, kb1 - 1, raw[b][0]);
#pragma unroll
        for (int j = 1; j < kSides; ++j) mx_load_scales(args.sb, n0 + 128 * (j - 1), lane, kb, kb1 - 1, raw[b][j]);
        kb += 4;
        if (kb >= kb1) { kb = kb0; tile += n_units; }
      }
#pragma unroll
      for (int b = 0; b < kMxScaleBatch; ++b) {
        if (g0 + b >= groups) break;
        const uint32_t buf = (g0 + b) % kMxScaleBufs;
        if (!mbar_wait(sfe_bar + 8u * buf, (((g0 + b) / kMxScaleBufs) & 1u) ^ 1u, args.wc, kDevTimeoutEmpty)) {
          ok = false;
          break;
        }
#pragma unroll
        for (int j = 0; j < kSides; ++j)
          mx_store_scales(base_ptr + sf_off + buf * kSfBytes + 512 * j, lane, raw[b][j]);
      }
      if (!ok) break;
      fence_proxy_async_smem();
      __syncwarp();
      if (lane < kMxScaleBatch && g0 + lane < groups) {
        const uint32_t at = 8u * ((g0 + lane) % kMxScaleBufs);
        if constexpr (PAIR) mbar_arrive_cluster(report + at);
        else mbar_arrive(report + at);
      }
      __syncwarp();
    }
    // (as wait_stages_free: the commits that free scales arrive at both CTAs)
    if (PAIR)
      for (uint32_t g = groups > kMxScaleBufs ? groups - kMxScaleBufs : 0; g < groups && ok; ++g)
        ok = mbar_wait(sfe_bar + 8u * (g % kMxScaleBufs), (g / kMxScaleBufs) & 1u, args.wc, kDevTimeoutEmpty);
  } else if (warp == 1) {
    // ------------------------------------------------------------ MMAs (the leader's, for both CTAs)
    if (leader) {
      // A block's four MMAs run for 270 ns (NT = 256): the loop around them has to be short.  It
      // walks whole scale groups, four blocks unrolled, so that the scale byte's number is a constant,
      // and asks for the next stage's barrier before it issues this one's MMAs.
      const uint64_t desc = make_smem_desc(0, 16384u, 1024u, 2u);
      const uint64_t step_a = (args.a_mn ? 4096u : 32u) >> 4;
      const uint64_t step_b = (args.b_mn ? 4096u : 32u) >> 4;
      const uint64_t desc_a = desc | (uint64_t)((base & 0x3FFFFu) >> 4);
      const uint64_t desc_b = desc | (uint64_t)(((base + b_off) & 0x3FFFFu) >> 4);
      const uint32_t b_stage = (uint32_t)args.b_stage_bytes >> 4;
      const int chunk = args.chunk;             // a multiple of four
      int stage = 0;
      uint32_t phase = 0, group = 0, acc_n = 0;
      bool ok = true, ready = false;
      for (int tile = unit; tile < n_tiles && ok; tile += n_units) {
        for (int c0 = kb0; c0 < kb1 && ok; c0 += chunk, ++acc_n) {
          const int c1 = min(c0 + chunk, kb1);
          const uint32_t acc = acc_n % kBuf;
          const uint32_t d = tmem_base + acc * NT;
          if (!mbar_wait(acce_bar + 8u * acc, ((acc_n / kBuf) & 1u) ^ 1u, args.wc, kDevTimeoutAccFree)) {
            ok = false;
            break;
          }
          for (int g0 = c0; g0 < c1 && ok; g0 += 4, ++group) {
            const uint32_t buf = group % kMxScaleBufs;
            const uint32_t sf = tmem_base + kBuf * NT + (group % kMxScaleTmem) * kSfCols;
            // the MMAs that read these tensor-memory columns last (four groups ago) have finished
            const uint32_t old = group - kMxScaleTmem;
            if ((group >= kMxScaleTmem &&
                 !mbar_wait(sfe_bar + 8u * (old % kMxScaleBufs), (old / kMxScaleBufs) & 1u, args.wc, kDevTimeoutDrain)) ||
                !mbar_wait(sff_bar + 8u * buf, (group / kMxScaleBufs) & 1u, args.wc, kDevTimeoutFull)) {
              ok = false;
              break;
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              if (g0 + i >= c1) break;
              if (!ready && !mbar_wait(full_bar + 8u * stage, phase, args.wc, kDevTimeoutFull)) {
                ok = false;
                break;
              }
              const int next = stage + 1 == stages ? 0 : stage + 1;
              const uint32_t next_phase = stage + 1 == stages ? phase ^ 1u : phase;
              ready = mbar_test_wait(full_bar + 8u * next, next_phase);
              tcgen05_fence_after();
              if (elect_one()) {
                if (i == 0) {
                  const uint32_t src = base + sf_off + buf * kSfBytes;
#pragma unroll
                  for (int j = 0; j < kSfCols; j += 4) tcgen05_copy_scales<PAIR>(sf + j, src + j * 128);
                }
                uint64_t a = desc_a + (uint64_t)((uint32_t)stage * (kAStage >> 4));
                uint64_t b = desc_b + (uint64_t)((uint32_t)stage * b_stage);
                // the byte of this block in the scale words of both operands
                const uint32_t idesc = args.idesc | ((uint32_t)i << 29) | ((uint32_t)i << 4);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                  tcgen05_mma_mx<PAIR>(d, a, b, idesc, sf, sf + 4, i > 0 || j > 0 || g0 > c0);
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
              if constexpr (PAIR) tcgen05_commit_pair(sfe_bar + 8u * buf);
              else tcgen05_commit(sfe_bar + 8u * buf);
            }
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
  } else {
    // ------------------------------------------------------------ totals and C
    const int q = warp & 3;                   // TMEM lanes this warp may read
    const int ew = warp - 4;
    const int u0 = (ew >> 2) * kUnits;        // its first unit of 32 columns
    const uint32_t release = PAIR ? map_to_cta(acce_bar, 0) : acce_bar;
    const uint32_t stg = base + st_off + (uint32_t)ew * stg_bytes;
    uint8_t* stg_ptr = base_ptr + st_off + (size_t)ew * stg_bytes;
    const uint64_t policy = l2_policy_evict_first();
    const int blocks = kb1 - kb0, chunks = (blocks + args.chunk - 1) / args.chunk;
    uint32_t acc_n = 0;
    bool ok = true;
    for (int tile = unit; tile < n_tiles && ok; tile += n_units) {
      int mt, nt;
      gemm8_tile(args.m_tiles, args.n_tiles, tile, &mt, &nt);
      const int m_warp = mt * tile_m + (PAIR ? rank * kGemm8TileM : 0) + q * 32;
      const int m = m_warp + lane;
      const int n0 = nt * NT + u0 * 32;
      float tot[kUnits][kUnitCols];
      for (int c = 0; c < chunks; ++c, ++acc_n) {
        const uint32_t acc = acc_n % kBuf;
        if (!mbar_wait(accf_bar + 8u * acc, (acc_n / kBuf) & 1u, args.wc, kDevTimeoutAccum)) {
          ok = false;
          break;
        }
        tcgen05_fence_after();
        const uint32_t t_row = tmem_base + ((uint32_t)(q * 32) << 16) + acc * NT + (uint32_t)(u0 * 32);
#pragma unroll
        for (int u = 0; u < kUnits; ++u) {
          if (u0 + u >= kAllUnits) continue;
#pragma unroll
          for (int h = 0; h < kUnitCols; h += 16) {
            uint32_t v[16];
            tmem_ld_32x16(t_row + (uint32_t)(32 * u + h), v);
            tmem_wait_ld();
            if (c == 0) {
#pragma unroll
              for (int i = 0; i < 16; ++i) tot[u][h + i] = __uint_as_float(v[i]);
            } else {
#pragma unroll
              for (int i = 0; i < 16; ++i) tot[u][h + i] += __uint_as_float(v[i]);
            }
          }
        }
        tcgen05_fence_before();
        __syncwarp();
        if (lane == 0) {
          if constexpr (PAIR) mbar_arrive_cluster(release + 8u * acc);
          else mbar_arrive(release + 8u * acc);
        }
      }
      if (!ok) break;
      if (!PAIR && split > 1) {
        // this CTA's totals where the ring was
        float* mine = reinterpret_cast<float*>(base_ptr);
#pragma unroll
        for (int u = 0; u < kUnits; ++u)
          if (u0 + u < kAllUnits) {
#pragma unroll
            for (int i = 0; i < kUnitCols; ++i)
              gemm8_keep_total<NT>(mine, args.c_row == 1, q * 32 + lane, (u0 + u) * 32 + i, tot[u][i]);
          }
      } else if (args.bulk_c) {
        if constexpr (NT >= 32) {
#pragma unroll
          for (int u = 0; u < kUnits; ++u) {
            if (u0 + u >= kAllUnits || n0 + 32 * u >= args.N || m_warp >= args.M) continue;
            // the staging tile must have been read by the store before
            if (lane == 0) bulk_wait_read<0>();
            __syncwarp();
            if (args.c_type == MAXDNN_F32) {
              uint8_t* row = stg_ptr + lane * 128;
#pragma unroll
              for (int i = 0; i < 8; ++i)
                *reinterpret_cast<float4*>(row + ((i ^ (lane & 7)) << 4)) =
                    make_float4(tot[u][4 * i], tot[u][4 * i + 1], tot[u][4 * i + 2], tot[u][4 * i + 3]);
            } else {
              uint8_t* row = stg_ptr + lane * 64;
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                uint32_t w[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                  const float x = tot[u][8 * i + 2 * k], y = tot[u][8 * i + 2 * k + 1];
                  if (args.c_type == MAXDNN_BF16) {
                    const __nv_bfloat162 t = __floats2bfloat162_rn(x, y);
                    w[k] = *reinterpret_cast<const uint32_t*>(&t);
                  } else {
                    const __half2 t = __floats2half2_rn(x, y);
                    w[k] = *reinterpret_cast<const uint32_t*>(&t);
                  }
                }
                *reinterpret_cast<uint4*>(row + ((i ^ ((lane >> 1) & 3)) << 4)) = make_uint4(w[0], w[1], w[2], w[3]);
              }
            }
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) {
              tma_store_2d_hint(&map_c, stg, n0 + 32 * u, m_warp, policy);
              bulk_commit();
            }
          }
        }
      } else if (args.staged_c) {
        // rows that bulk copies cannot store: through the staging tile (column c of row r at c ^ r,
        // which keeps both directions free of bank conflicts), a row of 32 neighbours at a time
        float* tile_f = reinterpret_cast<float*>(stg_ptr);
#pragma unroll
        for (int u = 0; u < kUnits; ++u) {
          if (u0 + u >= kAllUnits || n0 + 32 * u >= args.N) continue;
          __syncwarp();
#pragma unroll
          for (int i = 0; i < kUnitCols; ++i) tile_f[lane * 32 + (i ^ lane)] = tot[u][i];
          __syncwarp();
          const int n = n0 + 32 * u + lane;
          if (lane < kUnitCols && n < args.N) {
#pragma unroll 4
            for (int rr = 0; rr < 32 && m_warp + rr < args.M; ++rr)
              gemm8_store1(args.c, args.c_type, (int64_t)(m_warp + rr) * args.c_row + n, tile_f[rr * 32 + (lane ^ rr)]);
          }
        }
      } else if (m < args.M) {
        const int64_t at = (int64_t)m * args.c_row;
#pragma unroll
        for (int u = 0; u < kUnits; ++u)
          if (u0 + u < kAllUnits) {
#pragma unroll
            for (int i = 0; i < kUnitCols; ++i) {
              const int n = n0 + 32 * u + i;
              if (n < args.N) gemm8_store1(args.c, args.c_type, at + (int64_t)n * args.c_col, tot[u][i]);
            }
          }
      }
    }
    if (lane == 0) bulk_wait_all();
  }

  tcgen05_fence_before();
  __syncthreads();
  if constexpr (PAIR) {
    cluster_arrive();      // neither CTA leaves while its peer may still use its memory or barriers
    cluster_wait();
  } else if (split > 1) {
    cluster_arrive();
    cluster_wait();
    gemm8_add_split<NT, kMxThreads>(args, base, split, rank, unit);
    cluster_arrive();
    cluster_wait();
  }
  if (warp == 1) {
    tcgen05_fence_after();
    if constexpr (PAIR)
      asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base),
                   "r"((uint32_t)mx_tmem_cols(NT)) : "memory");
    else
      asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base),
                   "r"((uint32_t)mx_tmem_cols(NT)) : "memory");
  }
}

}  // namespace maxdnn
