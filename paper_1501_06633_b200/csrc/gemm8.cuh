// 8-bit matrix product with a scale for each block of 128 along the reduction (tcgen05 MMA, TMEM
// accumulators, bulk tensor copies):
//
//   C[m, n] = sum_kb sa[m, kb] sb[n, kb] D_kb[m, n],   D_kb[m, n] = sum_{k in block kb} a[m, k] b[n, k]
//
// The scales change along the reduction, so a block's product D_kb is finished on the tensor
// cores (four MMAs of 32 reduction steps into a TMEM accumulator that starts at zero), read back
// and added to totals in registers as fma(sa sb, D_kb, total): 32-bit sums with one rounding for
// each block, and no long run of the tensor core's truncating accumulator.
//
// Roles.  Warp 0 issues the copies of both operands, warp 1 the MMAs; the other warps hold the totals,
// 32 rows x up to 64 columns each (64 registers of a thread).  Two accumulators of tile_n columns
// alternate, so the MMAs of block kb + 1 run while block kb is scaled and added.  Operands are
// staged as rows of 128 bytes with the 128-byte swizzle, either along the reduction ("K-major") or
// along the rows / columns of C ("MN-major", 8 reduction steps of 128 values per swizzle atom):
// the MMA's descriptor covers both, so gradients read operands as the forward pass stored them.
//
// Few tiles.  A cluster of 2, 4 or 8 CTAs shares a tile's reduction: each leaves its totals in its
// shared memory and takes a part of the tile, adding the CTAs' totals in CTA order.
//
// This kernel serves scales that are fp32 numbers; E8M0 scales go to gemm8_mx.cuh.  Measured: 2048 x
// 4096 x 4096 45 us (1.5 PFLOP/s), bound by reading the products back from tensor memory and the
// multiply-adds; 16 x 4096 x 4096 7.4 us.
// Every wait on a barrier in shared memory is bounded and ends in a status code; TMEM is always freed.
// The waits without a limit are those for tensor memory and, at a cluster's end, for its CTAs: the
// first ends with the CTA before it on the SM (clusters whose CTAs could hold one another up do not
// fit an SM together: cluster_smem_floor), the second when the peers' bounded waits have.
#pragma once
#include "fp8_util.cuh"
#include "gemm8.h"
#include "umma_util.cuh"

namespace maxdnn {

// Where the scale of row (column) i and block kb of an operand is: p[(i >> shift) * step + kb * kstep].
struct Gemm8Scale {
  const void* p;
  int64_t step, kstep;
  int32_t shift;       // 0: one per row; 7: one per 128 rows
  int32_t is_float;    // 0: E8M0 bytes
  int32_t count;       // rows
  int32_t words;       // bytes of four neighbouring rows can be read as a word
};

struct Gemm8Args {
  Gemm8Scale sa, sb;
  void* c;
  int64_t c_row, c_col;        // element steps of the kernel's rows and columns in C
  int32_t M, N;                // the kernel's rows and columns
  int32_t m_tiles, n_tiles, k_blocks;
  int32_t split, stages;
  int32_t a_mn, b_mn;          // 1: MN-major
  int32_t b_stage_bytes;
  int32_t c_type;
  int32_t vec_c;               // columns are contiguous and rows start at multiples of 16 bytes
  uint32_t idesc;
  uint32_t test_missing_arrival;
  WaitCtx wc;
};

__host__ __device__ constexpr int gemm8_cols_per_warp(int nt) { return nt < 64 ? nt : 64; }
__host__ __device__ constexpr int gemm8_epi_warps(int nt) { return 4 * (nt < 64 ? 1 : nt / 64); }
__host__ __device__ constexpr int gemm8_threads(int nt) { return 64 + 32 * gemm8_epi_warps(nt); }

__device__ __forceinline__ void tcgen05_mma_f8(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc,
                                               uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
      "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}

__device__ __forceinline__ void tma_load_2d_hint(uint32_t dst, const CUtensorMap* m, uint32_t bar, int c0,
                                                 int c1, uint64_t policy) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.L2::cache_hint "
      "[%0], [%1, {%3, %4}], [%2], %5;" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(m)), "r"(bar), "r"(c0), "r"(c1), "l"(policy)
      : "memory");
}

__device__ __forceinline__ float4 ld_cluster_f32x4(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
               : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
  return v;
}

__device__ __forceinline__ float gemm8_scale(const Gemm8Scale& s, int i, int kb) {
  const int64_t at = (int64_t)(min(i, s.count - 1) >> s.shift) * s.step + (int64_t)kb * s.kstep;
  return s.is_float ? load_global(static_cast<const float*>(s.p) + at)
                    : e8m0_value(load_global(static_cast<const uint8_t*>(s.p) + at));
}

__device__ __forceinline__ void gemm8_store1(void* c, int c_type, int64_t at, float v) {
  if (c_type == MAXDNN_F32) static_cast<float*>(c)[at] = v;
  else if (c_type == MAXDNN_BF16) static_cast<__nv_bfloat16*>(c)[at] = __float2bfloat16_rn(v);
  else static_cast<__half*>(c)[at] = __float2half_rn(v);
}

// The tile (row tile, column tile) of index t: tiles that run at the same time share operand
// rows and columns (groups of eight row tiles, walked column by column).
__device__ __forceinline__ void gemm8_tile(int m_tiles, int n_tiles, int t, int* mt, int* nt) {
  const int per_group = 8 * n_tiles;
  const int group = t / per_group;
  const int first = group * 8;
  const int height = min(8, m_tiles - first);
  const int in = t - group * per_group;
  *mt = first + in % height;
  *nt = in / height;
}

// The end of a tile that `split` CTAs of a cluster share: CTA `rank` adds the CTAs' totals for its
// part of the tile, in CTA order, and stores them; all CTAs' loads are in flight at once.  The
// totals are at `base` of each CTA's shared memory, laid out so that neighbouring threads store
// neighbouring elements of C: [column][row] where C's rows are neighbours (exchanged roles), else
// [row][column] with rows 16 bytes apart from a power of two.
__host__ __device__ constexpr int gemm8_row_pitch(int nt) { return nt + 4; }        // floats

template <int NT>
__device__ __forceinline__ void gemm8_keep_total(float* mine, bool by_column, int row, int col, float v) {
  mine[by_column ? col * kGemm8TileM + row : row * gemm8_row_pitch(NT) + col] = v;
}

template <int NT, int THREADS, class Args>
__device__ __forceinline__ void gemm8_add_split(const Args& args, uint32_t base, int split, int rank, int unit) {
  const bool by_column = args.c_row == 1;
  const int cols = NT / split, rows = kGemm8TileM / split;      // this CTA's part: columns, or rows
  int mt, nt;
  gemm8_tile(args.m_tiles, args.n_tiles, unit, &mt, &nt);
  for (int e = threadIdx.x; e < kGemm8TileM * NT / 4 / split; e += THREADS) {
    // four neighbours: rows of a column, or columns of a row
    const int row = by_column ? 4 * (e & (kGemm8TileM / 4 - 1)) : rank * rows + e / (NT / 4);
    const int col = by_column ? rank * cols + e / (kGemm8TileM / 4) : 4 * (e % (NT / 4));
    const uint32_t off = base + 4u * (uint32_t)(by_column ? col * kGemm8TileM + row : row * gemm8_row_pitch(NT) + col);
    float4 part[kGemm8MaxSplit];
#pragma unroll
    for (int r = 0; r < kGemm8MaxSplit; ++r)
      if (r < split) part[r] = ld_cluster_f32x4(map_to_cta(off, (uint32_t)r));
    float v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int r = 0; r < kGemm8MaxSplit; ++r)
      if (r < split) {
        v[0] += part[r].x; v[1] += part[r].y; v[2] += part[r].z; v[3] += part[r].w;
      }
    const int m = mt * kGemm8TileM + row, n = nt * NT + col;
    const int64_t at = (int64_t)m * args.c_row + (int64_t)n * args.c_col;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (by_column ? (m + i < args.M && n < args.N) : (m < args.M && n + i < args.N))
        gemm8_store1(args.c, args.c_type, at + i, v[i]);
  }
}

// SBV: the columns have a scale each (else one for 128 of them).
template <int NT, bool SBV>
__global__ void __launch_bounds__(gemm8_threads(NT), 1)
gemm8_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
             const __grid_constant__ Gemm8Args args) {
  constexpr int CW = gemm8_cols_per_warp(NT);
  constexpr int kEpiWarps = gemm8_epi_warps(NT);
  constexpr uint32_t kAStage = kGemm8TileM * kGemm8BlockK;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* base_ptr = smem_raw + (base - smem_u32(smem_raw));
  const int stages = args.stages;
  const uint32_t b_off = (uint32_t)stages * kAStage;
  const uint32_t bar_off = b_off + (uint32_t)stages * (uint32_t)args.b_stage_bytes;
  const uint32_t full_bar = base + bar_off;
  const uint32_t empty_bar = full_bar + 8u * stages;
  const uint32_t accf_bar = empty_bar + 8u * stages;
  const uint32_t acce_bar = accf_bar + 16u;
  const uint32_t done_bar = acce_bar + 16u;
  const uint32_t tmem_slot = done_bar + 8u;
  volatile uint32_t* tmem_slot_ptr = reinterpret_cast<volatile uint32_t*>(base_ptr + bar_off + 16u * stages + 40u);
  // column scales of a block, per warp, two buffers
  float* col_scale = reinterpret_cast<float*>(base_ptr + bar_off + 16u * stages + 64u);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int split = args.split;
  const int rank = split > 1 ? (int)cluster_ctarank() : 0;
  const int unit = (int)blockIdx.x / split, n_units = (int)gridDim.x / split;
  const int n_tiles = args.m_tiles * args.n_tiles;
  const int kb0 = (int)((int64_t)args.k_blocks * rank / split);
  const int kb1 = (int)((int64_t)args.k_blocks * (rank + 1) / split);

  if (threadIdx.x == 0) {
    const uint32_t extra = (args.test_missing_arrival != 0 && blockIdx.x == 0) ? 1u : 0u;   // test hook
    for (int s = 0; s < stages; ++s) {
      mbar_init(full_bar + 8u * s, 1 + extra);
      mbar_init(empty_bar + 8u * s, 1);
    }
    for (int a = 0; a < 2; ++a) {
      mbar_init(accf_bar + 8u * a, 1);
      mbar_init(acce_bar + 8u * a, kEpiWarps);
    }
    mbar_init(done_bar, 1);
    fence_mbar_init();
    fence_proxy_async_smem();
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(tmem_slot),
                 "r"((uint32_t)gemm8_tmem_cols(NT)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tcgen05_fence_before();
  __syncthreads();
  tcgen05_fence_after();
  const uint32_t tmem_base = *tmem_slot_ptr;
  // Only now: a CTA of the next kernel that shares this SM takes its tensor memory after this one has
  // its own (it holds it while it waits for this kernel's end).
  let_next_start();
  wait_for_previous();

  if (warp == 0) {
    // ------------------------------------------------------------ copies
    if (lane == 0) {
      prefetch_tensormap(&map_a);
      prefetch_tensormap(&map_b);
    }
    const uint64_t policy = l2_policy_evict_last();
    const uint32_t tx = kAStage + (uint32_t)args.b_stage_bytes;
    int stage = 0;
    uint32_t phase = 0;
    bool ok = true;
    for (int tile = unit; tile < n_tiles && ok; tile += n_units) {
      int mt, nt;
      gemm8_tile(args.m_tiles, args.n_tiles, tile, &mt, &nt);
      const int m0 = mt * kGemm8TileM, n0 = nt * NT;
      for (int kb = kb0; kb < kb1; ++kb) {
        if (!mbar_wait(empty_bar + 8u * stage, phase ^ 1u, args.wc, kDevTimeoutEmpty)) {
          ok = false;
          break;
        }
        const uint32_t bar = full_bar + 8u * stage;
        const uint32_t a_dst = base + (uint32_t)stage * kAStage;
        const uint32_t b_dst = base + b_off + (uint32_t)stage * (uint32_t)args.b_stage_bytes;
        if (elect_one()) {
          mbar_arrive_expect_tx(bar, tx);
          const int k = kb * kGemm8BlockK;
          if (args.a_mn) tma_load_2d_hint(a_dst, &map_a, bar, m0, k, policy);
          else tma_load_2d_hint(a_dst, &map_a, bar, k, m0, policy);
          if (args.b_mn) {
            for (int b = 0; b < (NT + 127) / 128; ++b)
              tma_load_2d_hint(b_dst + (uint32_t)b * 16384u, &map_b, bar, n0 + 128 * b, k, policy);
          } else {
            tma_load_2d_hint(b_dst, &map_b, bar, k, n0, policy);
          }
        }
        __syncwarp();
        if (++stage == stages) { stage = 0; phase ^= 1u; }
      }
    }
    if (!ok) {
      // leaving early: give copies already issued time to land
      for (int s = 0; s < stages; ++s) mbar_wait_grace(full_bar + 8u * s, s < stage ? phase : (phase ^ 1u));
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------ MMAs
    // K-major: rows of 128 reduction steps, groups of 8 rows 1024 bytes apart, 32 steps = 32 bytes.
    // MN-major: rows of 128 values, 8 steps = 1024 bytes, the next 128 values one box (16 KB) on.
    const uint64_t desc_a = make_smem_desc(0, 16384u, 1024u, 2u);
    const uint64_t desc_b = desc_a;
    const uint64_t step_a = (args.a_mn ? 4096u : 32u) >> 4;
    const uint64_t step_b = (args.b_mn ? 4096u : 32u) >> 4;
    int stage = 0;
    uint32_t phase = 0, block = 0;
    bool ok = true;
    for (int tile = unit; tile < n_tiles && ok; tile += n_units) {
      for (int kb = kb0; kb < kb1; ++kb, ++block) {
        const uint32_t acc = block & 1u;
        if (!mbar_wait(acce_bar + 8u * acc, ((block >> 1) & 1u) ^ 1u, args.wc, kDevTimeoutAccFree) ||
            !mbar_wait(full_bar + 8u * stage, phase, args.wc, kDevTimeoutFull)) {
          ok = false;
          break;
        }
        tcgen05_fence_after();
        const uint32_t d = tmem_base + acc * NT;
        uint64_t a = desc_a | (uint64_t)(((base + (uint32_t)stage * kAStage) & 0x3FFFFu) >> 4);
        uint64_t b = desc_b | (uint64_t)(((base + b_off + (uint32_t)stage * (uint32_t)args.b_stage_bytes) & 0x3FFFFu) >> 4);
        if (elect_one()) {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            tcgen05_mma_f8(d, a, b, args.idesc, j > 0);
            a += step_a;
            b += step_b;
          }
          tcgen05_commit(empty_bar + 8u * stage);
          tcgen05_commit(accf_bar + 8u * acc);
        }
        __syncwarp();
        if (++stage == stages) { stage = 0; phase ^= 1u; }
      }
    }
    // every MMA issued so far has finished before TMEM is released
    if (elect_one()) tcgen05_commit(done_bar);
    mbar_wait(done_bar, 0, args.wc, kDevTimeoutDrain);
  } else {
    // ------------------------------------------------------------ totals
    const int q = warp & 3;                   // TMEM lanes this warp may read
    const int ew = warp - 2;
    const int part = ew >> 2;                 // which CW columns of the tile
    float* my_scale = col_scale + ew * 2 * CW;
    uint32_t block = 0;
    bool ok = true;
    for (int tile = unit; tile < n_tiles && ok; tile += n_units) {
      int mt, nt;
      gemm8_tile(args.m_tiles, args.n_tiles, tile, &mt, &nt);
      const int m = mt * kGemm8TileM + q * 32 + lane;
      const int n0 = nt * NT + part * CW;
      float tot[CW];
#pragma unroll
      for (int i = 0; i < CW; ++i) tot[i] = 0.f;
      float sa = gemm8_scale(args.sa, m, kb0);
      float sb = 1.f, sc0 = 1.f, sc1 = 1.f;
      if constexpr (SBV) {
        sc0 = gemm8_scale(args.sb, n0 + lane % CW, kb0);
        if constexpr (CW == 64) sc1 = gemm8_scale(args.sb, n0 + 32 + lane, kb0);
      } else {
        sb = gemm8_scale(args.sb, n0, kb0);
      }
      for (int kb = kb0; kb < kb1; ++kb, ++block) {
        const uint32_t acc = block & 1u;
        const float s = SBV ? sa : sa * sb;
        float* cs = my_scale + acc * CW;
        if constexpr (SBV) {
          if (lane < CW) cs[lane] = sc0;
          if constexpr (CW == 64) cs[32 + lane] = sc1;
          __syncwarp();
        }
        // the next block's scales are on their way while this one is added
        const int kn = min(kb + 1, kb1 - 1);
        sa = gemm8_scale(args.sa, m, kn);
        if constexpr (SBV) {
          sc0 = gemm8_scale(args.sb, n0 + lane % CW, kn);
          if constexpr (CW == 64) sc1 = gemm8_scale(args.sb, n0 + 32 + lane, kn);
        } else {
          sb = gemm8_scale(args.sb, n0, kn);
        }
        if (!mbar_wait(accf_bar + 8u * acc, (block >> 1) & 1u, args.wc, kDevTimeoutAccum)) {
          ok = false;
          break;
        }
        tcgen05_fence_after();
        const uint32_t t_row = tmem_base + ((uint32_t)(q * 32) << 16) + acc * NT + (uint32_t)(part * CW);
#pragma unroll
        for (int c = 0; c < CW; c += 16) {
          uint32_t v[16];
          tmem_ld_32x16(t_row + (uint32_t)c, v);
          tmem_wait_ld();
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const float d = __uint_as_float(v[i]);
            if constexpr (SBV) tot[c + i] = fmaf(s, d * cs[c + i], tot[c + i]);
            else tot[c + i] = fmaf(s, d, tot[c + i]);
          }
        }
        tcgen05_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(acce_bar + 8u * acc);
      }
      if (!ok) break;
      if (split == 1) {
        if (m < args.M) {
          const int64_t at = (int64_t)m * args.c_row;
          if (args.vec_c && n0 + CW <= args.N) {
#pragma unroll
            for (int c = 0; c < CW; c += 8) {
              float v[8];
#pragma unroll
              for (int i = 0; i < 8; ++i) v[i] = tot[c + i];
              if (args.c_type == MAXDNN_F32) store_float8<MAXDNN_F32, false>(static_cast<float*>(args.c) + at + n0 + c, v, 8);
              else if (args.c_type == MAXDNN_BF16) store_float8<MAXDNN_BF16, false>(static_cast<__nv_bfloat16*>(args.c) + at + n0 + c, v, 8);
              else store_float8<MAXDNN_F16, false>(static_cast<__half*>(args.c) + at + n0 + c, v, 8);
            }
          } else {
#pragma unroll
            for (int i = 0; i < CW; ++i)
              if (n0 + i < args.N) gemm8_store1(args.c, args.c_type, at + (int64_t)(n0 + i) * args.c_col, tot[i]);
          }
        }
      } else {
        // this CTA's totals where the ring was: it is no longer in use (every block that was
        // copied has been multiplied, and every product has been read)
        float* mine = reinterpret_cast<float*>(base_ptr);
#pragma unroll
        for (int i = 0; i < CW; ++i)
          gemm8_keep_total<NT>(mine, args.c_row == 1, q * 32 + lane, part * CW + i, tot[i]);
      }
    }
  }

  tcgen05_fence_before();
  __syncthreads();
  if (split > 1) {
    cluster_arrive();
    cluster_wait();
    gemm8_add_split<NT, gemm8_threads(NT)>(args, base, split, rank, unit);
    cluster_arrive();
    cluster_wait();
  }
  if (warp == 1) {
    tcgen05_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base),
                 "r"((uint32_t)gemm8_tmem_cols(NT)) : "memory");
  }
}

}  // namespace maxdnn
