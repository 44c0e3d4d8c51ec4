// Root-mean-square norm over the last axis with the residual's addition, forward and backward, with the
// packed forms that the 8-bit training step reads next.
//
//   h = x + residual,  rstd = 1 / sqrt(sum h^2 / C + eps),  hh = h rstd,  y = hh g
//   dx = rstd (g dy - hh s) + dsum,  s = sum(g dy hh) / C,  dg = sum over rows of dy hh
//
// A group of WR warps has a row: thread t holds the eight columns at 8 t and the eight at 8 (t + 32 WR), as
// 32-bit values, and the weights of the same columns for all of the group's rows.  Rows come through a ring in
// shared memory: one thread of the group fetches the row `depth` ahead with a bulk copy per input, whatever the
// row's alignment (the copy starts at the 16 bytes that hold the row's first value), so a row's loads cost no
// registers and no issue slots while the row before is packed.  The exchange of the row's one sum is also what
// tells that a stage has been read.  Few rows are read directly: a ring would only add its start.
// Rows that do not start at multiples of 16 bytes are shifted on their way from the stage to registers, and results go back
// into the stage as they will lie in memory, from where a bulk copy stores the row's whole 16-byte units (16-byte vectors in
// pieces of 2 and 4 bytes would be five times the stores; 8192 x 4095 bf16 forward 53.5 -> 47.3 us, backward 65.5 -> 60.7).
// Sums are in 32 bits; sixteen neighbouring lanes hold a block of 128 columns, so packing takes four shuffles
// for two blocks.
//
// Bound by memory for long aligned rows, and by instructions next to it (IPC 0.66 forward, 0.59 backward).  8192 x 4096 bf16 with
// residual: forward to packed y 44.4 us (235 MB, 5.3 TB/s; a copy has 6.56), backward from packed h 45.7 us (235 MB).  One row of
// 4096: 3.3 us, a launch.  1531 x 2309 fp16 backward: 16.7 us, of which 11 are two launches, the rows' latency and the fold.
#pragma once
#include "layer_norm.cuh"
#include "umma_util.cuh"

namespace maxdnn {

struct RmsNormArgs {
  const void *x, *res;         // fprop: x and residual; bprop: h (wide or packed) and dsum
  const uint8_t* x_scale;
  const void* gamma;           // null: 1
  void *sum, *y;               // fprop
  float* rstd;
  uint8_t *q, *s, *c, *sc;     // fprop: packed y, packed h
  const void* dy;              // bprop
  void* dx;
  float* partial;              // [grid][norm_sums_pitch(cols)] sums of a CTA's rows: dy hh
  int64_t ldx, ldr, ldy, ldq;
  int32_t rows, cols, w_type;
  int32_t q_e5m2;
  int32_t depth;               // stages of the ring
  float eps, inv_cols;
  WaitCtx wc;
};

constexpr int kRmsMaxDepth = 4;
__host__ __device__ constexpr int rms_threads(int wr) { return wr > 8 ? 32 * wr : 256; }
__host__ __device__ constexpr int rms_groups(int wr) { return wr > 8 ? 1 : 8 / wr; }
// Bytes of a row in a stage: the 16-byte units that hold it; anywhere: wherever its first value lies in one.
__host__ __device__ constexpr int64_t rms_stage_row(int64_t cols, int bytes, bool anywhere = true) {
  return (cols * bytes + 15) / 16 * 16 + (anywhere ? 16 : 0);
}

__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src),
               "r"(bytes), "r"(bar)
               : "memory");
}

// The 16 bytes that start `s` bytes (a multiple of 2, the same for a whole row) into 32.
__device__ __forceinline__ uint4 shifted16(uint4 lo, uint4 hi, uint32_t s) {
  if (s == 0) return lo;
  return words_at(lo, hi, s);
}

// One input of a ring stage: the units around `cols` values at `row`.  Rows that start at units are told apart when the kernel is
// built: one lane does this for each row and input, which a narrow row's other instructions do not hide (65536 x 256 bf16 backward
// 30.7 us with the general form, 28.5 so; 20000 x 1000 13.9 and 13.5 forward).
struct RmsRow {
  const void* from;
  uint32_t bytes, shift;
};
template <bool EDGE>
__device__ __forceinline__ RmsRow rms_row(const void* base, int64_t first, int cols, int elem) {
  const uintptr_t at = reinterpret_cast<uintptr_t>(base) + (uintptr_t)(first * elem);
  RmsRow r;
  if (!EDGE) {
    r.shift = 0;
    r.from = reinterpret_cast<const void*>(at);
    r.bytes = ((uint32_t)cols * (uint32_t)elem + 15u) & ~15u;
    return r;
  }
  r.shift = (uint32_t)(at & 15u);
  r.from = reinterpret_cast<const void*>(at - r.shift);
  r.bytes = (r.shift + (uint32_t)cols * (uint32_t)elem + 15u) & ~15u;
  return r;
}

// Eight values of a row in a stage: `at` is the first one's place.  Whole vectors without the masks that a row's end needs.
template <int DT, bool EDGE>
__device__ __forceinline__ Raw8<DT> stage_raw8(const uint8_t* at, int n) {
  typedef typename ElemOf<DT>::T T;
  if constexpr (EDGE && !is_fp8(DT)) {
    if (n == 8) {
      const uint32_t s = (uint32_t)(reinterpret_cast<uintptr_t>(at) & 15u);
      const uint4* q = reinterpret_cast<const uint4*>(at - s);
      Raw8<DT> r = {};
      const uint4 c0 = q[0], c1 = q[1];
      r.a = shifted16(c0, c1, s);
      if constexpr (DT == MAXDNN_F32) r.b = shifted16(c1, s ? q[2] : c1, s);
      return r;
    }
  }
  return load_raw8<DT, EDGE>(reinterpret_cast<const T*>(at), n);
}

// A row that the group's threads have written into a stage as it will lie in memory (`shift` bytes into the units at `from`, all
// of them behind a fence and a barrier): whole units by one bulk copy, which thread 0 has to wait for, and single values in
// front and behind (up to seven each) by the group's first threads.  A row without a whole unit, which may lie in two: up to 14
// values, all of them single.
template <class T>
__device__ __forceinline__ void store_staged(T* row, const uint8_t* from, uint32_t shift, int cols, int t) {
  const uint32_t end = shift + (uint32_t)cols * (uint32_t)sizeof(T), u0 = (shift + 15u) & ~15u, u1 = end & ~15u;
  uint8_t* to = reinterpret_cast<uint8_t*>(row) - shift;
  const bool whole = u1 > u0;
  if (t == 0 && whole) {
    asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(to + u0), "r"(smem_u32(from) + u0), "r"(u1 - u0)
                 : "memory");
  }
  const bool front = !whole || t < 8;
  const uint32_t at = front ? shift + t * (uint32_t)sizeof(T) : u1 + (t - 8) * (uint32_t)sizeof(T);
  if (t < 16 && at < (whole && front ? u0 : end)) *reinterpret_cast<T*>(to + at) = *reinterpret_cast<const T*>(from + at);
}

// Sum over the WR warps of a row's group.
template <int WR>
__device__ __forceinline__ float rms_total(float v, float (&slots)[2][WR], int flip, int group, int lane, int in_row) {
  v = warp_sum(v);
  if constexpr (WR > 1) {
    if (lane == 0) slots[flip][in_row] = v;
    asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "n"(WR * 32) : "memory");
    v = 0.f;
#pragma unroll
    for (int w = 0; w < WR; ++w) v += slots[flip][w];
  } else {
    __syncwarp();
  }
  return v;
}

// All threads of a row's group, and what they wrote for the copy engine.
template <int WR>
__device__ __forceinline__ void rms_group_barrier(int group) {
  fence_proxy_async_smem();
  if constexpr (WR > 1) asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "n"(WR * 32) : "memory");
  else __syncwarp();
}

template <int XT, int WR, bool EDGE, bool RING>
__global__ void __launch_bounds__(rms_threads(WR), WR > 8 ? 1 : 3)
rms_norm_fprop_kernel(const __grid_constant__ RmsNormArgs args) {
  typedef typename ElemOf<XT>::T T;
  constexpr int kGroups = rms_groups(WR), kStep = 256 * WR;      // columns from a thread's first vector to its second
  constexpr bool kStaged = EDGE && RING;
  __shared__ float slots[kGroups][2][WR];
  __shared__ __align__(8) uint64_t full[kGroups][kRmsMaxDepth];
  extern __shared__ __align__(16) uint8_t ring[];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int group = warp / WR, in_row = warp % WR, t = in_row * 32 + lane;
  const uint32_t bars = smem_u32(full[group]);
  if (RING && t == 0) {
    for (int i = 0; i < kRmsMaxDepth; ++i) mbar_init(bars + 8u * i, 1);
    fence_mbar_init();
    fence_proxy_async_smem();
  }
  if (RING) __syncthreads();
  let_next_start();
  wait_for_previous();
  const T* x = static_cast<const T*>(args.x);
  const T* res = static_cast<const T*>(args.res);
  const int64_t step = (int64_t)gridDim.x * kGroups, first = (int64_t)blockIdx.x * kGroups + group;
  const uint32_t part = (uint32_t)rms_stage_row(args.cols, sizeof(T), EDGE), stage = res ? 2 * part : part;
  uint8_t* mine = ring + (size_t)group * args.depth * stage;
  auto fetch = [&](int64_t r, int slot) {       // (one thread of the group)
    if (r >= args.rows) return;
    const RmsRow a = rms_row<EDGE>(x, r * args.ldx, args.cols, sizeof(T));
    const RmsRow b = rms_row<EDGE>(res, r * args.ldr, args.cols, sizeof(T));
    mbar_arrive_expect_tx(bars + 8u * slot, a.bytes + (res ? b.bytes : 0u));
    const uint32_t dst = smem_u32(mine) + (uint32_t)slot * stage;
    bulk_load(dst, a.from, a.bytes, bars + 8u * slot);
    if (res) bulk_load(dst + part, b.from, b.bytes, bars + 8u * slot);
  };
  if (RING && t == 0)
    for (int d = 0; d < args.depth; ++d) fetch(first + d * step, d);
  // whole warps without a second vector leave its work out, where that work is long or a row has many warps (elsewhere the
  // test costs more: 4096 x 8192 packed 38 -> 41 us)
  const bool second = !(EDGE || WR > 16) || 256 * in_row + kStep < args.cols;
  int n[2];
  F2 g[2][4];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int c = 8 * t + kStep * j;
    n[j] = vector_cols<EDGE>(args.cols, c);
    load_weights8<EDGE>(args.gamma, c, n[j], args.w_type, 1.f, g[j]);
  }
  int slot = 0, flip = 0;
  uint32_t phase = 0;
  bool ok = true;
  for (int64_t r = first; r < args.rows; r += step, flip ^= 1) {
    Raw8<XT> rx[2], rr[2];
    uint8_t* at_x = mine + (size_t)slot * stage;
    const uint32_t sr = (uint32_t)((uintptr_t)(r * args.ldr) * sizeof(T)) & 15u;
    if constexpr (RING) {
      // (a wait that ran out ends the launch's other waits too; its rows are then not valid)
      ok &= mbar_wait(bars + 8u * slot, phase, args.wc, kDevTimeoutFull);
      const uint32_t sx = (uint32_t)((uintptr_t)(r * args.ldx) * sizeof(T)) & 15u;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        if (j == 1 && !second) break;
        const uint32_t in = (uint32_t)(8 * t + kStep * j) * (uint32_t)sizeof(T);
        rx[j] = stage_raw8<XT, EDGE>(at_x + (EDGE ? sx : 0u) + in, n[j]);
        if (res) rr[j] = stage_raw8<XT, EDGE>(at_x + part + (EDGE ? sr : 0u) + in, n[j]);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        rx[j] = load_raw8<XT, EDGE>(x + r * args.ldx + 8 * t + kStep * j, n[j]);
        if (res) rr[j] = load_raw8<XT, EDGE>(res + r * args.ldr + 8 * t + kStep * j, n[j]);
      }
    }
    F2 h[2][4] = {}, sq = 0;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      if (j == 1 && !second) break;
      to_pairs<XT>(rx[j], h[j]);
      if (res) {
        F2 b[4];
        to_pairs<XT>(rr[j], b);
#pragma unroll
        for (int i = 0; i < 4; ++i) h[j][i] = add2(h[j][i], b[i]);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) sq = fma2(h[j][i], h[j][i], sq);
    }
    const float rstd = 1.f / sqrtf(rms_total<WR>(sum2(sq), slots[group], flip, group, lane, in_row) * args.inv_cols + args.eps);
    // every thread of the group has read this stage: the sum above needed its values
    if (RING && !kStaged) {
      if (t == 0) fetch(r + args.depth * step, slot);
      if (++slot == args.depth) { slot = 0; phase ^= 1u; }
    }
    if (t == 0 && args.rstd) args.rstd[r] = rstd;
    if (args.sum) {
      // (where there is a residual, its place in the stage is the sum's)
      T* to = kStaged && res ? reinterpret_cast<T*>(at_x + part + sr) : static_cast<T*>(args.sum) + r * args.ldr;
#pragma unroll
      for (int j = 0; j < 2; ++j)
        if (j == 0 || second) store_pairs<XT, EDGE>(to + 8 * t + kStep * j, h[j], n[j]);
    }
    const uint32_t sy = (uint32_t)((uintptr_t)(r * args.ldy) * sizeof(T)) & 15u;
    const int64_t at = r * args.ldq + 8 * t, scale_at = (int64_t)(t >> 4) * args.rows + r, scale_step = (int64_t)(kStep / kBlock8) * args.rows;
    if (args.c)
      norm_pack<kEitherFp8, EDGE>(h[0], h[1], args.q_e5m2, args.c + at, args.c + at + kStep, args.sc + scale_at, args.sc + scale_at + scale_step,
                                  n[0], n[1], lane);
    if (!kStaged && !args.y && !args.q) continue;
    if (!kStaged || args.y || args.q) {
      const F2 rs = f2(rstd);
      T* to = kStaged ? reinterpret_cast<T*>(at_x + sy) : static_cast<T*>(args.y) + r * args.ldy;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        if (j == 1 && !second) break;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          h[j][i] = mul2(mul2(h[j][i], rs), g[j][i]);
          // columns past the end take part in the block's maximum: zeros (0 x infinity is none)
          if (EDGE) {
            const float2 u = unf2(h[j][i]);
            h[j][i] = f2(2 * i < n[j] ? u.x : 0.f, 2 * i + 1 < n[j] ? u.y : 0.f);
          } else if (n[j] == 0) {
            h[j][i] = 0;
          }
        }
        if (args.y) store_pairs<XT, EDGE>(to + 8 * t + kStep * j, h[j], n[j]);
      }
      if (args.q)
        norm_pack<kEitherFp8, EDGE>(h[0], h[1], args.q_e5m2, args.q + at, args.q + at + kStep, args.s + scale_at, args.s + scale_at + scale_step,
                                    n[0], n[1], lane);
    }
    if constexpr (kStaged) {
      rms_group_barrier<WR>(group);
      if (args.sum && res) store_staged(static_cast<T*>(args.sum) + r * args.ldr, at_x + part, sr, args.cols, t);
      if (args.y) store_staged(static_cast<T*>(args.y) + r * args.ldy, at_x, sy, args.cols, t);
      if (t == 0) {
        // this row's copies may still be read; the row's before have been: its stage takes the next row
        bulk_commit();
        bulk_wait_read<1>();
        if (r > first) fetch(r - step + args.depth * step, slot == 0 ? args.depth - 1 : slot - 1);
      }
      if (++slot == args.depth) { slot = 0; phase ^= 1u; }
    }
  }
  if (kStaged && t == 0) bulk_wait_all();
  if (RING && !ok && t == 0)      // leaving early: give copies already issued time to land
    for (int i = 0; i < args.depth; ++i) mbar_wait_grace(bars + 8u * i, i < slot ? phase ^ 1u : phase);
}

// Rows too long for the registers of a CTA: read once for the sum, and again (from the second-level cache) for
// the results.  `sum` is written in the second reading, so that it may be the residual's own memory.
template <int XT>
__global__ void __launch_bounds__(1024) rms_norm_fprop_long_kernel(const __grid_constant__ RmsNormArgs args) {
  let_next_start();
  wait_for_previous();
  typedef typename ElemOf<XT>::T T;
  __shared__ float slots[2][kNormMaxWarps];
  const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
  const int steps = (int)(((int64_t)args.cols + 8191) / 8192);
  const T* x = static_cast<const T*>(args.x);
  const T* res = static_cast<const T*>(args.res);
  int flip = 0;
  for (int64_t r = blockIdx.x; r < args.rows; r += gridDim.x, flip ^= 1) {
    float acc = 0.f, rstd = 0.f;
    for (int pass = 0; pass < 2; ++pass) {
      for (int i = 0; i < steps; ++i) {
        const int c = 8 * t + 8192 * i;
        const int n = min(max(args.cols - c, 0), 8);
        F2 h[4], none[4] = {};
        to_pairs<XT>(load_raw8<XT, true>(x + r * args.ldx + c, n), h);
        if (res) {
          F2 b[4];
          to_pairs<XT>(load_raw8<XT, true>(res + r * args.ldr + c, n), b);
#pragma unroll
          for (int k = 0; k < 4; ++k) h[k] = add2(h[k], b[k]);
        }
        if (pass == 0) {
          F2 sq = 0;
#pragma unroll
          for (int k = 0; k < 4; ++k) sq = fma2(h[k], h[k], sq);
          acc += sum2(sq);
          continue;
        }
        if (args.sum) store_pairs<XT, true>(static_cast<T*>(args.sum) + r * args.ldr + c, h, n);
        const int64_t scale_at = (int64_t)(c >> 7) * args.rows + r;
        if (args.c)
          norm_pack<kEitherFp8, true>(h, none, args.q_e5m2, args.c + r * args.ldq + c, nullptr, args.sc + scale_at, nullptr, n, 0, lane);
        if (!args.y && !args.q) continue;
        F2 g[4];
        load_weights8<true>(args.gamma, c, n, args.w_type, 1.f, g);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float2 u = unf2(mul2(mul2(h[k], f2(rstd)), g[k]));
          h[k] = f2(2 * k < n ? u.x : 0.f, 2 * k + 1 < n ? u.y : 0.f);
        }
        if (args.y) store_pairs<XT, true>(static_cast<T*>(args.y) + r * args.ldy + c, h, n);
        if (args.q)
          norm_pack<kEitherFp8, true>(h, none, args.q_e5m2, args.q + r * args.ldq + c, nullptr, args.s + scale_at, nullptr, n, 0, lane);
      }
      if (pass == 1) break;
      rstd = 1.f / sqrtf(cta_sum(acc, slots[flip], lane, warp) * args.inv_cols + args.eps);
    }
    if (t == 0 && args.rstd) args.rstd[r] = rstd;
  }
}

// Backward.  A group has neighbouring rows (so that a packed row's scale bytes, which lie rows apart, come from
// the first-level cache); its threads keep dg of their columns for all of them.  With 32 warps to a row there are
// 64 registers to a thread: the row is then read from the stage again for dx, and released after that.
template <int XT, int YT, int WR, bool EDGE>
__global__ void __launch_bounds__(rms_threads(WR), WR > 8 ? 1 : 2)
rms_norm_bprop_kernel(const __grid_constant__ RmsNormArgs args) {
  typedef typename ElemOf<XT>::T TX;
  typedef typename ElemOf<YT>::T TY;
  constexpr int kGroups = rms_groups(WR), kStep = 256 * WR;
  constexpr bool kAgain = WR > 16;
  // dx goes through dy's place in the stage (not where dy is read again for it: other threads' shifted vectors overlap it)
  constexpr int kStagedAt = EDGE && !kAgain ? 1 : 0;
  const bool second = !(EDGE || WR > 16) || 256 * (int)((threadIdx.x >> 5) % WR) + kStep < args.cols;      // (see above)
  __shared__ float slots[kGroups][2][WR];
  __shared__ __align__(8) uint64_t full[kGroups][kRmsMaxDepth];
  __shared__ float fold[kGroups > 1 ? 512 * WR : 1];
  extern __shared__ __align__(16) uint8_t ring[];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int group = warp / WR, in_row = warp % WR, t = in_row * 32 + lane;
  const uint32_t bars = smem_u32(full[group]);
  if (t == 0) {
    for (int i = 0; i < kRmsMaxDepth; ++i) mbar_init(bars + 8u * i, 1);
    fence_mbar_init();
    fence_proxy_async_smem();
  }
  __syncthreads();
  let_next_start();
  wait_for_previous();
  const TX* x = static_cast<const TX*>(args.x);
  const TY* dy = static_cast<const TY*>(args.dy);
  const TY* ds = static_cast<const TY*>(args.res);
  const int64_t groups = (int64_t)gridDim.x * kGroups, me = (int64_t)blockIdx.x * kGroups + group;
  const int64_t r0 = args.rows * me / groups, r1 = args.rows * (me + 1) / groups;
  const uint32_t part_x = (uint32_t)rms_stage_row(args.cols, sizeof(TX)), part_y = (uint32_t)rms_stage_row(args.cols, sizeof(TY));
  const uint32_t stage = part_x + (ds ? 2 : 1) * part_y;
  uint8_t* mine = ring + (size_t)group * args.depth * stage;
  auto fetch = [&](int64_t r, int slot) {
    if (r >= r1) return;
    const RmsRow a = rms_row<EDGE>(x, r * args.ldx, args.cols, sizeof(TX));
    const RmsRow b = rms_row<EDGE>(dy, r * args.ldy, args.cols, sizeof(TY));
    const RmsRow d = rms_row<EDGE>(ds, r * args.ldr, args.cols, sizeof(TY));
    mbar_arrive_expect_tx(bars + 8u * slot, a.bytes + b.bytes + (ds ? d.bytes : 0u));
    const uint32_t dst = smem_u32(mine) + (uint32_t)slot * stage;
    bulk_load(dst, a.from, a.bytes, bars + 8u * slot);
    bulk_load(dst + part_x, b.from, b.bytes, bars + 8u * slot);
    if (ds) bulk_load(dst + part_x + part_y, d.from, d.bytes, bars + 8u * slot);
  };
  if (t == 0)
    for (int d = 0; d < args.depth; ++d) fetch(r0 + d, d);
  int n[2];
  F2 g[2][4], dg[2][4];
  const uint8_t* scales[2];
  float rstd_next = r0 < r1 ? args.rstd[r0] : 0.f;
  uint32_t byte_next[2] = {0, 0};
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int c = 8 * t + kStep * j;
    n[j] = vector_cols<EDGE>(args.cols, c);
    load_weights8<EDGE>(args.gamma, c, n[j], args.w_type, 1.f, g[j]);
#pragma unroll
    for (int i = 0; i < 4; ++i) dg[j][i] = 0;
    scales[j] = args.x_scale + (int64_t)(c >> 7) * args.rows;
    if (is_fp8(XT) && n[j] > 0 && r0 < r1) byte_next[j] = scales[j][r0];
  }
  int slot = 0, flip = 0;
  uint32_t phase = 0;
  bool ok = true;
  for (int64_t r = r0; r < r1; ++r, flip ^= 1) {
    const float rstd = rstd_next;
    F2 k[2];               // what a value of h is multiplied by to give hh
#pragma unroll
    for (int j = 0; j < 2; ++j) k[j] = f2(is_fp8(XT) ? (n[j] > 0 ? e8m0_value(byte_next[j]) : 0.f) : rstd);
    if (r + 1 < r1) {      // the next row's, on their way during this one
      rstd_next = args.rstd[r + 1];
#pragma unroll
      for (int j = 0; j < 2; ++j)
        if (is_fp8(XT) && n[j] > 0) byte_next[j] = scales[j][r + 1];
    }
    ok &= mbar_wait(bars + 8u * slot, phase, args.wc, kDevTimeoutFull);
    const uint8_t* at = mine + (size_t)slot * stage;
    const uint32_t sx = EDGE ? (uint32_t)((uintptr_t)(r * args.ldx) * sizeof(TX)) & 15u : 0u;
    const uint32_t sy = EDGE ? (uint32_t)((uintptr_t)(r * args.ldy) * sizeof(TY)) & 15u : 0u;
    const uint32_t sd = EDGE ? (uint32_t)((uintptr_t)(r * args.ldr) * sizeof(TY)) & 15u : 0u;
    // hh and dy of eight columns
    auto values = [&](int j, F2 (&hh)[4], F2 (&e)[4]) {
      const uint32_t in = (uint32_t)(8 * t + kStep * j);
      to_pairs<XT>(stage_raw8<XT, EDGE>(at + sx + in * (uint32_t)sizeof(TX), n[j]), hh);
      to_pairs<YT>(stage_raw8<YT, EDGE>(at + part_x + sy + in * (uint32_t)sizeof(TY), n[j]), e);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        hh[i] = mul2(hh[i], k[j]);
        if (is_fp8(XT)) hh[i] = mul2(hh[i], f2(rstd));
      }
    };
    const uint8_t* at_sums = at + part_x + part_y + sd;
    F2 hh[2][4], e[2][4], part = 0;
    Raw8<YT> rd[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      if (j == 1 && !second) break;
      values(j, hh[j], e[j]);
      if (!kAgain && ds) rd[j] = stage_raw8<YT, EDGE>(at_sums + (uint32_t)(8 * t + kStep * j) * (uint32_t)sizeof(TY), n[j]);
      if (n[j] > 0) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          dg[j][i] = fma2(e[j][i], hh[j][i], dg[j][i]);
          e[j][i] = mul2(e[j][i], g[j][i]);
          part = fma2(e[j][i], hh[j][i], part);
        }
      }
    }
    const float s = rms_total<WR>(sum2(part), slots[group], flip, group, lane, in_row) * args.inv_cols;
    if (!EDGE && !kAgain && t == 0) fetch(r + args.depth, slot);
    const F2 rs = f2(rstd), ms = f2(-s * rstd);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      if (j == 1 && !second) break;
      if (kAgain) {
        values(j, hh[j], e[j]);
        if (ds) rd[j] = stage_raw8<YT, EDGE>(at_sums + (uint32_t)(8 * t + kStep * j) * (uint32_t)sizeof(TY), n[j]);
#pragma unroll
        for (int i = 0; i < 4; ++i) e[j][i] = mul2(e[j][i], g[j][i]);
      }
      F2 o[4];
      if (ds) {
        to_pairs<YT>(rd[j], o);
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = add2(fma2(hh[j][i], ms, mul2(e[j][i], rs)), o[i]);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = fma2(hh[j][i], ms, mul2(e[j][i], rs));
      }
      if (kStagedAt == 0) store_pairs<YT, EDGE>(static_cast<TY*>(args.dx) + r * args.ldy + 8 * t + kStep * j, o, n[j]);
      else store_pairs<YT, EDGE>(reinterpret_cast<TY*>(mine + (size_t)slot * stage + part_x + sy) + 8 * t + kStep * j, o, n[j]);
    }
    if (kStagedAt != 0) {
      rms_group_barrier<WR>(group);
      store_staged(static_cast<TY*>(args.dx) + r * args.ldy, at + part_x, sy, args.cols, t);
      if (t == 0) {
        // this row's copy may still be read; the row's before has been: its stage takes the next row
        bulk_commit();
        bulk_wait_read<1>();
        if (r > r0) fetch(r - 1 + args.depth, slot == 0 ? args.depth - 1 : slot - 1);
      }
    } else if (EDGE || kAgain) {
      if (WR > 1) asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "n"(WR * 32) : "memory");
      else __syncwarp();
      if (t == 0) fetch(r + args.depth, slot);
    }
    if (++slot == args.depth) { slot = 0; phase ^= 1u; }
  }
  if (kStagedAt != 0 && t == 0) bulk_wait_all();
  if (!ok && t == 0)
    for (int i = 0; i < args.depth; ++i) mbar_wait_grace(bars + 8u * i, i < slot ? phase ^ 1u : phase);
  if (!args.partial) return;
  float* out = args.partial + (int64_t)blockIdx.x * norm_sums_pitch(args.cols);
  // the CTA's sum over its groups, in their order
  if constexpr (kGroups > 1) {
    for (int w = 0; w < kGroups; ++w) {
      if (group == w) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          float a[8];
          to_floats(dg[j], a);
#pragma unroll
          for (int i = 0; i < 8; ++i) {      // place i of vector (t, j)
            float& f = fold[(8 * j + i) * 32 * WR + t];
            f = w == 0 ? a[i] : f + a[i];
          }
        }
      }
      __syncthreads();
    }
    for (int c = threadIdx.x; c < args.cols; c += rms_threads(WR)) {
      const int j = c / kStep, in = c - kStep * j;
      out[c] = fold[(8 * j + (in & 7)) * 32 * WR + (in >> 3)];
    }
  } else {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int c = 8 * t + kStep * j;
      float a[8];
      to_floats(dg[j], a);
      if (c < args.cols) store_sums8(out + c, a);
    }
  }
}

// Long rows backward: the row's sum, then dx from a second reading; dg goes to the CTA's sums in memory (this CTA
// alone writes them, each thread always the same columns).
template <int XT, int YT>
__global__ void __launch_bounds__(1024) rms_norm_bprop_long_kernel(const __grid_constant__ RmsNormArgs args) {
  let_next_start();
  wait_for_previous();
  typedef typename ElemOf<XT>::T TX;
  typedef typename ElemOf<YT>::T TY;
  __shared__ float slots[2][kNormMaxWarps];
  const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
  const int steps = (int)(((int64_t)args.cols + 8191) / 8192);
  float* out = args.partial ? args.partial + (int64_t)blockIdx.x * norm_sums_pitch(args.cols) : nullptr;
  bool first = true;
  int flip = 0;
  for (int64_t r = blockIdx.x; r < args.rows; r += gridDim.x, flip ^= 1) {
    const float rstd = args.rstd[r];
    float s = 0.f;
    for (int pass = 0; pass < 2; ++pass) {
      for (int i = 0; i < steps; ++i) {
        const int c = 8 * t + 8192 * i;
        const int n = min(max(args.cols - c, 0), 8);
        F2 hh[4], e[4], g[4];
        to_pairs<XT>(load_raw8<XT, true>(static_cast<const TX*>(args.x) + r * args.ldx + c, n), hh);
        to_pairs<YT>(load_raw8<YT, true>(static_cast<const TY*>(args.dy) + r * args.ldy + c, n), e);
        load_weights8<true>(args.gamma, c, n, args.w_type, 1.f, g);
        float scale = 1.f;
        if (is_fp8(XT)) scale = n > 0 ? e8m0_value(args.x_scale[(int64_t)(c >> 7) * args.rows + r]) : 0.f;
        float pg[8] = {};
        const bool add = pass == 0 && out && n > 0;
        if (add && !first) load_sums8(out + c, pg);
        F2 part = 0, o[4] = {};
        if (pass == 1 && args.res) to_pairs<YT>(load_raw8<YT, true>(static_cast<const TY*>(args.res) + r * args.ldr + c, n), o);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          if (is_fp8(XT)) hh[k] = mul2(hh[k], f2(scale));
          hh[k] = mul2(hh[k], f2(rstd));
          const float2 u = unf2(mul2(e[k], hh[k]));
          pg[2 * k] += u.x;
          pg[2 * k + 1] += u.y;
          e[k] = mul2(e[k], g[k]);
          part = fma2(e[k], hh[k], part);
          o[k] = add2(fma2(hh[k], f2(-s * rstd), mul2(e[k], f2(rstd))), o[k]);
        }
        if (add) store_sums8(out + c, pg);
        if (pass == 0 && n > 0) s += sum2(part);
        if (pass == 1) store_pairs<YT, true>(static_cast<TY*>(args.dx) + r * args.ldy + c, o, n);
      }
      if (pass == 0) s = cta_sum(s, slots[flip], lane, warp) * args.inv_cols;
    }
    first = false;
  }
}

// dg from the CTAs' sums, in CTA order.  A CTA takes 32 columns; each of its 16 warps takes every sixteenth sum, four at a
// time, and the warps' results are added in warp order.  (Eight at a time behind tests of the end: 3 us more; 32 warps: 1 us more.)
__global__ void __launch_bounds__(512) rms_norm_fold_kernel(const float* partial, int parts, int cols, float* dgamma) {
  let_next_start();
  wait_for_previous();
  __shared__ float part[16][33];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t c = (int64_t)blockIdx.x * 32 + lane, pitch = norm_sums_pitch(cols);
  float s[4] = {0.f, 0.f, 0.f, 0.f};
  if (c < cols) {
    const float* at = partial + c;
    int p = warp;
    for (; p + 48 < parts; p += 64) {
#pragma unroll
      for (int i = 0; i < 4; ++i) s[i] += at[(int64_t)(p + 16 * i) * pitch];
    }
    for (; p < parts; p += 16) s[0] += at[(int64_t)p * pitch];
  }
  part[warp][lane] = (s[0] + s[1]) + (s[2] + s[3]);
  __syncthreads();
  if (warp != 0 || c >= cols) return;
  float total = 0.f;
#pragma unroll
  for (int w = 0; w < 16; ++w) total += part[w][lane];
  dgamma[c] = total;
}

}  // namespace maxdnn
