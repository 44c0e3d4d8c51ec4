// The orthogonalised update of matrices whose shorter side is at most 128 (see ortho.cuh for the formula and for what is
// kept in how many bits): a cluster has a matrix from its first reading to its result, and nothing goes through memory between.
//
// X is cut along its longer side, 256 rows or columns to a CTA: its entries stay in 32 bits in tensor memory, next to where the
// product that is added to them arrives, and their FP16 part lies in shared memory as the tensor core reads it.  One image serves both
// products that read X: rows of 128 bytes (64 entries along a row of X) are "K-major" where the reduction runs along X's rows and
// "MN-major" where it runs across them.  A step:
//
//   the CTA's part of X X^T                       MMA, 256 reduction steps
//   summed over the cluster's CTAs                each takes a share of the entries, from all CTAs' shared memory in their order,
//                                                 and writes it as FP16 into every CTA's copy of A
//   B = b A + c A A                               MMA, every CTA for itself
//   X' = a X + B X                                MMA
//
// With one launch and two cluster barriers a step instead of three products through memory with a wait for all CTAs after each
// (about 4 us apiece), 16 x 512 x 128 takes 48 us instead of 84, 128 x 128 30 instead of 69, 128 x 4096 65.  What bounds it is the step's
// chain of latencies: MMAs, reading tensor memory, the exchange of partial sums (4 us a step between two CTAs), two barriers.
// Where a device cannot place a matrix's cluster, the matrix goes through memory (ortho_api.cu).
// All waits on barriers in shared memory are bounded; a wait that runs out leaves the launch's results invalid and its status says so.
#pragma once
#include "ortho.cuh"

namespace maxdnn {

constexpr int kSmallN = 128;             // the shorter side, padded with zeros
constexpr int kSmallSlice = 256;         // of the longer side, to a CTA
constexpr int kSmallMaxCluster = 16;
constexpr int kSmallThreads = 512;
constexpr int kSmallPitch = kSmallN + 4; // floats of a row of partial sums (16 bytes off a power of two)
constexpr int kSmallImage = kSmallN * kSmallSlice * 2, kSmallSquare = kSmallN * kSmallN * 2;
constexpr int kSmallPartial = kSmallN * kSmallPitch * 4;
constexpr int kSmallTmem = 2 * kSmallSlice;      // columns: products, X
constexpr int kSmallSmem = 1024 + kSmallImage + 2 * kSmallSquare + kSmallPartial;
static_assert(2 * kSmallSquare + kSmallPartial >= 2 * kSmallImage, "a slice of X in 32 bits fits behind the image");

struct OrthoSmallArgs {
  const void* x;
  __nv_bfloat16* out;
  int64_t ldx, ldo, stride_x, stride_o;
  int32_t rows, cols, steps;
  float eps;
  float coefficients[kOrthoMaxSteps][3];
  uint32_t test_missing_arrival;
  WaitCtx wc;
};

__device__ __forceinline__ void st_cluster_u32x4(uint32_t addr, const uint32_t (&w)[4]) {
  asm volatile("st.shared::cluster.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]) : "memory");
}
__device__ __forceinline__ void st_cluster_f32(uint32_t addr, float v) {
  asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(addr), "f"(v) : "memory");
}
__device__ __forceinline__ float4 ld_cluster_float4(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ double ld_cluster_f64(uint32_t addr) {
  double v;
  asm volatile("ld.shared::cluster.f64 %0, [%1];" : "=d"(v) : "r"(addr) : "memory");
  return v;
}

__device__ __forceinline__ void tmem_st_32x32(uint32_t taddr, const float (&v)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
      "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};" ::"r"(taddr),
      "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]), "f"(v[8]), "f"(v[9]), "f"(v[10]),
      "f"(v[11]), "f"(v[12]), "f"(v[13]), "f"(v[14]), "f"(v[15]), "f"(v[16]), "f"(v[17]), "f"(v[18]), "f"(v[19]), "f"(v[20]),
      "f"(v[21]), "f"(v[22]), "f"(v[23]), "f"(v[24]), "f"(v[25]), "f"(v[26]), "f"(v[27]), "f"(v[28]), "f"(v[29]), "f"(v[30]), "f"(v[31])
      : "memory");
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Where eight entries (16 bytes) of an image lie: `row` of `rows`, columns 8 chunk.  Columns of 64 entries one after the other,
// rows of 128 bytes in each, 16-byte units exchanged as the 128-byte swizzle wants.
__device__ __forceinline__ uint32_t image_at(int rows, int row, int chunk) {
  return (uint32_t)((chunk >> 3) * rows * 128 + row * 128 + (((chunk & 7) ^ (row & 7)) << 4));
}

// TALL: rows > cols; the image's rows are X's rows either way.
template <int XT, bool TALL, bool EDGE>
__global__ void __launch_bounds__(kSmallThreads, 1) ortho_small_kernel(const __grid_constant__ OrthoSmallArgs args) {
  typedef typename ElemOf<XT>::T T;
  constexpr int kRows = TALL ? kSmallSlice : kSmallN;        // of the image
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t bar_mem[2];      // a product's end; after a wait that ran out: the end of all of them
  __shared__ uint32_t tmem_mem;
  __shared__ double norm_part, norm_factor;
  __shared__ double warp_part[kSmallThreads / 32];
  __shared__ __align__(16) float r_a[kSmallN], d_b[kSmallN], h_b[kSmallN];      // diagonals: what FP16 left of A's, B's, what of it FP16 holds
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* image = smem_raw + (base - smem_u32(smem_raw));
  uint8_t* square_a = image + kSmallImage;
  uint8_t* square_b = square_a + kSmallSquare;
  float* partial = reinterpret_cast<float*>(square_b + kSmallSquare);
  const uint32_t u_image = base, u_a = base + kSmallImage, u_b = u_a + kSmallSquare, u_partial = u_b + kSmallSquare;
  const uint32_t bar = smem_u32(bar_mem);
  const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
  const int q = warp & 3, group = warp >> 2;       // TMEM lanes; which quarter of the columns (TALL: tile of 128 rows and half)
  const int row = q * 32 + lane + (TALL ? 128 * (group >> 1) : 0);      // of the image
  const int rank = (int)cluster_ctarank();
  uint32_t parts;
  asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(parts));
  const int64_t matrix = blockIdx.x / parts;
  if (t == 0) {
    mbar_init(bar, 1 + (args.test_missing_arrival != 0 && blockIdx.x == 0 ? 1 : 0));      // (test hook)
    mbar_init(bar + 8u, 1);
    fence_mbar_init();
    fence_proxy_async_smem();
  }
  if (warp == 0) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_mem)), "r"((uint32_t)kSmallTmem) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tcgen05_fence_before();
  __syncthreads();
  tcgen05_fence_after();
  const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(&tmem_mem);
  let_next_start();
  wait_for_previous();

  // ---- G: a warp to a row (TALL: to two), kept as it lies until the norm is known
  constexpr int kPer = TALL ? 2 : 1;               // rows that a warp reads at once (16 lanes each where TALL)
  constexpr int kHeld = kRows / (kSmallThreads / 32) / kPer;
  const int first = rank * kSmallSlice;            // of the longer side
  const int rows_here = TALL ? min(max(args.rows - first, 0), kSmallSlice) : args.rows;
  const int cols_here = TALL ? args.cols : min(max(args.cols - first, 0), kSmallSlice);
  const int c_read = 8 * (TALL ? lane & 15 : lane);
  const int n_read = vector_cols<EDGE>(cols_here, c_read);
  auto row_read = [&](int i) { return TALL ? (warp * kHeld + i) * 2 + (lane >> 4) : warp * kHeld + i; };
  const T* x = static_cast<const T*>(args.x) + matrix * args.stride_x + (TALL ? first * args.ldx : first);
  {
    Raw8<XT> raw[kHeld];
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
      const int r = row_read(i);
      raw[i] = load_raw8<XT, EDGE>(x + r * args.ldx + c_read, r < rows_here ? n_read : 0);
    }
    // squares relative to the thread's largest entry (a power of two), then joined in 64 bits: they may leave the range of 32
    float most = 0.f;
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
      F2 v[4];
      to_pairs<XT>(raw[i], v);
      most = fmaxf(most, max8(v));
    }
    // (a subnormal one: by 2^127; from 2^127 on by 2^-126, the smallest unit; an infinity stays one)
    const int up = most > 0.f && !isinf(most) ? max(127 - (int)(__float_as_uint(most) >> 23), -126) : 0;
    const F2 unit = f2(__uint_as_float((uint32_t)min(127 + up, 254) << 23));
    F2 squares = 0;
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
      F2 v[4];
      convert_again(raw[i]);
      to_pairs<XT>(raw[i], v);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        v[k] = mul2(v[k], unit);
        squares = fma2(v[k], v[k], squares);
      }
    }
    double sum = ldexp((double)sum2(squares), -2 * min(up, 127));
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, d);
    if (lane == 0) warp_part[warp] = sum;
    __syncthreads();
    if (t == 0) {
      for (int w = 1; w < kSmallThreads / 32; ++w) sum += warp_part[w];
      norm_part = sum;
    }
    cluster_arrive();
    cluster_wait();
    if (t == 0) {
      double total = 0.0;
      for (uint32_t c = 0; c < parts; ++c) total += ld_cluster_f64(map_to_cta(smem_u32(&norm_part), c));
      // (a sum that is no number, or infinite: every entry becomes NaN)
      const double norm = sqrt(total);
      norm_factor = norm < 1e300 ? (double)(1 << kOrthoScaleBits) / (norm + (double)args.eps) : __longlong_as_double(0x7FF8000000000000ll);
    }
    __syncthreads();
    const double factor = norm_factor;
    const float narrow = (float)factor;
    const bool wide = !(narrow > 1e-30f && narrow < 1e30f);
    // through shared memory to the threads that keep the entries: in 32 bits where A, B and the partial sums will be, the first and the
    // last four of each eight laid out as the image.  (Not as two FP16 numbers: they end at 2^-35, where |G| is far below eps)
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
      float v[8];
      to_float8<XT>(raw[i], v);
      uint32_t hi[4];
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = wide ? (float)((double)v[k] * factor) : v[k] * narrow;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const __half2 h = __floats2half2_rn(v[2 * k], v[2 * k + 1]);
        hi[k] = *reinterpret_cast<const uint32_t*>(&h);
      }
      const uint32_t at = image_at(kRows, row_read(i), c_read / 8);
      *reinterpret_cast<uint4*>(image + at) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
      *reinterpret_cast<float4*>(square_a + at) = make_float4(v[0], v[1], v[2], v[3]);
      *reinterpret_cast<float4*>(square_a + kSmallImage + at) = make_float4(v[4], v[5], v[6], v[7]);
    }
  }
  __syncthreads();
  // this thread's 64 entries of its row: to tensor memory
  const int chunk0 = 8 * (TALL ? group & 1 : group);
  const uint32_t t_row = tmem + ((uint32_t)(q * 32) << 16), t_x = t_row + kSmallSlice + 64u * group;
#pragma unroll 1
  for (int u = 0; u < 2; ++u) {
    float v[32];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t at = image_at(kRows, row, chunk0 + 4 * u + i);
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const float4 f = *reinterpret_cast<const float4*>(square_a + k * kSmallImage + at);
        v[8 * i + 4 * k] = f.x; v[8 * i + 4 * k + 1] = f.y; v[8 * i + 4 * k + 2] = f.z; v[8 * i + 4 * k + 3] = f.w;
      }
    }
    tmem_st_32x32(t_x + 32u * u, v);
  }
  tmem_wait_st();

  // ---- products: one thread issues the MMAs when all have written what they read, and all wait for their end
  // (a CTA whose wait ran out goes on with its cluster's barriers, but issues no more)
  uint32_t phase = 0;
  bool ok = true;
  auto product = [&](auto issue) {
    tcgen05_fence_before();
    fence_proxy_async_smem();
    __syncthreads();
    if (warp == 0 && __all_sync(0xFFFFFFFFu, ok)) {
      tcgen05_fence_after();
      if (elect_one()) {
        fence_proxy_async_smem();
        issue();
        tcgen05_commit(bar);
      }
      __syncwarp();
    }
    ok = ok && mbar_wait(bar, phase, args.wc, kDevTimeoutAccum);
    phase ^= 1u;
    tcgen05_fence_after();
  };
  // instruction descriptors: fp32 accumulator, FP16 operands, majors, N / 8, M / 16
  auto idesc = [](int n, bool a_mn, bool b_mn) {
    return (1u << 4) | ((uint32_t)a_mn << 15) | ((uint32_t)b_mn << 16) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(kSmallN >> 4) << 24);
  };
  // start of reduction step j (16 entries) in an image of `rows` rows: along its rows, or across them
  auto along = [](uint32_t at, int rows, int j) { return make_smem_desc(at + (uint32_t)((j >> 2) * rows * 128 + (j & 3) * 32), 16384u, 1024u, 2u); };
  auto across = [](uint32_t at, int rows, int j) { return make_smem_desc(at + (uint32_t)(j * 2048), (uint32_t)rows * 128u, 1024u, 2u); };
  // the warps whose 32 x 32 entries of A and B hold part of the diagonal, and the others
  auto by_diagonal = [&](auto f) {
    if (group == q) f(OrthoKindOf<1>());
    else f(OrthoKindOf<0>());
  };

  for (int step = 0; step < args.steps; ++step) {
    const float ca = args.coefficients[step][0], cb = args.coefficients[step][1], cc = args.coefficients[step][2];
    // ---- A: this CTA's part
    product([&] {
#pragma unroll 1
      for (int j = 0; j < kSmallSlice / 16; ++j) {
        const uint64_t d = TALL ? across(u_image, kRows, j) : along(u_image, kRows, j);
        tcgen05_mma<true>(tmem, d, d, idesc(kSmallN, TALL, TALL), j > 0);
      }
    });
    const float scale = __int_as_float((127 - 2 * kOrthoScaleBits) << 23);
    const int m = q * 32 + lane;                    // this thread's row of A and B, columns from 32 group on
    {
      uint32_t v[32];
      tmem_ld_32x32(t_row + (uint32_t)(32 * group), v);
      tmem_wait_ld();
      if (parts == 1) {
        by_diagonal([&](auto diagonal) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            uint32_t w[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const float2 y = make_float2(__uint_as_float(v[8 * i + 2 * k]) * scale, __uint_as_float(v[8 * i + 2 * k + 1]) * scale);
              const __half2 h = __floats2half2_rn(y.x, y.y);
              w[k] = *reinterpret_cast<const uint32_t*>(&h);
              if (decltype(diagonal)::value && 8 * i + 2 * k == (lane & ~1)) {
                const float2 back = __half22float2(h);
                r_a[m] = lane & 1 ? y.y - back.y : y.x - back.x;
              }
            }
            *reinterpret_cast<uint4*>(square_a + image_at(kSmallN, m, 4 * group + i)) = make_uint4(w[0], w[1], w[2], w[3]);
          }
        });
      } else {
        float* to = partial + m * kSmallPitch + 32 * group;
#pragma unroll
        for (int i = 0; i < 8; ++i)
          *reinterpret_cast<float4*>(to + 4 * i) = make_float4(__uint_as_float(v[4 * i]), __uint_as_float(v[4 * i + 1]),
                                                               __uint_as_float(v[4 * i + 2]), __uint_as_float(v[4 * i + 3]));
      }
    }
    if (parts > 1) {
      cluster_arrive();
      cluster_wait();
      // its share of A's entries, four neighbours at a time and several of those at once: the CTAs' parts in their order
      // (neighbouring lanes join theirs to 16 bytes, which each writes to every other CTA: shares are whole eights)
      const int v0 = (int)(kSmallN * kSmallN / 8 * (uint32_t)rank / parts) * 2, v1 = (int)(kSmallN * kSmallN / 8 * ((uint32_t)rank + 1) / parts) * 2;
      auto share = [&](auto at_once) {
        constexpr int N = decltype(at_once)::value;
        for (int e0 = v0 + t; e0 - lane < v1; e0 += N * kSmallThreads) {      // (whole warps: lanes exchange)
          float4 s[N];
          uint32_t from[N];
#pragma unroll
          for (int k = 0; k < N; ++k) {
            const int e = min(e0 + k * kSmallThreads, v1 - 1);      // (past its share: the last one again, not written)
            from[k] = u_partial + 4u * (uint32_t)((e >> 5) * kSmallPitch + 4 * (e & 31));
            s[k] = ld_cluster_float4(map_to_cta(from[k], 0));
          }
#pragma unroll 2
          for (uint32_t c = 1; c < parts; ++c) {
            float4 p[N];
#pragma unroll
            for (int k = 0; k < N; ++k) p[k] = ld_cluster_float4(map_to_cta(from[k], c));
#pragma unroll
            for (int k = 0; k < N; ++k) {
              s[k].x += p[k].x; s[k].y += p[k].y; s[k].z += p[k].z; s[k].w += p[k].w;
            }
          }
#pragma unroll
          for (int k = 0; k < N; ++k) {
            const int e = e0 + k * kSmallThreads, em = e >> 5, en = 4 * (e & 31);
            const float x0 = s[k].x * scale, x1 = s[k].y * scale, x2 = s[k].z * scale, x3 = s[k].w * scale;
            const __half2 a = __floats2half2_rn(x0, x1), b = __floats2half2_rn(x2, x3);
            const uint32_t wa = *reinterpret_cast<const uint32_t*>(&a), wb = *reinterpret_cast<const uint32_t*>(&b);
            const uint32_t oa = __shfl_xor_sync(0xFFFFFFFFu, wa, 1), ob = __shfl_xor_sync(0xFFFFFFFFu, wb, 1);
            if (e >= v1) continue;
            const uint32_t to = u_a + image_at(kSmallN, em, en >> 3);
            const uint32_t w[4] = {lane & 1 ? oa : wa, lane & 1 ? ob : wb, lane & 1 ? wa : oa, lane & 1 ? wb : ob};
            for (uint32_t c = lane & 1; c < parts; c += 2) st_cluster_u32x4(map_to_cta(to, c), w);
            if ((em & ~3) == en) {
              const float2 fa = __half22float2(a), fb = __half22float2(b);
              const float rest = em == en ? x0 - fa.x : em == en + 1 ? x1 - fa.y : em == en + 2 ? x2 - fb.x : x3 - fb.y;
              for (uint32_t c = 0; c < parts; ++c) st_cluster_f32(map_to_cta(smem_u32(&r_a[em]), c), rest);
            }
          }
        }
      };
      // (a share is 2048 fours for two CTAs, 1024 for four)
      if (parts <= 2) share(OrthoKindOf<4>());
      else if (parts <= 4) share(OrthoKindOf<2>());
      else share(OrthoKindOf<1>());
      asm volatile("fence.proxy.async;" ::: "memory");      // (what went to the other CTAs is read by their MMAs)
      cluster_arrive();
      cluster_wait();
    }
    // ---- B
    product([&] {
#pragma unroll 1
      for (int j = 0; j < kSmallN / 16; ++j) {
        const uint64_t d = along(u_a, kSmallN, j);
        tcgen05_mma<true>(tmem, d, d, idesc(kSmallN, false, false), j > 0);
      }
    });
    {
      const float r_m = r_a[m];
      uint32_t v[32];
      tmem_ld_32x32(t_row + (uint32_t)(32 * group), v);
      tmem_wait_ld();
      const F2 rm2 = f2(r_m), cb2 = f2(cb), cc2 = f2(cc);
      by_diagonal([&](auto diagonal) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t at = image_at(kSmallN, m, 4 * group + i);
          Raw8<MAXDNN_F16> raw;
          raw.a = *reinterpret_cast<const uint4*>(square_a + at);
          F2 a[4];
          to_pairs<MAXDNN_F16>(raw, a);
          uint32_t w[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const F2 r2 = *reinterpret_cast<const F2*>(&r_a[32 * group + 8 * i + 2 * k]);
            const F2 acc = ((F2)v[8 * i + 2 * k + 1] << 32) | v[8 * i + 2 * k];
            float2 y = unf2(fma2(cb2, a[k], mul2(cc2, fma2(add2(rm2, r2), a[k], acc))));
            // the diagonal: A_mm has r besides, on both sides of its square too
            const bool mine = decltype(diagonal)::value && 8 * i + 2 * k == (lane & ~1);
            if (mine) (lane & 1 ? y.y : y.x) += r_m * fmaf(cc, r_m, cb);
            const __half2 h = __floats2half2_rn(y.x, y.y);
            w[k] = *reinterpret_cast<const uint32_t*>(&h);
            if (mine) {
              const float2 back = __half22float2(h);
              d_b[m] = lane & 1 ? y.y : y.x;
              h_b[m] = lane & 1 ? back.y : back.x;
            }
          }
          *reinterpret_cast<uint4*>(square_b + at) = make_uint4(w[0], w[1], w[2], w[3]);
        }
      });
    }
    // ---- X
    product([&] {
#pragma unroll 1
      for (int j = 0; j < kSmallN / 16; ++j) {
        const uint64_t b = along(u_b, kSmallN, j);
        if (TALL) {
          // rows from the left half's tile, then the right's (128 rows of 128 bytes further)
          tcgen05_mma<true>(tmem, along(u_image, kRows, j), b, idesc(kSmallN, false, false), j > 0);
          tcgen05_mma<true>(tmem + 128u, along(u_image + 16384u, kRows, j), b, idesc(kSmallN, false, false), j > 0);
        } else {
          tcgen05_mma<true>(tmem, b, across(u_image, kRows, j), idesc(kSmallSlice, false, true), j > 0);
        }
      }
    });
    // a x + (B x) with d lo + r hi for the diagonal: (a + d) x - h hi + the product, h = d - r what FP16 holds of it
    const F2 k_x = f2(ca + (TALL ? 0.f : d_b[row])), k_hi = f2(TALL ? 0.f : -h_b[row]);
#pragma unroll 1
    for (int u = 0; u < 2; ++u) {
      uint32_t v[32], old[32];
      tmem_ld_32x32(t_row + (uint32_t)(64 * group + 32 * u), v);
      tmem_ld_32x32(t_x + 32u * u, old);
      tmem_wait_ld();
      float fresh[32];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint32_t w[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int c = 8 * i + 2 * k, column = 8 * chunk0 + 32 * u + c;
          const F2 x2 = ((F2)old[c + 1] << 32) | old[c], acc = ((F2)v[c + 1] << 32) | v[c];
          const __half2 held = __floats2half2_rn(__uint_as_float(old[c]), __uint_as_float(old[c + 1]));
          const float2 hf = __half22float2(held);
          const F2 hi = f2(hf.x, hf.y);
          F2 kx = k_x, kh = k_hi;
          if (TALL) {
            kx = add2(kx, *reinterpret_cast<const F2*>(&d_b[column]));
            kh = mul2(f2(-1.f), *reinterpret_cast<const F2*>(&h_b[column]));
          }
          const float2 y = unf2(fma2(kx, x2, fma2(kh, hi, acc)));
          fresh[c] = y.x;
          fresh[c + 1] = y.y;
          const __half2 h = __floats2half2_rn(y.x, y.y);
          w[k] = *reinterpret_cast<const uint32_t*>(&h);
        }
        *reinterpret_cast<uint4*>(image + image_at(kRows, row, chunk0 + 4 * u + i)) = make_uint4(w[0], w[1], w[2], w[3]);
      }
      tmem_st_32x32(t_x + 32u * u, fresh);
    }
    tmem_wait_st();
    // (the next part of A overwrites `partial`, which the other CTAs read before the second cluster barrier)
  }

  // ---- the result: through the image in BF16, rows by warps
  const float out_scale = __int_as_float((127 - kOrthoScaleBits) << 23);
#pragma unroll 1
  for (int u = 0; u < 2; ++u) {
    uint32_t v[32];
    tmem_ld_32x32(t_x + 32u * u, v);
    tmem_wait_ld();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t w[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(__uint_as_float(v[8 * i + 2 * k]) * out_scale, __uint_as_float(v[8 * i + 2 * k + 1]) * out_scale);
        w[k] = *reinterpret_cast<const uint32_t*>(&h);
      }
      *reinterpret_cast<uint4*>(image + image_at(kRows, row, chunk0 + 4 * u + i)) = make_uint4(w[0], w[1], w[2], w[3]);
    }
  }
  __syncthreads();
  __nv_bfloat16* out = args.out + matrix * args.stride_o + (TALL ? first * args.ldo : first);
#pragma unroll 1
  for (int i = 0; i < kHeld; ++i) {
    const int r = row_read(i);
    Raw8<MAXDNN_BF16> raw;
    raw.a = *reinterpret_cast<const uint4*>(image + image_at(kRows, r, c_read / 8));
    float v[8];
    to_float8<MAXDNN_BF16>(raw, v);
    store_float8<MAXDNN_BF16, true>(out + r * args.ldo + c_read, v, r < rows_here ? min(max(cols_here - c_read, 0), 8) : 0);
  }
  tcgen05_fence_before();
  cluster_arrive();      // no CTA leaves while another may still read its shared memory
  cluster_wait();
  if (warp == 0) {
    if (!__all_sync(0xFFFFFFFFu, ok)) {      // every MMA issued so far has finished before TMEM is released
      if (elect_one()) tcgen05_commit(bar + 8u);
      __syncwarp();
      mbar_wait_grace(bar + 8u, 0);
    }
    tcgen05_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"((uint32_t)kSmallTmem) : "memory");
  }
}

}  // namespace maxdnn
