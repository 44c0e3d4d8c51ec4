// Element types of the 8-bit training operators: conversions between fp32 and the storage types,
// loads and stores of eight neighbouring values, and the scale of a block.
//
// Format.  A block of up to 128 values has one scale 2^E, kept as the byte E + 127 (E8M0).  With
// m the largest finite magnitude of the block and V = 1.75 2^8 (E4M3) or 1.75 2^15 (E5M2) the
// largest number of the type, E is the least integer with m <= V 2^E: the exponent of m less 8
// (15), plus one if m's mantissa is above 1.75.  It is clamped to [-126, 127], so that 2^E and
// 2^-E are normal numbers, and is 0 for a block of zeros.  Multiplying by a power of two is
// exact: a value is rounded once, to the 8-bit type, and the result does not depend on who
// computes it.  Infinities and NaN do not enter m; they are stored as NaN (E4M3, which has no
// infinity) or as themselves (E5M2).
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/maxdnn.h"

namespace maxdnn {

constexpr int kBlock8 = 128;       // values along a block
constexpr int kLanesPerBlock = 16; // lanes of eight values that cover a block

// Every kernel of these operators is launched so that it may start while the kernel before it in
// the stream still runs (programmatic dependent launch): it lets the next one do the same at once and, before
// it touches memory, waits until the one before has finished and its writes are visible.
__device__ __forceinline__ void let_next_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_for_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// What a kernel before this one may have written while this one was already resident is read by
// plain loads: the read-only path (ld.global.nc) is for memory that nobody writes during the
// kernel's life, which begins before that wait.
template <class T>
__device__ __forceinline__ T load_global(const T* p) { return *p; }
// The same loads (16 or 8 bytes), which stay behind that wait but which the compiler may move across this
// kernel's own stores: inputs and outputs do not overlap.
__device__ __forceinline__ uint4 load_global_free(const uint4* p) {
  uint4 v;
  asm volatile("ld.global.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}
__device__ __forceinline__ uint2 load_global_free(const uint2* p) {
  uint2 v;
  asm volatile("ld.global.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "l"(p));
  return v;
}
template <bool FREE, class T>
__device__ __forceinline__ T load_as(const T* p) {
  if constexpr (FREE) return load_global_free(p);
  else return load_global(p);
}

template <int DT> struct ElemOf;
template <> struct ElemOf<MAXDNN_F32> { typedef float T; };
template <> struct ElemOf<MAXDNN_BF16> { typedef __nv_bfloat16 T; };
template <> struct ElemOf<MAXDNN_F16> { typedef __half T; };
template <> struct ElemOf<MAXDNN_E4M3> { typedef uint8_t T; };
template <> struct ElemOf<MAXDNN_E5M2> { typedef uint8_t T; };

__host__ __device__ constexpr int elem_bytes(int dt) {
  return dt == MAXDNN_F32 ? 4 : (dt == MAXDNN_BF16 || dt == MAXDNN_F16) ? 2 : 1;
}
__host__ __device__ constexpr bool is_fp8(int dt) { return dt == MAXDNN_E4M3 || dt == MAXDNN_E5M2; }
__host__ __device__ constexpr bool is_wide(int dt) {
  return dt == MAXDNN_F32 || dt == MAXDNN_BF16 || dt == MAXDNN_F16;
}

// ---- pairs of fp32 values in one 64-bit register: two adds, multiplies or fused
// multiply-adds for one issue slot (each rounded as the single operation is) ----
typedef unsigned long long F2;
__device__ __forceinline__ F2 f2(float lo, float hi) {
  F2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ F2 f2(float both) { return f2(both, both); }
__device__ __forceinline__ float2 unf2(F2 v) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
  return r;
}
__device__ __forceinline__ F2 add2(F2 a, F2 b) {
  F2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ F2 mul2(F2 a, F2 b) {
  F2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ F2 fma2(F2 a, F2 b, F2 c) {
  F2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ float sum2(F2 v) {
  const float2 t = unf2(v);
  return t.x + t.y;
}
// The largest magnitude of three values; NaN do not count.
__device__ __forceinline__ float max3abs(float a, float b, float c) {
  float r;
  asm("max.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

// ---- two 8-bit values <-> fp32 (low byte first) ----
template <int QT>
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  uint16_t r;
  if constexpr (QT == MAXDNN_E4M3)
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  else
    asm("cvt.rn.satfinite.e5m2x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
template <int QT>
__device__ __forceinline__ float2 unpack2(uint32_t two) {
  uint32_t h;
  const uint16_t t = (uint16_t)two;
  if constexpr (QT == MAXDNN_E4M3)
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(t));
  else
    asm("cvt.rn.f16x2.e5m2x2 %0, %1;" : "=r"(h) : "h"(t));
  return __half22float2(*reinterpret_cast<const __half2*>(&h));
}

// The bytes of infinities among eight packed values: NaN (E4M3) or infinity (E5M2), where the
// conversion gives the largest number.  Out of line: few blocks hold one.
static __device__ __noinline__ uint2 infinities8(uint2 w, float v0, float v1, float v2, float v3, float v4, float v5,
                                                 float v6, float v7, uint32_t code) {
  const float v[8] = {v0, v1, v2, v3, v4, v5, v6, v7};
  uint32_t o[2] = {w.x, w.y};
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (isinf(v[i])) {
      const int sh = 8 * (i & 3);
      o[i >> 2] = (o[i >> 2] & ~(0xFFu << sh)) | ((code | (v[i] < 0 ? 0x80u : 0u)) << sh);
    }
  }
  return make_uint2(o[0], o[1]);
}

// Eight values times `inv` in 8 bytes.  fix: the block holds an infinity.
template <int QT>
__device__ __forceinline__ uint2 pack8(const F2 (&v)[4], const F2 (&inv)[4], bool fix) {
  uint32_t h[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 t = unf2(mul2(v[i], inv[i]));
    h[i] = pack2<QT>(t.x, t.y);
  }
  uint2 w = make_uint2(__byte_perm(h[0], h[1], 0x5410), __byte_perm(h[2], h[3], 0x5410));
  if (fix) {
    const float2 a = unf2(v[0]), b = unf2(v[1]), c = unf2(v[2]), d = unf2(v[3]);
    w = infinities8(w, a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y, QT == MAXDNN_E4M3 ? 0x7Fu : 0x7Cu);
  }
  return w;
}
template <int QT>
__device__ __forceinline__ uint2 pack8(const F2 (&v)[4], float inv, bool fix) {
  const F2 k = f2(inv), all[4] = {k, k, k, k};
  return pack8<QT>(v, all, fix);
}

// ---- scales ----
// The biased exponent byte for a largest magnitude `m` (finite, not negative).
template <int QT>
__device__ __forceinline__ uint32_t scale_byte(float m) {
  constexpr int kTop = QT == MAXDNN_E4M3 ? 8 : 15;
  const uint32_t b = __float_as_uint(m);
  // adding 0x1FFFFF carries into the exponent exactly where the mantissa is above 1.75
  const int e = (int)((b + 0x1FFFFFu) >> 23) - kTop;
  return b == 0 ? 127u : (uint32_t)max(e, 1);
}
// 2^E and 2^-E of a byte in [1, 253].
__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }
__device__ __forceinline__ float inv_scale_of(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }
// Any E8M0 byte: 0 is 2^-127, 255 is NaN.
__device__ __forceinline__ float e8m0_value(uint32_t byte) {
  return __uint_as_float(byte == 0 ? 0x00400000u : byte == 255 ? 0x7FC00000u : byte << 23);
}

__device__ __forceinline__ float max_over_block_lanes(float m) {
#pragma unroll
  for (int d = kLanesPerBlock / 2; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, d));
  return m;
}

// Largest magnitude of eight values; NaN do not count, infinities do (see finite_max8).
__device__ __forceinline__ float max8(const F2 (&v)[4]) {
  const float2 a = unf2(v[0]), b = unf2(v[1]), c = unf2(v[2]), d = unf2(v[3]);
  return max3abs(max3abs(a.x, a.y, b.x), max3abs(b.y, c.x, c.y), max3abs(d.x, d.y, 0.f));
}
static __device__ __noinline__ float finite_max8(F2 v0, F2 v1, F2 v2, F2 v3) {
  const F2 v[4] = {v0, v1, v2, v3};
  float m = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 t = unf2(v[i]);
    m = fmaxf(m, isinf(t.x) ? 0.f : fabsf(t.x));
    m = fmaxf(m, isinf(t.y) ? 0.f : fabsf(t.y));
  }
  return m;
}
// The scale bytes of two row blocks from the largest magnitudes of their lanes (16 lanes each, all
// lanes of the warp take part).  The exponent of a block's largest magnitude is the largest of its
// lanes' (rounded up where the mantissa is above 1.75: monotonic), so two blocks' exponents go
// through the shuffles as halves of one word.  rare: a block has exponent 0 (zeros or subnormals)
// or 255 (an infinity, or values near the largest); the caller then takes exact_byte.
template <int QT>
__device__ __forceinline__ bool block_bytes(float m0, float m1, uint32_t* b0, uint32_t* b1) {
  constexpr uint32_t kTop = QT == MAXDNN_E4M3 ? 8 : 15;
  const uint32_t e0 = (__float_as_uint(m0) + 0x1FFFFFu) >> 23, e1 = (__float_as_uint(m1) + 0x1FFFFFu) >> 23;
  uint32_t e = e0 | (e1 << 16);
#pragma unroll
  for (int d = kLanesPerBlock / 2; d > 0; d >>= 1) e = __vmaxu2(e, __shfl_xor_sync(0xFFFFFFFFu, e, d));
  const uint32_t lo = e & 0xFFFFu, hi = e >> 16;
  *b0 = (uint32_t)max((int)(lo - kTop), 1);
  *b1 = (uint32_t)max((int)(hi - kTop), 1);
  return __any_sync(0xFFFFFFFFu, lo - 1u >= 254u || hi - 1u >= 254u);
}

// The byte of one block from its lanes' values themselves; *fix: it holds an infinity.
template <int QT>
__device__ __forceinline__ uint32_t exact_byte(const F2 (&v)[4], bool* fix) {
  *fix = isinf(max_over_block_lanes(max8(v)));
  return scale_byte<QT>(max_over_block_lanes(finite_max8(v[0], v[1], v[2], v[3])));
}

// Columns of a vector of eight that starts at column c.
template <bool EDGE>
__device__ __forceinline__ int vector_cols(int cols, int c) {
  return EDGE ? min(max(cols - c, 0), 8) : c < cols ? 8 : 0;
}

// ---- eight neighbouring values as they lie in memory ----
template <int DT> struct Raw8;
template <> struct Raw8<MAXDNN_F32> { uint4 a, b; };
template <> struct Raw8<MAXDNN_BF16> { uint4 a; };
template <> struct Raw8<MAXDNN_F16> { uint4 a; };
template <> struct Raw8<MAXDNN_E4M3> { uint2 a; };
template <> struct Raw8<MAXDNN_E5M2> { uint2 a; };

// The four words that start `s` bytes (0..15) into eight.
__device__ __forceinline__ uint4 words_at(uint4 lo, uint4 hi, uint32_t s) {
  uint32_t w0 = lo.x, w1 = lo.y, w2 = lo.z, w3 = lo.w, w4 = hi.x;
  if (s & 8u) { w0 = lo.z; w1 = lo.w; w2 = hi.x; w3 = hi.y; w4 = hi.z; }
  if (s & 4u) { w0 = w1; w1 = w2; w2 = w3; w3 = w4; w4 = s & 8u ? hi.w : hi.y; }
  const uint32_t sh = 8u * (s & 3u);
  return make_uint4(__funnelshift_r(w0, w1, sh), __funnelshift_r(w1, w2, sh), __funnelshift_r(w2, w3, sh),
                    __funnelshift_r(w3, w4, sh));
}
// Bytes [0, n) of a word, n counted from the word's first byte; zeros beyond.
__device__ __forceinline__ uint32_t first_bytes(uint32_t w, int n) {
  return n >= 4 ? w : n <= 0 ? 0u : w & (0xFFFFFFFFu >> (32 - 8 * n));
}
__device__ __forceinline__ uint4 first_bytes(uint4 v, int n) {
  return make_uint4(first_bytes(v.x, n), first_bytes(v.y, n - 4), first_bytes(v.z, n - 8), first_bytes(v.w, n - 12));
}

// Loads `n` (0..8) values at `p`; the rest are zeros.
// EDGE = false: vectors are whole (n is 0 or 8) and aligned.  Kernels are built for both: a branch
// between the two forms makes the loaded registers move when the branches join, which waits for each load in
// turn (a layer norm with 16 loads a lane took 9.7 us a row that way).
// EDGE = true: the aligned 16 (8-bit types: 8) bytes that hold the first and the last value are
// loaded and shifted; no load touches an aligned unit that holds none of the n values.
template <int DT, bool EDGE, bool FREE = false>
__device__ __forceinline__ Raw8<DT> load_raw8(const typename ElemOf<DT>::T* p, int n) {
  Raw8<DT> r;
  if constexpr (!EDGE) {
    if constexpr (DT == MAXDNN_F32) {
      r.a = r.b = make_uint4(0, 0, 0, 0);
      if (n) {
        r.a = load_as<FREE>(reinterpret_cast<const uint4*>(p));
        r.b = load_as<FREE>(reinterpret_cast<const uint4*>(p) + 1);
      }
    } else if constexpr (is_fp8(DT)) {
      r.a = make_uint2(0, 0);
      if (n) r.a = load_as<FREE>(reinterpret_cast<const uint2*>(p));
    } else {
      r.a = make_uint4(0, 0, 0, 0);
      if (n) r.a = load_as<FREE>(reinterpret_cast<const uint4*>(p));
    }
  } else {
    const uintptr_t at = reinterpret_cast<uintptr_t>(p);
    const int bytes = n * (int)sizeof(typename ElemOf<DT>::T);
    if constexpr (is_fp8(DT)) {
      const uint32_t s = (uint32_t)(at & 7u);
      const uint2* q = reinterpret_cast<const uint2*>(at - s);
      uint2 lo = make_uint2(0, 0), hi = make_uint2(0, 0);
      if (bytes > 0) lo = load_as<FREE>(q);
      if ((int)s + bytes > 8) hi = load_as<FREE>(q + 1);
      const uint4 v = words_at(make_uint4(lo.x, lo.y, hi.x, hi.y), make_uint4(0, 0, 0, 0), s);
      r.a = make_uint2(first_bytes(v.x, bytes), first_bytes(v.y, bytes - 4));
    } else {
      const uint32_t s = (uint32_t)(at & 15u);
      const uint4* q = reinterpret_cast<const uint4*>(at - s);
      uint4 c0 = make_uint4(0, 0, 0, 0), c1 = c0;
      if (bytes > 0) c0 = load_as<FREE>(q);
      if ((int)s + bytes > 16) c1 = load_as<FREE>(q + 1);
      r.a = first_bytes(words_at(c0, c1, s), bytes);
      if constexpr (DT == MAXDNN_F32) {
        uint4 c2 = make_uint4(0, 0, 0, 0);
        if ((int)s + bytes > 32) c2 = load_as<FREE>(q + 2);
        r.b = first_bytes(words_at(c1, c2, s), bytes - 16);
      }
    }
  }
  return r;
}

template <int DT>
__device__ __forceinline__ void to_float8(const Raw8<DT>& r, float (&v)[8]) {
  if constexpr (DT == MAXDNN_F32) {
    v[0] = __uint_as_float(r.a.x); v[1] = __uint_as_float(r.a.y);
    v[2] = __uint_as_float(r.a.z); v[3] = __uint_as_float(r.a.w);
    v[4] = __uint_as_float(r.b.x); v[5] = __uint_as_float(r.b.y);
    v[6] = __uint_as_float(r.b.z); v[7] = __uint_as_float(r.b.w);
  } else if constexpr (DT == MAXDNN_BF16) {
    const uint32_t w[4] = {r.a.x, r.a.y, r.a.z, r.a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(w[i] << 16);
      v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
  } else if constexpr (DT == MAXDNN_F16) {
    const uint32_t w[4] = {r.a.x, r.a.y, r.a.z, r.a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
      v[2 * i] = f.x;
      v[2 * i + 1] = f.y;
    }
  } else {
    const uint32_t w[2] = {r.a.x, r.a.y};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 f = unpack2<DT>(w[i >> 1] >> (16 * (i & 1)));
      v[2 * i] = f.x;
      v[2 * i + 1] = f.y;
    }
  }
}

// The same values as pairs.
template <int DT>
__device__ __forceinline__ void to_pairs(const Raw8<DT>& r, F2 (&v)[4]) {
  if constexpr (DT == MAXDNN_F32) {
    v[0] = ((F2)r.a.y << 32) | r.a.x;
    v[1] = ((F2)r.a.w << 32) | r.a.z;
    v[2] = ((F2)r.b.y << 32) | r.b.x;
    v[3] = ((F2)r.b.w << 32) | r.b.z;
  } else {
    float f[8];
    to_float8<DT>(r, f);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = f2(f[2 * i], f[2 * i + 1]);
  }
}
__device__ __forceinline__ void to_floats(const F2 (&v)[4], float (&f)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 t = unf2(v[i]);
    f[2 * i] = t.x;
    f[2 * i + 1] = t.y;
  }
}

// Hides that the registers are what an earlier conversion saw, so that the values are converted
// again where they are used instead of being kept as fp32.
template <int DT>
__device__ __forceinline__ void convert_again(Raw8<DT>& r) {
  if constexpr (DT == MAXDNN_BF16 || DT == MAXDNN_F16)
    asm volatile("" : "+r"(r.a.x), "+r"(r.a.y), "+r"(r.a.z), "+r"(r.a.w));
}

template <int DT>
__device__ __forceinline__ typename ElemOf<DT>::T from_float(float v) {
  if constexpr (DT == MAXDNN_F32) return v;
  else if constexpr (DT == MAXDNN_BF16) return __float2bfloat16_rn(v);
  else return __float2half_rn(v);
}

// Stores the first `n` values.  EDGE = false: n is 0 or 8 and p is aligned.  EDGE = true: whole
// vectors in the widest pieces that p's alignment allows.
template <int DT, bool EDGE>
__device__ __forceinline__ void store_float8(typename ElemOf<DT>::T* p, const float (&v)[8], int n) {
  static_assert(!is_fp8(DT), "8-bit values are stored by store_bytes8");
  constexpr int kWords = 2 * (int)sizeof(typename ElemOf<DT>::T);
  uint32_t w[kWords];
  if constexpr (DT == MAXDNN_F32) {
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = __float_as_uint(v[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (DT == MAXDNN_BF16) {
        const __nv_bfloat162 t = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t*>(&t);
      } else {
        const __half2 t = __floats2half2_rn(v[2 * i], v[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t*>(&t);
      }
    }
  }
  if (n == 0) return;
  const uint32_t s = EDGE ? (uint32_t)(reinterpret_cast<uintptr_t>(p) & 15u) : 0u;
  if (!EDGE || (n == 8 && s == 0)) {
#pragma unroll
    for (int i = 0; i < kWords; i += 4)
      reinterpret_cast<uint4*>(p)[i / 4] = make_uint4(w[i], w[i + 1], w[i + 2], w[i + 3]);
  } else if (n == 8 && (s & 7u) == 0) {
#pragma unroll
    for (int i = 0; i < kWords; i += 2) reinterpret_cast<uint2*>(p)[i / 2] = make_uint2(w[i], w[i + 1]);
  } else if (n == 8 && (s & 3u) == 0) {
#pragma unroll
    for (int i = 0; i < kWords; ++i) reinterpret_cast<uint32_t*>(p)[i] = w[i];
  } else if (n == 8) {               // 16-bit values at an odd place
    uint16_t* h = reinterpret_cast<uint16_t*>(p);
    h[0] = (uint16_t)w[0];
#pragma unroll
    for (int i = 0; i + 1 < kWords; ++i) *reinterpret_cast<uint32_t*>(h + 1 + 2 * i) = __funnelshift_r(w[i], w[i + 1], 16);
    h[7] = (uint16_t)(w[kWords - 1] >> 16);
  } else {
#pragma unroll 1
    for (int i = 0; i < n; ++i) {
      if constexpr (DT == MAXDNN_F32) {
        reinterpret_cast<uint32_t*>(p)[i] = w[0];
#pragma unroll
        for (int k = 0; k + 1 < kWords; ++k) w[k] = w[k + 1];
      } else {
        reinterpret_cast<uint16_t*>(p)[i] = (uint16_t)w[0];
#pragma unroll
        for (int k = 0; k + 1 < kWords; ++k) w[k] = __funnelshift_r(w[k], w[k + 1], 16);
        w[kWords - 1] >>= 16;
      }
    }
  }
}

template <int DT, bool EDGE>
__device__ __forceinline__ void store_pairs(typename ElemOf<DT>::T* p, const F2 (&v)[4], int n) {
  float f[8];
  to_floats(v, f);
  store_float8<DT, EDGE>(p, f, n);
}

// The first `n` of eight bytes; EDGE as above.
template <bool EDGE>
__device__ __forceinline__ void store_bytes8(uint8_t* p, uint2 w, int n) {
  if (n == 0) return;
  const uint32_t s = EDGE ? (uint32_t)(reinterpret_cast<uintptr_t>(p) & 7u) : 0u;
  if (!EDGE || (n == 8 && s == 0)) {
    *reinterpret_cast<uint2*>(p) = w;
  } else if (n == 8 && s == 4) {
    reinterpret_cast<uint32_t*>(p)[0] = w.x;
    reinterpret_cast<uint32_t*>(p)[1] = w.y;
  } else {
#pragma unroll 1
    for (int i = 0; i < n; ++i) {
      p[i] = (uint8_t)w.x;
      w.x = __funnelshift_r(w.x, w.y, 8);
      w.y >>= 8;
    }
  }
}

}  // namespace maxdnn
