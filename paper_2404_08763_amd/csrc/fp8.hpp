// e4m3 values with a scale for each block: what the 8-bit kernels share.
#pragma once

#include "device.hpp"

namespace cats {

constexpr int kFp8Block = 128;  // columns (and, for weights, rows) of a scale's block

// Row pitch of a matrix of `cols` columns.
inline __host__ __device__ int fp8_ld(int cols) { return (cols + kFp8Block - 1) / kFp8Block * kFp8Block; }

// The magnitude's bit pattern, 0 for an infinity or NaN (which order as
// unsigned numbers as the magnitudes do).
__device__ __forceinline__ uint32_t finite_bits(float f) {
  const uint32_t u = __float_as_uint(f) & 0x7fffffffu;
  return u < 0x7f800000u ? u : 0u;
}

template <int CTRL> __device__ __forceinline__ uint32_t dpp_u32(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, false);
}

// Largest over each row of 16 lanes, on all of them (the steps of wave_sum).
__device__ __forceinline__ uint32_t max16(uint32_t v) {
  v = max(v, dpp_u32<0xb1>(v));
  v = max(v, dpp_u32<0x4e>(v));
  v = max(v, dpp_u32<0x141>(v));
  return max(v, dpp_u32<0x140>(v));
}

// How a block's values become e4m3: the values are f * m (m = hi + lo, a row's
// RMSNorm, or 1), A is the largest finite |f| (bit pattern), the scale as it is
// stored goes by a = A m, and e4m3 gets f * k (k = hi + lo).  448 is e4m3's
// largest value.
//
// fp32: scale a / 448, so f m / scale = f (448 / A): the row's factor drops out,
// and with the quotient to twice fp32's precision the one rounding left is that
// of f k.  Where a / 448 is below 2^-126, f (m / 2^-126).
// E8M0: the smallest power of two 2^e, e >= -126, with a <= 448 2^e (448 = 1.75 *
// 2^8), stored as e + 127, whose division is exact.
// A block of zeros has the scale 1, and so has one whose m makes zeros,
// infinities or NaN of its values, with e4m3's zero or NaN.
// Below A = 2^-100 a factor could overflow: there f is to be multiplied by 2^64
// before (`tiny`).  `plain`: none of these exceptions.
struct Fp8Factor { float hi, lo; };
constexpr uint32_t kFp8Tiny = 0x0d800000u;  // 2^-100
constexpr float kFp8Lift = 0x1p64f;
__device__ __forceinline__ float times(float f, const Fp8Factor& k) { return fmaf(f, k.hi, f * k.lo); }

template <bool E8M0> struct Fp8Scale;
template <> struct Fp8Scale<false> {
  typedef float type;
  template <bool TWO>
  static __device__ __forceinline__ float stored(uint32_t A, const Fp8Factor& m, Fp8Factor& k, bool& tiny, bool& plain) {
    const float top = __uint_as_float(A), a = times(top, m);
    tiny = false;
    plain = A >= kFp8Tiny && a >= 448.f * 0x1p-126f && a < __builtin_inff();
    if (__builtin_expect(plain, 1)) {
      // the quotients as the reciprocal's (of a number whose own is in the normal
      // range) and what is left
      const float r = __builtin_amdgcn_rcpf(top * 0x1p-14f), q = a * (1.f / 448.f);
      k.hi = 448.f * 0x1p-14f * r;
      k.lo = TWO ? fmaf(-k.hi, top, 448.f) * (0x1p-14f * r) : 0.f;
      return fmaf(fmaf(-448.f, q, a), 1.f / 448.f, q);
    }
    const float s = a / 448.f;
    k.lo = 0.f;
    k.hi = m.hi;
    if (!(a > 0.f && a < __builtin_inff())) return 1.f;
    const float t = fmaxf(s, 0x1p-126f);
    tiny = A < kFp8Tiny;
    k.hi = (tiny ? m.hi * (1.f / kFp8Lift) : m.hi) / t;
    return t;
  }
  // the same from the block's largest in 64 bits
  static __device__ __forceinline__ float exact(double a, double& k) {
    k = a > 0.0 ? 448.0 / a : 1.0;
    return a > 0.0 ? (float)(a / 448.0) : 1.f;
  }
};
template <> struct Fp8Scale<true> {
  typedef uint8_t type;
  template <bool TWO>
  static __device__ __forceinline__ uint8_t stored(uint32_t A, const Fp8Factor& m, Fp8Factor& k, bool& tiny, bool& plain) {
    const uint32_t a = __float_as_uint(times(__uint_as_float(A), m));
    int e = (int)(a >> 23) - 8 + ((a & 0x7fffffu) > 0x600000u ? 1 : 0);
    const bool none = a == 0u || a >= 0x7f800000u;
    plain = !none && e >= 1 && A >= kFp8Tiny;
    e = none ? 127 : max(e, 1);
    tiny = A < kFp8Tiny && !none;
    const float inv = __uint_as_float((uint32_t)(254 - e) << 23), lift = tiny ? 1.f / kFp8Lift : 1.f;
    k.hi = m.hi * lift * inv;
    k.lo = m.lo * lift * inv;
    return (uint8_t)e;
  }
  static __device__ __forceinline__ uint8_t exact(double a, double& k) {
    const uint64_t b = (uint64_t)__double_as_longlong(a);
    const int e = !(a > 0.0) ? 0 : max((int)(b >> 52) - 1023 - 8 + ((b & 0xfffffffffffffull) > 0xc000000000000ull ? 1 : 0), -126);
    k = __longlong_as_double((long long)(1023 - e) << 52);
    return (uint8_t)(e + 127);
  }
};

// The scale and factor of a block, its lane's N values made ready for it.  TWO: the
// factor to twice fp32's precision (else its hi alone counts, two of fp32's steps off).
template <bool E8M0, bool TWO, int N>
__device__ __forceinline__ typename Fp8Scale<E8M0>::type fp8_scale(uint32_t A, const Fp8Factor& m, Fp8Factor& k, float* f, bool& plain) {
  bool tiny;
  const typename Fp8Scale<E8M0>::type s = Fp8Scale<E8M0>::template stored<TWO>(A, m, k, tiny, plain);
  if (__builtin_expect(__any(tiny), 0)) {
#pragma unroll
    for (int e = 0; e < N; ++e) f[e] *= tiny ? kFp8Lift : 1.f;
  }
  return s;
}

// Eight values to nearest e4m3 (ties to even).  An infinity or NaN
// becomes e4m3's NaN: the conversion makes it of what lies beyond its range, and
// no finite value of a block does.
__device__ __forceinline__ uint2 fp8x8(const float (&v)[8]) {
  int a = __builtin_amdgcn_cvt_pk_fp8_f32(v[0], v[1], 0, false), b = __builtin_amdgcn_cvt_pk_fp8_f32(v[4], v[5], 0, false);
  a = __builtin_amdgcn_cvt_pk_fp8_f32(v[2], v[3], a, true);
  b = __builtin_amdgcn_cvt_pk_fp8_f32(v[6], v[7], b, true);
  return uint2{(uint32_t)a, (uint32_t)b};
}

// An error of fp32's size moves a value to the wrong e4m3 neighbour only where it
// lies next to the middle of two: 20 bits below the kept three of the
// significand, 0x80000.  Whether one of eight lies within W of fp32's steps of it.
// Such values, one in 2^19 / W, are looked at again in 64 bits, so that q is the
// nearest value and not one of the two nearest.  (Below 2^-6, e4m3's
// subnormals, of which fp32 has 2^14 steps to one and more, values are left as they are.)
__device__ __forceinline__ bool near_tie(const float (&v)[8], uint32_t W) {
  uint32_t a = ~0u;
#pragma unroll
  for (int e = 0; e < 8; ++e) a = min(a, (__float_as_uint(v[e]) << 12) + (0x80000000u + (W << 12)));
  return a < (2u * W << 12);
}
// v, rounded from a number `above` or `below` it, rounded to odd instead: on the side
// of any middle that the number is on.
__device__ __forceinline__ float to_odd(float v, bool above, bool below) {
  const uint32_t b = __float_as_uint(v);
  if (above == below || (b & 1u) || v == 0.f) return v;
  return __uint_as_float(above == (v > 0.f) ? b + 1u : b - 1u);
}
__device__ __forceinline__ float to_odd(double x) {
  const float v = (float)x;
  const double off = x - (double)v, few = fabs(x) * 0x1p-46;  // (x's own error: a middle may be meant)
  return to_odd(v, off > few, off < -few);
}
// Quantisation of fp32 alone: v = f 448 / A to one rounding, and f 448 beside v A is
// exact in 64 bits.  (Of bf16 no f 448 / A lies next to a middle but on it.)
__device__ __forceinline__ void fix_ties(float (&v)[8], const float (&f)[8], uint32_t A, bool plain) {
  if (__builtin_expect(__any(plain && near_tie(v, 1)), 0)) {
    const double a = __uint_as_float(A);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const double x = (double)f[e] * 448.0, y = (double)v[e] * a;
      if (plain) v[e] = to_odd(v[e], x > y, x < y);
    }
  }
}
template <int CTRL> __device__ __forceinline__ double dpp_f64(double v) {
  const uint64_t b = (uint64_t)__double_as_longlong(v);
  return __longlong_as_double((long long)((uint64_t)dpp_u32<CTRL>((uint32_t)(b >> 32)) << 32 | dpp_u32<CTRL>((uint32_t)b)));
}
__device__ __forceinline__ double max16(double v) {
  v = fmax(v, dpp_f64<0xb1>(v));
  v = fmax(v, dpp_f64<0x4e>(v));
  v = fmax(v, dpp_f64<0x141>(v));
  return fmax(v, dpp_f64<0x140>(v));
}
// Over the wave (the steps of wave_sum).
__device__ __forceinline__ double wave_sum64(double v) {
  v += dpp_f64<0xb1>(v);
  v += dpp_f64<0x4e>(v);
  v += dpp_f64<0x141>(v);
  v += dpp_f64<0x140>(v);
  const uint64_t b = (uint64_t)__double_as_longlong(v);
  const uint32_t l = (uint32_t)b, h = (uint32_t)(b >> 32);
  double sum = 0.0;
#pragma unroll
  for (int i = 0; i < 64; i += 16)
    sum += __longlong_as_double((long long)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)h, i) << 32 |
                                            (uint32_t)__builtin_amdgcn_readlane((int)l, i)));
  return sum;
}

// Eight consecutive elements of a row from column c on, as fp32, zeros from
// column `cols` on.  One or two 16-byte loads; rows need no more than their
// elements' alignment (global loads of 16 bytes take any), so odd widths read as
// wide ones do.
struct __attribute__((packed, aligned(4))) f32x4u { float v[4]; };
struct __attribute__((packed, aligned(2))) u16x8u { uint16_t v[8]; };
__device__ __forceinline__ float as_f32(float v) { return v; }
__device__ __forceinline__ float as_f32(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }
template <typename T> struct Raw8;
template <> struct Raw8<float> {
  f32x4u a, b;
  __device__ __forceinline__ void load(const float* p) {
    a = *reinterpret_cast<const f32x4u*>(p);
    b = *reinterpret_cast<const f32x4u*>(p + 4);
  }
  __device__ __forceinline__ float get(int e) const { return e < 4 ? a.v[e & 3] : b.v[e & 3]; }
};
template <> struct Raw8<uint16_t> {
  u16x8u a;
  __device__ __forceinline__ void load(const uint16_t* p) { a = *reinterpret_cast<const u16x8u*>(p); }
  __device__ __forceinline__ float get(int e) const { return as_f32(a.v[e]); }
};
template <typename T> __device__ __forceinline__ void load8(const T* row, int c, int cols, float (&f)[8]) {
  if (c + 8 <= cols) {
    Raw8<T> a;
    a.load(row + c);
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = a.get(e);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = c + e < cols ? as_f32(row[c + e]) : 0.f;
  }
}
// The same of two rows, both on their way before either is waited for.
template <typename T, typename U>
__device__ __forceinline__ void load8(const T* row, const U* other, int c, int cols, float (&f)[8], float (&g)[8]) {
  if (c + 8 <= cols) {
    Raw8<T> a;
    Raw8<U> b;
    a.load(row + c);
    b.load(other + c);
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = a.get(e), g[e] = b.get(e);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      f[e] = c + e < cols ? as_f32(row[c + e]) : 0.f;
      g[e] = c + e < cols ? as_f32(other[c + e]) : 0.f;
    }
  }
}
__device__ __forceinline__ void store8(float* row, int c, int cols, const float (&f)[8]) {
  if (c + 8 <= cols) {
    f32x4u a, b;
#pragma unroll
    for (int e = 0; e < 4; ++e) a.v[e] = f[e], b.v[e] = f[4 + e];
    *reinterpret_cast<f32x4u*>(row + c) = a;
    *reinterpret_cast<f32x4u*>(row + c + 4) = b;
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (c + e < cols) row[c + e] = f[e];
  }
}

// Largest magnitude (bit pattern) of N values, infinities and NaN among them, and
// of the finite ones alone.
template <int N> __device__ __forceinline__ uint32_t max_bits(const float* f) {
  uint32_t a = 0;
#pragma unroll
  for (int e = 0; e < N; ++e) a = max(a, __float_as_uint(f[e]) & 0x7fffffffu);
  return a;
}
template <int N> __device__ __forceinline__ uint32_t finite_max_bits(const float* f) {
  uint32_t a = 0;
#pragma unroll
  for (int e = 0; e < N; ++e) a = max(a, finite_bits(f[e]));
  return a;
}
// Largest finite magnitude over 16 lanes' N values each: blocks with an infinity
// or NaN, which are looked at a second time, are rare.
template <int N> __device__ __forceinline__ uint32_t block_max(const float* f) {
  const uint32_t a = max16(max_bits<N>(f));
  if (__builtin_expect(__any(a >= 0x7f800000u), 0)) return max16(finite_max_bits<N>(f));
  return a;
}

}  // namespace cats
