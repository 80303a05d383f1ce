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
// of f k (2^-20 of an e4m3 step; a value is off its neighbour's side only where
// it lies that near to the middle of two).  Where a / 448 is below 2^-126, f (m / 2^-126).
// E8M0: the smallest power of two 2^e, e >= -126, with a <= 448 2^e (448 = 1.75 *
// 2^8), stored as e + 127, whose division is exact.
// A block of zeros has the scale 1, and so has one whose m makes zeros,
// infinities or NaN of its values, with e4m3's zero or NaN.
// Below A = 2^-100 a factor could overflow: there f is to be multiplied by 2^64
// before (`tiny`).
struct Fp8Factor { float hi, lo; };
constexpr uint32_t kFp8Tiny = 0x0d800000u;  // 2^-100
constexpr float kFp8Lift = 0x1p64f;
__device__ __forceinline__ float times(float f, const Fp8Factor& k) { return fmaf(f, k.hi, f * k.lo); }

template <bool E8M0> struct Fp8Scale;
template <> struct Fp8Scale<false> {
  typedef float type;
  static __device__ __forceinline__ float stored(uint32_t A, const Fp8Factor& m, Fp8Factor& k, bool& tiny) {
    const float top = __uint_as_float(A), a = times(top, m), s = a / 448.f;
    tiny = false;
    if (__builtin_expect(A >= kFp8Tiny && s >= 0x1p-126f && s < __builtin_inff(), 1)) {
      k.hi = 448.f / top;
      k.lo = fmaf(-k.hi, top, 448.f) * (k.hi * (1.f / 448.f));
      return s;
    }
    k.lo = 0.f;
    k.hi = m.hi;
    if (!(a > 0.f && a < __builtin_inff())) return 1.f;
    const float t = fmaxf(s, 0x1p-126f);
    tiny = A < kFp8Tiny;
    k.hi = (tiny ? m.hi * (1.f / kFp8Lift) : m.hi) / t;
    return t;
  }
};
template <> struct Fp8Scale<true> {
  typedef uint8_t type;
  static __device__ __forceinline__ uint8_t stored(uint32_t A, const Fp8Factor& m, Fp8Factor& k, bool& tiny) {
    const uint32_t a = __float_as_uint(times(__uint_as_float(A), m));
    int e = (int)(a >> 23) - 8 + ((a & 0x7fffffu) > 0x600000u ? 1 : 0);
    const bool none = a == 0u || a >= 0x7f800000u;
    e = none ? 127 : max(e, 1);
    tiny = A < kFp8Tiny && !none;
    const float inv = __uint_as_float((uint32_t)(254 - e) << 23), lift = tiny ? 1.f / kFp8Lift : 1.f;
    k.hi = m.hi * lift * inv;
    k.lo = m.lo * lift * inv;
    return (uint8_t)e;
  }
};

// The scale and factor of a block, its lane's N values made ready for it.
template <bool E8M0, int N>
__device__ __forceinline__ typename Fp8Scale<E8M0>::type fp8_scale(uint32_t A, const Fp8Factor& m, Fp8Factor& k, float* f) {
  bool tiny;
  const typename Fp8Scale<E8M0>::type s = Fp8Scale<E8M0>::stored(A, m, k, tiny);
  if (__builtin_expect(__any(tiny), 0)) {
#pragma unroll
    for (int e = 0; e < N; ++e) f[e] *= tiny ? kFp8Lift : 1.f;
  }
  return s;
}

// Four values times k, to nearest e4m3 (ties to even).  An infinity or NaN
// becomes e4m3's NaN: the conversion makes it of what lies beyond its range, and
// no finite value of the block does.
__device__ __forceinline__ uint32_t fp8x4(const float* f, const Fp8Factor& k) {
  int v = __builtin_amdgcn_cvt_pk_fp8_f32(times(f[0], k), times(f[1], k), 0, false);
  v = __builtin_amdgcn_cvt_pk_fp8_f32(times(f[2], k), times(f[3], k), v, true);
  return (uint32_t)v;
}

// Eight consecutive elements of a row from column c on, as fp32, zeros from
// column `cols` on.  One or two 16-byte loads; rows need no more than their
// elements' alignment (global loads of 16 bytes take any), so odd widths read as
// wide ones do.
struct __attribute__((packed, aligned(4))) f32x4u { float v[4]; };
struct __attribute__((packed, aligned(2))) u16x8u { uint16_t v[8]; };
__device__ __forceinline__ void load8(const float* row, int c, int cols, float (&f)[8]) {
  if (c + 8 <= cols) {
    const f32x4u a = *reinterpret_cast<const f32x4u*>(row + c), b = *reinterpret_cast<const f32x4u*>(row + c + 4);
#pragma unroll
    for (int e = 0; e < 4; ++e) f[e] = a.v[e], f[4 + e] = b.v[e];
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = c + e < cols ? row[c + e] : 0.f;
  }
}
__device__ __forceinline__ void load8(const uint16_t* row, int c, int cols, float (&f)[8]) {
  if (c + 8 <= cols) {
    const u16x8u a = *reinterpret_cast<const u16x8u*>(row + c);
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = __uint_as_float((uint32_t)a.v[e] << 16);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = c + e < cols ? __uint_as_float((uint32_t)row[c + e] << 16) : 0.f;
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
