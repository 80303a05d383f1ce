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

// A block's scale from its largest finite magnitude a (bit pattern), as it is
// stored, and its reciprocal, which the values are multiplied by.  448 is e4m3's
// largest value.  fp32: a / 448, at least 2^-126 so that the reciprocal is
// finite; the values are then off their quotient by 1.5 fp32 steps, 2^-19 of
// an e4m3 step, and a itself stays below 464, where 448 ends.  E8M0: the
// smallest power of two 2^e, e >= -126, with a <= 448 2^e (448 = 1.75 * 2^8),
// stored as e + 127; its reciprocal is exact.  A block of zeros has the scale 1.
template <bool E8M0> struct Fp8Scale;
template <> struct Fp8Scale<false> {
  typedef float type;
  static __device__ __forceinline__ float stored(uint32_t a, float& inv) {
    const float s = a == 0u ? 1.f : fmaxf(__uint_as_float(a) / 448.f, 0x1p-126f);
    inv = 1.f / s;
    return s;
  }
};
template <> struct Fp8Scale<true> {
  typedef uint8_t type;
  static __device__ __forceinline__ uint8_t stored(uint32_t a, float& inv) {
    int e = (int)(a >> 23) - 8 + ((a & 0x7fffffu) > 0x600000u ? 1 : 0);
    e = a == 0u ? 127 : max(e, 1);
    inv = __uint_as_float((uint32_t)(254 - e) << 23);
    return (uint8_t)e;
  }
};

// Four values times inv, to nearest e4m3 (ties to even).  An infinity or NaN
// becomes e4m3's NaN: the conversion makes it of what lies beyond its range, and
// no finite value of the block does.
__device__ __forceinline__ uint32_t fp8x4(const float* f, float inv) {
  int v = __builtin_amdgcn_cvt_pk_fp8_f32(f[0] * inv, f[1] * inv, 0, false);
  v = __builtin_amdgcn_cvt_pk_fp8_f32(f[2] * inv, f[3] * inv, v, true);
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

__device__ __forceinline__ uint32_t finite_max8(const float (&f)[8]) {
  uint32_t a = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) a = max(a, finite_bits(f[e]));
  return a;
}

}  // namespace cats
