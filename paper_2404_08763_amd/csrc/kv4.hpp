// The cache of keys and values in 4 bits: its layout and what its kernels share.
//
// A record holds 16 tokens of one head, 17 D bytes: keys, values, the keys'
// scales, the values' scales.  It is laid out for the attention kernel's matrix
// operands, so that each lane reads its part of a record with one wide load and
// needs no exchange with other lanes:
//   key   (t, c)  byte t D/2 + c/2, even columns in the low half.  Lane (m, g) =
//                 (lane % 16, lane / 16) is token m's columns [g D/4, (g+1) D/4).
//   value (t, c)  byte 8 D + ((t/4 * 16 + n) * 4 + t%4) * D/32 + r/2, n = c / (D/16),
//                 r = c % (D/16).  Lane (n, g) is columns [n D/16, (n+1) D/16) of the
//                 tokens 4 g .. 4 g + 3, D/4 bytes in one piece.
//   scales        bytes 16 D + t D/32 + c/32 (keys) and 16 D + D/2 + (t/4 * D/32 + c/32)
//                 * 4 + t%4 (values: the four tokens of a lane side by side).
#pragma once

#include "device.hpp"

namespace cats {

constexpr int kKvGroup = 16;  // tokens of a record
constexpr int kKvMinExp = -125, kKvMaxExp = 125;

__host__ __device__ constexpr int kv_record_bytes(int d) { return 17 * d; }

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

// Scale byte of a block whose largest magnitude has the bit pattern A: the
// smallest 2^e with |x| <= 6 2^e (6 = 1.5 * 2^2), e + 127 stored; 255 (NaN) where
// the block holds an infinity or NaN, 127 (1) where it is zero.
__device__ __forceinline__ uint32_t kv_scale_byte(uint32_t A) {
  if (A >= 0x7f800000u) return 255u;
  if (A == 0u) return 127u;
  // exponent of A, one more where its mantissa is above 1.5 (for a subnormal the clamp decides)
  const int e = (int)(A >> 23) - 127 - 2 + ((A & 0x7fffffu) > 0x400000u ? 1 : 0);
  return (uint32_t)(min(max(e, kKvMinExp), kKvMaxExp) + 127);
}

// The scale a byte stands for; 255 is an infinity here, of which the conversion
// instructions make NaN for every code, as of any scale with that exponent.
__device__ __forceinline__ float kv_scale(uint32_t byte) { return __uint_as_float(byte << 23); }

}  // namespace cats
