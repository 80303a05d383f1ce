// Linear layer on e4m3 operands with a scale for each block:
//   y[r, c] = residual[r, c] + sum_b xs[r, b] ws[c / 128, b] sum_{k in b} xq[r, k] wq[c, k]
// with blocks b of 128 columns: just one matrix instruction's depth.
#include "fp8.hpp"
#include "internal.hpp"

namespace cats {

typedef __bf16 fp_bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 fp_bf16x2 __attribute__((ext_vector_type(2)));

constexpr int kFewWaves = 8;  // waves of a block, each taking every eighth column block

// Eight e4m3 values times 2^e (scale = 2^e) as bf16, which holds them exactly.
__device__ __forceinline__ fp_bf16x8 widen8(uint32_t lo, uint32_t hi, float scale) {
  const fp_bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false);
  const fp_bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
  const fp_bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false);
  const fp_bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
  return fp_bf16x8{a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y};
}

// A scale as fp32.
template <bool E8M0> __device__ __forceinline__ float scale_at(const void* s, size_t i) {
  if constexpr (E8M0) {
    const uint32_t e = static_cast<const uint8_t*>(s)[i];
    return e == 255u ? __uint_as_float(0x7fc00000u) : e == 0u ? 0x1p-127f : __uint_as_float(e << 23);
  } else {
    return static_cast<const float*>(s)[i];
  }
}

// The products of one column block, 16 weights by 16 rows: weights are the first
// operand and rows of x the second, so a lane's four results are four
// consecutive outputs of one row.  Which of the block's columns sit in which
// lane does not matter as long as both operands agree: lane l holds bytes
// 16 (l / 16) .. + 15 and 64 more of row l % 16.
// The values go through the bf16 instructions, whose sums are exact to fp32;
// the 8-bit ones drop what lies 2^-13 below the largest of each eight products
// (4e-5 of the result on rows with outliers, in the mean square).
__device__ __forceinline__ f32x4 block_product(const u32x4 (&w)[2], const u32x4 (&x)[2]) {
  f32x4 p = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    p = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen8(w[h].x, w[h].y, 1.f), widen8(x[h].x, x[h].y, 1.f), p, 0, 0, 0);
    p = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen8(w[h].z, w[h].w, 1.f), widen8(x[h].z, x[h].w, 1.f), p, 0, 0, 0);
  }
  return p;
}

__device__ __forceinline__ float bf16_value(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }

// y[i] = v + residual[i]; bf16 rounds once, here.
__device__ __forceinline__ void put_y(const LinearFp8Args& a, size_t i, float v) {
  if (a.ybf16) {
    if (a.residual) v += bf16_value(static_cast<const uint16_t*>(a.residual)[i]);
    static_cast<uint16_t*>(a.y)[i] = (uint16_t)bf16_bits(v);
  } else {
    if (a.residual) v += static_cast<const float*>(a.residual)[i];
    static_cast<float*>(a.y)[i] = v;
  }
}

// 16 outputs x 16 rows per block, its waves splitting the column blocks.
template <bool E8M0>
__global__ __launch_bounds__(kFewWaves * kWaveSize) void k_fp8_few(LinearFp8Args a) {
  __shared__ f32x4 red[kFewWaves][kWaveSize];
  const int tid = threadIdx.x, lane = tid & (kWaveSize - 1);
  const int w = __builtin_amdgcn_readfirstlane(tid / kWaveSize);
  const int r16 = lane & 15, g = lane >> 4;
  const int c0 = blockIdx.x * 16, t0 = blockIdx.y * 16;
  const int KB = a.ld / kFp8Block;
  const int nc = min(16, a.n - c0), nt = min(16, a.N - t0);
  const __amdgpu_buffer_rsrc_t rw = make_rsrc(a.wq + (size_t)c0 * a.ld, (uint32_t)nc * a.ld);
  const __amdgpu_buffer_rsrc_t rx = make_rsrc(a.xq + (size_t)t0 * a.ld, (uint32_t)nt * a.ld);
  const uint32_t woff = r16 < nc ? (uint32_t)r16 * a.ld + g * 16u : kOOB;
  const uint32_t xoff = r16 < nt ? (uint32_t)r16 * a.ld + g * 16u : kOOB;
  const size_t xsrow = (size_t)(t0 + (r16 < nt ? r16 : 0)) * KB, wsrow = (size_t)(c0 / kFp8Block) * KB;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  for (int b = w; b < KB; b += kFewWaves) {
    const uint32_t k = (uint32_t)b * kFp8Block;
    const u32x4 wv[2] = {ld_buf16_stream(rw, woff + k), ld_buf16_stream(rw, woff + k + 64u)};
    const u32x4 xv[2] = {ld_buf16(rx, xoff + k), ld_buf16(rx, xoff + k + 64u)};
    const f32x4 p = block_product(wv, xv);
    const float scale = scale_at<E8M0>(a.xs, xsrow + b) * scale_at<E8M0>(a.ws, wsrow + b);
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[e] = fmaf(p[e], scale, acc[e]);
  }
  red[w][lane] = acc;
  __syncthreads();
  if (tid < 256) {
    const int t = tid >> 4, c = tid & 15;
    if (t < nt && c < nc) {
      const int l = t + 16 * (c >> 2), e = c & 3;
      float v = 0.f;
#pragma unroll
      for (int i = 0; i < kFewWaves; ++i) v += red[i][l][e];
      put_y(a, (size_t)(t0 + t) * a.n + c0 + c, v);
    }
  }
}

hipError_t launch_linear_fp8(const LinearFp8Args& a, hipStream_t s) {
  const dim3 grid((a.n + 15) / 16, (a.N + 15) / 16);
  KernelTimer timer("linear_fp8_few", s);
  if (a.e8m0)
    hipExtLaunchKernelGGL((k_fp8_few<true>), grid, dim3(kFewWaves * kWaveSize), 0, s, timer.start(), timer.stop(), 0, a);
  else
    hipExtLaunchKernelGGL((k_fp8_few<false>), grid, dim3(kFewWaves * kWaveSize), 0, s, timer.start(), timer.stop(), 0, a);
  return hipGetLastError();
}

}  // namespace cats
