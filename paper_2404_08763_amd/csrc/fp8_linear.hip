// Linear layer on e4m3 operands with a scale for each block:
//   y[r, c] = residual[r, c] + sum_b xs[r, b] ws[c / 128, b] sum_{k in b} xq[r, k] wq[c, k]
// with column blocks b of 128.
//
// Weights are the matrix instructions' first operand and rows of x the second, so a
// lane's results are fours of consecutive outputs of one row.  Which of a
// block's columns sit in which lane does not matter as long as both operands agree.
//
// Precision.  The 8-bit matrix instructions cut each product at 2^-13 of the
// power of two in the largest of its group of eight (measured: 256 * 256 beside
// 2^2 gives 65536, beside 2^3 65544): 3e-5 to 5e-5 of the outputs in the mean
// square on rows with outlier channels.  That is below bf16's rounding (2^-8) but
// not fp32's, so they are used where y is bf16 and the products, not the reads,
// bound the call (k_fp8_tile of bf16 outputs).  Elsewhere the values are widened
// to bf16, which holds them exactly, on their way from the registers to the bf16
// instructions, whose sums are exact to fp32.
#include <algorithm>

#include "fp8.hpp"
#include "internal.hpp"
#include "stream.hpp"

namespace cats {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 fp_bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 fp_bf16x2 __attribute__((ext_vector_type(2)));

// Eight e4m3 values as bf16.
__device__ __forceinline__ fp_bf16x8 widen8(uint32_t lo, uint32_t hi) {
  const fp_bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, false);
  const fp_bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, true);
  const fp_bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, false);
  const fp_bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, true);
  return fp_bf16x8{a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y};
}

// A scale as fp32.
__device__ __forceinline__ float e8m0_value(uint32_t e) {
  // (0 is 2^-127, a subnormal, and 255 NaN: both have the uppermost mantissa bit)
  return __uint_as_float((e << 23) | (e - 1u < 254u ? 0u : 0x400000u));
}

// A scale as it is stored, from a buffer, and as a number.
template <bool E8M0> __device__ __forceinline__ uint32_t scale_load(const __amdgpu_buffer_rsrc_t& r, uint32_t at) {
  if constexpr (E8M0) return __builtin_amdgcn_raw_buffer_load_b8(r, (int)at, 0, 0);
  else return __builtin_amdgcn_raw_buffer_load_b32(r, (int)at, 0, 0);
}
template <bool E8M0> __device__ __forceinline__ float scale_value(uint32_t s) {
  return E8M0 ? e8m0_value(s) : __uint_as_float(s);
}

// From two loads of eight rows' whole lines (lane r + 16 g: piece g, or g + 4 for
// r >= 8, of row r % 8, and of row r % 8 + 8) pieces g and g + 4 of row r.
__device__ __forceinline__ void whole_rows(const u32x4 (&l)[2], u32x4 (&v)[2]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {  // row_ror:8, into lanes 8 .. 15 and 0 .. 7 of each 16
    v[0][e] = (uint32_t)__builtin_amdgcn_update_dpp((int)l[0][e], (int)l[1][e], 0x128, 0xf, 0xc, false);
    v[1][e] = (uint32_t)__builtin_amdgcn_update_dpp((int)l[1][e], (int)l[0][e], 0x128, 0xf, 0x3, false);
  }
}

// A value the compiler knows nothing about: that it is the same for all lanes (it
// would move what is loaded through it to a scalar register, and wait for it at
// once), or what addresses made from it could be kept.
__device__ __forceinline__ uint32_t fresh(uint32_t v) {
  asm volatile("" : "+v"(v));
  return v;
}

// Values 8 k .. 8 k + 7 of a lane's 16.
__device__ __forceinline__ fp_bf16x8 widen_part(const u32x4& v, int k) {
  return k ? widen8(v.z, v.w) : widen8(v.x, v.y);
}

__device__ __forceinline__ i32x8 join8(const u32x4& a, const u32x4& b) {
  return i32x8{(int)a.x, (int)a.y, (int)a.z, (int)a.w, (int)b.x, (int)b.y, (int)b.z, (int)b.w};
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

// The same for four consecutive outputs (i a multiple of four).
__device__ __forceinline__ void put_y4(const LinearFp8Args& a, size_t i, f32x4 v) {
  if (a.ybf16) {
    if (a.residual) {
      const uint2 r = *reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(a.residual) + i);
      v += f32x4{__uint_as_float(r.x << 16), __uint_as_float(r.x & 0xffff0000u), __uint_as_float(r.y << 16),
                 __uint_as_float(r.y & 0xffff0000u)};
    }
    *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.y) + i) =
        uint2{bf16_bits(v.x) | (bf16_bits(v.y) << 16), bf16_bits(v.z) | (bf16_bits(v.w) << 16)};
  } else {
    if (a.residual) v += *reinterpret_cast<const f32x4*>(static_cast<const float*>(a.residual) + i);
    *reinterpret_cast<f32x4*>(static_cast<float*>(a.y) + i) = v;
  }
}

// A wave's results through LDS, so that memory sees whole stretches of rows and not
// the 16 bytes of many that a lane holds (303 rows 384 -> 21645 25.7 us, 32.3 without;
// 512 rows 4096 -> 22016 70 and 72): T rows of x by 4 CH outputs, chunk c (four
// outputs) of row t at c ^ (t % 16) of its row's, so that reads and writes of 16 rows
// or chunks hit distinct banks.
template <int CH> __device__ __forceinline__ f32x4& staged(f32x4* stage, int t, int c) {
  return stage[t * CH + (c ^ (t & (CH < 16 ? CH - 1 : 15)))];
}
// Writes them out: to y from row t0 and output c0 on, or to a part's sums.
template <int T, int CH>
__device__ __forceinline__ void put_staged(const LinearFp8Args& a, f32x4* stage, int lane, int t0, int c0, float* part) {
  wait_lds();  // (the wave's own writes)
  if (part || (a.n & 3) == 0) {
#pragma unroll
    for (int i = 0; i < T * CH / kWaveSize; ++i) {
      const int j = i * kWaveSize + lane, t = t0 + j / CH, c = c0 + j % CH * 4;
      if (t >= a.N || c >= a.n) continue;
      const f32x4 v = staged<CH>(stage, j / CH, j % CH);
      if (part) *reinterpret_cast<f32x4*>(part + (size_t)t * a.pitch + c) = v;
      else put_y4(a, (size_t)t * a.n + c, v);
    }
  } else {
#pragma unroll 4
    for (int i = 0; i < T * CH / kWaveSize * 4; ++i) {
      const int j = i * kWaveSize + lane, r = j / (4 * CH), e = j % (4 * CH);
      if (t0 + r < a.N && c0 + e < a.n) put_y(a, (size_t)(t0 + r) * a.n + c0 + e, staged<CH>(stage, r, e >> 2)[e & 3]);
    }
  }
  wait_lds();
}

// Up to 16 rows (32 with NB = 2) whose C column blocks a wave can keep: a block a
// compute unit goes through the tiles of 16 outputs.  Its 16 waves split the column
// blocks (wave w takes w, w + 16, ..), keep x's in registers for all tiles and
// always have the next tile's weights under way, also while the waves add up a
// tile (a barrier that waits for LDS alone).  Bound by the weights' stream: a load
// instruction reads whole 128-byte lines, of eight rows (rows r and r + 8 in two
// loads, then lanes r and r + 8 exchange halves: 4096 -> 22016 of one row 16.6 us,
// 22.1 with 64 bytes of 16 rows).  4096 -> 22016: 5.4 TB/s, launch included, of
// the 7.2 that a large plain read reaches.  Short streams pay the latencies one after the
// other: 4096 -> 6144 is 192 blocks of two tiles, the second asked for when the first is there
// (7.6 us, 3.3 TB/s).  With C = 4 six to nine registers spill (8192 -> 28672 47 us, 5.0 TB/s).
constexpr int kStreamWaves = 16;
template <int C, int NB, bool E8M0, bool RES>
__global__ __launch_bounds__(64 * kStreamWaves) void k_fp8_stream(LinearFp8Args a, int CT) {
  constexpr int W = kStreamWaves;
  __shared__ f32x4 red[2][W][NB][kWaveSize];
  const int tid = threadIdx.x, lane = tid & (kWaveSize - 1);
  const int w = __builtin_amdgcn_readfirstlane(tid / kWaveSize);
  const int r16 = lane & 15, g = lane >> 4;
  const int KB = a.ld / kFp8Block;
  constexpr uint32_t SB = E8M0 ? 1 : 4;
  // x: rows past the last, and column blocks past the last, read as zero
  u32x4 x[C][NB][2];
  float sx[C][NB];
  {
    const __amdgpu_buffer_rsrc_t rx = make_rsrc(a.xq, (uint32_t)a.N * a.ld);
    const __amdgpu_buffer_rsrc_t rsx = make_rsrc(a.xs, (uint32_t)a.N * KB * SB);
#pragma unroll
    for (int u = 0; u < C; ++u) {
      const int b = w + W * u;
      const uint32_t out = b < KB ? 0u : kOOB;
#pragma unroll
      for (int j = 0; j < NB; ++j) {
        const uint32_t at = out + (uint32_t)(16 * j + r16) * a.ld + (uint32_t)b * kFp8Block + g * 16u;
#pragma unroll
        for (int h = 0; h < 2; ++h) x[u][j][h] = ld_buf16(rx, at + 64u * h);
        sx[u][j] = scale_value<E8M0>(scale_load<E8M0>(rsx, out + ((uint32_t)(16 * j + r16) * KB + b) * SB));
      }
    }
  }
  u32x4 wl[C][2];
  uint32_t sw[C];
  const uint32_t woff = (uint32_t)(r16 & 7) * a.ld + (uint32_t)(g + 4 * (r16 >> 3)) * 16u;
  const int ot = tid >> 4, oc = tid & 15;  // the output this thread adds up (256 or 512 of them)
  auto load = [&](int u, int ct) {
    const int b = w + W * u, c0 = ct * 16;
    const bool in = b < KB && ct < CT;
    const __amdgpu_buffer_rsrc_t rw = make_rsrc(a.wq + (size_t)(in ? c0 : 0) * a.ld, (uint32_t)min(16, a.n - (in ? c0 : 0)) * a.ld);
    const uint32_t at = woff + (in ? (uint32_t)b * kFp8Block : kOOB);
    wl[u][0] = ld_buf16_stream(rw, at);
    wl[u][1] = ld_buf16_stream(rw, at + 8u * a.ld);
    const __amdgpu_buffer_rsrc_t rsw =
        make_rsrc(static_cast<const uint8_t*>(a.ws) + (size_t)((in ? c0 : 0) / kFp8Block) * KB * SB, (uint32_t)KB * SB);
    sw[u] = scale_load<E8M0>(rsw, fresh(in ? (uint32_t)b * SB : kOOB));
  };
  const uint32_t yb = a.ybf16 ? 2 : 4, ybytes = (uint32_t)a.N * a.n * yb;
  const __amdgpu_buffer_rsrc_t ry = make_rsrc(a.y, ybytes), rr = make_rsrc(a.residual, ybytes);
  auto y_at = [&](int ct) { return ot < a.N && ct * 16 + oc < a.n ? (uint32_t)(ot * a.n + ct * 16 + oc) * yb : kOOB; };
  int ct = blockIdx.x;
#pragma unroll
  for (int u = 0; u < C; ++u) {
    __builtin_amdgcn_sched_barrier(0);
    load(u, ct);
  }
  __builtin_amdgcn_sched_barrier(0);
  for (int turn = 0; ct < CT; ct += gridDim.x, turn ^= 1) {
    f32x4 acc[NB];
#pragma unroll
    for (int j = 0; j < NB; ++j) acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int u = 0; u < C; ++u) {
      u32x4 v[2];
      fp_bf16x8 wv[4];
      whole_rows(wl[u], v);
#pragma unroll
      for (int k = 0; k < 4; ++k) wv[k] = widen_part(v[k >> 1], k & 1);
      float s[NB];
#pragma unroll
      for (int j = 0; j < NB; ++j) s[j] = sx[u][j] * scale_value<E8M0>(sw[u]);
      // the next tile's loads go out before the products, into the registers that
      // the exchange has just left (into others, a copy would wait for them)
      __builtin_amdgcn_sched_barrier(0);
      load(u, ct + gridDim.x);
      __builtin_amdgcn_sched_barrier(0);
      f32x4 p[NB];
#pragma unroll
      for (int j = 0; j < NB; ++j) p[j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < 4; ++k) {
#pragma unroll
        for (int j = 0; j < NB; ++j)
          p[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wv[k], widen_part(x[u][j][k >> 1], k & 1), p[j], 0, 0, 0);
      }
#pragma unroll
      for (int j = 0; j < NB; ++j) {
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[j][e] = fmaf(p[j][e], s[j], acc[j][e]);
      }
    }
#pragma unroll
    for (int j = 0; j < NB; ++j) red[turn][w][j][lane] = acc[j];
    wait_lds();
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    if (tid < NB * 256) {
      float part[W], v = 0.f;
#pragma unroll
      for (int q = 0; q < W; ++q) part[q] = red[turn][q][ot >> 4][(ot & 15) + 16 * (oc >> 2)][oc & 3];
#pragma unroll
      for (int q = 0; q < W; ++q) v += part[q];
      const uint32_t at = y_at(ct);
      if constexpr (RES)
        v += a.ybf16 ? bf16_value((uint16_t)__builtin_amdgcn_raw_buffer_load_b16(rr, (int)at, 0, 0))
                     : __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(rr, (int)at, 0, 0));
      if (a.ybf16) __builtin_amdgcn_raw_buffer_store_b16((short)bf16_bits(v), ry, (int)at, 0, 0);
      else __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(v), ry, (int)at, 0, 0);
    }
  }
}

template <int C, int NB>
static hipError_t launch_stream(const LinearFp8Args& a, hipStream_t s) {
  const int CT = (a.n + 15) / 16, each = (CT + 255) / 256;
  const dim3 grid((CT + each - 1) / each), block(64 * kStreamWaves);
  KernelTimer timer("linear_fp8_stream", s);
  if (a.e8m0 && a.residual)
    hipExtLaunchKernelGGL((k_fp8_stream<C, NB, true, true>), grid, block, 0, s, timer.start(), timer.stop(), 0, a, CT);
  else if (a.e8m0)
    hipExtLaunchKernelGGL((k_fp8_stream<C, NB, true, false>), grid, block, 0, s, timer.start(), timer.stop(), 0, a, CT);
  else if (a.residual)
    hipExtLaunchKernelGGL((k_fp8_stream<C, NB, false, true>), grid, block, 0, s, timer.start(), timer.stop(), 0, a, CT);
  else
    hipExtLaunchKernelGGL((k_fp8_stream<C, NB, false, false>), grid, block, 0, s, timer.start(), timer.stop(), 0, a, CT);
  return hipGetLastError();
}

// Up to 16 rows of more column blocks than that: a block owns 16 outputs, its
// waves split the column blocks the same way, weights and x two column blocks
// ahead in registers.  14336 -> 4096 of 16 rows 20 us, 11008 -> 4096 of one row 13 (2.9 and 3.4
// TB/s; nothing is fetched twice): a wave has five to seven column blocks, two of them under
// way, between the first loads of its block and the sum over 16 waves.
template <bool E8M0>
__global__ __launch_bounds__(64 * kStreamWaves) void k_fp8_split(LinearFp8Args a) {
  constexpr int W = kStreamWaves, D = 2;
  __shared__ f32x4 red[W][kWaveSize];
  const int tid = threadIdx.x, lane = tid & (kWaveSize - 1);
  const int w = __builtin_amdgcn_readfirstlane(tid / kWaveSize);
  const int r16 = lane & 15, g = lane >> 4;
  const int c0 = blockIdx.x * 16, KB = a.ld / kFp8Block;
  const int nc = min(16, a.n - c0);
  constexpr uint32_t SB = E8M0 ? 1 : 4;
  const __amdgpu_buffer_rsrc_t rw = make_rsrc(a.wq + (size_t)c0 * a.ld, (uint32_t)nc * a.ld);
  const __amdgpu_buffer_rsrc_t rx = make_rsrc(a.xq, (uint32_t)a.N * a.ld);
  const __amdgpu_buffer_rsrc_t rsx = make_rsrc(a.xs, (uint32_t)a.N * KB * SB);
  const __amdgpu_buffer_rsrc_t rsw =
      make_rsrc(static_cast<const uint8_t*>(a.ws) + (size_t)(c0 / kFp8Block) * KB * SB, (uint32_t)KB * SB);
  const uint32_t woff = (uint32_t)(r16 & 7) * a.ld + (uint32_t)(g + 4 * (r16 >> 3)) * 16u;
  const uint32_t xoff = (uint32_t)r16 * a.ld + g * 16u, soff = (uint32_t)r16 * KB * SB;
  u32x4 wl[D][2], x[D][2];
  uint32_t sw[D], sx[D];
  auto load = [&](int u, int b) {
    const uint32_t k = b < KB ? (uint32_t)b * kFp8Block : kOOB, s = b < KB ? (uint32_t)b * SB : kOOB;
    wl[u][0] = ld_buf16_stream(rw, woff + k);
    wl[u][1] = ld_buf16_stream(rw, woff + k + 8u * a.ld);
    x[u][0] = ld_buf16(rx, xoff + k);
    x[u][1] = ld_buf16(rx, xoff + k + 64u);
    sx[u] = scale_load<E8M0>(rsx, soff + s);
    sw[u] = scale_load<E8M0>(rsw, fresh(s));
  };
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int u = 0; u < D; ++u) {
    __builtin_amdgcn_sched_barrier(0);
    load(u, w + u * W);
  }
  __builtin_amdgcn_sched_barrier(0);
  for (int b = w; b < KB; b += D * W) {
#pragma unroll
    for (int u = 0; u < D; ++u) {
      u32x4 v[2];
      whole_rows(wl[u], v);
      const float s = scale_value<E8M0>(sx[u]) * scale_value<E8M0>(sw[u]);
      f32x4 p = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < 4; ++k)
        p = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen_part(v[k >> 1], k & 1), widen_part(x[u][k >> 1], k & 1), p, 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
      load(u, b + (u + D) * W);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e] = fmaf(p[e], s, acc[e]);
    }
  }
  red[w][lane] = acc;
  __syncthreads();
  if (tid < 256) {
    const int t = tid >> 4, c = tid & 15;
    if (t < a.N && c < nc) {
      float v = 0.f;
#pragma unroll
      for (int q = 0; q < W; ++q) v += red[q][t + 16 * (c >> 2)][c & 3];
      put_y(a, (size_t)t * a.n + c0 + c, v);
    }
  }
}

static hipError_t launch_split(const LinearFp8Args& a, hipStream_t s) {
  const dim3 grid((a.n + 15) / 16), block(64 * kStreamWaves);
  KernelTimer timer("linear_fp8_split", s);
  if (a.e8m0)
    hipExtLaunchKernelGGL((k_fp8_split<true>), grid, block, 0, s, timer.start(), timer.stop(), 0, a);
  else
    hipExtLaunchKernelGGL((k_fp8_split<false>), grid, block, 0, s, timer.start(), timer.stop(), 0, a);
  return hipGetLastError();
}

// The scales of four consecutive steps of a row, in registers.  Where fewer than
// four are left, the row's last four; a row of fewer takes load_few.
inline __device__ int scale_start(int st, int KB) { return max(0, min(st, KB - 4)); }
struct __attribute__((packed, aligned(1))) u32u { uint32_t v; };
template <bool E8M0> struct Fp8ScaleRun;
template <> struct Fp8ScaleRun<false> {
  f32x4u v;
  __device__ __forceinline__ void load(const uint8_t* row, int st, int KB) {
    v = *reinterpret_cast<const f32x4u*>(reinterpret_cast<const float*>(row) + scale_start(st, KB));
  }
  __device__ __forceinline__ void load_few(const uint8_t* row, int KB) {
#pragma unroll
    for (int j = 0; j < 4; ++j) v.v[j] = j < KB ? reinterpret_cast<const float*>(row)[j] : 0.f;
  }
  template <bool HW> __device__ __forceinline__ uint32_t get(int j) const { return __float_as_uint(v.v[j]); }
};
template <> struct Fp8ScaleRun<true> {
  uint32_t v;
  __device__ __forceinline__ void load(const uint8_t* row, int st, int KB) {
    v = reinterpret_cast<const u32u*>(row + scale_start(st, KB))->v;
  }
  __device__ __forceinline__ void load_few(const uint8_t* row, int KB) {
    v = 0u;
#pragma unroll
    for (int j = 0; j < 4; ++j) v |= j < KB ? (uint32_t)row[j] << (8 * j) : 0u;
  }
  // the byte for the matrix instruction, or the number
  template <bool HW> __device__ __forceinline__ uint32_t get(int j) const {
    const uint32_t e = (v >> (8 * j)) & 255u;
    return HW ? e : __float_as_uint(e8m0_value(e));
  }
};

constexpr int kTileGroup = 6;  // (whole columns: 5% slower for 2048 rows 4096 -> 22016, 4 and 6 alike)

// Many rows: a block of eight waves owns TM = 256 outputs x TN rows of x.
//
// The waves form two groups, one wave of each on every SIMD, that alternate: while
// one multiplies the operands it holds in registers (step s in phase 2 s, the
// second group's in phase 2 s + 1), the other reads its next ones from LDS; a
// barrier ends each phase.  Memory goes straight to LDS, two buffers of a step
// each, and its loads are sent between products: sent all at once they hold up
// the wave that sends them for as long as the 64 KB of a step take.  The first
// group's outputs are the lower half of the weights (W0), the second's the upper
// (W1), x is everyone's:
//   phase 2 s      first group multiplies s, sends W1 of s + 1 and W0 of s + 2;
//                  second reads W1 and x of s
//   phase 2 s + 1  second group multiplies s, sends x of s + 2; first reads W0
//                  and x of s + 1
// so each part is overwritten once its readers are through with it, and has one
// to three phases to arrive.  (All of a step's loads as its reads begin: 2048
// rows 4096 -> 22016 in bf16 292 us with fp32 scales and 199 with E8M0, in place of
// 211 and 162; one group of waves, multiplying and reading by turns in each: 352 and 256.)
//
// bf16 outputs: 256 x 256, the 8-bit instructions, one a tile and step, E8M0 scales
// applied by them, fp32 ones on the vector ALUs, whose sums lie between the
// products.  Bound by what of the reading phases, loads and sums does not overlap with the
// products: of a busy compute unit's cycles the matrix cores work 0.66 with E8M0 scales and
// 0.43 with fp32 ones, the vector ALUs 0.35 and 0.40 (fp32 scales are 128 multiply-adds a wave
// and step, half as long as its 32 products, and use products three instructions
// back).  4096 rows 14336 -> 4096 172 to 175 us, 2.8 PFLOP/s (fp32 scales 225 us, 2.1), where the
// library's product of one scale for all takes 153.
// EXACT, fp32 outputs: 256 x 128, the bf16 instructions; operands are widened in the
// reading phase, under the other group's products (in the multiplying phase:
// 410 us).  The same size 371 to 412 us by the card, 1.17 to 1.30 PFLOP/s; the library's bf16 product, whose
// operands have twice the bytes, takes 305.  Tiles of 32 x 32 had the same time or more.
template <bool EXACT> struct TileGeom;
template <> struct TileGeom<false> {
  static constexpr int WM = 2, WN = 4, MI = 8, NB = 4;  // waves, and 16 x 16 tiles of a wave
};
template <> struct TileGeom<true> {
  static constexpr int WM = 4, WN = 2, MI = 4, NB = 4;
};

template <bool EXACT, bool E8M0>
__global__ __launch_bounds__(512, 2) void k_fp8_tile(LinearFp8Args a, int MT, int NT) {
  typedef TileGeom<EXACT> G;
  constexpr int MI = G::MI, NB = G::NB;
  constexpr int TM = 16 * MI * G::WM, TN = 16 * NB * G::WN;
  static_assert(TM == 256 && MI * G::WM / 2 == 8, "a group's outputs are 128");
  constexpr int WQ = 4, XQ = TN / 32;  // 1 KB loads (8 rows) of a wave: of a half of the weights, of x
  constexpr bool HW = E8M0 && !EXACT;   // scales applied by the matrix instruction
  // one array per part in flight: the compiler then sees that a load into one
  // does not touch what is read from another
  __shared__ __attribute__((aligned(1024))) uint8_t wlo0[128 * 128], wlo1[128 * 128], whi0[128 * 128], whi1[128 * 128];
  __shared__ __attribute__((aligned(1024))) uint8_t xb0[TN * 128], xb1[TN * 128];
  // scales of eight steps: of the tile's rows, and of the weights' two blocks
  __shared__ uint32_t ring[8][TN + 2];
  const int tid = threadIdx.x, lane = tid & (kWaveSize - 1);
  const int w = __builtin_amdgcn_readfirstlane(tid / kWaveSize);
  const int wm = w / G::WN, wn = w % G::WN, grp = w / 4, gw = w % 4;
  const int r16 = lane & 15, g = lane >> 4;

  // Each XCD takes a consecutive run of tiles, in columns of kTileGroup tiles of
  // outputs, so that the 32 tiles an XCD works on share operands both ways.
  const int total = MT * NT;
  const int xcd = blockIdx.x % 8, ix = blockIdx.x / 8, per = total / 8, rem = total % 8;
  const int tile = xcd * per + (xcd < rem ? xcd : rem) + ix;
  const int first = tile / (kTileGroup * NT) * kTileGroup, in = tile - first * NT;
  const int high = min(kTileGroup, MT - first);
  const int c0 = (first + in % high) * TM, t0 = in / high * TN;
  const int KB = a.ld / kFp8Block;
  const int nc = min(TM, a.n - c0), nt = min(TN, a.N - t0);
  const __amdgpu_buffer_rsrc_t rw = make_rsrc(a.wq + (size_t)c0 * a.ld, (uint32_t)nc * a.ld);
  const __amdgpu_buffer_rsrc_t rx = make_rsrc(a.xq + (size_t)t0 * a.ld, (uint32_t)nt * a.ld);

  // Piece c (16 bytes) of row r lies at slot c ^ (r & 7) of its 128 bytes, so
  // that eight lanes that read the same piece of eight rows hit distinct banks.
  // Rows past the tile's last lie past the buffer and read as zero, and so do
  // steps past the last.
  const uint32_t loff = (uint32_t)((lane & 7) ^ (lane >> 3)) * 16u;
  const uint32_t woff = (uint32_t)(8 * WQ * gw + (lane >> 3)) * a.ld + loff;
  const uint32_t xoff = (uint32_t)(8 * XQ * gw + (lane >> 3)) * a.ld + loff;
  auto at = [&](int st) { return st < KB ? (uint32_t)st * kFp8Block : kOOB; };
  auto send_w = [&](uint8_t* dst, int half, int st) {
#pragma unroll
    for (int q = 0; q < WQ; ++q)
      dma16(rw, dst + (WQ * gw + q) * 1024, fresh(woff) + (at(st) + (128u * half + 8u * q) * a.ld));
  };
  auto send_x = [&](uint8_t* dst, int st) {
#pragma unroll
    for (int q = 0; q < XQ; ++q) dma16(rx, dst + (XQ * gw + q) * 1024, fresh(xoff) + (at(st) + 8u * q * a.ld));
  };

  // Scales: each wave of the first group fetches those of 64 of the tile's rows and
  // of the two weight blocks, four steps at a time (some lanes the same), and puts
  // them into LDS a step later.  Not a load where they are used: its wait would be
  // one for the operands under way too (2048 rows 4096 -> 22016: 351 us against 292).
  constexpr uint32_t SB = E8M0 ? 1 : 4;
  typedef Fp8ScaleRun<E8M0> Run;
  const int wb = min(c0 / kFp8Block + (lane >> 5), (a.n - 1) / kFp8Block), srow = (64 * gw + lane) % TN;
  const uint8_t* swp = static_cast<const uint8_t*>(a.ws) + (size_t)wb * KB * SB;
  const uint8_t* sxp = static_cast<const uint8_t*>(a.xs) + (size_t)min(t0 + srow, a.N - 1) * KB * SB;
  Run px, pw;
  auto fetch_scales = [&](int st) {
    px.load(sxp, st, KB);
    pw.load(swp, st, KB);
  };
  auto put_scales = [&](int st) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int slot = (scale_start(st, KB) + j) & 7;
      const uint32_t row = fresh((uint32_t)(64 * gw + lane) % TN);
      ring[slot][row] = px.template get<HW>(j);
      ring[slot][TN + (lane >> 5)] = pw.template get<HW>(j);
    }
  };
  uint32_t xe[NB], we;
  fp_bf16x8 xw[EXACT ? NB : 1][4], ww[EXACT ? MI : 1][4];

  f32x4 acc[MI][NB];
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int b = 0; b < NB; ++b) acc[i][b] = f32x4{0.f, 0.f, 0.f, 0.f};
  u32x4 fa[MI][2], fb[NB][2];
  const uint32_t fslot = (uint32_t)(g ^ (r16 & 7)) * 16u;
  const uint32_t abase = (uint32_t)(16 * MI * (wm % (G::WM / 2)) + r16) * 128u + fslot, bbase = (uint32_t)(16 * NB * wn + r16) * 128u + fslot;
  auto read = [&](const uint8_t* sw, const uint8_t* sx, int st) {
    const uint32_t* ss = ring[st & 7];
    const uint32_t rb = fresh((uint32_t)(16 * NB * wn + r16));
#pragma unroll
    for (int b = 0; b < NB; ++b) xe[b] = ss[rb + 16 * b];
    we = ss[TN + grp];
    const uint8_t *pb = sx + fresh(bbase), *pbx = sx + fresh(bbase ^ 64u);
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      fb[b][0] = *reinterpret_cast<const u32x4*>(pb + b * 2048);
      fb[b][1] = *reinterpret_cast<const u32x4*>(pbx + b * 2048);
    }
    const uint8_t *pa = sw + fresh(abase), *pax = sw + fresh(abase ^ 64u);
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      fa[i][0] = *reinterpret_cast<const u32x4*>(pa + i * 2048);
      fa[i][1] = *reinterpret_cast<const u32x4*>(pax + i * 2048);
    }
    if constexpr (EXACT) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
#pragma unroll
        for (int b = 0; b < NB; ++b) xw[b][k] = widen_part(fb[b][k >> 1], k & 1);
#pragma unroll
        for (int i = 0; i < MI; ++i) ww[i][k] = widen_part(fa[i][k >> 1], k & 1);
      }
    }
  };
  // The products of outputs I0 .. I1 - 1 of the wave's MI, and between them SENDS
  // loads, sent by `send` before.
  float sc[NB];
  auto multiply = [&](auto i0, auto i1, auto sends) {
    constexpr int I0 = decltype(i0)::v, I1 = decltype(i1)::v, SENDS = decltype(sends)::v;
    constexpr int TILES = (I1 - I0) * NB;
    if constexpr (I0 == 0 && !HW) {
#pragma unroll
      for (int b = 0; b < NB; ++b) sc[b] = __uint_as_float(xe[b]) * __uint_as_float(we);
    }
    if constexpr (EXACT) {
#pragma unroll
      for (int i = I0; i < I1; ++i) {
        f32x4 p[NB];
#pragma unroll
        for (int b = 0; b < NB; ++b) p[b] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
#pragma unroll
          for (int b = 0; b < NB; ++b) p[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ww[i][k], xw[b][k], p[b], 0, 0, 0);
        }
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[i][b][e] = fmaf(p[b][e], sc[b], acc[i][b][e]);
      }
      // the sums of one row of tiles among the products of the next
      if (I0 == 0) __builtin_amdgcn_sched_group_barrier(0x002, NB, 0);
#pragma unroll
      for (int k = 0; k < 4 * TILES; ++k) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        if (k >= 4 * NB) __builtin_amdgcn_sched_group_barrier(0x002, 1, 0);
        if (SENDS > 0 && k % (4 * TILES / SENDS) == 0) __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);
      }
      __builtin_amdgcn_sched_group_barrier(0x002, 4 * NB, 0);
    } else {
#pragma unroll
      for (int i = I0; i < I1; ++i)
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          const i32x8 wv = join8(fa[i][0], fa[i][1]), xv = join8(fb[b][0], fb[b][1]);
          if constexpr (HW) {
            acc[i][b] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wv, xv, acc[i][b], 0, 0, 0, (int)we, 0, (int)xe[b]);
          } else {
            const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
            const f32x4 p = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wv, xv, zero, 0, 0, 0, 0, 0, 0);
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[i][b][e] = fmaf(p[e], sc[b], acc[i][b][e]);
          }
        }
      if constexpr (HW) {
#pragma unroll
        for (int k = 0; k < TILES; ++k) {
          __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
          if (SENDS > 0 && k % (TILES / SENDS) == 0) __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);
        }
      } else {
        // a few products ahead of the sums that use them
        if (I0 == 0) __builtin_amdgcn_sched_group_barrier(0x002, NB, 0);
        __builtin_amdgcn_sched_group_barrier(0x008, 3, 0);
#pragma unroll
        for (int k = 0; k < TILES - 3; ++k) {
          __builtin_amdgcn_sched_group_barrier(0x002, 4, 0);
          __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
          if (SENDS > 0 && k % (TILES / SENDS) == 0) __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x002, 12, 0);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  auto phase_end = [&]() {
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  };

  constexpr Const<0> none;
  constexpr Const<MI / 2> half;
  constexpr Const<MI> all;
  // A step of the first group, FETCH: with the loads of the scales of steps st + 4
  // on, which step st + 1 (PUT) puts into the ring.  Loads complete in order: with
  // st's W1 there, st + 1's W0 (and the two of scales) may be under way; with that
  // there too, the parts sent in this step.
  auto first_step = [&](uint8_t* wlo, uint8_t* next_whi, const uint8_t* xb, int st, auto fetch, auto put) {
    constexpr int F = decltype(fetch)::v ? 2 : 0;
    if constexpr (decltype(fetch)::v) fetch_scales(st + 4);
    read(wlo, xb, st);
    wait_vm<WQ + F>();
    if constexpr (decltype(put)::v) put_scales(st + 3);
    wait_lds();
    phase_end();
    __builtin_amdgcn_s_setprio(1);  // (products before the other group's widening: up to 3%)
    send_w(next_whi, 1, st + 1);
    if constexpr (EXACT) {
      asm volatile("" ::: "memory");  // (in this order)
      send_w(wlo, 0, st + 2);
      multiply(none, all, Const<2 * WQ>());
    } else {
      multiply(none, half, Const<WQ>());
      send_w(wlo, 0, st + 2);
      multiply(half, all, Const<WQ>());
    }
    __builtin_amdgcn_s_setprio(0);
    wait_vm<2 * WQ + F>();
    phase_end();
  };
  auto second_step = [&](const uint8_t* whi, uint8_t* xb, int st) {
    read(whi, xb, st);
    wait_lds();
    wait_vm<0>();
    phase_end();
    __builtin_amdgcn_s_setprio(1);
    send_x(xb, st + 2);
    if constexpr (EXACT) {
      multiply(none, all, Const<XQ>());
    } else {
      multiply(none, half, Const<XQ>());
      multiply(half, all, none);
    }
    __builtin_amdgcn_s_setprio(0);
    phase_end();
  };
  constexpr Const<1> yes;
  int st = 0;
  if (grp == 0) {
    if (KB >= 4) {
      fetch_scales(0);
    } else {
      px.load_few(sxp, KB);
      pw.load_few(swp, KB);
    }
    send_w(wlo0, 0, 0);
    send_w(whi0, 1, 0);
    __builtin_amdgcn_sched_barrier(0);
    send_w(wlo1, 0, 1);
    __builtin_amdgcn_sched_barrier(0);
    wait_vm<WQ>();
    put_scales(0);
    wait_lds();
    phase_end();
    for (; st + 4 <= KB; st += 4) {
      first_step(wlo0, whi1, xb0, st, yes, none);
      first_step(wlo1, whi0, xb1, st + 1, none, yes);
      first_step(wlo0, whi1, xb0, st + 2, none, none);
      first_step(wlo1, whi0, xb1, st + 3, none, none);
    }
    if (st < KB) first_step(wlo0, whi1, xb0, st, none, none);
    if (st + 1 < KB) first_step(wlo1, whi0, xb1, st + 1, none, none);
    if (st + 2 < KB) first_step(wlo0, whi1, xb0, st + 2, none, none);
    phase_end();
  } else {
    send_x(xb0, 0);
    __builtin_amdgcn_sched_barrier(0);
    send_x(xb1, 1);
    __builtin_amdgcn_sched_barrier(0);
    wait_vm<XQ>();
    phase_end();
    phase_end();
    for (; st + 2 <= KB; st += 2) {
      second_step(whi0, xb0, st);
      second_step(whi1, xb1, st + 1);
    }
    if (st < KB) second_step(whi0, xb0, st);
  }
  wait_vm<0>();  // no load is on its way to LDS when the block ends

  wait_lds();
  __builtin_amdgcn_s_barrier();  // every wave is through with the operands in LDS
  asm volatile("" ::: "memory");
  // D[i][j] sits in lane j + 16 (i / 4), register i % 4.
  constexpr int CH = 4 * MI;
  f32x4* stage = reinterpret_cast<f32x4*>(w < 2 ? wlo0 : w < 4 ? wlo1 : w < 6 ? whi0 : whi1) + (w & 1) * 512;
#pragma unroll
  for (int b = 0; b < NB; ++b) {
#pragma unroll
    for (int i = 0; i < MI; ++i) staged<CH>(stage, r16, 4 * i + g) = acc[i][b];
    put_staged<16, CH>(a, stage, lane, t0 + 16 * NB * wn + 16 * b, c0 + 16 * MI * wm, nullptr);
  }
}

template <bool EXACT>
static hipError_t launch_tile(const LinearFp8Args& a, hipStream_t s) {
  typedef TileGeom<EXACT> G;
  constexpr int TM = 16 * G::MI * G::WM, TN = 16 * G::NB * G::WN;
  const int MT = (a.n + TM - 1) / TM, NT = (a.N + TN - 1) / TN;
  KernelTimer timer(EXACT ? "linear_fp8_tile_f32" : "linear_fp8_tile", s);
  if (a.e8m0)
    hipExtLaunchKernelGGL((k_fp8_tile<EXACT, true>), dim3(MT * NT), dim3(512), 0, s, timer.start(), timer.stop(), 0, a, MT, NT);
  else
    hipExtLaunchKernelGGL((k_fp8_tile<EXACT, false>), dim3(MT * NT), dim3(512), 0, s, timer.start(), timer.stop(), 0, a, MT, NT);
  return hipGetLastError();
}

// Rows between: a block of four waves owns 128 outputs x TN rows of x and one of S
// parts of the column blocks; parts meet in k_fp8_join.  Values are widened
// between LDS and the bf16 instructions for every output type.  A step's operands
// go from memory straight to LDS while the step before is multiplied, one barrier
// a step.  Bound by a step's chain of reads, widening and products (0.9, 1.0 and 1.2 us of
// a lone block of 32, 64 and 128 rows, 0.5, 0.6 and 1.0 each of several on a compute unit),
// by the parts' traffic and the second launch where there are many parts: 300 rows
// 4096 -> 4096 23 us, 101 rows 7001 -> 2857 17, 312 rows 256 -> 3106 6.7.
template <int TN> struct MidGeom;
template <> struct MidGeom<128> { static constexpr int WN = 2, MI = 2, NB = 2; };  // waves along x's rows, 32 x 32 tiles of a wave
template <> struct MidGeom<64> { static constexpr int WN = 2, MI = 2, NB = 1; };
template <> struct MidGeom<32> { static constexpr int WN = 1, MI = 1, NB = 1; };

template <int TN, bool E8M0>
__global__ __launch_bounds__(256, TN == 128 ? 2 : 3) void k_fp8_mid(LinearFp8Args a, int MT, int NT) {
  typedef MidGeom<TN> G;
  constexpr int T = 128, MI = G::MI, NB = G::NB, XQ = TN / 32;
  __shared__ __attribute__((aligned(1024))) uint8_t w0[T * 128], w1[T * 128], x0[TN * 128], x1[TN * 128];
  __shared__ float ring[8][TN + 1];  // scales of eight steps: of the tile's rows, and the weight's
  const int tid = threadIdx.x, lane = tid & (kWaveSize - 1);
  const int w = __builtin_amdgcn_readfirstlane(tid / kWaveSize);
  const int wm = w / G::WN, wn = w % G::WN;
  const int r32 = lane & 31, h = lane >> 5;
  // blocks of one weight tile (and part) run on one XCD, one after the other
  const int ix = blockIdx.x / 8, unit = (ix / NT) * 8 + blockIdx.x % 8;
  if (unit >= MT * a.S) return;
  const int part = unit / MT, c0 = (unit - part * MT) * T, t0 = ix % NT * TN;
  const int KB = a.ld / kFp8Block;
  const int first = (int)((int64_t)part * KB / a.S), last = (int)((int64_t)(part + 1) * KB / a.S);
  const int nc = min(T, a.n - c0), nt = min(TN, a.N - t0);
  const __amdgpu_buffer_rsrc_t rw = make_rsrc(a.wq + (size_t)c0 * a.ld, (uint32_t)nc * a.ld);
  const __amdgpu_buffer_rsrc_t rx = make_rsrc(a.xq + (size_t)t0 * a.ld, (uint32_t)nt * a.ld);
  // (LDS layout, rows and steps past the last: as k_fp8_tile)
  const uint32_t loff = (uint32_t)((lane & 7) ^ (lane >> 3)) * 16u;
  const uint32_t woff = (uint32_t)(32 * w + (lane >> 3)) * a.ld + loff, xoff = (uint32_t)(8 * XQ * w + (lane >> 3)) * a.ld + loff;
  auto send = [&](uint8_t* sw, uint8_t* sx, int st) {
    const uint32_t k = st < last ? (uint32_t)st * kFp8Block : kOOB;
#pragma unroll
    for (int q = 0; q < 4; ++q) dma16(rw, sw + (4 * w + q) * 1024, fresh(woff) + (k + 8u * q * a.ld));
#pragma unroll
    for (int q = 0; q < XQ; ++q) dma16(rx, sx + (XQ * w + q) * 1024, fresh(xoff) + (k + 8u * q * a.ld));
  };
  // Scales, four steps at a time, into registers and a step later into LDS.
  constexpr uint32_t SB = E8M0 ? 1 : 4;
  const int srow = tid & (TN - 1);
  const uint8_t* swp = static_cast<const uint8_t*>(a.ws) + (size_t)(c0 / kFp8Block) * KB * SB;
  const uint8_t* sxp = static_cast<const uint8_t*>(a.xs) + (size_t)min(t0 + srow, a.N - 1) * KB * SB;
  Fp8ScaleRun<E8M0> px, pw;
  auto fetch_scales = [&](int st) {
    px.load(sxp, st, KB);
    pw.load(swp, st, KB);
  };
  auto put_scales = [&](int st) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float* slot = ring[(scale_start(st, KB) + j) & 7];
      slot[srow] = __uint_as_float(px.template get<false>(j));
      slot[TN] = __uint_as_float(pw.template get<false>(j));
    }
  };

  f32x16 acc[MI][NB];
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][b][e] = 0.f;
  // Lane (r32, h) holds pieces h, h + 2, h + 4, h + 6 of its row: 16 columns each,
  // two instructions' depth of eight.
  const uint32_t fslot = (uint32_t)(h ^ (r32 & 7)) * 16u;
  const uint32_t abase = (uint32_t)(32 * MI * wm + r32) * 128u + fslot, bbase = (uint32_t)(32 * NB * wn + r32) * 128u + fslot;
  auto step = [&](uint8_t* sw, uint8_t* sx, uint8_t* nw, uint8_t* nx, int st, auto fetch, auto put) {
    wait_vm<0>();
    if constexpr (decltype(put)::v) put_scales(st + 3);
    wait_lds();
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    u32x4 fb[NB][4], fa[MI][4];
    float sc[NB];
    const float* ss = ring[st & 7];
    const float swv = ss[TN];
#pragma unroll
    for (int b = 0; b < NB; ++b) sc[b] = ss[32 * NB * wn + 32 * b + r32];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
#pragma unroll
      for (int b = 0; b < NB; ++b) fb[b][q] = *reinterpret_cast<const u32x4*>(sx + (fresh(bbase) ^ (32u * q)) + b * 4096);
#pragma unroll
      for (int i = 0; i < MI; ++i) fa[i][q] = *reinterpret_cast<const u32x4*>(sw + (fresh(abase) ^ (32u * q)) + i * 4096);
    }
    // (the loads behind the reads: a read behind a load waits for it)
    __builtin_amdgcn_sched_barrier(0);
    send(nw, nx, st + 1);
    if constexpr (decltype(fetch)::v) fetch_scales(st + 4);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int b = 0; b < NB; ++b) sc[b] *= swv;
    fp_bf16x8 xw[NB][8];
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        xw[b][2 * q] = widen_part(fb[b][q], 0);
        xw[b][2 * q + 1] = widen_part(fb[b][q], 1);
      }
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      f32x16 p[NB];
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int e = 0; e < 16; ++e) p[b][e] = 0.f;
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const fp_bf16x8 wv = widen_part(fa[i][k >> 1], k & 1);
#pragma unroll
        for (int b = 0; b < NB; ++b) p[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wv, xw[b][k], p[b], 0, 0, 0);
      }
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[i][b][e] = fmaf(p[b][e], sc[b], acc[i][b][e]);
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  constexpr Const<1> yes;
  constexpr Const<0> none;
  if (KB >= 4) {
    fetch_scales(first);
  } else {
    px.load_few(sxp, KB);
    pw.load_few(swp, KB);
  }
  send(w0, x0, first);
  put_scales(first);
  int st = first;
  for (; st + 4 <= last; st += 4) {
    step(w0, x0, w1, x1, st, yes, none);
    step(w1, x1, w0, x0, st + 1, none, yes);
    step(w0, x0, w1, x1, st + 2, none, none);
    step(w1, x1, w0, x0, st + 3, none, none);
  }
  if (st < last) step(w0, x0, w1, x1, st, none, none);
  if (st + 1 < last) step(w1, x1, w0, x0, st + 1, none, none);
  if (st + 2 < last) step(w0, x0, w1, x1, st + 2, none, none);
  wait_vm<0>();  // no load is on its way to LDS when the block ends

  wait_lds();
  __builtin_amdgcn_s_barrier();  // every wave is through with the operands in LDS
  asm volatile("" ::: "memory");
  // D[i][j] sits in lane j + 32 ((i / 4) % 2), register i % 4 + 4 (i / 8).
  constexpr int CH = 8 * MI;
  f32x4* stage = reinterpret_cast<f32x4*>(w < 2 ? w0 : w1) + (w & 1) * 512;
  float* part_out = a.S > 1 ? a.partial + (size_t)part * a.N * a.pitch : nullptr;
#pragma unroll
  for (int b = 0; b < NB; ++b) {
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        staged<CH>(stage, r32, 8 * i + 2 * q + h) =
            f32x4{acc[i][b][4 * q], acc[i][b][4 * q + 1], acc[i][b][4 * q + 2], acc[i][b][4 * q + 3]};
    put_staged<32, CH>(a, stage, lane, t0 + 32 * NB * wn + 32 * b, c0 + 32 * MI * wm, part_out);
  }
}

// y = residual + the parts' sums, in part order.
__global__ __launch_bounds__(256) void k_fp8_join(LinearFp8Args a) {
  const uint32_t per = (uint32_t)a.pitch / 4, i = blockIdx.x * 256u + threadIdx.x;
  if (i >= (uint32_t)a.N * per) return;
  const uint32_t t = i / per, c = (i - t * per) * 4u;
  const size_t stride = (size_t)a.N * a.pitch;
  const float* p = a.partial + (size_t)t * a.pitch + c;
  f32x4 v = *reinterpret_cast<const f32x4*>(p);
#pragma unroll 4
  for (int s = 1; s < a.S; ++s) v += *reinterpret_cast<const f32x4*>(p + s * stride);
  const size_t at = (size_t)t * a.n + c;
  if ((a.n & 3) == 0) {
    put_y4(a, at, v);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (c + e < (uint32_t)a.n) put_y(a, at + e, v[e]);
  }
}

template <int TN>
static hipError_t launch_mid(const LinearFp8Args& a, hipStream_t s) {
  const int MT = (a.n + 127) / 128, NT = (a.N + TN - 1) / TN;
  const dim3 grid((unsigned)((MT * a.S + 7) / 8 * 8) * (unsigned)NT);
  {
    KernelTimer timer("linear_fp8_mid", s);
    if (a.e8m0)
      hipExtLaunchKernelGGL((k_fp8_mid<TN, true>), grid, dim3(256), 0, s, timer.start(), timer.stop(), 0, a, MT, NT);
    else
      hipExtLaunchKernelGGL((k_fp8_mid<TN, false>), grid, dim3(256), 0, s, timer.start(), timer.stop(), 0, a, MT, NT);
  }
  if (a.S > 1) {
    KernelTimer timer("linear_fp8_join", s);
    hipExtLaunchKernelGGL(k_fp8_join, dim3(((unsigned)a.N * (a.pitch / 4) + 255) / 256), dim3(256), 0, s, timer.start(), timer.stop(), 0, a);
  }
  return hipGetLastError();
}

// How a call is run.
enum LinearPath { kStreamPath, kSplitPath, kMidPath, kTilePath };
struct LinearPlan {
  LinearPath path;
  int rows;  // of x, of a tile (stream and mid)
  int S;     // parts of the reduction
};

// What a column block's step takes, in 1/100 us, measured on 112 steps with the weights
// from memory: of a round of 256 tiles (one a compute unit) of the two-group kernel by
// output and type of scale; of k_fp8_mid's blocks of 32, 64 and 128 rows, one on a compute
// unit and each of several, and what larger tiles take longer to start and end.
constexpr int kTileStepF32 = 172, kTileStepE8m0 = 160, kTileStep = 210;
constexpr int kMidParts[] = {1, 2, 3, 4, 5, 6, 8, 12, 16, 24};
constexpr int kMidBlocks = 768;  // most blocks of a call in parts: three a compute unit
inline bool mid_parts_ok(int S, int KB, int64_t blocks) { return S == 1 || (2 * S <= KB && blocks * S <= kMidBlocks); }
constexpr int kMidStepOne[3] = {95, 97, 123}, kMidStepEach[3] = {46, 62, 99}, kMidStart[3] = {0, 40, 100};
// The second launch; bytes of the parts' sums, written and read, and of weights, which two
// blocks that run beside each other both fetch, in 1/100 us.
constexpr int kJoin = 400, kJoinBytes = 40000, kFetchBytes = 55000;

// Up to 16 rows, and up to 32 of no more than 32 column blocks: the streaming kernel
// (32 rows 4096 -> 22016 22 us against 26 of the 128 x 32 tiles; 1 row 8192 -> 28672 46, split
// 50), unless a wave had more than four column blocks of x to keep.
// Above: what takes least by the steps and rounds of its blocks, of 128 outputs x 32, 64
// or 128 rows in S parts and of the two-group kernel, whose larger tiles need a filled
// chip (us, weights from memory; 128 rows from 65 on, in parts of six column blocks and more,
// and this rule: 304 rows 3240 -> 286 14.4 / 10.3; 96 rows 1128 -> 3304 14.0 / 8.5; 312 rows
// 256 -> 3106 10.4 / 6.7; 300 rows 4096 -> 4096 29.5 / 24.1; 200 rows 14336 -> 512 18.0 / 15.2;
// 1743 rows 9346 -> 852 51.8 / 54.3.  Two-group / 128 x 128: 512
// rows 4096 -> 22016, bf16 71 / 102, fp32 111 / 104; 256 rows, bf16 with fp32 scales 70 / 62,
// with E8M0 52 / 62; 2048 rows 4096 -> 4096, fp32 60 / 74; 1024 rows 11008 -> 4096, fp32
// 128 / 102; 4096 rows 512 -> 4096, bf16 21 / 34).
static LinearPlan linear_plan(int N, int n, int KB, bool bf16, bool e8m0) {
  const int each = (KB + kStreamWaves - 1) / kStreamWaves;  // column blocks of a wave
  if (N <= 16) return {each <= 4 ? kStreamPath : kSplitPath, 16, 1};
  if (N <= 32 && each <= 2) return {kStreamPath, 32, 1};
  LinearPlan best = {kMidPath, 0, 1};
  int64_t least = INT64_MAX;
  const int64_t columns = (n + 127) / 128;
  for (int i = 0; i < 3; ++i) {
    const int rows = 32 << i;
    if (i > 0 && rows >= 2 * N) break;
    const int64_t high = (N + rows - 1) / rows, blocks = columns * high;
    const int64_t fetch = columns * KB * (128 * 128) * (high > 1 ? 2 : 1);
    for (const int S : kMidParts) {
      if (!mid_parts_ok(S, KB, blocks)) break;
      const int64_t all = blocks * S, rounds = (all + 255) / 256;
      // (a last round that fills part of the chip goes with less traffic beside it)
      const int64_t step = std::max<int64_t>(kMidStepOne[i], kMidStepEach[i] * (3 * 256 * rounds + all) / 1024);
      const int64_t steps = std::max((KB + S - 1) / S * step, fetch / kFetchBytes);
      const int64_t us = kMidStart[i] + steps + (S > 1 ? kJoin + (int64_t)S * N * n * 8 / kJoinBytes : 0);
      if (us < least) least = us, best.rows = rows, best.S = S;
    }
  }
  const int wide = bf16 ? 256 : 128;
  const int64_t tiles = (int64_t)((n + 255) / 256) * ((N + wide - 1) / wide);
  const int step = !bf16 ? kTileStepF32 : e8m0 ? kTileStepE8m0 : kTileStep;
  if (N > 64 && KB * step * ((tiles + 255) / 256) < least) return {kTilePath, wide, 1};
  return best;
}

static int partial_pitch(int n) { return (n + 3) / 4 * 4; }

size_t linear_fp8_partial_bytes(int N, int n, int KB, bool bf16, bool e8m0) {
  const LinearPlan p = linear_plan(N, n, KB, bf16, e8m0);
  return p.S > 1 ? (size_t)p.S * N * partial_pitch(n) * sizeof(float) : 0;
}

// The plan's own parts go up and down with N and n (4096 -> 4096: 16 MB at 256 rows, none
// at 512), so the bound is on what any of the smaller calls may take: the most parts that
// KB allows, and kMidBlocks blocks of 128 outputs and the most rows that N allows.
size_t linear_fp8_partial_most(int N, int n, int KB) {
  if (N <= 16 || (N <= 32 && KB <= 2 * kStreamWaves)) return 0;
  int parts = 1;
  for (const int S : kMidParts) parts = mid_parts_ok(S, KB, 1) ? S : parts;
  if (parts == 1) return 0;
  const int rows = N <= 32 ? 32 : N <= 64 ? 64 : 128;
  return std::min((size_t)parts * N * partial_pitch(n), (size_t)kMidBlocks * 128 * rows) * sizeof(float);
}

hipError_t launch_linear_fp8(LinearFp8Args a, hipStream_t s) {
  const int KB = a.ld / kFp8Block;
  const LinearPlan p = linear_plan(a.N, a.n, KB, a.ybf16 != 0, a.e8m0 != 0);
  a.S = p.S;
  a.pitch = partial_pitch(a.n);
  switch (p.path) {
    case kStreamPath:
      if (p.rows == 32) return KB <= 16 ? launch_stream<1, 2>(a, s) : launch_stream<2, 2>(a, s);
      if (KB <= 16) return launch_stream<1, 1>(a, s);
      if (KB <= 32) return launch_stream<2, 1>(a, s);
      return KB <= 48 ? launch_stream<3, 1>(a, s) : launch_stream<4, 1>(a, s);
    case kSplitPath: return launch_split(a, s);
    case kMidPath: return p.rows == 32 ? launch_mid<32>(a, s) : p.rows == 64 ? launch_mid<64>(a, s) : launch_mid<128>(a, s);
    case kTilePath: return a.ybf16 ? launch_tile<false>(a, s) : launch_tile<true>(a, s);
  }
  return hipErrorInvalidValue;
}

}  // namespace cats
