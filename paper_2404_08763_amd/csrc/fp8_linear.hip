// Linear layer on e4m3 operands with a scale for each block:
//   y[r, c] = residual[r, c] + sum_b xs[r, b] ws[c / 128, b] sum_{k in b} xq[r, k] wq[c, k]
// with blocks b of 128 columns: just one matrix instruction's depth.
#include "fp8.hpp"
#include "internal.hpp"
#include "stream.hpp"

namespace cats {

typedef int i32x8 __attribute__((ext_vector_type(8)));
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
__device__ __forceinline__ float e8m0_value(uint32_t e) {
  return e == 255u ? __uint_as_float(0x7fc00000u) : e == 0u ? 0x1p-127f : __uint_as_float(e << 23);
}
template <bool E8M0> __device__ __forceinline__ float scale_at(const void* s, size_t i) {
  return E8M0 ? e8m0_value(static_cast<const uint8_t*>(s)[i]) : static_cast<const float*>(s)[i];
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

// Many rows: a block of eight waves owns TM outputs x TN rows of x.
//
// The waves form two groups, one wave of each on every SIMD, that alternate: while
// one multiplies the operands it holds in registers, the other reads its next
// ones from LDS (a barrier ends each such phase), so the matrix cores never wait
// for a read of the wave they work for.  Memory goes straight to LDS
// two phases ahead: step s + 2 overwrites step s once both groups have read it.
template <bool PREC> struct TileGeom;
template <> struct TileGeom<false> {
  static constexpr int WM = 2, WN = 4, MI = 8, NB = 4;  // waves, and 16 x 16 tiles of a wave
};
template <> struct TileGeom<true> {
  static constexpr int WM = 4, WN = 2, MI = 4, NB = 4;
};

template <bool PREC, bool E8M0>
__global__ __launch_bounds__(512, 2) void k_fp8_tile(LinearFp8Args a, int MT, int NT) {
  typedef TileGeom<PREC> G;
  constexpr int MI = G::MI, NB = G::NB;
  constexpr int TM = 16 * MI * G::WM, TN = 16 * NB * G::WN;
  constexpr int WQ = TM / 64, XQ = TN / 64;  // loads of a wave and step: 1 KB (8 rows) each
  constexpr int WB = TM / kFp8Block;         // the weight's scales of a step
  constexpr bool HW = E8M0 && !PREC;         // scales applied by the matrix instruction
  __shared__ __attribute__((aligned(1024))) uint8_t sw0[TM * 128], sx0[TN * 128], sw1[TM * 128], sx1[TN * 128];
  __shared__ uint32_t ss0[TN + WB], ss1[TN + WB];
  const int tid = threadIdx.x, lane = tid & (kWaveSize - 1);
  const int w = __builtin_amdgcn_readfirstlane(tid / kWaveSize);
  const int wm = w / G::WN, wn = w % G::WN;
  const int r16 = lane & 15, g = lane >> 4;

  // Each XCD takes a consecutive run of tiles, rows of x fastest.
  const int total = MT * NT;
  const int xcd = blockIdx.x % 8, ix = blockIdx.x / 8, per = total / 8, rem = total % 8;
  const int tile = xcd * per + (xcd < rem ? xcd : rem) + ix;
  const int mt = tile / NT, c0 = mt * TM, t0 = (tile - mt * NT) * TN;
  const int KB = a.ld / kFp8Block;
  const int nc = min(TM, a.n - c0), nt = min(TN, a.N - t0);
  const __amdgpu_buffer_rsrc_t rw = make_rsrc(a.wq + (size_t)c0 * a.ld, (uint32_t)nc * a.ld);
  const __amdgpu_buffer_rsrc_t rx = make_rsrc(a.xq + (size_t)t0 * a.ld, (uint32_t)nt * a.ld);

  // Piece c (16 bytes) of row r lies at slot c ^ (r & 7) of its 128 bytes, so
  // that eight lanes that read the same piece of eight rows hit distinct banks.
  const uint32_t loff = (uint32_t)((lane & 7) ^ (lane >> 3)) * 16u;
  // Rows past the tile's last lie past the buffer and read as zero.
  const uint32_t woff = (uint32_t)(8 * WQ * w + (lane >> 3)) * a.ld + loff;
  const uint32_t xoff = (uint32_t)(8 * XQ * w + (lane >> 3)) * a.ld + loff;
  auto issue = [&](uint8_t* sw, uint8_t* sx, int st) {
    const uint32_t k = st < KB ? (uint32_t)st * kFp8Block : kOOB;
#pragma unroll
    for (int q = 0; q < WQ; ++q) dma16(rw, sw + (WQ * w + q) * 1024, woff + (k + 8u * q * a.ld));
#pragma unroll
    for (int q = 0; q < XQ; ++q) dma16(rx, sx + (XQ * w + q) * 1024, xoff + (k + 8u * q * a.ld));
  };
  // The scales of a step: each wave of the first group fetches those of 64 of the
  // tile's rows and one of the weight's into registers and, a phase later, puts them
  // into LDS (some waves the same).  Not a load where they are used: its wait
  // would be one for the step's operands too.
  constexpr uint32_t SB = E8M0 ? 1 : 4;
  const int wb = min(c0 / kFp8Block + w % WB, (a.n - 1) / kFp8Block), srow = (64 * w + lane) % TN;
  const __amdgpu_buffer_rsrc_t rsw = make_rsrc(static_cast<const uint8_t*>(a.ws) + (size_t)wb * KB * SB, (uint32_t)KB * SB);
  const __amdgpu_buffer_rsrc_t rsx =
      make_rsrc(static_cast<const uint8_t*>(a.xs) + (size_t)t0 * KB * SB, (uint32_t)nt * KB * SB);
  const uint32_t soff = (uint32_t)srow * KB * SB;
  uint32_t px = 0, pw = 0;
  auto fetch_scales = [&](int st) {
    if constexpr (E8M0) {
      px = __builtin_amdgcn_raw_buffer_load_b8(rsx, (int)(soff + (uint32_t)st), 0, 0);
      pw = __builtin_amdgcn_raw_buffer_load_b8(rsw, st, 0, 0);
    } else {
      px = __builtin_amdgcn_raw_buffer_load_b32(rsx, (int)(soff + (uint32_t)st * 4u), 0, 0);
      pw = __builtin_amdgcn_raw_buffer_load_b32(rsw, st * 4, 0, 0);
    }
  };
  auto put_scales = [&](uint32_t* ss) {
    ss[srow] = E8M0 && !HW ? __float_as_uint(e8m0_value(px)) : px;
    ss[TN + w % WB] = E8M0 && !HW ? __float_as_uint(e8m0_value(pw)) : pw;
  };
  uint32_t xe[NB], we;

  f32x4 acc[MI][NB];
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int b = 0; b < NB; ++b) acc[i][b] = f32x4{0.f, 0.f, 0.f, 0.f};
  u32x4 fa[MI][2], fb[NB][2];
  const uint32_t fslot = (uint32_t)(g ^ (r16 & 7)) * 16u;
  const uint32_t abase = (uint32_t)(16 * MI * wm + r16) * 128u + fslot, bbase = (uint32_t)(16 * NB * wn + r16) * 128u + fslot;
  auto read = [&](const uint8_t* sw, const uint8_t* sx, const uint32_t* ss) {
#pragma unroll
    for (int b = 0; b < NB; ++b) xe[b] = ss[16 * NB * wn + 16 * b + r16];
    we = ss[TN + 16 * MI * wm / kFp8Block];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      fb[b][0] = *reinterpret_cast<const u32x4*>(sx + bbase + b * 2048);
      fb[b][1] = *reinterpret_cast<const u32x4*>(sx + (bbase ^ 64u) + b * 2048);
    }
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      fa[i][0] = *reinterpret_cast<const u32x4*>(sw + abase + i * 2048);
      fa[i][1] = *reinterpret_cast<const u32x4*>(sw + (abase ^ 64u) + i * 2048);
    }
  };
  auto multiply = [&]() {
    float sc[NB];
    if constexpr (!HW) {
#pragma unroll
      for (int b = 0; b < NB; ++b) sc[b] = __uint_as_float(xe[b]) * __uint_as_float(we);
    }
    if constexpr (PREC) {
      fp_bf16x8 xb[NB][4];
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          xb[b][2 * h] = widen8(fb[b][h].x, fb[b][h].y, 1.f);
          xb[b][2 * h + 1] = widen8(fb[b][h].z, fb[b][h].w, 1.f);
        }
#pragma unroll
      for (int i = 0; i < MI; ++i) {
        f32x4 p[NB];
#pragma unroll
        for (int b = 0; b < NB; ++b) p[b] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const u32x4 v = fa[i][k >> 1];
          const fp_bf16x8 wb = (k & 1) ? widen8(v.z, v.w, 1.f) : widen8(v.x, v.y, 1.f);
#pragma unroll
          for (int b = 0; b < NB; ++b) p[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wb, xb[b][k], p[b], 0, 0, 0);
        }
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[i][b][e] = fmaf(p[b][e], sc[b], acc[i][b][e]);
      }
      // the first outputs' products among x's conversions, then each outputs'
      // conversions and the sums of those before among the products
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        __builtin_amdgcn_sched_group_barrier(0x002, 4 + 4 * NB, 0);
        __builtin_amdgcn_sched_group_barrier(0x008, NB, 0);
      }
#pragma unroll
      for (int k = 0; k < 4 * MI - 4; ++k) {
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          __builtin_amdgcn_sched_group_barrier(0x002, 1 + 4 / NB, 0);
          __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        }
      }
      __builtin_amdgcn_sched_group_barrier(0x002, 4 * NB, 0);
    } else {
#pragma unroll
      for (int i = 0; i < MI; ++i)
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
      if constexpr (!HW) {
        // a few products ahead of the sums that use them
        __builtin_amdgcn_sched_group_barrier(0x002, NB, 0);
        __builtin_amdgcn_sched_group_barrier(0x008, 3, 0);
#pragma unroll
        for (int i = 0; i < MI * NB - 3; ++i) {
          __builtin_amdgcn_sched_group_barrier(0x002, 4, 0);
          __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x002, 12, 0);
      }
    }
  };
  auto phase_end = [&]() {
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  };

  // A step of the first group: it sends step s + 1's loads as it reads step s (its
  // multiply phase of the step before and the second group's read phase of
  // that step are over), and waits for them in its multiply phase.
  auto first_step = [&](uint8_t* sw, uint8_t* sx, uint32_t* ss, uint8_t* nw, uint8_t* nx, uint32_t* ns, int st) {
    issue(nw, nx, st + 1);
    fetch_scales(st + 1);
    read(sw, sx, ss);
    wait_lds();
    phase_end();
    multiply();
    __builtin_amdgcn_sched_barrier(0);
    wait_vm<0>();
    put_scales(ns);
    wait_lds();
    phase_end();
  };
  // The second group, a phase behind: step s + 2's loads as it multiplies step s,
  // waited for after it has read step s + 1.
  auto second_step = [&](uint8_t* sw, uint8_t* sx, uint32_t* ss, int st) {
    read(sw, sx, ss);
    wait_lds();
    wait_vm<0>();
    phase_end();
    issue(sw, sx, st + 2);
    __builtin_amdgcn_sched_barrier(0);
    multiply();
    phase_end();
  };
  issue(sw0, sx0, 0);
  int st = 0;
  if (w < 4) {
    fetch_scales(0);
    wait_vm<0>();
    put_scales(ss0);
    wait_lds();
    phase_end();
    for (; st + 2 <= KB; st += 2) {
      first_step(sw0, sx0, ss0, sw1, sx1, ss1, st);
      first_step(sw1, sx1, ss1, sw0, sx0, ss0, st + 1);
    }
    if (st < KB) first_step(sw0, sx0, ss0, sw1, sx1, ss1, st);
    phase_end();
  } else {
    issue(sw1, sx1, 1);
    wait_vm<WQ + XQ>();
    phase_end();
    phase_end();
    for (; st + 2 <= KB; st += 2) {
      second_step(sw0, sx0, ss0, st);
      second_step(sw1, sx1, ss1, st + 1);
    }
    if (st < KB) second_step(sw0, sx0, ss0, st);
  }
  wait_vm<0>();  // no load is on its way to LDS when the block ends

  // D[i][j] sits in lane j + 16 (i / 4), register i % 4: four consecutive
  // outputs of one row.
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    const int t = t0 + 16 * NB * wn + 16 * b + r16;
    if (t >= a.N) continue;
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      const int c = c0 + 16 * MI * wm + 16 * i + 4 * g;
      const size_t at = (size_t)t * a.n + c;
      if ((a.n & 3) == 0) {
        if (c < a.n) put_y4(a, at, acc[i][b]);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (c + e < a.n) put_y(a, at + e, acc[i][b][e]);
      }
    }
  }
}

template <bool PREC>
static hipError_t launch_tile(const LinearFp8Args& a, hipStream_t s) {
  typedef TileGeom<PREC> G;
  constexpr int TM = 16 * G::MI * G::WM, TN = 16 * G::NB * G::WN;
  const int MT = (a.n + TM - 1) / TM, NT = (a.N + TN - 1) / TN;
  KernelTimer timer(PREC ? "linear_fp8_tile_f32" : "linear_fp8_tile", s);
  if (a.e8m0)
    hipExtLaunchKernelGGL((k_fp8_tile<PREC, true>), dim3(MT * NT), dim3(512), 0, s, timer.start(), timer.stop(), 0, a, MT, NT);
  else
    hipExtLaunchKernelGGL((k_fp8_tile<PREC, false>), dim3(MT * NT), dim3(512), 0, s, timer.start(), timer.stop(), 0, a, MT, NT);
  return hipGetLastError();
}

hipError_t launch_linear_fp8(const LinearFp8Args& a, hipStream_t s) {
  if (a.N > 64) return a.ybf16 ? launch_tile<false>(a, s) : launch_tile<true>(a, s);
  const dim3 grid((a.n + 15) / 16, (a.N + 15) / 16);
  KernelTimer timer("linear_fp8_few", s);
  if (a.e8m0)
    hipExtLaunchKernelGGL((k_fp8_few<true>), grid, dim3(kFewWaves * kWaveSize), 0, s, timer.start(), timer.stop(), 0, a);
  else
    hipExtLaunchKernelGGL((k_fp8_few<false>), grid, dim3(kFewWaves * kWaveSize), 0, s, timer.start(), timer.stop(), 0, a);
  return hipGetLastError();
}

}  // namespace cats
