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

// A lane's 32 values of a column block.
__device__ __forceinline__ void widen32(const u32x4 (&v)[2], fp_bf16x8 (&f)[4]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    f[2 * h] = widen8(v[h].x, v[h].y, 1.f);
    f[2 * h + 1] = widen8(v[h].z, v[h].w, 1.f);
  }
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

constexpr int kTileGroup = 6;

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
// to three phases to arrive.
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
  static_assert(TM == 256 && MI * G::WM / 2 == 8, "a group's outputs are 128");
  constexpr int WQ = 4, XQ = TN / 32;  // 1 KB loads (8 rows) of a wave: of a half of the weights, of x
  constexpr bool HW = E8M0 && !PREC;   // scales applied by the matrix instruction
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
  // (addresses made anew for each load: kept, they cost the registers of a tile)
  auto fresh = [](uint32_t v) {
    asm volatile("" : "+v"(v));
    return v;
  };
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
  // of the two weight blocks, four steps at a time (some lanes the same), and puts them into LDS a step later.  Not a load where they are used: its wait
  // would be one for the operands under way too.  Where fewer than four steps are
  // left, the last four of the row; where there are fewer, zeros past its end.
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
      const uint32_t srow = fresh((uint32_t)(64 * gw + lane) % TN);
      ring[slot][srow] = px.template get<HW>(j);
      ring[slot][TN + (lane >> 5)] = pw.template get<HW>(j);
    }
  };
  uint32_t xe[NB], we;
  fp_bf16x8 xw[PREC ? NB : 1][4], ww[PREC ? MI : 1][4];

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
    if constexpr (PREC) {
#pragma unroll
      for (int b = 0; b < NB; ++b) widen32(fb[b], xw[b]);
#pragma unroll
      for (int i = 0; i < MI; ++i) widen32(fa[i], ww[i]);
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
    if constexpr (PREC) {
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
    send_w(next_whi, 1, st + 1);
    multiply(none, half, Const<WQ>());
    send_w(wlo, 0, st + 2);
    multiply(half, all, Const<WQ>());
    wait_vm<2 * WQ + F>();
    phase_end();
  };
  auto second_step = [&](const uint8_t* whi, uint8_t* xb, int st) {
    read(whi, xb, st);
    wait_lds();
    wait_vm<0>();
    phase_end();
    send_x(xb, st + 2);
    multiply(none, half, Const<XQ>());
    multiply(half, all, none);
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
