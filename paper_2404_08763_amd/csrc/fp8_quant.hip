// The kernels that write 8-bit rows: quantisation alone, RMSNorm with the
// residual's addition, and the SiLU gate with the CATS cutoff.
//
// A scale covers 128 columns: 16 lanes of eight columns, one DPP row, so a
// block's largest magnitude is four DPP steps away and no value leaves its
// lane's registers between the load and the 8-byte store of its e4m3 values.
// All of them are bound by memory, each input read once and each output written
// once, and reach the rate of a large copy (5.1 TB/s): the gate of 2048 x 14336 in
// bf16 148 MB in 29.1 us (its vector instructions take about as long), 11008 x 4096 bf16
// weights 135 MB in 27.5, RMSNorm of 4096 x 4096 bf16 with the residual and its new value 185
// MB in 36.8.
#include "fp8.hpp"
#include "internal.hpp"

namespace cats {

// Stores a lane's eight values (times m) of block (row, cb), A the block's largest
// finite one, and from the group's first lane its scale.
//   kAgain: where one of the block's values, known to `steps` of fp32, may lie on either
//     side of the middle of two e4m3 values (or its largest of an E8M0 scale's limit),
//     `exact` gives all eight (m included) in 64 bits;
//   kFp32: the values are fp32 numbers and m, with fp32 scales, counts for the scale alone;
//   kAsIs: no second look.
enum Fp8Look { kAsIs, kFp32, kAgain };
template <bool E8M0, Fp8Look LOOK, typename F>
__device__ __forceinline__ void put_block(const Fp8Out& o, size_t row, int cb, int sub, uint32_t A, const Fp8Factor& m,
                                          float (&f)[8], uint32_t steps, const F& exact) {
  Fp8Factor k;
  bool plain;
  typename Fp8Scale<E8M0>::type s = fp8_scale<E8M0, LOOK != kAgain, 8>(A, m, k, f, plain);
  float v[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = LOOK == kAgain ? f[e] * k.hi : times(f[e], k);
  if constexpr (LOOK == kFp32) {
    fix_ties(v, f, A, plain);
  } else if constexpr (LOOK == kAgain) {
    bool doubt = near_tie(v, steps);
    if constexpr (E8M0) doubt |= ((__float_as_uint(times(__uint_as_float(A), m)) + steps - 0x600000u) & 0x7fffffu) <= 2u * steps;
    const uint64_t who = __ballot(doubt && plain);
    if (__builtin_expect(who != 0, 0)) {
      double x[8], top = 0.0, kx;
      exact(x);
#pragma unroll
      for (int e = 0; e < 8; ++e) top = fabsf(f[e]) < __builtin_inff() ? fmax(top, fabs(x[e])) : top;
      top = max16(top);
      // (of the block alone: a row's result does not depend on the rows beside it)
      if ((who >> (threadIdx.x & 48)) & 0xffffu) {
        s = Fp8Scale<E8M0>::exact(top, kx);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = fabsf(f[e]) < __builtin_inff() ? to_odd(x[e] * kx) : __builtin_nanf("");
      }
    }
  }
  *reinterpret_cast<uint2*>(o.q + row * o.ld + (size_t)cb * kFp8Block + sub * 8) = fp8x8(v);
  if (sub == 0) reinterpret_cast<typename Fp8Scale<E8M0>::type*>(o.scale)[row * (o.ld / kFp8Block) + cb] = s;
}

// SiLU with the reciprocal instruction (one fp32 step off) in place of a division,
// whose instructions the gate's kernel would otherwise be bound by; the same
// infinities and NaN.  Below -87.3, where SiLU is less than 1.2e-36, the reciprocal
// leaves the normal range and the result may be 0.
// e^-z with what its argument rounds off (-z log2 e = a + r): within 4.4 2^-24 of
// SiLU, measured over every z.  Without it 10 2^-24 at z = -10, 30 from -22 on and 65 at -87: no
// few steps find the values next to a middle or the cutoff then (2048 x 14336 bf16 28.5
// us, with it 29.8).
__device__ __forceinline__ float silu_fast(float z) {
  constexpr float L = 0x1.715476p+0f, LLO = 0x1.4ae0cp-26f, LN2 = 0x1.62e43p-1f;  // log2 e = L + LLO
  const float c = __builtin_amdgcn_fmed3f(z, -3e38f, 100.f);  // (past 100 e^-z counts for nothing)
  const float a = c * -L, r = fmaf(c, -LLO, fmaf(c, -L, -a));
  return z * __builtin_amdgcn_rcpf(fmaf(__builtin_amdgcn_exp2f(a), fmaf(r, LN2, 1.f), 1.f));
}

// One group of 16 lanes per block of 128 columns of a row.  GATE: the row
// holds m gate values, then m up values; h = SiLU(g) u where |SiLU(g)| is not below t.
// A value next to the cutoff is found by 2^-21.  A product is off by SiLU's error and its own
// rounding, with fp32 scales the quotient by the largest's too and by four half steps
// of the factor and its use: 6 and 15 (0.6 and 1.5% of the waves).
template <typename T, bool E8M0, bool GATE>
__global__ __launch_bounds__(256) void k_fp8_rows(const T* __restrict__ x, int cols, float t, uint32_t blocks, Fp8Out o) {
  const uint32_t b = blockIdx.x * 16u + threadIdx.x / 16u;
  if (b >= blocks) return;
  const uint32_t nb = (uint32_t)o.ld / kFp8Block, row = b / nb;
  const int cb = (int)(b - row * nb), sub = threadIdx.x & 15, c = cb * kFp8Block + sub * 8;
  const T* xr = x + (size_t)row * cols * (GATE ? 2 : 1);
  float f[8];
  const Fp8Factor one = {1.f, 0.f};
  if constexpr (GATE) {
    float u[8], h[8];
    load8(xr, xr + cols, c, cols, f, u);
    const float lo = t * (1.f - 0x1p-21f), hi = t * (1.f + 0x1p-21f);  // between them: 64 bits decide
    bool off = false;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float v = silu_fast(f[e]);
      off |= (fabsf(v) < lo) != (fabsf(v) < hi);
      h[e] = fabsf(v) < lo ? 0.f : v * u[e];
    }
    if (__builtin_expect(__any(off), 0)) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const double z = f[e];
        if (fabs(z / (1.0 + exp(-z))) < (double)t) h[e] = 0.f;
      }
    }
    put_block<E8M0, kAgain>(o, row, cb, sub, block_max<8>(h), one, h, E8M0 ? 6 : 15, [&](double (&x)[8]) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const double z = f[e], v = z / (1.0 + exp(-z));
        x[e] = fabs(v) < (double)t ? 0.0 : v * (double)u[e];
      }
    });
  } else {
    load8(xr, c, cols, f);
    put_block<E8M0, sizeof(T) == 4 && !E8M0 ? kFp32 : kAsIs>(o, row, cb, sub, block_max<8>(f), one, f, 0, 0);
  }
}

// One block of 512 threads per 128 x 128 weights, 32 of them per thread, in
// registers between the block's largest and the quotients.
template <typename T, bool E8M0>
__global__ __launch_bounds__(512) void k_fp8_tiles(const T* __restrict__ x, int rows, int cols, Fp8Out o) {
  constexpr int R = 4;  // rows of a thread
  __shared__ uint32_t red[32];
  const int nb = o.ld / kFp8Block;
  const int rb = blockIdx.x / nb, cb = blockIdx.x - rb * nb;
  const int grp = threadIdx.x / 16, sub = threadIdx.x & 15, c = cb * kFp8Block + sub * 8;
  const int r0 = rb * kFp8Block + grp;
  float f[R][8];
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int r = r0 + 32 * i;
    if (r < rows) {
      load8(x + (size_t)r * cols, c, cols, f[i]);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) f[i][e] = 0.f;
    }
  }
  uint32_t a = block_max<8 * R>(&f[0][0]);
  if (sub == 0) red[grp] = a;
  __syncthreads();
  a = max16(max(red[sub], red[sub + 16]));
  Fp8Factor k;
  bool plain;
  const typename Fp8Scale<E8M0>::type s = fp8_scale<E8M0, true, 8 * R>(a, Fp8Factor{1.f, 0.f}, k, &f[0][0], plain);
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int r = r0 + 32 * i;
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = times(f[i][e], k);
    if constexpr (sizeof(T) == 4 && !E8M0) fix_ties(v, f[i], a, plain);
    if (r < rows) *reinterpret_cast<uint2*>(o.q + (size_t)r * o.ld + c) = fp8x8(v);
  }
  if (threadIdx.x == 0) reinterpret_cast<typename Fp8Scale<E8M0>::type*>(o.scale)[(size_t)rb * nb + cb] = s;
}

// One block per row, the row in registers (NV chunks of eight columns per thread):
// one read of x and the residual, all under way together.  One row of 4096 takes 2.8 us:
// the loads, the sum over the block and the second reduction of its blocks' largest.
// BARE: x alone, without residual and gain, and fp32 scales.  Its quotients are
// quantisation's, f 448 / A, of which bf16 numbers often lie on the middle of two values and
// never next to it: 4096 x 4096 bf16 16.2 us, 29.1 with the others' second look, which two waves
// of three took.
template <typename T, bool E8M0, int NV, bool BARE>
__global__ __launch_bounds__(1024, NV == 1 ? 8 : 4) void k_rmsnorm_fp8(RmsnormFp8Args a) {
  __shared__ double red[16];
  const int d = a.d, tid = threadIdx.x, T0 = blockDim.x;
  const size_t row = blockIdx.x;
  const T* xr = static_cast<const T*>(a.x) + row * d;
  // What the additions round off is kept for values next to a middle.  Rows of more than
  // 8192 columns have no registers for it without fewer waves (2048 rows of 12288, bf16 with
  // residual: 56 us, 48 without), and no second look.
  constexpr bool LO = NV == 1 && !BARE;
  float f[NV][8], lo[LO ? NV : 1][8] = {};
  // The row's factor reaches q with E8M0 scales alone: there the squares are those of 64
  // bits (4096 x 4096 bf16 17.3 -> 18.2 us).
  double ss = 0.0;
  const float *residual = BARE ? nullptr : a.residual, *gain = BARE ? nullptr : a.gain;
  if (NV > 1 || !residual) {
#pragma unroll
    for (int i = 0; i < NV; ++i) load8(xr, (tid + T0 * i) * 8, d, f[i]);
  }
  if (residual) {
    float r[NV][8];
    if constexpr (NV == 1) {
      load8(xr, residual + row * d, tid * 8, d, f[0], r[0]);
    } else {
#pragma unroll
      for (int i = 0; i < NV; ++i) load8(residual + row * d, (tid + T0 * i) * 8, d, r[i]);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float x = f[i][e], sum = x + r[i][e], b = sum - x;
        if constexpr (LO) lo[i][e] = (x - (sum - b)) + (r[i][e] - b);
        f[i][e] = sum;
      }
  }
  if (a.sum) {
#pragma unroll
    for (int i = 0; i < NV; ++i) store8(a.sum + row * d, (tid + T0 * i) * 8, d, f[i]);
  }
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if constexpr (E8M0) {
        double v = f[i][e];
        if constexpr (LO) v += (double)__builtin_amdgcn_fmed3f(lo[i][e], -1e38f, 1e38f);  // (NaN beside an infinite sum)
        ss = fma(v, v, ss);
      } else {
        ss += (double)(f[i][e] * f[i][e]);
      }
    }
  double sum = wave_sum64(ss);
  const int nw = T0 / kWaveSize;
  if (nw > 1) {
    if ((tid & (kWaveSize - 1)) == 0) red[tid / kWaveSize] = sum;
    __syncthreads();
    sum = red[0];
    for (int w = 1; w < nw; ++w) sum += red[w];
  }
  // (a sum of squares past fp32's range makes zeros of the row, one below it counts as 0)
  const double r = sum >= 0x1p128 ? 0.0 : 1.0 / sqrt((sum < 0x1p-149 ? 0.0 : sum / d) + (double)a.eps);
  Fp8Factor m;
  m.hi = (float)r;
  m.lo = m.hi < __builtin_inff() ? (float)(r - m.hi) : 0.f;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (tid + T0 * i) * 8;
    if (c >= a.o.ld) continue;
    float g[8], y[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = f[i][e], g[e] = 1.f;
    if (gain) {
      load8(gain, c, d, g);
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] *= g[e];
    }
    // (the sum's and the product's roundings, of the value and of the largest, and the
    // factor's: 10 steps)
    constexpr Fp8Look look = LO ? kAgain : BARE && sizeof(T) == 4 ? kFp32 : kAsIs;
    put_block<E8M0, look>(a.o, row, c / kFp8Block, (c / 8) & 15, block_max<8>(y), m, y, 10, [&](double (&x)[8]) {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = ((double)f[i][e] + (double)lo[LO ? i : 0][e]) * (double)g[e] * r;
    });
  }
}

namespace {
// A launch's threads are counted in 32 bits, 16 to a block: larger calls are
// several launches, of 2^31 elements each (a millisecond of work).
constexpr uint32_t kLaunchBlocks = 1u << 24;

template <typename T, bool GATE>
hipError_t rows_launch(const char* name, const void* x, int N, int cols, float t, const Fp8Out& out, hipStream_t s) {
  const uint32_t nb = (uint32_t)out.ld / kFp8Block;
  const int most = (int)(kLaunchBlocks / nb);  // rows of a launch
  for (int r = 0; r < N; r += most) {
    const uint32_t blocks = (uint32_t)(N - r < most ? N - r : most) * nb;
    const dim3 grid((blocks + 15) / 16);
    const T* xr = static_cast<const T*>(x) + (size_t)r * cols * (GATE ? 2 : 1);
    Fp8Out o = out;
    o.q += (size_t)r * o.ld;
    o.scale = static_cast<uint8_t*>(o.scale) + (size_t)r * nb * (o.e8m0 ? 1 : 4);
    KernelTimer timer(name, s);
    if (o.e8m0)
      hipExtLaunchKernelGGL((k_fp8_rows<T, true, GATE>), grid, dim3(256), 0, s, timer.start(), timer.stop(), 0, xr, cols, t, blocks, o);
    else
      hipExtLaunchKernelGGL((k_fp8_rows<T, false, GATE>), grid, dim3(256), 0, s, timer.start(), timer.stop(), 0, xr, cols, t, blocks, o);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <typename T>
hipError_t tiles_launch(const void* x, int rows, int cols, const Fp8Out& o, hipStream_t s) {
  const dim3 grid((unsigned)((rows + kFp8Block - 1) / kFp8Block) * (unsigned)(o.ld / kFp8Block));
  KernelTimer timer("quantize_fp8_tiles", s);
  if (o.e8m0)
    hipExtLaunchKernelGGL((k_fp8_tiles<T, true>), grid, dim3(512), 0, s, timer.start(), timer.stop(), 0,
                          static_cast<const T*>(x), rows, cols, o);
  else
    hipExtLaunchKernelGGL((k_fp8_tiles<T, false>), grid, dim3(512), 0, s, timer.start(), timer.stop(), 0,
                          static_cast<const T*>(x), rows, cols, o);
  return hipGetLastError();
}

template <typename T, bool E8M0, int NV, bool BARE = false>
hipError_t norm_launch_nv(const RmsnormFp8Args& a, int threads, hipStream_t s) {
  KernelTimer timer("rmsnorm_fp8", s);
  hipExtLaunchKernelGGL((k_rmsnorm_fp8<T, E8M0, NV, BARE>), dim3(a.N), dim3(threads), 0, s, timer.start(), timer.stop(), 0, a);
  return hipGetLastError();
}

template <typename T, bool E8M0>
hipError_t norm_launch(const RmsnormFp8Args& a, hipStream_t s) {
  const int chunks = a.o.ld / 8;
  const int nv = chunks <= 1024 ? 1 : chunks <= 2048 ? 2 : chunks <= 4096 ? 4 : 8;
  const int threads = ((chunks + nv - 1) / nv + kWaveSize - 1) / kWaveSize * kWaveSize;
  if constexpr (!E8M0) {
    if (nv == 1 && !a.residual && !a.gain) return norm_launch_nv<T, false, 1, true>(a, threads, s);
  }
  switch (nv) {
    case 1: return norm_launch_nv<T, E8M0, 1>(a, threads, s);
    case 2: return norm_launch_nv<T, E8M0, 2>(a, threads, s);
    case 4: return norm_launch_nv<T, E8M0, 4>(a, threads, s);
    default: return norm_launch_nv<T, E8M0, 8>(a, threads, s);
  }
}
}  // namespace

hipError_t launch_quantize_fp8(const void* x, int bf16, int rows, int cols, int block_rows, const Fp8Out& o, hipStream_t s) {
  if (block_rows == 1)
    return bf16 ? rows_launch<uint16_t, false>("quantize_fp8_rows", x, rows, cols, 0.f, o, s)
                : rows_launch<float, false>("quantize_fp8_rows", x, rows, cols, 0.f, o, s);
  return bf16 ? tiles_launch<uint16_t>(x, rows, cols, o, s) : tiles_launch<float>(x, rows, cols, o, s);
}

hipError_t launch_silu_fp8(const void* gu, int bf16, int N, int m, float t, const Fp8Out& o, hipStream_t s) {
  return bf16 ? rows_launch<uint16_t, true>("silu_mul_fp8", gu, N, m, t, o, s)
              : rows_launch<float, true>("silu_mul_fp8", gu, N, m, t, o, s);
}

hipError_t launch_rmsnorm_fp8(const RmsnormFp8Args& a, int bf16, hipStream_t s) {
  if (bf16) return a.o.e8m0 ? norm_launch<uint16_t, true>(a, s) : norm_launch<uint16_t, false>(a, s);
  return a.o.e8m0 ? norm_launch<float, true>(a, s) : norm_launch<float, false>(a, s);
}

}  // namespace cats
