// Norms of queries and keys for each head, with the position rotation in the
// same pass: n = x / sqrt(mean(x^2) + eps) * gain, then each pair (u, w) of the
// first `rot` columns turned by the angle pos * freq.
//
// Bound by memory for a prompt: every element is read and written once.  A lane
// has 8 elements, of which the two of a pair are its own, so nothing is
// exchanged but the sum of squares, and the lanes of a head are a power of two
// side by side.  A row's angles are the same for all heads: a wave takes several
// heads of a row and computes them once.  The angle is reduced in 64 bits (at
// position 10^6 fp32's product alone is off by 0.03), sine and cosine are fp32, with what the reduced
// angle's rounding to fp32 cuts off (0.2 us of a prompt of 4096 rows; half the error of fp32 rows).
// The next heads' loads are under way before the angles: 4096 rows of 32 + 8 heads of
// 128 columns (bf16, norms and rotation, 84 MB) take 18.3 us, 4.6 TB/s, with the vector
// ALUs busy 0.97 of the time; one row, 3 us, its launch and one chain of loads.
#include <algorithm>

#include "device.hpp"
#include "internal.hpp"

namespace cats {
namespace {

constexpr int kThreads = 256;
constexpr float kTiny = 0x1p-100f;

// Four elements as they are in memory.
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
template <bool BF16> struct Quad;
template <> struct Quad<true> {
  u32x2 v;
  __device__ __forceinline__ void load(const void* p, size_t at) {
    v = *reinterpret_cast<const u32x2*>(static_cast<const uint16_t*>(p) + at);
  }
  __device__ __forceinline__ void get(float* f) const {
    f[0] = __uint_as_float(v.x << 16);
    f[1] = __uint_as_float(v.x & 0xffff0000u);
    f[2] = __uint_as_float(v.y << 16);
    f[3] = __uint_as_float(v.y & 0xffff0000u);
  }
};
template <> struct Quad<false> {
  u32x4 v;
  __device__ __forceinline__ void load(const void* p, size_t at) {
    v = *reinterpret_cast<const u32x4*>(static_cast<const float*>(p) + at);
  }
  __device__ __forceinline__ void get(float* f) const { widen<wf32>(v, f); }
};

typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
template <bool BF16> __device__ __forceinline__ void store4(void* p, size_t at, const float* f) {
  if (BF16) {
    const bf16x4 v = {(__bf16)f[0], (__bf16)f[1], (__bf16)f[2], (__bf16)f[3]};
    *reinterpret_cast<bf16x4*>(static_cast<uint16_t*>(p) + at) = v;
  } else {
    *reinterpret_cast<f32x4*>(static_cast<float*>(p) + at) = f32x4{f[0], f[1], f[2], f[3]};
  }
}

// Sum over each L lanes side by side, the same bits on all of them.
template <int L> __device__ __forceinline__ float lanes_sum(float v) {
  v += dpp_f32<0xb1>(v);
  v += dpp_f32<0x4e>(v);
  if (L >= 8) v += dpp_f32<0x141>(v);
  if (L >= 16) v += dpp_f32<0x140>(v);
  if (L >= 32) v += __shfl_xor(v, 16);
  if (L >= 64) v += __shfl_xor(v, 32);
  return v;
}

// L lanes have a head (the power of two from d / 8 on); a wave takes 64 / L
// heads at a time, `passes` times.
template <int L, bool XB, bool YB> __global__ __launch_bounds__(kThreads) void k_qk_rope(QkRopeArgs a) {
  constexpr int HW = 64 / L;
  const int wave = uniform_u32(blockIdx.x * (kThreads / 64) + threadIdx.x / 64), lane = threadIdx.x % 64;
  const int row = wave / a.chunks, chunk = wave % a.chunks;
  if (row >= a.N) return;
  const int s = lane % L, H = a.hq + a.hkv;
  const bool mine = 8 * s < a.d, turns = 8 * s < a.rot;
  // columns of the lane's two quads
  const int ca = turns && !a.interleaved ? 4 * s : 8 * s, cb = turns && !a.interleaved ? 4 * s + a.rot / 2 : 8 * s + 4;
  const int h0 = chunk * a.passes * HW + lane / L, end = min(H, (chunk + 1) * a.passes * HW);
  const size_t x0 = (size_t)row * a.ld;
  Quad<XB> nu, nw;  // the next pass's, loaded before this one's are used
  if (mine && h0 < end) {
    nu.load(a.x, x0 + (size_t)h0 * a.d + ca);
    nw.load(a.x, x0 + (size_t)h0 * a.d + cb);
  }
  float co[4] = {1.f, 1.f, 1.f, 1.f}, si[4] = {0.f, 0.f, 0.f, 0.f};
  if (turns) {
    const double pos = (double)a.pos[row];
    const f32x4 fr = *reinterpret_cast<const f32x4*>(a.freq + 4 * s);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      double half = pos * (double)fr[i] * 0.31830988618379067154;  // in half turns
      half -= 2.0 * rint(0.5 * half);
      const float near = (float)half;
      float sn, cs;
      sincospif(near, &sn, &cs);
      // what fp32 cuts off, 2^-25 at most, by the first terms of the series
      const float rest = (float)(half - (double)near) * 3.14159265f;
      si[i] = fmaf(cs, rest, sn);
      co[i] = fmaf(-sn, rest, cs);
    }
  }
  for (int h = h0; h - lane / L < end; h += HW) {
    const bool on = mine && h < end;
    float u[4] = {0.f, 0.f, 0.f, 0.f}, w[4] = {0.f, 0.f, 0.f, 0.f};
    if (on) {
      nu.get(u);
      nw.get(w);
    }
    if (mine && h + HW < end) {
      nu.load(a.x, x0 + (size_t)(h + HW) * a.d + ca);
      nw.load(a.x, x0 + (size_t)(h + HW) * a.d + cb);
    }
    if (a.norm) {
      float q = 0.f;
#pragma unroll
      for (int i = 0; i < 4; ++i) q = fmaf(u[i], u[i], fmaf(w[i], w[i], q));
      q = lanes_sum<L>(q);
      float eps = a.eps;
      if (a.eps < kTiny) {
        // squares below 2^-100 in all lose digits, which only so small an eps shows: those of 2^100 x
        const float up = q < kTiny ? 0x1p100f : 1.f;
        q = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          u[i] *= up;
          w[i] *= up;
          q = fmaf(u[i], u[i], fmaf(w[i], w[i], q));
        }
        q = lanes_sum<L>(q);
        eps = eps * up * up;
      }
      const float r = 1.f / sqrtf(q / (float)a.d + eps);
      const float* gain = h < a.hq ? a.gq : a.gk;
      if (gain && on) {
        const f32x4 ga = *reinterpret_cast<const f32x4*>(gain + ca), gb = *reinterpret_cast<const f32x4*>(gain + cb);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          u[i] = u[i] * r * ga[i];
          w[i] = w[i] * r * gb[i];
        }
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          u[i] *= r;
          w[i] *= r;
        }
      }
    }
    if (turns) {
      if (a.interleaved) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const float p = u[2 * i], q = u[2 * i + 1], c = w[2 * i], d = w[2 * i + 1];
          u[2 * i] = p * co[i] - q * si[i];
          u[2 * i + 1] = q * co[i] + p * si[i];
          w[2 * i] = c * co[i + 2] - d * si[i + 2];
          w[2 * i + 1] = d * co[i + 2] + c * si[i + 2];
        }
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float p = u[i], q = w[i];
          u[i] = p * co[i] - q * si[i];
          w[i] = q * co[i] + p * si[i];
        }
      }
    }
    if (on) {
      void* out = h < a.hq ? a.q : a.k;
      const size_t at = h < a.hq ? ((size_t)row * a.hq + h) * a.d : ((size_t)row * a.hkv + (h - a.hq)) * a.d;
      store4<YB>(out, at + ca, u);
      store4<YB>(out, at + cb, w);
    }
  }
}

template <int L> void go(const QkRopeArgs& a, int blocks, bool xb, bool yb, const KernelTimer& tm, hipStream_t s) {
#define CATS_GO(X, Y) hipExtLaunchKernelGGL((k_qk_rope<L, X, Y>), dim3(blocks), dim3(kThreads), 0, s, tm.start(), tm.stop(), 0, a)
  if (xb) {
    if (yb) CATS_GO(true, true);
    else CATS_GO(true, false);
  } else {
    if (yb) CATS_GO(false, true);
    else CATS_GO(false, false);
  }
#undef CATS_GO
}

}  // namespace

hipError_t launch_qk_rope(QkRopeArgs a, bool xbf16, bool ybf16, hipStream_t s) {
  int L = 4;
  while (8 * L < a.d) L *= 2;
  const int all = (a.hq + a.hkv + 64 / L - 1) / (64 / L);  // passes that a row takes
  // one pass to a wave until the chip is full of waves, then more of a row's, for its angles
  const long long waves = (long long)a.N * all;
  a.passes = (int)std::min<long long>(all, std::max<long long>(1, waves / 8192));
  a.chunks = (all + a.passes - 1) / a.passes;
  const int blocks = (int)(((long long)a.N * a.chunks + kThreads / 64 - 1) / (kThreads / 64));
  KernelTimer tm("qk_norm_rope", s);
  switch (L) {
    case 4: go<4>(a, blocks, xbf16, ybf16, tm, s); break;
    case 8: go<8>(a, blocks, xbf16, ybf16, tm, s); break;
    case 16: go<16>(a, blocks, xbf16, ybf16, tm, s); break;
    case 32: go<32>(a, blocks, xbf16, ybf16, tm, s); break;
    default: go<64>(a, blocks, xbf16, ybf16, tm, s); break;
  }
  return hipGetLastError();
}

}  // namespace cats
