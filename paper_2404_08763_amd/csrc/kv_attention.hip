// Attention over the cache in 4 bits: o = sum_j softmax_j(scale q k_j) v_j.
//
// One pass over the keys with a running maximum and sum.  A wave has a tile of
// 16 QT rows (the query heads of a key head side by side, then the next query)
// and takes 32 tokens a step; everything stays in its registers:
//   - S^T = K Q^T: the records' layout (kv4.hpp) gives each lane its part of the
//     matrix operand in one load; the conversion instructions make bf16 of the
//     codes and scales, exactly, so the products are exact and their sums fp32.
//   - a column of S^T, a query row, is in the lanes of equal lane % 16: its
//     softmax needs no exchange but for a new maximum, and P is the operand of
//     O^T = V^T P^T as it lies, as the order of the tokens within a step is free.
//   - V^T needs two tokens side by side where a conversion gives two columns: one
//     byte permutation per pair.
// The scores, P before its split, the statistics and O are fp32.  P goes into the
// products as two bf16 parts (16 bits of it) for bf16 rows, as three (all 24 bits)
// for fp32 rows, whose q is split in three as well.
// A row's maximum is only moved when a score is 2^8 above it, so that O is rarely
// multiplied; p is then up to 2^8.
//
// A block's four waves take every fourth step of its tokens and add their sums
// through LDS.  The blocks share all (head, tile, 128 tokens) units of the call
// evenly, each a run of them, whatever the sequences' lengths: what is split over
// blocks is joined by a second kernel.
#include <algorithm>

#include "internal.hpp"
#include "kv4.hpp"

namespace cats {
namespace {

constexpr int kThreads = 256, kWaves = 4;
constexpr int kStep = 32;                // tokens of a wave's step
constexpr int kUnit = kWaves * kStep;    // tokens of a block's
constexpr float kLow = -3.402823466e+38f;  // maximum of a row that has seen no key
constexpr float kLazy = 8.f;

// Keys a tile reads: [lo, hi), from the record of lo on in units.
struct Span {
  int lo, hi, units;
};
__device__ __forceinline__ Span span_of(const KvAttentionArgs& a, int len, int nq, int G, int row0, int rows) {
  const int first = len - nq + row0 / G, last = len - nq + (row0 + rows - 1) / G;
  Span s;
  s.hi = min(max(last + 1, 0), len);
  s.lo = a.window > 0 ? min(max(first - a.window + 1, 0), s.hi) : 0;
  s.lo &= ~(kKvGroup - 1);
  s.units = max(1, (s.hi - s.lo + kUnit - 1) / kUnit);
  return s;
}

__device__ __forceinline__ int length_of(const KvAttentionArgs& a, int b) { return min(max(a.lens[b], 0), a.limit); }

// Queries [start, start + nq) of a sequence, whatever q_start holds.
__device__ __forceinline__ int queries_of(const KvAttentionArgs& a, int b, int& start) {
  if (!a.q_start) {
    start = b;
    return 1;
  }
  start = min(max(a.q_start[b], 0), a.N);
  return max(min(max(a.q_start[b + 1], 0), a.N) - start, 0);
}

// Exclusive prefix of v over the block's threads and its total.
template <int THREADS> __device__ __forceinline__ int block_scan(int v, int& total, int* sh) {
  const int lane = threadIdx.x % 64, w = threadIdx.x / 64;
  int x = v;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int y = __shfl_up(x, d);
    if (lane >= d) x += y;
  }
  __syncthreads();
  if (lane == 63) sh[w] = x;
  __syncthreads();
  int before = 0;
  total = 0;
#pragma unroll
  for (int i = 0; i < THREADS / 64; ++i) {
    if (i < w) before += sh[i];
    total += sh[i];
  }
  total = (int)uniform_u32(total);
  return before + x - v;
}

// ---- the plan: tiles of ragged queries --------------------------------------

constexpr int kPlanThreads = 1024;
__global__ __launch_bounds__(kPlanThreads) void k_kv_plan(KvAttentionArgs a, int R, int most) {
  __shared__ int sh[kPlanThreads / 64];
  const int G = a.hq / a.hkv;
  int tiles = 0;
  for (int base = 0; base < a.B; base += kPlanThreads) {
    const int b = base + threadIdx.x;
    int start, n = 0, total;
    if (b < a.B) n = (queries_of(a, b, start) * G + R - 1) / R;
    const int at = block_scan<kPlanThreads>(n, total, sh) + tiles;
    if (b < a.B) a.first[b] = at;
    tiles += total;
  }
  tiles = min(tiles, most);  // (more only where q_start overlaps: refused rows)
  __syncthreads();           // makes first[] visible to the block
  int units = 0;
  for (int base = 0; base < tiles; base += kPlanThreads) {
    const int e = base + threadIdx.x;
    int u = 0, total, b = 0, row0 = 0;
    if (e < tiles) {
      int lo = 0, n = a.B;  // the last sequence with first[b] <= e: it has tiles
      while (n > 1) {
        const int half = n / 2;
        if (a.first[lo + half] <= e) lo += half, n -= half;
        else n = half;
      }
      b = lo;
      row0 = (e - a.first[b]) * R;
      int start;
      const int nq = queries_of(a, b, start);
      u = span_of(a, length_of(a, b), nq, G, row0, min(R, nq * G - row0)).units;
    }
    const int at = block_scan<kPlanThreads>(u, total, sh) + units;
    if (e < tiles) {
      a.plan[e] = KvPlanEntry{b, row0};
      a.prefix[e] = at;
    }
    units += total;
  }
  if (threadIdx.x == 0) {
    a.head[0] = tiles;
    a.head[1] = units;
  }
}

// ---- the products ----------------------------------------------------------------

// A wave's part of two records: what one step needs.
template <int D> struct Step {
  uint32_t k[2][D / 32], v[2][D / 32];
  uint32_t ks[2], vs[2];
  uint32_t bad[2];  // all ones where the page is none of the cache's
};

template <int W> __device__ __forceinline__ void load_words(const uint8_t* p, uint32_t* w) {
  if constexpr (W == 2) {
    const u32x2 v = *reinterpret_cast<const u32x2*>(p);
    w[0] = v.x;
    w[1] = v.y;
  } else {
#pragma unroll
    for (int i = 0; i < W / 4; ++i) {
      const u32x4 v = reinterpret_cast<const u32x4*>(p)[i];
      w[4 * i] = v.x;
      w[4 * i + 1] = v.y;
      w[4 * i + 2] = v.z;
      w[4 * i + 3] = v.w;
    }
  }
}

__device__ __forceinline__ bf16x8 as_bf16x8(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  const u32x4 v = {a, b, c, d};
  return __builtin_bit_cast(bf16x8, v);
}

template <int SEL> __device__ __forceinline__ uint32_t two_of(uint32_t w, float s) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, SEL));
}
__device__ __forceinline__ bf16x8 eight_of(uint32_t w, float s) {
  return as_bf16x8(two_of<0>(w, s), two_of<1>(w, s), two_of<2>(w, s), two_of<3>(w, s));
}
// Byte c of the lane's D / 32 bytes of token i.
template <int D, int C> __device__ __forceinline__ uint32_t value_pair(const uint32_t* v, int i, float s) {
  if constexpr (D == 64) {
    return i % 2 ? two_of<2 + C>(v[i / 2], s) : two_of<C>(v[i / 2], s);
  } else {
    return two_of<C % 4>(v[i * (D / 128) + C / 4], s);
  }
}

__device__ __forceinline__ uint32_t low_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }
__device__ __forceinline__ uint32_t high_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }

// f as NP bf16 parts: 8 bits each, the last rounded to nearest.
__device__ __forceinline__ float cut(float f) { return __uint_as_float(__float_as_uint(f) & 0xffff0000u); }

template <int NP> __device__ __forceinline__ void split8(const float* f, bf16x8* out) {
  float r[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) r[i] = f[i];
#pragma unroll
  for (int p = 0; p < NP; ++p) {
    if (p == NP - 1) {
#pragma unroll
      for (int i = 0; i < 8; ++i) out[p][i] = (__bf16)r[i];
    } else {
      uint32_t w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = high_halves(__float_as_uint(r[2 * i]), __float_as_uint(r[2 * i + 1]));
      out[p] = as_bf16x8(w[0], w[1], w[2], w[3]);
#pragma unroll
      for (int i = 0; i < 8; ++i) r[i] -= cut(r[i]);
    }
  }
}

template <int D, int QT, bool BF16> struct Wave {
  static constexpr int NQ = BF16 ? 1 : 3, NP = BF16 ? 2 : 3;  // bf16 parts of q and of P
  bf16x8 q[QT][NQ][D / 32];
  f32x4 o[QT][D / 16];  // o[t][j][i]: row lane % 16, column g D/4 + i D/16 + j
  float m[QT], l[QT];   // maximum (times c), the lane's part of the sum
  int pos[QT];          // the row's position, -1 and less: sees nothing
};

// Rows `row0 .. row0 + rows` of key head h of the sequence; q rows as bf16 parts.
template <int D, int QT, bool BF16>
__device__ __forceinline__ void load_q(Wave<D, QT, BF16>& w, const KvAttentionArgs& a, int h, int start, int nq, int len,
                                       int row0, int rows) {
  const int lane = threadIdx.x % 64, g = lane / 16, G = a.hq / a.hkv;
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const int r = min(t * 16 + lane % 16, rows - 1);  // (rows behind the last repeat it and are not stored)
    const int i = (row0 + r) / G, head = h * G + (row0 + r) % G;
    w.pos[t] = len - nq + i;
    w.m[t] = kLow;
    w.l[t] = 0.f;
    const size_t at = ((size_t)(start + i) * a.hq + head) * D + g * (D / 4);
#pragma unroll
    for (int j = 0; j < D / 32; ++j) {
      if constexpr (BF16) {
        w.q[t][0][j] = *reinterpret_cast<const bf16x8*>(static_cast<const uint16_t*>(a.q) + at + 8 * j);
      } else {
        const f32x4* p = reinterpret_cast<const f32x4*>(static_cast<const float*>(a.q) + at + 8 * j);
        const f32x4 x = p[0], y = p[1];
        const float f[8] = {x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
        bf16x8 part[3];
        split8<3>(f, part);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          // an infinity or NaN is in the first part alone
          const bool whole = (__float_as_uint(f[e]) & 0x7f800000u) == 0x7f800000u;
          w.q[t][0][j][e] = whole ? (__bf16)f[e] : part[0][e];
          w.q[t][1][j][e] = whole ? (__bf16)0.f : part[1][e];
          w.q[t][2][j][e] = whole ? (__bf16)0.f : part[2][e];
        }
      }
    }
#pragma unroll
    for (int j = 0; j < D / 16; ++j) w.o[t][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
}

template <int D, int C, int QT, bool BF16>
__device__ __forceinline__ void value_products(Wave<D, QT, BF16>& w, const Step<D>& s, const float (&sc)[2][4],
                                               const bf16x8 (&p)[QT][Wave<D, QT, BF16>::NP]) {
  uint32_t e[2][4];
#pragma unroll
  for (int u = 0; u < 2; ++u)
#pragma unroll
    for (int i = 0; i < 4; ++i) e[u][i] = value_pair<D, C>(s.v[u], i, sc[u][i]);
  const bf16x8 lo = as_bf16x8(low_halves(e[0][0], e[0][1]), low_halves(e[0][2], e[0][3]), low_halves(e[1][0], e[1][1]),
                              low_halves(e[1][2], e[1][3]));
  const bf16x8 hi = as_bf16x8(high_halves(e[0][0], e[0][1]), high_halves(e[0][2], e[0][3]),
                              high_halves(e[1][0], e[1][1]), high_halves(e[1][2], e[1][3]));
#pragma unroll
  for (int t = 0; t < QT; ++t) {
#pragma unroll
    for (int n = 0; n < Wave<D, QT, BF16>::NP; ++n) {
      w.o[t][2 * C] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(lo, p[t][n], w.o[t][2 * C], 0, 0, 0);
      w.o[t][2 * C + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(hi, p[t][n], w.o[t][2 * C + 1], 0, 0, 0);
    }
  }
  if constexpr (C + 1 < D / 32) value_products<D, C + 1, QT, BF16>(w, s, sc, p);
}

// Tokens [tok, tok + 32): scores, softmax and the sum.  MASK: not every row sees all of them.
template <int D, int QT, bool BF16, bool MASK>
__device__ __forceinline__ void step(Wave<D, QT, BF16>& w, const KvAttentionArgs& a, const Step<D>& s, int tok, int len) {
  typedef Wave<D, QT, BF16> W;
  const int lane = threadIdx.x % 64, g = lane / 16;
  f32x4 z[QT][2];
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    bf16x8 k[D / 32];
    const uint32_t ks = s.ks[u] | s.bad[u];
#pragma unroll
    for (int j = 0; j < D / 32; ++j)
      k[j] = eight_of(s.k[u][j], D == 256 && j >= 4 ? kv_scale(ks >> 8 & 0xffu) : kv_scale(ks & 0xffu));
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      f32x4 c = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int n = W::NQ - 1; n >= 0; --n)
#pragma unroll
        for (int j = 0; j < D / 32; ++j) c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[j], w.q[t][n][j], c, 0, 0, 0);
      z[t][u] = c;
    }
  }
  uint32_t vs[2] = {s.vs[0], s.vs[1]};
  uint32_t nan = 0;  // MASK: bit t: the row sees a NaN among its columns' values
  if constexpr (MASK) {
    uint32_t odd = 0;
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int j = tok + 16 * u + 4 * g + i;
#pragma unroll
        for (int t = 0; t < QT; ++t) {
          const bool seen = j <= w.pos[t] && (a.window <= 0 || j > w.pos[t] - a.window);
          z[t][u][i] = seen ? z[t][u][i] : -__builtin_inff();
        }
        // A hidden token's p is 0, but 0 times NaN is not: scales of NaN (and the two
        // whose values leave fp32, which are in a cache only where nothing was written)
        // become 1, and those of tokens that some row sees are looked at below.
        if ((vs[u] >> (8 * i) & 0xffu) > kKvMaxExp + 127) {
          vs[u] = (vs[u] & ~(0xffu << (8 * i))) | 0x7fu << (8 * i);
          odd |= j < len ? 1u << (4 * u + i) : 0u;
        }
      }
    if (__ballot(odd != 0)) {
      // Token 16 u + 4 g' + i is NaN in the columns of lane (n', g').  A lane's columns
      // of o are those of all n' with n' D/16 in [g D/4, (g+1) D/4): four of them.
      for (int u = 0; u < 2; ++u)
        for (int gg = 0; gg < 4; ++gg)
          for (int i = 0; i < 4; ++i) {
            const int j = tok + 16 * u + 4 * gg + i;
            for (int n = 0; n < 4; ++n) {
              const uint32_t there = __shfl(odd, gg * 16 + 4 * g + n);
              if (there >> (4 * u + i) & 1u) {
                for (int t = 0; t < QT; ++t)
                  if (j <= w.pos[t] && (a.window <= 0 || j > w.pos[t] - a.window)) nan |= 1u << (4 * t + n);
              }
            }
          }
    }
  }
  bf16x8 p[QT][W::NP];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    float top = z[t][0][0];
#pragma unroll
    for (int i = 1; i < 8; ++i) top = fmaxf(top, z[t][i / 4][i % 4]);
    top *= a.c;
    if (__ballot(top > w.m[t] + kLazy)) {  // (kLow + 8 is kLow)
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      const float m = fmaxf(w.m[t], top), f = __builtin_amdgcn_exp2f(w.m[t] - m);
      w.m[t] = m;
      w.l[t] *= f;
#pragma unroll
      for (int j = 0; j < D / 16; ++j) w.o[t][j] *= f;
    }
    float e[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      e[i] = __builtin_amdgcn_exp2f(fmaf(z[t][i / 4][i % 4], a.c, -w.m[t]));
      w.l[t] += e[i];
    }
    split8<W::NP>(e, p[t]);
  }
  float sc[2][4];
#pragma unroll
  for (int u = 0; u < 2; ++u)
#pragma unroll
    for (int i = 0; i < 4; ++i) sc[u][i] = kv_scale(vs[u] >> (8 * i) & 0xffu);
  value_products<D, 0, QT, BF16>(w, s, sc, p);
  if constexpr (MASK) {
    if (__ballot(nan != 0)) {
#pragma unroll
      for (int t = 0; t < QT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (nan >> (4 * t + i) & 1u) {
#pragma unroll
            for (int j = 0; j < D / 16; ++j) w.o[t][j][i] = __builtin_nanf("");
          }
    }
  }
}

template <int D, int QT, bool BF16> struct Sizes {
  static constexpr int WAVES = D * QT >= 256 ? 1 : 2;  // of a SIMD: what the registers allow
  static constexpr int R = 16 * QT;
  static constexpr int PITCH = D + 4;
  static constexpr int PART = R * (D + 2);  // floats of a partial sum: o, then m, then l
};

template <bool BF16> __device__ __forceinline__ void store_out(void* out, size_t at, const f32x4& v) {
  if (BF16) {
    typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
    *reinterpret_cast<bf16x4*>(static_cast<uint16_t*>(out) + at) = bf16x4{(__bf16)v[0], (__bf16)v[1], (__bf16)v[2], (__bf16)v[3]};
  } else {
    *reinterpret_cast<f32x4*>(static_cast<float*>(out) + at) = v;
  }
}

template <int D, int QT, bool BF16, bool PLAN>
__global__ __launch_bounds__(kThreads, (Sizes<D, QT, BF16>::WAVES)) void k_kv_attention(KvAttentionArgs a) {
  typedef Sizes<D, QT, BF16> Z;
  constexpr int R = Z::R;
  __shared__ float so[kWaves][16][Z::PITCH];
  __shared__ float sm[kWaves][R], sl[kWaves][R];
  __shared__ int sh[8];
  const int wave = uniform_u32(threadIdx.x / 64), lane = threadIdx.x % 64, g = lane / 16;
  const int G = a.hq / a.hkv;
  // units of a head, and the block's run of all heads' units
  long long W = 0;
  const int tiles = PLAN ? a.head[0] : a.tiles;
  if constexpr (PLAN) {
    W = a.head[1];
  } else {
    for (int base = 0; base < a.B; base += kThreads) {
      const int b = base + threadIdx.x;
      int total;
      block_scan<kThreads>(b < a.B ? tiles * span_of(a, length_of(a, b), 1, G, 0, 1).units : 0, total, sh);
      W += total;
    }
  }
  // Every block has a unit or more, but those behind the last unit: a sum's parts are in
  // blocks without a gap.  Runs next to each other are on one XCD, which shares their keys.
  const long long T = W * a.hkv;
  const int nb = (int)min(T, (long long)a.blocks);
  const int lb = nb < a.blocks ? (int)blockIdx.x : (int)(blockIdx.x % 8) * (nb / 8) + (int)(blockIdx.x / 8);
  if (threadIdx.x == 0) a.desc[lb] = int4{0, 0, 0, 0};
  if (lb >= nb) return;
  const long long p0 = T * lb / nb, p1 = T * (lb + 1) / nb;

  // where the run begins: head, tile (sequence and rows) and unit within it
  int h = (int)(p0 / W);
  const int x = (int)(p0 - h * W);
  int b = 0, e = 0, before = 0;
  if constexpr (PLAN) {
    int lo = 0, n = tiles;
    while (n > 1) {
      const int stride = (n + kThreads - 1) / kThreads, at = threadIdx.x * stride;
      const int last = (int)uniform_u32(__syncthreads_count(at < n && a.prefix[lo + at] <= x)) - 1;
      lo += last * stride;
      n = min(stride, n - last * stride);
    }
    e = lo;
    before = a.prefix[e];
  } else {
    int sum = 0;
    for (int base = 0; base < a.B; base += kThreads) {
      const int bb = base + threadIdx.x;
      const int u = bb < a.B ? tiles * span_of(a, length_of(a, bb), 1, G, 0, 1).units : 0;
      int total;
      const int at = block_scan<kThreads>(u, total, sh) + sum;
      if (at <= x && x < at + u) {
        sh[4] = bb;
        sh[5] = at;
      }
      sum += total;
      if (x < sum) break;
    }
    __syncthreads();
    b = (int)uniform_u32(sh[4]);
    before = (int)uniform_u32(sh[5]);
    const int units = span_of(a, length_of(a, b), 1, G, 0, 1).units;
    e = (x - before) / units;  // (the sequence's tile)
    before += e * units;
  }
  int skip = x - before;

  for (long long p = p0; p < p1;) {
    int row0, rows, start, nq;
    if constexpr (PLAN) {
      const KvPlanEntry t = a.plan[e];
      b = t.b;
      row0 = t.row0;
      nq = queries_of(a, b, start);
      rows = min(R, nq * G - row0);
    } else {
      nq = 1;
      start = b;
      row0 = e * R;
      rows = min(R, G - row0);
    }
    const int len = length_of(a, b);
    const Span sp = span_of(a, len, nq, G, row0, rows);
    const int u1 = (int)min((long long)sp.units, skip + (p1 - p));
    const bool head = skip == 0, tail = u1 == sp.units;

    Wave<D, QT, BF16> w;
    load_q<D, QT, BF16>(w, a, h, start, nq, len, row0, rows);
    const int first = len - nq + row0 / G, last = len - nq + (row0 + rows - 1) / G;
    const int* table = a.table + (size_t)b * a.width;
    const int end = min(sp.hi, sp.lo + u1 * kUnit), most = (max(sp.hi, 1) - 1) / kKvGroup;

    const auto page_of = [&](int rec) { return (int)__umulhi((uint32_t)rec << 1, a.magic); };
    const auto entry = [&](int tok, int u) { return table[page_of(min(tok / kKvGroup + u, most))]; };
    const auto load = [&](Step<D>& s, int tok, const int (&page)[2]) {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int rec = min(tok / kKvGroup + u, most), in = rec - page_of(rec) * a.groups;
        const bool ok = (uint32_t)page[u] < (uint32_t)a.pages;
        const uint8_t* r = a.cache + (((size_t)(ok ? page[u] : 0) * a.hkv + h) * a.groups + in) * kv_record_bytes(D);
        s.bad[u] = ok ? 0u : 0xffffu;
        load_words<D / 32>(r + (lane % 16) * (D / 2) + g * (D / 8), s.k[u]);
        load_words<D / 32>(r + 8 * D + lane * (D / 8), s.v[u]);
        const uint8_t* ks = r + 16 * D + (lane % 16) * (D / 32);
        if constexpr (D == 256) s.ks[u] = *reinterpret_cast<const uint16_t*>(ks + 2 * g);
        else s.ks[u] = ks[D == 128 ? g : g / 2];
        s.vs[u] = *reinterpret_cast<const uint32_t*>(r + 16 * D + D / 2 + g * (D / 8) + (lane % 16) * D / 512 * 4);
      }
    };

    int tok = sp.lo + skip * kUnit + wave * kStep;
    if (tok < end) {
      Step<D> cur, next;
      int page[2] = {entry(tok, 0), entry(tok, 1)};
      load(cur, tok, page);
      page[0] = entry(tok + kUnit, 0);
      page[1] = entry(tok + kUnit, 1);
      for (;;) {
        load(next, tok + kUnit, page);
        page[0] = entry(tok + 2 * kUnit, 0);
        page[1] = entry(tok + 2 * kUnit, 1);
        const bool all = tok + kStep - 1 <= first && (a.window <= 0 || tok > last - a.window);
        if (all) step<D, QT, BF16, false>(w, a, cur, tok, len);
        else step<D, QT, BF16, true>(w, a, cur, tok, len);
        tok += kUnit;
        if (tok >= end) break;
        cur = next;
      }
    }

    // the waves' sums together, 16 rows at a time
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      float l = w.l[t];
      l += __shfl_xor(l, 16);
      l += __shfl_xor(l, 32);
      if (g == 0) {
        sm[wave][t * 16 + lane] = w.m[t];
        sl[wave][t * 16 + lane] = l;
      }
    }
    float* part = a.part + ((size_t)lb * 2 + (head ? 1 : 0)) * Z::PART;
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      __syncthreads();
      const int r16 = t * 16 + lane % 16;
      const float top = fmaxf(fmaxf(sm[0][r16], sm[1][r16]), fmaxf(sm[2][r16], sm[3][r16]));
      const float f = __builtin_amdgcn_exp2f(w.m[t] - top);
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < D / 16; j += 4)
          *reinterpret_cast<f32x4*>(&so[wave][lane % 16][g * (D / 4) + i * (D / 16) + j]) =
              f32x4{w.o[t][j][i] * f, w.o[t][j + 1][i] * f, w.o[t][j + 2][i] * f, w.o[t][j + 3][i] * f};
      __syncthreads();
      for (int v = threadIdx.x; v < 16 * (D / 4); v += kThreads) {
        const int r = v / (D / 4), c = v % (D / 4) * 4, row = t * 16 + r;
        if (row >= rows) break;
        f32x4 o = {0.f, 0.f, 0.f, 0.f};
        float m = kLow, l = 0.f;
#pragma unroll
        for (int i = 0; i < kWaves; ++i) {
          o += *reinterpret_cast<const f32x4*>(&so[i][r][c]);
          m = fmaxf(m, sm[i][row]);
        }
#pragma unroll
        for (int i = 0; i < kWaves; ++i) l += sl[i][row] * __builtin_amdgcn_exp2f(sm[i][row] - m);
        const int qi = (row0 + row) / G;
        const bool empty = len - nq + qi < 0;  // sees no key: zeros
        if (head && tail) {
          const float inv = 1.f / l;
          o *= inv;
          if (empty) o = f32x4{0.f, 0.f, 0.f, 0.f};
          store_out<BF16>(a.out, ((size_t)(start + qi) * a.hq + h * G + (row0 + row) % G) * D + c, o);
        } else {
          *reinterpret_cast<f32x4*>(part + row * D + c) = o;
          if (c == 0) {
            part[R * D + row] = empty ? -__builtin_inff() : m;
            part[R * D + R + row] = l;
          }
        }
      }
    }
    if (head && !tail && threadIdx.x == 0) {
      const long long stop = p + sp.units - 1;  // the tile's last unit, and the block that has it
      const int until = (int)(((stop + 1) * nb - 1) / T);
      a.desc[lb] = int4{until - lb + 1, h, b, row0};
    }
    __syncthreads();

    p += u1 - skip;
    skip = 0;
    // the next tile
    ++e;
    if constexpr (PLAN) {
      if (e == tiles) e = 0, ++h;
    } else {
      if (e == tiles) {
        e = 0;
        if (++b == a.B) b = 0, ++h;
      }
    }
  }
}

// Joins the sum that begins in block lb: its first part there, the others in the blocks behind it.
template <int D, int QT, bool BF16> __global__ __launch_bounds__(kThreads) void k_kv_join(KvAttentionArgs a) {
  typedef Sizes<D, QT, BF16> Z;
  constexpr int R = Z::R;
  const int lb = blockIdx.x, lane = threadIdx.x % 64;
  const int4 d = a.desc[lb];
  if (d.x == 0) return;
  const int n = d.x, h = d.y, b = d.z, row0 = d.w, G = a.hq / a.hkv;
  int start;
  const int nq = queries_of(a, b, start);
  const int row = blockIdx.y * (kThreads / 64) + threadIdx.x / 64;
  if (row >= R || row >= nq * G - row0) return;
  const float* base = a.part + (size_t)lb * 2 * Z::PART;
  const auto part = [&](int i) { return base + (size_t)(i == 0 ? 1 : 2 * i) * Z::PART; };
  float m = -__builtin_inff();
  for (int i = lane; i < n; i += 64) m = fmaxf(m, part(i)[R * D + row]);
#pragma unroll
  for (int s = 1; s < 64; s *= 2) m = fmaxf(m, __shfl_xor(m, s));
  constexpr int C = D / 64;  // columns of a lane
  float o[C], l = 0.f;
#pragma unroll
  for (int c = 0; c < C; ++c) o[c] = 0.f;
  const bool empty = m == -__builtin_inff();
  if (!empty) {
#pragma unroll 4
    for (int i = 0; i < n; ++i) {
      const float* p = part(i);
      const float f = __builtin_amdgcn_exp2f(p[R * D + row] - m);
      l += p[R * D + R + row] * f;
#pragma unroll
      for (int c = 0; c < C; ++c) o[c] += p[row * D + lane * C + c] * f;
    }
  }
  const float inv = 1.f / l;
  const size_t at = ((size_t)(start + (row0 + row) / G) * a.hq + h * G + (row0 + row) % G) * D + lane * C;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const float v = empty ? 0.f : o[c] * inv;
    if (BF16) reinterpret_cast<__bf16*>(a.out)[at + c] = (__bf16)v;
    else static_cast<float*>(a.out)[at + c] = v;
  }
}

// Rows of a tile, and what a call takes of the workspace.
struct Shape {
  int qt;                // tiles of 16 rows
  int blocks;            // blocks at most
  size_t tiles;          // entries of the plan at most (0: none)
  size_t off_plan, off_prefix, off_first, off_desc, off_part, bytes;
};
constexpr size_t up256(size_t v) { return (v + 255) / 256 * 256; }

// One to a compute unit, or two: all run at once.
int blocks_of(int d, int qt) { return d * qt >= 256 ? 256 : 512; }
size_t part_bytes(int d, int qt) { return (size_t)blocks_of(d, qt) * 2 * 16 * qt * (d + 2) * 4; }

Shape shape_of(int N, int B, int hq, int hkv, int d, bool planned) {
  Shape s{};
  const int G = hq / hkv;
  // 16 rows to a tile while they hold all of a sequence's rows, 32 beyond
  const long long per = planned ? ((long long)N * G + B - 1) / B : G;
  s.qt = per > 16 && d < 256 ? 2 : 1;
  const int R = 16 * s.qt;
  s.blocks = blocks_of(d, s.qt);
  s.tiles = planned ? (size_t)(((long long)N * G + R - 1) / R + B) : 0;
  s.off_plan = 256;
  s.off_prefix = s.off_plan + up256(s.tiles * sizeof(KvPlanEntry));
  s.off_first = s.off_prefix + up256(s.tiles * 4);
  s.off_desc = s.off_first + (planned ? up256((size_t)(B + 1) * 4) : 0);
  s.off_part = s.off_desc + up256((size_t)s.blocks * 16);
  s.bytes = s.off_part + part_bytes(d, s.qt);
  return s;
}

template <int D, int QT, bool BF16> hipError_t go(const KvAttentionArgs& a, bool join, hipStream_t s) {
  constexpr int R = 16 * QT;
  const dim3 th(kThreads);
  if (a.q_start) {
    {
      KernelTimer tm("kv_plan", s);
      const int G = a.hq / a.hkv;
      const int most = (int)(((long long)a.N * G + R - 1) / R + a.B);
      hipExtLaunchKernelGGL((k_kv_plan), dim3(1), dim3(kPlanThreads), 0, s, tm.start(), tm.stop(), 0, a, R, most);
    }
    KernelTimer tm("kv_attention", s);
    hipExtLaunchKernelGGL((k_kv_attention<D, QT, BF16, true>), dim3(a.blocks), th, 0, s, tm.start(), tm.stop(), 0, a);
  } else {
    KernelTimer tm("kv_attention", s);
    hipExtLaunchKernelGGL((k_kv_attention<D, QT, BF16, false>), dim3(a.blocks), th, 0, s, tm.start(), tm.stop(), 0, a);
  }
  if (join) {
    KernelTimer tm("kv_join", s);
    hipExtLaunchKernelGGL((k_kv_join<D, QT, BF16>), dim3(a.blocks, (R + 3) / 4), th, 0, s, tm.start(), tm.stop(), 0, a);
  }
  return hipGetLastError();
}

}  // namespace

size_t kv_attention_bytes(int N, int B, int hq, int hkv, int d, bool /*bf16*/, bool planned) {
  return shape_of(N, B, hq, hkv, d, planned).bytes;
}

size_t kv_attention_most(int N, int B, int hq, int hkv, int d) {
  const size_t tiles = ((size_t)N * (hq / hkv) + 15) / 16 + B;
  return 256 + up256(tiles * sizeof(KvPlanEntry)) + up256(tiles * 4) + up256((size_t)(B + 1) * 4) + up256(512 * 16) +
         std::max(part_bytes(d, 1), part_bytes(d, d < 256 ? 2 : 1));
}

hipError_t launch_kv_attention(KvAttentionArgs a, int d, bool bf16, hipStream_t s) {
  const Shape sh = shape_of(a.N, a.B, a.hq, a.hkv, d, a.q_start != nullptr);
  uint8_t* ws = reinterpret_cast<uint8_t*>(a.head);
  a.plan = reinterpret_cast<KvPlanEntry*>(ws + sh.off_plan);
  a.prefix = reinterpret_cast<int*>(ws + sh.off_prefix);
  a.first = reinterpret_cast<int*>(ws + sh.off_first);
  a.desc = reinterpret_cast<int4*>(ws + sh.off_desc);
  a.part = reinterpret_cast<float*>(ws + sh.off_part);
  const int R = 16 * sh.qt, G = a.hq / a.hkv;
  a.tiles = (G + R - 1) / R;
  // no more blocks than units; tiles of one unit need no join
  const long long per = (a.limit + kUnit - 1 + (a.window > 0 ? kKvGroup : 0)) / kUnit;
  const long long units = (a.q_start ? (long long)sh.tiles : (long long)a.B * a.tiles) * a.hkv * std::max(1ll, per);
  a.blocks = (int)std::min<long long>(sh.blocks, (units + 7) / 8 * 8);
  const bool join = per > 1;
#define CATS_D(D, Q) return bf16 ? go<D, Q, true>(a, join, s) : go<D, Q, false>(a, join, s)
  if (d == 256) CATS_D(256, 1);
  if (sh.qt == 1) {
    if (d == 64) CATS_D(64, 1);
    CATS_D(128, 1);
  }
  if (d == 64) CATS_D(64, 2);
  CATS_D(128, 2);
#undef CATS_D
}

}  // namespace cats
