// Attention over the cache in 4 bits for few rows of each sequence: single tokens.
//
// Bound by the cache's bytes.  A wave takes 32 tokens a step for a tile of 16 QT rows (the
// query heads of a key head side by side, then the next query) and keeps all of it in its
// registers: no step waits for another wave.  Two steps' loads are under way; a block's
// four waves take every fourth step of its tokens and add their sums through LDS.
// 8 key heads of 128 columns with 4 query heads each, 32 sequences (311 MB of cache in all):
// 57.5 us, 5.4 TB/s; 32 heads of their own, 16 sequences (95 MB): 27.2 us, of which the bytes
// would be 13 at a plain read's rate.  The rest is the launch, and what a tile's end and the next one's start
// leave empty: no key is under way while the sums are joined and the next tile's length, table and q
// are read, and a tile's last two steps load its last record again for nothing.
#pragma once

#include "kv_attention.hpp"
#include "ticket.hpp"

namespace cats {
namespace {

constexpr int kThreads = kKvThreads, kWaves = kKvWaves;
constexpr int kStep = 32;              // tokens of a wave's step
constexpr int kUnit = kWaves * kStep;  // tokens of a block's
static_assert(kUnit == kKvRowsUnit, "the host shares out the kernel's units");
constexpr int kLeadUnits = kKvRowsLead;

// A wave's part of two records: what one step needs.
template <int D> struct Step {
  uint32_t k[2][D / 32], v[2][D / 32];
  uint32_t ks[2], vs[2];
  uint32_t bad[2];  // all ones where the page is none of the cache's
};

// How a kernel of D columns, QT tiles of 16 rows and this type is laid out.
template <int D, int QT, bool BF16> struct Sizes {
  static constexpr int R = 16 * QT;
  static constexpr int NQ = BF16 ? 1 : 3;  // bf16 parts of q
  static constexpr int NP = BF16 ? 1 : 2;  // f16 parts of P
  // q's operands are in registers, or where they would take too many in LDS, for all waves
  static constexpr bool QLDS = QT * NQ * D > 3 * 128 || QT * D >= 256;
  static constexpr int QBYTES = QLDS ? QT * NQ * (D / 32) * 64 * 16 : 0;
  static constexpr int PITCH = D + 4;
  static constexpr int SOBYTES = kWaves * 16 * PITCH * 4;
  static constexpr int POOL = QBYTES > SOBYTES ? QBYTES : SOBYTES;
  static constexpr int WAVES = kv_rows_waves(D, QT, BF16);
  static constexpr int DEPTH = 2;  // steps whose loads are under way
  static constexpr int PART = R * (D + 2);  // floats of a partial sum: o, then m, then l
};

template <int D, int QT, bool BF16> struct Wave : KvSums<D, QT> {
  typedef Sizes<D, QT, BF16> Z;
  bf16x8 q[Z::QLDS ? 1 : QT][Z::NQ][D / 32];
};

// A tile's rows of key head h; sq: LDS for their operands.
template <int D, int QT, bool BF16>
__device__ __forceinline__ void load_q(Wave<D, QT, BF16>& w, const KvAttentionArgs& a, int h, const KvTile& tile, bf16x8* sq) {
  typedef Sizes<D, QT, BF16> Z;
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, g = lane / 16, G = a.hq / a.hkv;
  clear<D, QT>(w, a);
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const int r = min(t * 16 + lane % 16, tile.rows - 1);  // (rows behind the last repeat it and are not stored)
    const int i = (tile.row0 + r) / G, head = h * G + (tile.row0 + r) % G;
    w.pos[t] = tile.len - tile.nq + i;
    const size_t at = ((size_t)(tile.start + i) * a.hq + head) * D + g * (D / 4);
    if constexpr (Z::QLDS) {
#pragma unroll
      for (int j = 0; j < D / 32 / kWaves + (D / 32 < kWaves); ++j) {
        const int jj = j * kWaves + (D / 32 < kWaves ? wave % (D / 32) : wave);
        bf16x8 part[Z::NQ];
        load_q8<Z::NQ>(a.q, at + 8 * jj, part);
#pragma unroll
        for (int n = 0; n < Z::NQ; ++n) sq[((t * Z::NQ + n) * (D / 32) + jj) * 64 + lane] = part[n];
      }
    } else {
#pragma unroll
      for (int j = 0; j < D / 32; ++j) {
        bf16x8 part[Z::NQ];
        load_q8<Z::NQ>(a.q, at + 8 * j, part);
#pragma unroll
        for (int n = 0; n < Z::NQ; ++n) w.q[t][n][j] = part[n];
      }
    }
  }
  if constexpr (Z::QLDS) __syncthreads();
}

// Tokens [tok, tok + 32): scores, softmax and the sum.  `masked`: not every row sees all of
// them; no row sees one from hi on.  `keys` and `values` load the step after next's into s as
// soon as its registers are free.
template <int D, int QT, bool BF16, typename Keys, typename Values>
__device__ __forceinline__ void step(Wave<D, QT, BF16>& w, const KvAttentionArgs& a, Step<D>& s, int tok, int hi,
                                     bool masked, const bf16x8* sq, const Keys& keys, const Values& values) {
  typedef Sizes<D, QT, BF16> Z;
  const int lane = threadIdx.x % 64, g = lane / 16;
  f32x4 z[QT][2];
  if constexpr (Z::QLDS) asm volatile("" ::: "memory");  // (q is read from LDS in each step, not kept)
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
      for (int n = Z::NQ - 1; n >= 0; --n)
#pragma unroll
        for (int j = 0; j < D / 32; ++j) {
          bf16x8 q;
          if constexpr (Z::QLDS) q = sq[((t * Z::NQ + n) * (D / 32) + j) * 64 + lane];
          else q = w.q[t][n][j];
          c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[j], q, c, 0, 0, 0);
        }
      z[t][u] = c;
    }
  }
  keys(s);
  uint32_t vs[2] = {s.vs[0], s.vs[1]};
  if (__builtin_expect(masked, 0)) {
    asm volatile("");
#pragma unroll
    for (int u = 0; u < 2; ++u) vs[u] = hidden_as_one(vs[u], tok + 16 * u + 4 * g, hi);
  }
  weights<D, QT, 2>(w, a, z, tok, masked);
  if (__builtin_expect(__ballot((not_narrow(vs[0]) | not_narrow(vs[1])) != 0) != 0, 0)) {
    asm volatile("");
    wide_values<D, QT, 2>(w, a, s.v, vs, z, 0, tok);
    no_values(s.v[0], vs[0]);
    no_values(s.v[1], vs[1]);
  }
  f16x8 part[QT][Z::NP];
  weight_operands<QT, Z::NP, 2>(z, 0, part);
  float sc[2][4];
#pragma unroll
  for (int u = 0; u < 2; ++u)
#pragma unroll
    for (int i = 0; i < 4; ++i) sc[u][i] = kv_scale(vs[u] >> (8 * i) & 0xffu);
  products<D, 0, QT, Z::NP>(w, s.v, sc, part);
  values(s);
}

// The block that arrives last joins a tile's n parts: the first in block `first`, the others in
// those behind it.  D / 4 threads have a row of a part; rows are side by side, and where there
// are few of them, parts.
template <int D, bool BF16>
__device__ __forceinline__ void join_parts(const KvAttentionArgs& a, __amdgpu_buffer_rsrc_t parts, int first, int n, int size, int R,
                                           const KvTile& tile, int h, uint8_t* lds) {
  constexpr int L = D / 4, S = kThreads / L;
  float (*so)[D] = reinterpret_cast<float (*)[D]>(lds);
  float* sm = reinterpret_cast<float*>(lds) + S * D;
  float* sl = sm + S;
  const int s = threadIdx.x / L, c = threadIdx.x % L * 4, G = a.hq / a.hkv;
  int side = 1;  // rows side by side
  while (side < S && side < tile.rows) side *= 2;
  const int sub = s / side, subs = S / side;
  for (int r0 = 0; r0 < tile.rows; r0 += side) {
    const int row = r0 + s % side;
    float m = -__builtin_inff(), l = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    if (row < tile.rows) {
      // four parts' loads under way; one behind the last reads as zeros, and counts for none
      for (int i0 = sub; i0 < n; i0 += 4 * subs) {
        f32x4 po[4];
        float pm[4], pl[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int i = i0 + k * subs;
          const uint32_t p = i < n ? (uint32_t)(2 * (first + i) + (i == 0 ? 1 : 0)) * (uint32_t)(size * 4) : kOOB;
          po[k] = __builtin_bit_cast(f32x4, ld_buf16_coherent(parts, p + (row * D + c) * 4));
          pm[k] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(parts, (int)(p + (R * D + row) * 4), 0, kCachePolicySc1));
          pl[k] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(parts, (int)(p + (R * D + R + row) * 4), 0, kCachePolicySc1));
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float is_m = i0 + k * subs < n ? pm[k] : -__builtin_inff();
          const float top = fmaxf(m, is_m);
          const float was = m == top ? 1.f : __builtin_amdgcn_exp2f(m - top);
          const float is = is_m == top ? 1.f : __builtin_amdgcn_exp2f(is_m - top);
          m = top;
          l = l * was + pl[k] * is;
          o = o * was + po[k] * is;
        }
      }
    }
    __syncthreads();
    *reinterpret_cast<f32x4*>(&so[s][c]) = o;
    if (c == 0) {
      sm[s] = m;
      sl[s] = l;
    }
    __syncthreads();
    if (sub == 0 && row < tile.rows) {
      float top = m;
      for (int i = 1; i < subs; ++i) top = fmaxf(top, sm[s + i * side]);
      l = 0.f;
      o = f32x4{0.f, 0.f, 0.f, 0.f};
      for (int i = 0; i < subs; ++i) {
        const int from = s + i * side;
        if (sm[from] == -__builtin_inff()) continue;  // (fewer parts than that, or a row that sees no key)
        const float f = __builtin_amdgcn_exp2f(sm[from] - top);
        l += sl[from] * f;
        o += *reinterpret_cast<const f32x4*>(&so[from][c]) * f;
      }
      o *= 1.f / l;
      if (top == -__builtin_inff()) o = f32x4{0.f, 0.f, 0.f, 0.f};
      const int i = (tile.row0 + row) / G;
      store_out<BF16>(a.out, ((size_t)(tile.start + i) * a.hq + h * G + (tile.row0 + row) % G) * D + c, o);
    }
  }
}

template <int D, int QT, bool BF16, bool PLAN>
__global__ __launch_bounds__(kThreads, (Sizes<D, QT, BF16>::WAVES)) void k_kv_rows(KvAttentionArgs a) {
  typedef Sizes<D, QT, BF16> Z;
  constexpr int R = Z::R;
  __shared__ __attribute__((aligned(16))) uint8_t pool[Z::POOL];  // q's operands, then the waves' sums
  bf16x8* sq = reinterpret_cast<bf16x8*>(pool);
  float (*so)[16][Z::PITCH] = reinterpret_cast<float (*)[16][Z::PITCH]>(pool);
  __shared__ float sm[kWaves][R], sl[kWaves][R];
  __shared__ int sh[13];
  const int wave = uniform_u32(threadIdx.x / 64), lane = threadIdx.x % 64, g = lane / 16;
  const int G = a.hq / a.hkv;
  const KvLane<D> off;
  KvOwnPlan* own = nullptr;
  if constexpr (PLAN) {
    __shared__ KvOwnPlan of_block;
    own = &of_block;
  }
  KvRun run;
  if (!kv_run<PLAN, kUnit, kLeadUnits, R>(a, run, sh, own)) return;

  while (run.p < run.p1) {
    const KvTile tile = kv_tile_of<PLAN, kUnit, R>(a, G, run, own);
    const KvPart p = kv_part<kLeadUnits>(run, tile);
    if (p.u0 >= p.u1) {
      kv_next<PLAN, kLeadUnits>(a, run, tile, p);
      continue;
    }
    const int h = run.h, row0 = tile.row0, rows = tile.rows, start = tile.start;
    // (the ticket's word is read now, so that arriving costs one atomic)
    int n = 1, first_block = run.lb;
    unsigned long long peek = 0;
    if (!PLAN && a.parts > 0 && !p.whole) {
      first_block = kv_parts_of<kLeadUnits>(run, tile, p, n);
      if (threadIdx.x == 0) peek = ticket_peek(a.tickets + first_block);
    }
    Wave<D, QT, BF16> w;
    load_q<D, QT, BF16>(w, a, h, tile, sq);
    const KvRecords<D> records(a, tile.b, h, tile.hi);
    const int end = min(tile.hi, tile.lo + p.u1 * kUnit);

    // The places of a step's records are read a step before these are.
    typename KvRecords<D>::Place at[2];
    const auto find = [&](int tok) {
#pragma unroll
      for (int u = 0; u < 2; ++u) at[u] = records.find((uint32_t)tok / kKvGroup + u);
    };
    const auto keys = [&](Step<D>& s) {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const __amdgpu_buffer_rsrc_t r = records.at(at[u]);
        s.bad[u] = records.bad(at[u]);
        load_words<D / 32, !PLAN>(r, off.k, s.k[u]);
        s.ks[u] = load_key_scales<D>(r, off.ks);
      }
    };
    const auto values = [&](Step<D>& s, int tok) {  // (behind keys(), whose places they are)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const __amdgpu_buffer_rsrc_t r = records.at(at[u]);
        load_words<D / 32, !PLAN>(r, off.v, s.v[u]);
        s.vs[u] = __builtin_amdgcn_raw_buffer_load_b32(r, (int)off.vs, 0, 0);
      }
      find(tok + kUnit);
    };

    int tok = tile.lo + p.u0 * kUnit + wave * kStep;
    if (tok < end) {
      Step<D> s[Z::DEPTH];
      find(tok);
#pragma unroll
      for (int i = 0; i < Z::DEPTH; ++i) {
        keys(s[i]);
        values(s[i], tok + i * kUnit);
      }
      do {
#pragma unroll
        for (int i = 0; i < Z::DEPTH; ++i) {
          if (i > 0 && tok >= end) break;
          const bool all = tok + kStep - 1 <= tile.first && (a.window <= 0 || tok > tile.last - a.window);
          step<D, QT, BF16>(w, a, s[i], tok, tile.hi, !all, sq, keys,
                            [&](Step<D>& t) { values(t, tok + Z::DEPTH * kUnit); });
          tok += kUnit;
        }
      } while (tok < end);
    }

    if (__builtin_expect(uniform_u32(w.large ? 1 : 0) != 0, 0))
      large_values<D, QT, Z::NQ>(w, a, records, tile.lo + p.u0 * kUnit + wave * kStep, end, kUnit, tile.hi, [&](int t, int n, int j) {
        if constexpr (Z::QLDS) return sq[((t * Z::NQ + n) * (D / 32) + j) * 64 + lane];
        else return w.q[t][n][j];
      });

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
    // where the part goes, in bytes from the first block's
    const uint32_t part = (uint32_t)(run.lb * 2 + (p.head ? 1 : 0)) * (Z::PART * 4);
    const __amdgpu_buffer_rsrc_t parts = make_rsrc(a.part, (uint32_t)(a.blocks * 2 - 1) * (Z::PART * 4));
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
        const bool empty = tile.len - tile.nq + qi < 0;  // sees no key: zeros
        if (p.whole) {
          o *= 1.f / l;
          if (empty) o = f32x4{0.f, 0.f, 0.f, 0.f};
          store_out<BF16>(a.out, ((size_t)(start + qi) * a.hq + h * G + (row0 + row) % G) * D + c, o);
        } else {
          const uint32_t at = part + (row * D + c) * 4;
          if (empty) m = -__builtin_inff();
          if (PLAN || a.parts == 0) {
            float* to = a.part + part / 4;
            *reinterpret_cast<f32x4*>(to + row * D + c) = o;
            if (c == 0) {
              to[R * D + row] = m;
              to[R * D + R + row] = l;
            }
          } else {
            st_buf16_coherent(parts, at, __builtin_bit_cast(u32x4, o));
            if (c == 0) {
              __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(m), parts, (int)(part + (R * D + row) * 4), 0, kCachePolicySc1);
              __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(l), parts, (int)(part + (R * D + R + row) * 4), 0, kCachePolicySc1);
            }
          }
        }
      }
    }
    if (!PLAN && a.parts > 0 && !p.whole) {
      __builtin_amdgcn_s_waitcnt(0);  // this thread's stores have completed
      __syncthreads();
      if (threadIdx.x == 0) sh[12] = take_ticket(a.tickets + first_block, a.epoch, (uint32_t)n, peek) ? 1 : 0;
      __syncthreads();
      if (sh[12]) join_parts<D, BF16>(a, parts, first_block, n, Z::PART, R, tile, h, pool);
    }
    __syncthreads();
    kv_next<PLAN, kLeadUnits>(a, run, tile, p);
  }
}

template <int D, int QT, bool BF16> hipError_t go_rows(const KvAttentionArgs& a, hipStream_t s) {
  KernelTimer tm("kv_attention", s);
  const dim3 grid(a.blocks), th(kThreads);
  if (a.q_start)
    hipExtLaunchKernelGGL((k_kv_rows<D, QT, BF16, true>), grid, th, 0, s, tm.start(), tm.stop(), 0, a);
  else
    hipExtLaunchKernelGGL((k_kv_rows<D, QT, BF16, false>), grid, th, 0, s, tm.start(), tm.stop(), 0, a);
  return hipGetLastError();
}

}  // namespace

template <int D> hipError_t launch_kv_rows_attention(const KvAttentionArgs& a, int qt, bool bf16, hipStream_t s) {
  if constexpr (D < 256) {
    if (qt == 2) return bf16 ? go_rows<D, 2, true>(a, s) : go_rows<D, 2, false>(a, s);
  }
  return bf16 ? go_rows<D, 1, true>(a, s) : go_rows<D, 1, false>(a, s);
}

}  // namespace cats
