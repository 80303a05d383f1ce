// Attention over the cache in 4 bits for many rows of each sequence: a prompt.
//
// A block has a tile of 64 or 128 rows, each wave 16 QT of its own.  What a step of the keys
// (64 tokens, or 32 of 256 columns) costs besides the products is the conversion of the cache,
// so it is done once for the tile: each wave makes the operands of one record and puts them
// into LDS as its readers take them, 16 bytes to a lane side by side, while the step before
// is multiplied (two buffers, one barrier a step).  Bound by issue: matrix cores work 0.33, vector ALUs (softmax,
// the weights' rounding, the conversion) 0.47 of a busy compute unit's cycles, and the two waves
// of a SIMD hide only a part of one behind the other.  4096 rows of one sequence, 32 heads of
// 128 columns on 8 (137 GFLOP): 180 us, 0.76 PFLOP/s; in fp32 288.
#pragma once

#include "kv_attention.hpp"
#include "ticket.hpp"

namespace cats {
namespace {

constexpr int kPromptLead = kKvPromptLead;

template <int D, bool BF16> struct PromptSizes {
  static constexpr int QT = kv_prompt_qt(D, BF16);
  static constexpr int R = kv_prompt_rows(D, BF16);
  static constexpr int RECS = D == 256 ? 2 : 4;  // records of a step
  static constexpr int UNIT = RECS * kKvGroup;
  static_assert(UNIT == kv_prompt_unit(D), "the host shares out the kernel's units");
  static constexpr int NQ = BF16 ? 1 : 3, NP = BF16 ? 1 : 2;
  static constexpr int SIDE = QT == 1 && RECS == 4 ? 4 : 2;  // records, with QT four sums, whose products alternate
  static constexpr int KOPS = RECS * (D / 32), VOPS = RECS / 2 * (D / 16);  // operands of a step, 1 KB each
  static constexpr int PART = R * (D + 2);
};

// One record's words, or (two records a step) the keys' or the values' of one.
template <int D> struct Raw {
  uint32_t k[D / 32], v[D / 32];
  uint32_t ks, vs, bad;
};

// The values' operands of a record: the lower or upper half of each of a pair's.
template <int D, int C> __device__ __forceinline__ void put_values(const uint32_t (&v)[D / 32], const float (&sc)[4], uint8_t* to) {
  uint32_t e[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) e[i] = value_pair<D, C, true>(v, i, sc[i]);
  *reinterpret_cast<u32x2*>(to + 2 * C * 1024) = u32x2{low_halves(e[0], e[1]), low_halves(e[2], e[3])};
  *reinterpret_cast<u32x2*>(to + (2 * C + 1) * 1024) = u32x2{high_halves(e[0], e[1]), high_halves(e[2], e[3])};
  if constexpr (C + 1 < D / 32) put_values<D, C + 1>(v, sc, to);
}

// A barrier that waits for LDS alone: the next records stay under way.
__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// A block's part of a sum that n blocks from `first` on share, its own the idx-th.  True where
// the whole sum is in w: in the block that arrives last.  Four parts side by side are joined by the
// last of their blocks, which has its own in registers, and four such sums again: the other
// blocks write theirs and go on.  Parts are added in their order, whoever does it.  A block's last
// tile is the next one's first, which is done long before: the part is mostly not written at all.
constexpr int kJoin = 4;
static_assert(kJoin * kJoin * kJoin * kJoin * kJoin >= 512, "five words of tickets for each block");
template <int D, bool BF16>
__device__ __forceinline__ bool join_prompt(const KvAttentionArgs& a, KvSums<D, kv_prompt_qt(D, BF16)>& w, int first, int idx, int n,
                                            int rows, int* sh) {
  typedef PromptSizes<D, BF16> Z;
  constexpr int QT = Z::QT, J = D / 16;
  int me = threadIdx.x;
  asm volatile("" : "+v"(me));  // (nothing of this is computed in front of the loop and kept over it)
  const int lane = me % 64, mine = me / 64 * 16 * QT;
  const __amdgpu_buffer_rsrc_t parts = make_rsrc(a.part, (uint32_t)(a.blocks * 2 - 1) * (Z::PART * 4));
  const auto slot = [&](int i) { return (uint32_t)(2 * (first + i) + (i == 0 ? 1 : 0)) * (Z::PART * 4); };
  // a thread's words of a part: its sums, then m and l
  const auto word = [&](int t, int j) { return (uint32_t)((t * J + j) * kKvThreads + me) * 16; };
  const auto stat = [&](int t) { return (uint32_t)(Z::R * D + mine + t * 16 + lane % 16) * 4; };
  int level = 0;
  for (int stride = 1;; stride *= kJoin, ++level) {
    const int base = idx / (stride * kJoin) * (stride * kJoin), count = min(kJoin, (n - base + stride - 1) / stride);
    if (count > 1) {
      unsigned long long* ticket = a.tickets + level * a.blocks + first + base;
      unsigned long long peek = 0;
      if (threadIdx.x == 0) {
        peek = ticket_peek(ticket);
        sh[10] = peek == ((unsigned long long)a.epoch << 32 | (uint32_t)(count - 1)) ? 1 : 0;
      }
      __syncthreads();
      const bool alone = sh[10] != 0;  // (the others have written theirs)
      if (!alone) {
        const uint32_t to = slot(idx);
#pragma unroll
        for (int t = 0; t < QT; ++t) {
          if (mine + t * 16 + lane % 16 >= rows) continue;
#pragma unroll
          for (int j = 0; j < J; ++j) st_buf16_coherent(parts, to + word(t, j), __builtin_bit_cast(u32x4, w.o[t][j]));
          if (lane < 16) {
            __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(w.m[t]), parts, (int)(to + stat(t)), 0, kCachePolicySc1);
            __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(w.l[t]), parts, (int)(to + stat(t) + Z::R * 4), 0, kCachePolicySc1);
          }
        }
        __builtin_amdgcn_s_waitcnt(0);  // this thread's stores have completed
      }
      __syncthreads();
      if (threadIdx.x == 0) sh[11] = take_ticket(ticket, a.epoch, (uint32_t)count, peek) ? 1 : 0;
      __syncthreads();
      if (sh[11] == 0) return false;
      // (a part that is not there, and the block's own, reads as zeros)
      uint32_t from[kJoin];
      int own = 0;
#pragma unroll
      for (int k = 0; k < kJoin; ++k) {
        const int i = base + k * stride;
        own = i == idx ? k : own;
        from[k] = k < count && i != idx ? slot(i) : kOOB;
      }
#pragma unroll
      for (int t = 0; t < QT; ++t) {
        float f[kJoin], l[kJoin], top = w.m[t];
#pragma unroll
        for (int k = 0; k < kJoin; ++k) {
          f[k] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(parts, (int)(from[k] + stat(t)), 0, kCachePolicySc1));
          l[k] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(parts, (int)(from[k] + stat(t) + Z::R * 4), 0, kCachePolicySc1));
        }
#pragma unroll
        for (int k = 0; k < kJoin; ++k) {
          f[k] = k == own ? w.m[t] : k < count ? f[k] : kLow;
          l[k] = k == own ? w.l[t] : l[k];
          top = fmaxf(top, f[k]);
        }
        float sum = 0.f;
#pragma unroll
        for (int k = 0; k < kJoin; ++k) {
          f[k] = __builtin_amdgcn_exp2f(f[k] - top);
          sum += l[k] * f[k];
        }
        w.m[t] = top;
        w.l[t] = sum;
#pragma unroll
        for (int j = 0; j < J; ++j) {
          f32x4 po[kJoin], o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int k = 0; k < kJoin; ++k) po[k] = __builtin_bit_cast(f32x4, ld_buf16_coherent(parts, from[k] + word(t, j)));
#pragma unroll
          for (int k = 0; k < kJoin; ++k) o += (k == own ? w.o[t][j] : po[k]) * f[k];
          w.o[t][j] = o;
          if (j % 4 == 3) __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
    idx = base;
    if (stride * kJoin >= n) return true;
  }
}

template <int D, bool BF16> __global__ __launch_bounds__(kKvThreads, 2) void k_kv_prompt(KvAttentionArgs a) {
  typedef PromptSizes<D, BF16> Z;
  constexpr int QT = Z::QT, R = Z::R;
  __shared__ __attribute__((aligned(16))) uint8_t lds[2][(Z::KOPS + Z::VOPS) * 1024];
  __shared__ uint32_t wide[2][Z::RECS];
  __shared__ int sh[12];
  const int wave = uniform_u32(threadIdx.x / 64), lane = threadIdx.x % 64, g = lane / 16;
  const int G = a.hq / a.hkv;
  const KvLane<D> off;
  const int rec = wave % Z::RECS;  // the wave's record of a step
  const bool with_k = Z::RECS == 4 || wave < 2, with_v = Z::RECS == 4 || wave >= 2;
  __shared__ KvOwnPlan own;
  KvRun run;
  if (!kv_run<true, Z::UNIT, kPromptLead, R>(a, run, sh, &own)) return;

  while (run.p < run.p1) {
    const KvTile tile = kv_tile_of<true, Z::UNIT, R>(a, G, run, &own);
    const KvPart p = kv_part<kPromptLead>(run, tile);
    if (p.u0 >= p.u1) {
      kv_next<true, kPromptLead>(a, run, tile, p);
      continue;
    }
    const int h = run.h;

    // the wave's rows
    KvSums<D, QT> w;
    clear<D, QT>(w, a);
    bf16x8 q[QT][Z::NQ][D / 32];
    const int mine = wave * 16 * QT;
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      const int r = min(mine + t * 16 + lane % 16, tile.rows - 1);  // (rows behind the last repeat it and are not stored)
      const int i = (tile.row0 + r) / G, head = h * G + (tile.row0 + r) % G;
      w.pos[t] = tile.len - tile.nq + i;
      const size_t at = ((size_t)(tile.start + i) * a.hq + head) * D + g * (D / 4);
#pragma unroll
      for (int j = 0; j < D / 32; ++j) {
        bf16x8 part[Z::NQ];
        load_q8<Z::NQ>(a.q, at + 8 * j, part);
#pragma unroll
        for (int n = 0; n < Z::NQ; ++n) q[t][n][j] = part[n];
      }
    }
    // positions of its first and last row; none: a last one that sees nothing
    const int base = tile.len - tile.nq;
    const int first = base + (tile.row0 + min(mine, tile.rows - 1)) / G;
    const int last = mine < tile.rows ? base + (tile.row0 + min(mine + 16 * QT, tile.rows) - 1) / G : -1;

    const KvRecords<D> records(a, tile.b, h, tile.hi);
    const uint32_t rec0 = (uint32_t)tile.lo / kKvGroup + rec;
    typename KvRecords<D>::Place place = records.find_later(rec0 + p.u0 * Z::RECS);
    Raw<D> raw;
    const auto load = [&](int u) {  // unit u, whose place is known; then the next one's place
      place.page = uniform_u32(place.page);
      const __amdgpu_buffer_rsrc_t r = records.at(place);
      raw.bad = records.bad(place);
      if (with_k) {
        load_words<D / 32, false>(r, off.k, raw.k);
        raw.ks = load_key_scales<D>(r, off.ks);
      }
      if (with_v) {
        load_words<D / 32, false>(r, off.v, raw.v);
        raw.vs = __builtin_amdgcn_raw_buffer_load_b32(r, (int)off.vs, 0, 0);
      }
      place = records.find_later(rec0 + (u + 1) * Z::RECS);
    };
    const auto put = [&](int u, int b) {
      uint8_t* to = lds[b];
      if (with_k) {
        const uint32_t ks = raw.ks | raw.bad;
#pragma unroll
        for (int j = 0; j < D / 32; ++j)
          reinterpret_cast<bf16x8*>(to)[(rec * (D / 32) + j) * 64 + lane] =
              eight_of(raw.k[j], D == 256 && j >= 4 ? kv_scale(ks >> 8 & 0xffu) : kv_scale(ks & 0xffu));
      }
      if (with_v) {
        const int tok = tile.lo + (u * Z::RECS + rec) * kKvGroup;
        uint32_t vs = raw.vs;
        if (tok + kKvGroup > tile.hi) vs = hidden_as_one(vs, tok + 4 * g, tile.hi);
        const uint64_t odd = __ballot(not_narrow(vs) != 0);
        if (lane == 0) wide[b][rec] = odd != 0 ? 1u : 0u;
        if (__builtin_expect(odd != 0, 0)) no_values(raw.v, vs);
        float sc[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) sc[i] = kv_scale(vs >> (8 * i) & 0xffu);
        put_values<D, 0>(raw.v, sc, to + Z::KOPS * 1024 + rec / 2 * (D / 16) * 1024 + lane * 16 + rec % 2 * 8);
      }
    };

    load(p.u0);
    put(p.u0, 0);
    load(p.u0 + 1);
    lds_barrier();
    for (int u = p.u0; u < p.u1; ++u) {
      const int b = (u - p.u0) & 1;
      if (u + 1 < p.u1) {
        put(u + 1, b ^ 1);
        load(u + 2);
      }
      const int tok = tile.lo + u * Z::UNIT;
      if (tok <= last && (a.window <= 0 || tok + Z::UNIT - 1 > first - a.window)) {  // (else none of the wave's rows sees them)
        const bf16x8* ko = reinterpret_cast<const bf16x8*>(lds[b]) + lane;
        const f16x8* vo = reinterpret_cast<const f16x8*>(lds[b] + Z::KOPS * 1024) + lane;
        f32x4 z[QT][Z::RECS];
#pragma unroll
        for (int t = 0; t < QT; ++t)
#pragma unroll
          for (int s = 0; s < Z::RECS; ++s) z[t][s] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s0 = 0; s0 < Z::RECS; s0 += Z::SIDE)
#pragma unroll
          for (int j = 0; j < D / 32; ++j)
#pragma unroll
            for (int n = Z::NQ - 1; n >= 0; --n)
#pragma unroll
              for (int s = s0; s < s0 + Z::SIDE; ++s)
#pragma unroll
                for (int t = 0; t < QT; ++t)  // (a sum's next product waits for its last)
                  z[t][s] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ko[(s * (D / 32) + j) * 64], q[t][n][j], z[t][s], 0, 0, 0);
        __builtin_amdgcn_s_setprio(1);  // (the other wave's products need no issue while they run)
        uint32_t odd = 0;
#pragma unroll
        for (int s = 0; s < Z::RECS; ++s) odd |= wide[b][s];
        weights<D, QT, Z::RECS>(w, a, z, tok, !(tok + Z::UNIT - 1 <= first && (a.window <= 0 || tok > last - a.window)));
#pragma unroll
        for (int s0 = 0; s0 < Z::RECS; s0 += 2) {
          f16x8 part[QT][Z::NP];
          weight_operands<QT, Z::NP, Z::RECS>(z, s0, part);
#pragma unroll
          for (int j0 = 0; j0 < D / 16; j0 += 4 / QT)
#pragma unroll
            for (int n = Z::NP - 1; n >= 0; --n)
#pragma unroll
              for (int j = j0; j < j0 + 4 / QT; ++j)
#pragma unroll
                for (int t = 0; t < QT; ++t)
                  w.o[t][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vo[(s0 / 2 * (D / 16) + j) * 64], part[t][n], w.o[t][j], 0, 0, 0);
        }
        __builtin_amdgcn_s_setprio(0);
        if (__builtin_expect(uniform_u32(odd) != 0, 0)) {
          asm volatile("");
#pragma unroll
          for (int s0 = 0; s0 < Z::RECS; s0 += 2) {
            uint32_t v[2][D / 32], vs[2];
#pragma unroll
            for (int s = 0; s < 2; ++s) {
              const __amdgpu_buffer_rsrc_t r = records.at(records.find((uint32_t)tok / kKvGroup + s0 + s));
              load_words<D / 32, false>(r, off.v, v[s]);
              vs[s] = hidden_as_one(__builtin_amdgcn_raw_buffer_load_b32(r, (int)off.vs, 0, 0), tok + 16 * (s0 + s) + 4 * g, tile.hi);
              if (wide[b][s0 + s] == 0u) no_values(v[s], vs[s]);  // (its operands are in LDS)
            }
            wide_values<D, QT, Z::RECS>(w, a, v, vs, z, s0, tok + 16 * s0);
          }
        }
      }
      lds_barrier();
    }
    if (__builtin_expect(w.large, 0))
      large_values<D, QT, Z::NQ>(w, a, records, tile.lo + p.u0 * Z::UNIT, min(tile.hi, tile.lo + p.u1 * Z::UNIT), 2 * kKvGroup, tile.hi,
                                 [&](int t, int n, int j) {
                                   if constexpr (Z::NQ * D <= 512) return q[t][n][j];
                                   // (no registers for them there)
                                   int r = mine + t * 16 + lane % 16;
                                   asm volatile("" : "+v"(r));
                                   const int row = tile.row0 + min(r, tile.rows - 1);
                                   bf16x8 part[Z::NQ];
                                   load_q8<Z::NQ>(a.q, ((size_t)(tile.start + row / G) * a.hq + h * G + row % G) * D + g * (D / 4) + 8 * j, part);
                                   return part[n];
                                 });

#pragma unroll
    for (int t = 0; t < QT; ++t) {
      w.l[t] += __shfl_xor(w.l[t], 16);
      w.l[t] += __shfl_xor(w.l[t], 32);
    }
    if (!p.whole && a.parts > 0) {
      int n;
      const int first_block = kv_parts_of<kPromptLead>(run, tile, p, n);
      if (!join_prompt<D, BF16>(a, w, first_block, run.lb - first_block, n, tile.rows, sh)) {
        kv_next<true, kPromptLead>(a, run, tile, p);
        continue;
      }
    }
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      const int r = mine + t * 16 + lane % 16;
      if (r >= tile.rows) continue;
      const int i = (tile.row0 + r) / G;
      const bool empty = w.pos[t] < 0;  // sees no key: zeros
      const size_t at = ((size_t)(tile.start + i) * a.hq + h * G + (tile.row0 + r) % G) * D + g * (D / 4);
      float* part = a.part + ((size_t)run.lb * 2 + (p.head ? 1 : 0)) * Z::PART;
      const bool last_kernel = !p.whole && a.parts == 0;  // joins the parts
      const float inv = last_kernel ? 1.f : 1.f / w.l[t];
#pragma unroll
      for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int j = 0; j < D / 16; j += 4) {
          f32x4 o = f32x4{w.o[t][j][c], w.o[t][j + 1][c], w.o[t][j + 2][c], w.o[t][j + 3][c]} * inv;
          if (last_kernel) {
            *reinterpret_cast<f32x4*>(part + r * D + g * (D / 4) + c * (D / 16) + j) = o;
          } else {
            if (empty) o = f32x4{0.f, 0.f, 0.f, 0.f};
            store_out<BF16>(a.out, at + c * (D / 16) + j, o);
          }
        }
      if (last_kernel && g == 0) {
        part[R * D + r] = empty ? -__builtin_inff() : w.m[t];
        part[R * D + R + r] = w.l[t];
      }
    }
    kv_next<true, kPromptLead>(a, run, tile, p);
  }
}

template <int D, bool BF16> hipError_t go_prompt(const KvAttentionArgs& a, hipStream_t s) {
  KernelTimer tm("kv_attention", s);
  hipExtLaunchKernelGGL((k_kv_prompt<D, BF16>), dim3(a.blocks), dim3(kKvThreads), 0, s, tm.start(), tm.stop(), 0, a);
  return hipGetLastError();
}

}  // namespace

template <int D> hipError_t launch_kv_prompt_attention(const KvAttentionArgs& a, bool bf16, hipStream_t s) {
  return bf16 ? go_prompt<D, true>(a, s) : go_prompt<D, false>(a, s);
}

}  // namespace cats
