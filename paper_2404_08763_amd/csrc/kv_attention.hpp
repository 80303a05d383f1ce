// What the attention kernels over the cache in 4 bits share: the keys a tile of rows reads,
// how the blocks share the work, the operands of the matrix products.
#pragma once

#include "internal.hpp"
#include "kv4.hpp"

namespace cats {

constexpr int kKvThreads = 256, kKvWaves = 4;
constexpr float kLow = -3.402823466e+38f;  // maximum of a row that has seen no key
// A row's exponents are counted from its maximum less kLead, which is moved only when a
// score is kLazy above that, so that O is rarely multiplied: p is 2^15 at most, and f16's
// least number 2^-31 of the largest.
constexpr float kLead = 7.f, kLazy = 8.f;
// Up to here a maximum is off by half at most: the exponents, which are exact, stay below 16.
constexpr float kFar = 8388608.f;
// A cached value is below 2^127.6 (6 * 2^125), a weight 2^15 at most, a sequence has 2^30 tokens at
// most: with scales below 2^65 O stays below 2^(67.6 + 15 + 30), whatever is joined.  Where there are larger
// ones O is looked at behind a wave's last step.  If some rows left fp32, the wave's are done once more,
// these and those of kTall and more with weights 2^-kLift of what they were (O is below 2^(127.6 +
// 15 + 30 - 48) then), which loses what is below 2^-84 of each token's: fp32's least normal number by a
// largest weight of 2^(7 - 48).  Else O of kTall or more is made 2^-kLower as large, so that the
// sum of a row's parts (four waves of 768 blocks at most) stays in range.
constexpr uint32_t kHighScale = 192;  // 2^65
constexpr int kLift = 48, kLower = 16;
constexpr uint32_t kTall = (127u + 112u) << 23;  // 2^112

// ---- the work of a call -------------------------------------------------------------

__device__ __forceinline__ int kv_length(const KvAttentionArgs& a, int b) { return min(max(a.lens[b], 0), a.limit); }

// Queries [start, start + nq) of a sequence, whatever q_start holds.
__device__ __forceinline__ int kv_queries(const KvAttentionArgs& a, int b, int& start) {
  if (!a.q_start) {
    start = b;
    return 1;
  }
  start = min(max(a.q_start[b], 0), a.N);
  return max(min(max(a.q_start[b + 1], 0), a.N) - start, 0);
}

// A tile: rows [row0, row0 + rows) of a sequence, counted over its queries and a key head's
// query heads, and the keys [lo, hi) it reads, from the record of lo on, in units of UNIT tokens.
struct KvTile {
  int b, row0, rows, start, nq, len;
  int first, last;  // positions of its first and last row
  int lo, hi, units;
};
template <int UNIT> __device__ __forceinline__ void kv_span(const KvAttentionArgs& a, int G, KvTile& t) {
  t.first = t.len - t.nq + t.row0 / G;
  t.last = t.len - t.nq + (t.row0 + t.rows - 1) / G;
  t.hi = min(max(t.last + 1, 0), t.len);
  t.lo = a.window > 0 ? min(max(t.first - a.window + 1, 0), t.hi) : 0;
  t.lo &= ~(kKvGroup - 1);
  t.units = max(1, (t.hi - t.lo + UNIT - 1) / UNIT);
}
template <int UNIT> __device__ __forceinline__ KvTile kv_tile(const KvAttentionArgs& a, int G, int b, int row0, int R, int len) {
  KvTile t;
  t.b = b;
  t.row0 = row0;
  t.nq = kv_queries(a, b, t.start);
  t.rows = min(R, t.nq * G - row0);
  t.len = len;
  kv_span<UNIT>(a, G, t);
  return t;
}

// Inclusive prefix over a wave.
__device__ __forceinline__ int wave_prefix(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);  // row_shr 1, 2, 4, 8
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // row_bcast 15 into rows 1 and 3
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);  // row_bcast 31 into rows 2 and 3
  return x;
}

__device__ __forceinline__ int wave_max(int x) {
  x = max(x, __builtin_amdgcn_update_dpp(x, x, 0x111, 0xf, 0xf, false));
  x = max(x, __builtin_amdgcn_update_dpp(x, x, 0x112, 0xf, 0xf, false));
  x = max(x, __builtin_amdgcn_update_dpp(x, x, 0x114, 0xf, 0xf, false));
  x = max(x, __builtin_amdgcn_update_dpp(x, x, 0x118, 0xf, 0xf, false));
  x = max(x, __builtin_amdgcn_update_dpp(x, x, 0x142, 0xa, 0xf, false));
  return max(x, __builtin_amdgcn_update_dpp(x, x, 0x143, 0xc, 0xf, false));  // lane 63 has it
}

// Exclusive prefix of v over the block's threads, its total and (sh for twice as many) the largest.
template <int THREADS> __device__ __forceinline__ int block_prefix(int v, int& total, int* sh, int* top = nullptr) {
  constexpr int W = THREADS / 64;
  const int w = threadIdx.x / 64, x = wave_prefix(v), m = top ? wave_max(v) : 0;
  __syncthreads();
  if (threadIdx.x % 64 == 63) {
    sh[w] = x;
    if (top) sh[W + w] = m;
  }
  __syncthreads();
  int before = 0, most = 0;
  total = 0;
#pragma unroll
  for (int i = 0; i < W; ++i) {
    if (i < w) before += sh[i];
    total += sh[i];
    if (top) most = max(most, sh[W + i]);
  }
  total = (int)uniform_u32(total);
  if (top) *top = max(*top, (int)uniform_u32(most));
  return before + x - v;
}

// n / d for a quotient below 2^32.
__device__ __forceinline__ uint32_t quotient(uint64_t n, uint32_t d) {
  return (n >> 32) == 0 ? (uint32_t)n / d : (uint32_t)(n / d);
}

// The tiles of ragged queries, made by each block for itself where they are few (a.plan is null).
constexpr int kKvOwnTiles = 1024, kKvOwnSequences = kKvThreads;
struct KvOwnPlan {
  int prefix[kKvOwnTiles];     // what is in front of each tile
  int first[kKvOwnSequences];  // first tile of each sequence
  uint16_t seq[kKvOwnTiles];
};
template <int UNIT, int LEAD, int R>
__device__ __forceinline__ int kv_own_plan(const KvAttentionArgs& a, KvOwnPlan& own, uint32_t& W, int* sh) {
  const int G = a.hq / a.hkv, me = threadIdx.x;
  int start, n = 0, tiles;
  if (me < a.B) n = (kv_queries(a, me, start) * G + R - 1) / R;
  own.first[me] = block_prefix<kKvThreads>(n, tiles, sh);
  tiles = min(tiles, a.tiles);  // (there are more only where q_start decreases)
  __syncthreads();
  W = 0;
  for (int base = 0; base < tiles; base += kKvThreads) {
    const int e = base + me;
    int u = 0, total, lo = 0;
    if (e < tiles) {
      int left = a.B;  // the last sequence with first[b] <= e: it has tiles
      while (left > 1) {
        const int half = left / 2;
        if (own.first[lo + half] <= e) lo += half, left -= half;
        else left = half;
      }
      u = kv_tile<UNIT>(a, G, lo, (e - own.first[lo]) * R, R, kv_length(a, lo)).units + LEAD;
    }
    const int at = block_prefix<kKvThreads>(u, total, sh);
    if (e < tiles) {
      own.prefix[e] = (int)W + at;
      own.seq[e] = (uint16_t)lo;
    }
    W += (uint32_t)total;
  }
  __syncthreads();
  return tiles;
}

// A block's share.  The tiles of a head lie one behind the other, the heads behind each other,
// each tile as its units and LEAD more, which stand for what a tile costs besides; each
// block has a run of that line, all of one length but for one, whatever the sequences' lengths.
// Runs next to each other are on one XCD, which shares their keys.  A tile's parts are in
// consecutive blocks: none is empty but those behind the last.
struct KvRun {
  int lb;              // the block's place on the line
  uint32_t base, rem;  // length of a run, and how many are one longer
  uint64_t p, p1;      // the run
  int tiles;           // of a head, or (no plan) of a sequence
  int h, e, b, skip;   // head, tile (no plan: of sequence b), and where in the tile
  int len;             // of the first tile's sequence, while it is known; -1
};

template <bool PLAN, int UNIT, int LEAD, int R>
__device__ __forceinline__ bool kv_run(const KvAttentionArgs& a, KvRun& r, int* sh, KvOwnPlan* own = nullptr) {
  const int G = a.hq / a.hkv;
  r.tiles = a.tiles;
  int len = 0;
  const auto cost = [&](int b) {
    if (b >= a.B) return 0;
    len = kv_length(a, b);
    return r.tiles * (kv_tile<UNIT>(a, G, b, 0, R, len).units + LEAD);
  };
  r.len = -1;
  uint32_t W = 0;  // of a head
  int mine = 0, before = 0, top = 0;
  if constexpr (PLAN) {
    if (a.plan) {
      r.tiles = a.head[0];
      W = (uint32_t)a.head[1];
    } else {
      r.tiles = kv_own_plan<UNIT, LEAD, R>(a, *own, W, sh);
    }
  } else {
    for (int base = 0; base < a.B; base += kKvThreads) {
      int total;
      mine = cost(base + threadIdx.x);
      before = block_prefix<kKvThreads>(mine, total, sh, &top);
      W += (uint32_t)total;
    }
  }
  const uint64_t T = (uint64_t)W * (uint32_t)a.hkv;
  uint32_t nb = T < (uint32_t)a.blocks ? (uint32_t)T : (uint32_t)a.blocks;
  if (!PLAN && a.parts > 0) {
    // A tile in a.parts parts at most, or, where it is long, in as many as it takes about as long
    // to join (0.04 us a KB) as to read the keys of one of them (0.5 us a unit).
    const uint32_t one = (uint32_t)(top / r.tiles);
    const float longest = __builtin_sqrtf((float)one * (float)a.parts * (1.f / 5.f));
    const uint64_t most = T * (uint32_t)(max(a.parts, (int)longest) - 1);
    if ((uint64_t)nb * one > most) nb = quotient(most, one);
  }
  r.lb = nb < (uint32_t)a.blocks ? (int)blockIdx.x : (int)((blockIdx.x % 8) * (nb / 8) + blockIdx.x / 8);
  if (a.parts == 0 && a.by_tile) {  // (each tile there is notes itself)
    for (int i = r.tiles * (PLAN ? 1 : a.B) * a.hkv + blockIdx.x * kKvThreads + threadIdx.x; i < a.sums; i += a.blocks * kKvThreads)
      a.desc[i] = int4{0, 0, 0, 0};
  } else if (a.parts == 0 && threadIdx.x == 0) {
    a.desc[r.lb] = int4{0, 0, 0, 0};
  }
  if ((uint32_t)r.lb >= nb) return false;
  r.base = quotient(T, nb);
  r.rem = (uint32_t)(T - (uint64_t)r.base * nb);
  r.p = (uint64_t)r.lb * r.base + min((uint32_t)r.lb, r.rem);
  r.p1 = r.p + r.base + ((uint32_t)r.lb < r.rem ? 1 : 0);
  r.h = (int)quotient(r.p, W);
  const uint32_t x = (uint32_t)(r.p - (uint64_t)(uint32_t)r.h * W);
  if constexpr (PLAN) {
    int lo = 0, n = r.tiles;  // the last tile whose prefix is not behind x
    while (n > 1) {
      const int stride = (n + kKvThreads - 1) / kKvThreads, at = threadIdx.x * stride;
      const bool before_x = at < n && (uint32_t)(a.plan ? a.prefix[lo + at] : own->prefix[lo + at]) <= x;
      const int last = (int)uniform_u32(__syncthreads_count(before_x)) - 1;
      lo += last * stride;
      n = min(stride, n - last * stride);
    }
    r.e = lo;
    r.b = 0;
    r.skip = (int)(x - (uint32_t)(a.plan ? a.prefix[lo] : own->prefix[lo]));
  } else {
    uint32_t sum = 0;
    for (int base = 0;; base += kKvThreads) {
      int total = 0;
      if (a.B > kKvThreads) {  // (else as it was counted above)
        mine = cost(base + threadIdx.x);
        before = block_prefix<kKvThreads>(mine, total, sh);
      }
      const uint32_t at = sum + (uint32_t)before;
      if (at <= x && x < at + (uint32_t)mine) {
        sh[8] = base + threadIdx.x;
        sh[9] = (int)(x - at);
        sh[10] = mine;
        sh[11] = len;
      }
      sum += (uint32_t)total;
      if (a.B <= kKvThreads || x < sum) break;
    }
    __syncthreads();
    r.b = (int)uniform_u32(sh[8]);
    const uint32_t in = uniform_u32(sh[9]), one = uniform_u32(sh[10]) / r.tiles;
    r.e = (int)(in / one);
    r.len = (int)uniform_u32(sh[11]);
    r.skip = (int)(in - r.e * one);
  }
  r.h = (int)uniform_u32(r.h);
  r.skip = (int)uniform_u32(r.skip);
  return true;
}

// The run's present tile.
template <bool PLAN, int UNIT, int R>
__device__ __forceinline__ KvTile kv_tile_of(const KvAttentionArgs& a, int G, const KvRun& r, const KvOwnPlan* own = nullptr) {
  if constexpr (PLAN) {
    KvPlanEntry t;
    if (a.plan) {
      t = a.plan[r.e];
    } else {
      t.b = own->seq[r.e];
      t.row0 = (r.e - own->first[t.b]) * R;
    }
    const int b = (int)uniform_u32(t.b);
    return kv_tile<UNIT>(a, G, b, (int)uniform_u32(t.row0), R, kv_length(a, b));
  } else {
    return kv_tile<UNIT>(a, G, r.b, r.e * R, R, r.len >= 0 ? r.len : kv_length(a, r.b));
  }
}

// The part of the tile that is in the run: units [u0, u1), possibly none.
struct KvPart {
  int u0, u1;
  bool head, whole;  // begins the tile; is all of it
};
template <int LEAD> __device__ __forceinline__ KvPart kv_part(const KvRun& r, const KvTile& t) {
  const uint64_t left = r.p1 - r.p;
  const int all = t.units + LEAD, c1 = left < (uint64_t)(all - r.skip) ? r.skip + (int)left : all;
  KvPart p;
  p.u0 = max(0, r.skip - LEAD);
  p.u1 = max(0, c1 - LEAD);
  p.head = r.skip <= LEAD && p.u1 > 0;
  p.whole = p.head && c1 == all;
  return p;
}

// The block that has a place on the line.
__device__ __forceinline__ int block_at(const KvRun& r, uint64_t x) {
  const uint64_t big = (uint64_t)r.rem * (r.base + 1);
  return (int)(x < big ? quotient(x, r.base + 1) : r.rem + quotient(x - big, r.base));
}

// The first of the blocks that have parts of the tile, and how many.
template <int LEAD> __device__ __forceinline__ int kv_parts_of(const KvRun& r, const KvTile& t, const KvPart& p, int& n) {
  const uint64_t from = r.p - (uint32_t)r.skip;
  const int head = p.head ? r.lb : block_at(r, from + LEAD);
  n = block_at(r, from + (uint32_t)(t.units + LEAD) - 1) - head + 1;
  return head;
}

// Goes on to the next tile; before, notes for the last kernel (without tickets) a sum that
// begins in this block and ends in a later one (by tile: any that begins here).
template <bool PLAN, int LEAD>
__device__ __forceinline__ void kv_next(const KvAttentionArgs& a, KvRun& r, const KvTile& t, const KvPart& p) {
  const uint64_t end = r.p - (uint32_t)r.skip + (uint32_t)(t.units + LEAD);  // of the tile, on the line
  if (a.parts == 0 && p.head && (a.by_tile || !p.whole) && threadIdx.x == 0) {
    int n = 0;
    if (!p.whole) kv_parts_of<LEAD>(r, t, p, n);
    const int at = !a.by_tile ? r.lb : PLAN ? r.h * r.tiles + r.e : (r.h * a.B + r.b) * r.tiles + r.e;
    a.desc[at] = int4{n | r.lb << 16, r.h, t.b, t.row0};
  }
  r.p = end < r.p1 ? end : r.p1;
  r.skip = 0;
  r.len = -1;
  ++r.e;
  if constexpr (PLAN) {
    if (r.e == r.tiles) r.e = 0, ++r.h;
  } else {
    if (r.e == r.tiles) {
      r.e = 0;
      if (++r.b == a.B) r.b = 0, ++r.h;
    }
  }
}

// ---- the cache's records ----------------------------------------------------------------

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// Words that no kernel of the call writes, at an address equal on all lanes: a scalar load.
__device__ __forceinline__ int scalar_load(const int* p, size_t i) {
  return reinterpret_cast<const __attribute__((address_space(4))) int*>(reinterpret_cast<uintptr_t>(p))[i];
}

// The lane's parts of a record (kv4.hpp).
template <int D> struct KvLane {
  uint32_t k, v, ks, vs;
  __device__ __forceinline__ KvLane() {
    const uint32_t lane = threadIdx.x % 64, m = lane % 16, g = lane / 16;
    k = m * (D / 2) + g * (D / 8);
    v = 8 * D + lane * (D / 8);
    ks = 16 * D + m * (D / 32) + (D == 256 ? 2 * g : D == 128 ? g : g / 2);
    vs = 16 * D + D / 2 + g * (D / 8) + m * D / 512 * 4;
  }
};

// The records of a key head of a sequence.
template <int D> struct KvRecords {
  const int* table;
  const uint8_t* base;
  uint32_t stride, most, magic, groups, pages;
  __device__ __forceinline__ KvRecords(const KvAttentionArgs& a, int b, int h, int hi) {
    table = a.table + (size_t)b * a.width;
    base = a.cache + (size_t)h * a.groups * kv_record_bytes(D);
    stride = (uint32_t)(a.hkv * a.groups) * kv_record_bytes(D);
    most = (uint32_t)(max(hi, 1) - 1) / kKvGroup;  // the last record some row sees
    magic = a.magic;
    groups = (uint32_t)a.groups;
    pages = (uint32_t)a.pages;
  }
  // A record's page and its place there; what is behind the last one is that once more.
  struct Place {
    uint32_t page, in;
  };
  __device__ __forceinline__ Place find(uint32_t rec) const {
    rec = min(rec, most);
    const uint32_t at = __umulhi(rec << 1, magic);
    return Place{(uint32_t)scalar_load(table, at), (rec - at * groups) * kv_record_bytes(D)};
  }
  // The same by a vector load, for a kernel whose waits for LDS would wait for scalar loads too;
  // page is to be made uniform where it is used.
  __device__ __forceinline__ Place find_later(uint32_t rec) const {
    rec = min(rec, most);
    const uint32_t at = __umulhi(rec << 1, magic);
    const __amdgpu_buffer_rsrc_t t = make_rsrc(table, (at + 1) * 4);
    return Place{(uint32_t)__builtin_amdgcn_raw_buffer_load_b32(t, (int)(at * 4), 0, 0),
                 (rec - at * groups) * kv_record_bytes(D)};
  }
  // All ones where the page is none of the cache's (whose first page is read for it).
  __device__ __forceinline__ uint32_t bad(const Place& p) const { return p.page < pages ? 0u : 0xffffu; }
  __device__ __forceinline__ __amdgpu_buffer_rsrc_t at(const Place& p) const {
    return make_rsrc(base + (uint64_t)(p.page < pages ? p.page : 0u) * stride + p.in, kv_record_bytes(D));
  }
};

// The lane's words at an offset in a record, whose address is equal on all lanes: a buffer
// load adds the two (and reads nothing behind the record).
// ONCE: for no later reader (non-temporal).
template <int W, bool ONCE>
__device__ __forceinline__ void load_words(__amdgpu_buffer_rsrc_t record, uint32_t off, uint32_t* w) {
  if constexpr (W == 2) {
    const auto v = __builtin_amdgcn_raw_buffer_load_b64(record, (int)off, 0, ONCE ? 2 : 0);
    w[0] = v[0];
    w[1] = v[1];
  } else {
#pragma unroll
    for (int i = 0; i < W / 4; ++i) {
      const u32x4 v = ONCE ? ld_buf16_stream(record, off + 16 * i) : ld_buf16(record, off + 16 * i);
      w[4 * i] = v.x;
      w[4 * i + 1] = v.y;
      w[4 * i + 2] = v.z;
      w[4 * i + 3] = v.w;
    }
  }
}

// The scales of a lane's keys: one, or two of 256 columns.
template <int D> __device__ __forceinline__ uint32_t load_key_scales(__amdgpu_buffer_rsrc_t record, uint32_t off) {
  if constexpr (D == 256) return (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(record, (int)off, 0, 0);
  else return (uint8_t)__builtin_amdgcn_raw_buffer_load_b8(record, (int)off, 0, 0);
}

template <typename T> __device__ __forceinline__ T as_eight(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  const u32x4 v = {a, b, c, d};
  return __builtin_bit_cast(T, v);
}

// The two values of byte SEL, as bf16 (exact for every scale) or f16 (exact where kNarrow says so).
template <int SEL> __device__ __forceinline__ uint32_t two_bf16(uint32_t w, float s) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, SEL));
}
template <int SEL> __device__ __forceinline__ uint32_t two_f16(uint32_t w, float s) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, s, SEL));
}
__device__ __forceinline__ bf16x8 eight_of(uint32_t w, float s) {
  return as_eight<bf16x8>(two_bf16<0>(w, s), two_bf16<1>(w, s), two_bf16<2>(w, s), two_bf16<3>(w, s));
}
// Byte C of the lane's D / 32 bytes of token i.
template <int D, int C, bool F16> __device__ __forceinline__ uint32_t value_pair(const uint32_t* v, int i, float s) {
  if constexpr (D == 64) {
    if (F16) return i % 2 ? two_f16<2 + C>(v[i / 2], s) : two_f16<C>(v[i / 2], s);
    return i % 2 ? two_bf16<2 + C>(v[i / 2], s) : two_bf16<C>(v[i / 2], s);
  } else {
    const uint32_t w = v[i * (D / 128) + C / 4];
    return F16 ? two_f16<C % 4>(w, s) : two_bf16<C % 4>(w, s);
  }
}

__device__ __forceinline__ uint32_t low_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }
__device__ __forceinline__ uint32_t high_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }

// V^T's operands of columns 2 C and 2 C + 1 (of each lane's D / 16): the tokens of two records side by side.
template <int D, int C, bool F16, typename T>
__device__ __forceinline__ void value_operands(const uint32_t (&v)[2][D / 32], const float (&sc)[2][4], T (&out)[2]) {
  uint32_t e[2][4];
#pragma unroll
  for (int u = 0; u < 2; ++u)
#pragma unroll
    for (int i = 0; i < 4; ++i) e[u][i] = value_pair<D, C, F16>(v[u], i, sc[u][i]);
  out[0] = as_eight<T>(low_halves(e[0][0], e[0][1]), low_halves(e[0][2], e[0][3]), low_halves(e[1][0], e[1][1]),
                       low_halves(e[1][2], e[1][3]));
  out[1] = as_eight<T>(high_halves(e[0][0], e[0][1]), high_halves(e[0][2], e[0][3]), high_halves(e[1][0], e[1][1]),
                       high_halves(e[1][2], e[1][3]));
}
// Whether a value scale's byte is outside [109, 140], 2^-18 to 2^13, for which f16 has all
// of the codes' values: bits of the four bytes that say so.  (The sum of a byte above
// 236 carries into the next, but is itself outside.)
__device__ __forceinline__ uint32_t not_narrow(uint32_t vs) { return ((vs + 0x13131313u) ^ 0x80808080u) & 0xe0e0e0e0u; }

// Codes of 0 with scales of 1.
template <int W> __device__ __forceinline__ void no_values(uint32_t (&v)[W], uint32_t& vs) {
#pragma unroll
  for (int i = 0; i < W; ++i) v[i] = 0u;
  vs = 0x7f7f7f7fu;
}

// f as three bf16 parts, all 24 bits of it.
__device__ __forceinline__ float cut(float f) { return __uint_as_float(__float_as_uint(f) & 0xffff0000u); }
__device__ __forceinline__ void split8(const float* f, bf16x8* out) {
  float r[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) r[i] = f[i];
#pragma unroll
  for (int p = 0; p < 3; ++p) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = high_halves(__float_as_uint(r[2 * i]), __float_as_uint(r[2 * i + 1]));
    out[p] = as_eight<bf16x8>(w[0], w[1], w[2], w[3]);
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] -= cut(r[i]);
  }
}

__device__ __forceinline__ bool sees(const KvAttentionArgs& a, int pos, int j) {
  return j <= pos && (a.window <= 0 || j > pos - a.window);
}

template <bool BF16> __device__ __forceinline__ void store_out(void* out, size_t at, const f32x4& v) {
  if (BF16) {
    typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
    *reinterpret_cast<bf16x4*>(static_cast<uint16_t*>(out) + at) = bf16x4{(__bf16)v[0], (__bf16)v[1], (__bf16)v[2], (__bf16)v[3]};
  } else {
    *reinterpret_cast<f32x4*>(static_cast<float*>(out) + at) = v;
  }
}

// Eight columns of a row of q as bf16 parts.
template <int NQ> __device__ __forceinline__ void load_q8(const void* q, size_t at, bf16x8* out) {
  if constexpr (NQ == 1) {
    out[0] = *reinterpret_cast<const bf16x8*>(static_cast<const uint16_t*>(q) + at);
  } else {
    const f32x4* p = reinterpret_cast<const f32x4*>(static_cast<const float*>(q) + at);
    const f32x4 x = p[0], y = p[1];
    const float f[8] = {x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
    split8(f, out);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      // an infinity or NaN is in the first part alone
      const bool whole = (__float_as_uint(f[e]) & 0x7f800000u) == 0x7f800000u;
      out[0][e] = whole ? (__bf16)f[e] : out[0][e];
      out[1][e] = whole ? (__bf16)0.f : out[1][e];
      out[2][e] = whole ? (__bf16)0.f : out[2][e];
    }
  }
}

// ---- a step ----------------------------------------------------------------------------------

// A wave's rows, QT tiles of 16, one to a lane of 16: their sums.
template <int D, int QT> struct KvSums {
  f32x4 o[QT][D / 16];  // o[t][j][i]: row lane % 16, column g D/4 + i D/16 + j
  float m[QT], l[QT];   // what the exponents are counted from, the lane's part of the sum
  int pos[QT];          // the row's position, -1 and less: sees nothing
  bool far;             // some row's m is beyond kFar; then c is 1 and off 0, else a.c and m
  float c, off[QT];
  bool large;           // there were value scales of kHighScale and more
};

template <int D, int QT> __device__ __forceinline__ void clear(KvSums<D, QT>& w, const KvAttentionArgs& a) {
  w.far = w.large = false;
  w.c = a.c;
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    w.m[t] = w.off[t] = kLow;
    w.l[t] = 0.f;
#pragma unroll
    for (int j = 0; j < D / 16; ++j) w.o[t][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
}

// The softmax of a step: scores z of the tokens of U records from tok on become weights, the
// sums what they are counted from.  `masked`: not every row sees all of the tokens.
template <int D, int QT, int U>
__device__ __forceinline__ void weights(KvSums<D, QT>& w, const KvAttentionArgs& a, f32x4 (&z)[QT][U], int tok, bool masked) {
  const int g = threadIdx.x % 64 / 16;
  if (__builtin_expect(masked, 0)) {
    asm volatile("");  // (a branch: these cost a step a third more where no row needs them)
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int t = 0; t < QT; ++t)
          z[t][u][i] = sees(a, w.pos[t], tok + 16 * u + 4 * g + i) ? z[t][u][i] : -__builtin_inff();
  }
  float top[QT];
  bool rise = false;
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    top[t] = z[t][0][0];
#pragma unroll
    for (int i = 1; i < 4 * U; ++i) top[t] = fmaxf(top[t], z[t][i / 4][i % 4]);
    top[t] *= a.c;
    rise |= top[t] > w.m[t] + (kLead + kLazy);  // (kLow plus that is kLow)
  }
  if (__builtin_expect(__ballot(rise) != 0, 0)) {
    asm volatile("");
    bool far = false;
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      float x = fmaxf(top[t], __shfl_xor(top[t], 16));
      x = fmaxf(x, __shfl_xor(x, 32));
      const float m = fmaxf(w.m[t], x - kLead), f = __builtin_amdgcn_exp2f(w.m[t] - m);
      w.m[t] = m;
      w.l[t] *= f;
      far |= fabsf(m) > kFar && m != kLow;
#pragma unroll
      for (int j = 0; j < D / 16; ++j) w.o[t][j] *= f;
    }
    w.far = __ballot(far) != 0;
    w.c = w.far ? 1.f : a.c;
#pragma unroll
    for (int t = 0; t < QT; ++t) w.off[t] = w.far ? 0.f : w.m[t];
  }
  if (__builtin_expect(w.far, 0)) {  // the exponents of rounded products, not of exact ones
    asm volatile("");
#pragma unroll
    for (int t = 0; t < QT; ++t)
#pragma unroll
      for (int i = 0; i < 4 * U; ++i) {
        float x = z[t][i / 4][i % 4] * a.c;
        asm volatile("" : "+v"(x));  // (no fused operation)
        x -= w.m[t];
        z[t][i / 4][i % 4] = x > kLead + kLazy ? kLead + kLazy : x;
      }
  }
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    float l = 0.f;
#pragma unroll
    for (int i = 0; i < 4 * U; ++i) {
      z[t][i / 4][i % 4] = __builtin_amdgcn_exp2f(fmaf(z[t][i / 4][i % 4], w.c, -w.off[t]));
      l += z[t][i / 4][i % 4];
    }
    w.l[t] += l;
  }
}

// The weights of records `first` and the next as NP f16 parts, the second product's operands.
template <int QT, int NP, int U>
__device__ __forceinline__ void weight_operands(const f32x4 (&z)[QT][U], int first, f16x8 (&part)[QT][NP]) {
#pragma unroll
  for (int t = 0; t < QT; ++t)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float r = z[t][first + i / 4][i % 4];
#pragma unroll
      for (int n = 0; n < NP; ++n) {
        part[t][n][i] = (_Float16)r;
        r -= (float)part[t][n][i];
      }
    }
}

// The value scales of tokens from `hi` on, of which no row sees any, as 1: a hidden token's
// weight is 0, but 0 times an infinity or NaN is not.  first: of the lane's four.
__device__ __forceinline__ uint32_t hidden_as_one(uint32_t vs, int first, int hi) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (first + i >= hi) vs = (vs & ~(0xffu << (8 * i))) | 0x7fu << (8 * i);
  return vs;
}

template <int D, int C, int QT>
__device__ __forceinline__ void wide_products(KvSums<D, QT>& w, const uint32_t (&v)[2][D / 32], const float (&sc)[2][4],
                                              const bf16x8 (&part)[QT][3]) {
  bf16x8 f[2];
  value_operands<D, C, false>(v, sc, f);
#pragma unroll
  for (int t = 0; t < QT; ++t)
#pragma unroll
    for (int n = 2; n >= 0; --n)
#pragma unroll
      for (int j = 0; j < 2; ++j)
        w.o[t][2 * C + j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f[j], part[t][n], w.o[t][2 * C + j], 0, 0, 0);
  if constexpr (C + 1 < D / 32) wide_products<D, C + 1, QT>(w, v, sc, part);
}

// The second product where a value scale is outside f16's range or NaN: bf16 values, whose
// range is the scales', and P in three bf16 parts.  A hidden token's p is 0, but 0 times NaN
// is not: scales of NaN (and the two whose values leave fp32, which are in a cache only
// where nothing was written) become 1, and the rows that see such a token NaN in its columns.
// The product of f16 operands follows in every step, here with values of 0 (no_values): where
// it followed in other steps alone, every step copied the sums.  lost: bit t: the lane's row has
// weights 2^-kLift as large.
template <int D, int QT, int U>
__device__ __forceinline__ void wide_values(KvSums<D, QT>& w, const KvAttentionArgs& a, const uint32_t (&v)[2][D / 32],
                                            const uint32_t (&scales)[2], const f32x4 (&p)[QT][U], int first, int tok,
                                            uint32_t lost = 0) {
  const int lane = threadIdx.x % 64, g = lane / 16;
  uint32_t odd = 0, vs[2] = {scales[0], scales[1]};
  bool large = false;  // (those of NaN are none: such rows are NaN however they are done)
  float sc[2][4];
#pragma unroll
  for (int u = 0; u < 2; ++u)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t byte = vs[u] >> (8 * i) & 0xffu;
      const bool nan = byte > kKvMaxExp + 127;
      odd |= nan ? 1u << (4 * u + i) : 0u;
      large |= byte >= kHighScale && !nan;
      sc[u][i] = kv_scale(nan ? 127u : byte);
    }
  if (__ballot(large)) w.large = true;
  uint32_t nan = 0;  // bit 4 t + i: the row sees a NaN in the columns o[t][..][i]
  if (__ballot(odd != 0)) {
    // Token 16 u + 4 g' + i is NaN in the columns of lane (n', g').  The columns o[..][..][n] of a
    // lane are those of n' = 4 g + n.
    for (int u = 0; u < 2; ++u)
      for (int gg = 0; gg < 4; ++gg)
        for (int i = 0; i < 4; ++i) {
          const int j = tok + 16 * u + 4 * gg + i;
          for (int n = 0; n < 4; ++n) {
            const uint32_t there = __shfl(odd, gg * 16 + 4 * g + n);
            if (there >> (4 * u + i) & 1u) {
#pragma unroll
              for (int t = 0; t < QT; ++t)
                if (sees(a, w.pos[t], j)) nan |= 1u << (4 * t + n);
            }
          }
        }
  }
  bf16x8 part[QT][3];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const float as = lost >> t & 1u ? 0x1p-48f : 1.f;
    const f32x4 x = p[t][first] * as, y = p[t][first + 1] * as;
    const float e[8] = {x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
    split8(e, part[t]);
  }
  wide_products<D, 0, QT>(w, v, sc, part);
#pragma unroll
  for (int t = 0; t < QT; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (nan >> (4 * t + i) & 1u) {
#pragma unroll
        for (int j = 0; j < D / 16; ++j) w.o[t][j][i] = __builtin_nanf("");
      }
}

template <int D, int C, int QT, int NP>
__device__ __forceinline__ void products(KvSums<D, QT>& w, const uint32_t (&v)[2][D / 32], const float (&sc)[2][4],
                                         const f16x8 (&part)[QT][NP]) {
  f16x8 f[2];
  value_operands<D, C, true>(v, sc, f);
#pragma unroll
  for (int t = 0; t < QT; ++t)
#pragma unroll
    for (int n = NP - 1; n >= 0; --n)
#pragma unroll
      for (int j = 0; j < 2; ++j)
        w.o[t][2 * C + j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(f[j], part[t][n], w.o[t][2 * C + j], 0, 0, 0);
  if constexpr (C + 1 < D / 32) products<D, C + 1, QT, NP>(w, v, sc, part);
}

// ---- large values -----------------------------------------------------------------------------

// The largest magnitude of a row's O, as bits (an infinity, or above it NaN); 0 for a row that is NaN by
// its scores.
template <int D, int QT> __device__ __forceinline__ uint32_t tallest(const KvSums<D, QT>& w, int t) {
  uint32_t top = w.l[t] != w.l[t] ? ~0u : 0u;
#pragma unroll
  for (int j = 0; j < D / 16; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i) top = max(top, __float_as_uint(w.o[t][j][i]) & 0x7fffffffu);
  top = max(top, (uint32_t)__shfl_xor((int)top, 16));
  top = max(top, (uint32_t)__shfl_xor((int)top, 32));
  return top == ~0u ? 0u : top;
}

// Makes m of a row whose O is smaller (lost), or is to be, what O is counted from; l follows, so that
// whoever joins sums need not know.  m is rounded up in front of the addition, which is exact then,
// and what that moves it by goes into l and O alike.  (Beyond 2^28 the sum may not be a float: O is
// as it would be without; weights are 0 or equal there, and only sums of equal ones can pass fp32.)
template <int D, int QT> __device__ __forceinline__ void settle(KvSums<D, QT>& w, uint32_t lost) {
  static_assert(kLift == 48, "the power below, and wide_values'");
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const bool small = lost >> t & 1u;
    const uint32_t top = tallest<D, QT>(w, t);
    const float add = small ? (float)kLift : top >= kTall && top < 0x7f800000u ? (float)kLower : 0.f;
    const float to = ceilf(w.m[t]) + add, by = w.m[t] - to;
    const bool can = add > 0.f && by <= -add && by >= -(add + 1.f);  // (m next to the integer below rounds to the latter)
    const float f = can ? __builtin_amdgcn_exp2f(by) : 1.f;
    w.m[t] = can ? to : w.m[t];
    w.l[t] *= f;
#pragma unroll
    for (int j = 0; j < D / 16; ++j) w.o[t][j] *= small ? f * 0x1p48f : f;
  }
}

// Behind a wave's steps, where there were large values (w.large).  The second time a wave is by itself: it
// reads the records for tokens tok, tok + stride .. below end, 32 at a time, and has wide_values do all
// values; q(t, n, j) is an operand of its rows.  Calls without large values take 0 to 2% longer for the code
// that is jumped over; 16 tokens behind 2048, all values near 2^124, 32 us instead of 17, a prompt of
// 2048 rows 239 instead of 71.
template <int D, int QT, int NQ, typename Q>
__device__ __forceinline__ void large_values(KvSums<D, QT>& w, const KvAttentionArgs& a, const KvRecords<D>& records, int tok, int end,
                                             int stride, int hi, const Q& q) {
  asm volatile("");
  uint32_t lost = 0;  // (what a row's weights are counted from may differ by 2^8 the second time: tall ones too)
  bool any = false;
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const uint32_t top = tallest<D, QT>(w, t);
    lost |= top >= kTall ? 1u << t : 0u;
    any |= top >= 0x7f800000u;
  }
  if (__ballot(any) == 0) lost = 0;
  if (__ballot(any)) {
    const int g = threadIdx.x % 64 / 16;
    const KvLane<D> off;
    clear(w, a);
#pragma unroll 1
    for (; tok < end; tok += stride) {
      f32x4 z[QT][2];
      uint32_t v[2][D / 32], vs[2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const typename KvRecords<D>::Place at = records.find((uint32_t)tok / kKvGroup + u);
        const __amdgpu_buffer_rsrc_t r = records.at(at);
        uint32_t k[D / 32];
        load_words<D / 32, false>(r, off.k, k);
        load_words<D / 32, false>(r, off.v, v[u]);
        const uint32_t ks = load_key_scales<D>(r, off.ks) | records.bad(at);
        vs[u] = hidden_as_one(__builtin_amdgcn_raw_buffer_load_b32(r, (int)off.vs, 0, 0), tok + 16 * u + 4 * g, hi);
#pragma unroll
        for (int t = 0; t < QT; ++t) z[t][u] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int n = NQ - 1; n >= 0; --n)
#pragma unroll
          for (int j = 0; j < D / 32; ++j) {
            const bf16x8 key = eight_of(k[j], D == 256 && j >= 4 ? kv_scale(ks >> 8 & 0xffu) : kv_scale(ks & 0xffu));
#pragma unroll
            for (int t = 0; t < QT; ++t) z[t][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(key, q(t, n, j), z[t][u], 0, 0, 0);
          }
      }
      weights<D, QT, 2>(w, a, z, tok, true);
      wide_values<D, QT, 2>(w, a, v, vs, z, 0, tok, lost);
    }
  }
  settle<D, QT>(w, lost);
}

// ---- kernels ----------------------------------------------------------------------------------

// Waves of a SIMD of the rows' kernel, which is blocks of a compute unit: what its registers
// allow.  (A kernel that spills any takes 6 us longer to start: with two waves the widest fp32 rows
// take 14.4 us instead of 8.8 for 200 tiles of 4 tokens, 49 instead of 28.5 behind 16 times 8192.)
constexpr int kv_rows_waves(int d, int qt, bool bf16) { return d * qt == 64 ? 3 : d * qt == 256 && !bf16 ? 1 : 2; }
// Tokens of a unit, and the units that a tile costs besides its own.
constexpr int kKvRowsUnit = 128, kKvRowsLead = 3, kKvPromptLead = 3;
constexpr int kv_prompt_unit(int d) { return d == 256 ? 32 : 64; }
// Tiles of 16 rows of a wave of the prompt's kernel.
constexpr int kv_prompt_qt(int d, bool bf16) { return d == 64 || (d == 128 && bf16) ? 2 : 1; }
constexpr int kv_prompt_rows(int d, bool bf16) { return kKvWaves * 16 * kv_prompt_qt(d, bf16); }

template <int D> hipError_t launch_kv_rows_attention(const KvAttentionArgs& a, int qt, bool bf16, hipStream_t s);
template <int D> hipError_t launch_kv_prompt_attention(const KvAttentionArgs& a, bool bf16, hipStream_t s);

}  // namespace cats
