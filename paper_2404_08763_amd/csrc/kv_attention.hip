// Attention over the cache in 4 bits: o = sum_j softmax_j(scale q k_j) v_j.
//
// One pass over the keys with a running maximum and sum.  A wave has a tile of
// 16 QT rows (the query heads of a key head side by side, then the next query)
// and takes 32 or 64 tokens a step; its sums stay in registers:
//   - S^T = K Q^T: the records' layout (kv4.hpp) gives each lane its part of the
//     matrix operand in one load; the conversion instructions make bf16 of the
//     codes and scales, exactly, so the products are exact and their sums fp32.
//   - a column of S^T, a query row, is in the lanes of equal lane % 16: its
//     softmax needs no exchange but for a new maximum, and P is the operand of
//     O^T = V^T P^T as it lies, as the order of the tokens within a step is free.
//   - V^T needs two tokens side by side where a conversion gives two columns: one
//     byte permutation per pair.
// The scores, P before its rounding, the statistics and O are fp32.  The second product
// is one of f16, which has the cache's values exactly (but for scales far out, see
// wide_values) and P with 11 bits for bf16 rows, an eighth of their own rounding, and in
// two parts with 22 for fp32 rows, whose q is split in three bf16 parts, all 24 bits.  P's
// steps end at f16's least, 2^-24 of weights that are 2^7 or more where they are largest: its
// error is 2^-32 of a row's largest weight for each token where that is more.
//
// One kernel takes few rows of each sequence (kv_rows.hpp), another many (kv_prompt.hpp).
// The blocks share all of a call's keys evenly, whatever the sequences' lengths (KvRun): what
// is split over blocks is joined by a last kernel (few rows in few parts: by the block that
// arrives last), and where ragged queries make many tiles a first one lists them.
#include <algorithm>

#include "kv_attention.hpp"

namespace cats {
namespace {

// ---- the plan: tiles of ragged queries --------------------------------------

constexpr int kPlanThreads = 1024;
template <int UNIT, int LEAD>
__global__ __launch_bounds__(kPlanThreads) void k_kv_plan(KvAttentionArgs a, int R, int most) {
  __shared__ int sh[kPlanThreads / 64];
  const int G = a.hq / a.hkv;
  int tiles = 0;
  for (int base = 0; base < a.B; base += kPlanThreads) {
    const int b = base + threadIdx.x;
    int start, n = 0, total;
    if (b < a.B) n = (kv_queries(a, b, start) * G + R - 1) / R;
    const int at = block_prefix<kPlanThreads>(n, total, sh) + tiles;
    if (b < a.B) a.first[b] = at;
    tiles += total;
  }
  tiles = min(tiles, most);  // (there are more only where q_start decreases)
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
      u = kv_tile<UNIT>(a, G, b, row0, R, kv_length(a, b)).units + LEAD;
    }
    const int at = block_prefix<kPlanThreads>(u, total, sh) + units;
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

// ---- parts into one -----------------------------------------------------------

// Joins a sum that desc notes: its first part in block lb, the others in the blocks
// behind it.  D / 4 threads have a row of a part.  ROW: a block has one row and takes its parts
// side by side (few rows, many parts); else it has as many rows as it holds.
template <int D, bool BF16, bool ROW> __global__ __launch_bounds__(kKvThreads) void k_kv_join(KvAttentionArgs a, int R) {
  constexpr int L = D / 4, S = kKvThreads / L;
  const int PART = R * (D + 2);
  const int s = threadIdx.x / L, c = threadIdx.x % L * 4;
  const int row = ROW ? blockIdx.y : blockIdx.y * S + s;
  const int4 d = a.desc[blockIdx.x];
  const int n = d.x & 0xffff, lb = d.x >> 16, h = d.y, b = d.z, row0 = d.w, G = a.hq / a.hkv;
  if (n == 0) return;
  int start;
  const int nq = kv_queries(a, b, start);
  if (row >= min(R, nq * G - row0)) return;
  const float* base = a.part + (size_t)lb * 2 * PART;
  // a running maximum again, so that each part is read once
  float m = -__builtin_inff(), l = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int i = ROW ? s : 0; i < n; i += ROW ? S : 1) {
    const float* p = base + (size_t)(i == 0 ? 1 : 2 * i) * PART;
    const float pm = p[R * D + row], pl = p[R * D + R + row];
    const f32x4 po = *reinterpret_cast<const f32x4*>(p + row * D + c);
    const float top = fmaxf(m, pm);
    const float was = m == top ? 1.f : __builtin_amdgcn_exp2f(m - top), is = pm == top ? 1.f : __builtin_amdgcn_exp2f(pm - top);
    m = top;
    l = l * was + pl * is;
    o = o * was + po * is;
  }
  if constexpr (ROW) {
    __shared__ float so[S][D];
    __shared__ float sm[S], sl[S];
    *reinterpret_cast<f32x4*>(&so[s][c]) = o;
    if (c == 0) {
      sm[s] = m;
      sl[s] = l;
    }
    __syncthreads();
    if (s != 0) return;
    float top = -__builtin_inff();
#pragma unroll
    for (int i = 0; i < S; ++i) top = fmaxf(top, sm[i]);
    l = 0.f;
    o = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < S; ++i) {
      if (sm[i] == -__builtin_inff()) continue;  // (fewer parts than S, or a row that sees no key)
      const float f = __builtin_amdgcn_exp2f(sm[i] - top);
      l += sl[i] * f;
      o += *reinterpret_cast<const f32x4*>(&so[i][c]) * f;
    }
    m = top;
  }
  o *= 1.f / l;
  if (m == -__builtin_inff()) o = f32x4{0.f, 0.f, 0.f, 0.f};
  store_out<BF16>(a.out, ((size_t)(start + (row0 + row) / G) * a.hq + h * G + (row0 + row) % G) * D + c, o);
}

// ---- the host's side ----------------------------------------------------------

// How a call is done, and what it takes of the workspace.
struct Shape {
  bool prompt;           // the prompt's kernel
  int qt;                // the rows' kernel: tiles of 16 rows of a wave
  int R, unit, lead;     // rows of a tile, tokens of a unit, units that a tile costs besides
  int blocks;            // blocks at most: all run at once
  size_t tiles;          // of a head, at most
  size_t off_plan, off_prefix, off_first, off_desc, off_part, bytes;
};
constexpr size_t up256(size_t v) { return (v + 255) / 256 * 256; }
constexpr int kMostBlocks = 768;
// Partial sums: two a block, but for the first block's first and the last block's second, which no tile has.
size_t part_bytes(int d, int R, int blocks) { return (size_t)(2 * blocks - 2) * R * (d + 2) * 4; }

// Two to a compute unit; fewer where a workspace without its lists would pass 64 MiB: 504 for bf16 rows of
// 128 columns and for 256 columns.  (23 bf16 prompts of 512 to 8192 rows of 128 columns take 0.957 of the time
// of 480 blocks with 512, 0.976 with 504, single ones up to 5% more or 5% less by how tiles fall on blocks;
// fp32 rows 0.959 with 512; 256 columns 0.996 with 512, 1.01 with 504.)
constexpr size_t kMostWorkspace = (size_t)64 << 20;
int prompt_blocks(int d, bool bf16) {
  int blocks = 512;
  while (256 + up256(kMostBlocks * 40) + part_bytes(d, kv_prompt_rows(d, bf16), blocks) > kMostWorkspace) blocks -= 8;
  return blocks;
}

Shape shape_of(int N, int B, int hq, int hkv, int d, bool bf16, bool planned) {
  Shape s{};
  const int G = hq / hkv;
  // A tile of 16 rows while it holds all of a sequence's rows, then 32; the prompt's kernel
  // for more.
  const long long per = planned ? ((long long)N * G + B - 1) / B : G;
  s.prompt = planned && per > 32;
  s.qt = per <= 16 || d == 256 ? 1 : 2;
  s.R = s.prompt ? kv_prompt_rows(d, bf16) : 16 * s.qt;
  s.unit = s.prompt ? kv_prompt_unit(d) : kKvRowsUnit;
  s.lead = s.prompt ? kKvPromptLead : kKvRowsLead;
  s.blocks = s.prompt ? prompt_blocks(d, bf16) : 256 * kv_rows_waves(d, s.qt, bf16);
  s.tiles = planned ? (size_t)(((long long)N * G + s.R - 1) / s.R + B) : (size_t)B * ((G + s.R - 1) / s.R);
  const size_t listed = planned ? s.tiles : 0;
  s.off_plan = 256;
  s.off_prefix = s.off_plan + up256(listed * sizeof(KvPlanEntry));
  s.off_first = s.off_prefix + up256(listed * 4);
  s.off_desc = s.off_first + (planned ? up256((size_t)(B + 1) * 4) : 0);
  s.off_part = s.off_desc + up256((size_t)s.blocks * (s.prompt ? 40 : 16));
  s.bytes = s.off_part + part_bytes(d, s.R, s.blocks);
  return s;
}

// Units of a tile at most: of a table's row.
long long units_most(const KvAttentionArgs& a, int unit) { return ((long long)a.limit + unit - 1) / unit + 1; }

template <int D> hipError_t join(const KvAttentionArgs& a, const Shape& sh, bool bf16, hipStream_t s) {
  KernelTimer tm("kv_join", s);
  const int at_once = sh.prompt ? kKvThreads / (D / 4) : 1, rows = a.q_start ? sh.R : std::min(sh.R, a.hq / a.hkv);
  const dim3 grid(a.sums, (rows + at_once - 1) / at_once), th(kKvThreads);
#define CATS_GO(B, ROW) hipExtLaunchKernelGGL((k_kv_join<D, B, ROW>), grid, th, 0, s, tm.start(), tm.stop(), 0, a, sh.R)
  if (bf16) {
    if (sh.prompt) CATS_GO(true, false);
    else CATS_GO(true, true);
  } else {
    if (sh.prompt) CATS_GO(false, false);
    else CATS_GO(false, true);
  }
#undef CATS_GO
  return hipGetLastError();
}

template <int D> hipError_t go(const KvAttentionArgs& a, const Shape& sh, bool bf16, bool split, hipStream_t s) {
  hipError_t e = sh.prompt ? launch_kv_prompt_attention<D>(a, bf16, s) : launch_kv_rows_attention<D>(a, sh.qt, bf16, s);
  if (e == hipSuccess && split) e = join<D>(a, sh, bf16, s);
  return e;
}

}  // namespace

size_t kv_attention_bytes(int N, int B, int hq, int hkv, int d, bool bf16, bool planned) {
  return shape_of(N, B, hq, hkv, d, bf16, planned).bytes;
}

size_t kv_attention_most(int N, int B, int hq, int hkv, int d) {
  const size_t tiles = ((size_t)N * (hq / hkv) + 15) / 16 + B;
  size_t part = 0;
  for (int qt = 1; qt <= 2; ++qt) part = std::max(part, part_bytes(d, 16 * qt, 256 * kv_rows_waves(d, qt, true)));
  for (const bool bf16 : {false, true}) part = std::max(part, part_bytes(d, kv_prompt_rows(d, bf16), prompt_blocks(d, bf16)));
  return 256 + up256(tiles * sizeof(KvPlanEntry)) + up256(tiles * 4) + up256((size_t)(B + 1) * 4) + up256(kMostBlocks * 40) + part;
}

// (the prefixes of a head's tiles are 32-bit numbers)
bool kv_attention_fits(const KvAttentionArgs& a, int d, bool bf16) {
  const Shape sh = shape_of(a.N, a.B, a.hq, a.hkv, d, bf16, a.q_start != nullptr);
  return (double)sh.tiles * (double)(units_most(a, sh.unit) + sh.lead) < 2147483648.0;
}

hipError_t launch_kv_attention(KvAttentionArgs a, int d, bool bf16, hipStream_t s) {
  const Shape sh = shape_of(a.N, a.B, a.hq, a.hkv, d, bf16, a.q_start != nullptr);
  uint8_t* ws = reinterpret_cast<uint8_t*>(a.head);
  a.plan = reinterpret_cast<KvPlanEntry*>(ws + sh.off_plan);
  a.prefix = reinterpret_cast<int*>(ws + sh.off_prefix);
  a.first = reinterpret_cast<int*>(ws + sh.off_first);
  a.desc = reinterpret_cast<int4*>(ws + sh.off_desc);
  a.part = reinterpret_cast<float*>(ws + sh.off_part - (size_t)sh.R * (d + 2) * 4);
  a.tiles = a.q_start ? (int)sh.tiles : (a.hq / a.hkv + sh.R - 1) / sh.R;
  // The last block to arrive joins a tile's parts where they are 64 KB at most if all tiles are
  // as long as the tables (tiles of very different lengths: KvRun); more of them a kernel of their own.
  const int row_bytes = std::min(sh.R, a.hq / a.hkv) * d * 4;
  const long long split_in = std::min<long long>(units_most(a, sh.unit), sh.blocks / ((long long)sh.tiles * a.hkv) + 2);
  a.parts = !a.q_start && split_in * row_bytes <= (64 << 10) ? (64 << 10) / row_bytes : 0;
  // So do the blocks of a prompt with a tile for every other block or more, whose tiles are in
  // three parts or less where they are alike, in tens where one is far longer (1024 tiles for 480
  // blocks 186 us instead of 195, 256 tiles 37 instead of 44; 188 tiles 49 instead of 45, 128 tiles 33
  // instead of 32).
  if (sh.prompt && (long long)a.N * (a.hq / a.hkv) / sh.R * a.hkv >= sh.blocks / 2) a.parts = 1;
  a.tickets = reinterpret_cast<unsigned long long*>(a.desc);
  a.epoch = call_epoch();
  // no more blocks than units
  const double most = (double)sh.tiles * a.hkv * (double)(units_most(a, sh.unit) + sh.lead);
  a.blocks = most < sh.blocks ? ((int)most + 7) / 8 * 8 : sh.blocks;
  a.by_tile = sh.tiles * a.hkv <= (size_t)a.blocks ? 1 : 0;
  a.sums = a.by_tile ? (int)sh.tiles * a.hkv : a.blocks;
  if (a.q_start && sh.tiles <= (size_t)kKvOwnTiles && a.B <= kKvOwnSequences) {
    a.plan = nullptr;  // (each block makes it: 2 us of each instead of a launch of 4)
  } else if (a.q_start) {
    KernelTimer tm("kv_plan", s);
    const int listed = (int)sh.tiles;
#define CATS_GO(U, L) \
  hipExtLaunchKernelGGL((k_kv_plan<U, L>), dim3(1), dim3(kPlanThreads), 0, s, tm.start(), tm.stop(), 0, a, sh.R, listed)
    if (!sh.prompt) CATS_GO(kKvRowsUnit, kKvRowsLead);
    else if (sh.unit == 64) CATS_GO(64, kKvPromptLead);
    else CATS_GO(32, kKvPromptLead);
#undef CATS_GO
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  const bool split = a.parts == 0 && a.limit > sh.unit;  // (else every tile is one unit)
  return d == 64 ? go<64>(a, sh, bf16, split, s) : d == 128 ? go<128>(a, sh, bf16, split, s) : go<256>(a, sh, bf16, split, s);
}

}  // namespace cats
