// Quantising rows of keys and values into the cache, and reading rows back.
//
// Both are bound by memory at many rows and by their launch at few: a lane has 8
// columns of one token (16 bytes of bf16, 4 of codes), four lanes share a scale,
// and a block has consecutive rows of one head, whose records they fill or read
// together while their lines are in the L2.  The codes come from the conversion
// instructions: nearest value, ties to even, largest 6, scales powers of two, so
// nothing is rounded but the value to its code.
// 4096 rows of 32 heads of 128 columns in bf16, 85 MB: written in 18.6 us (4.6 TB/s),
// read back in 14.0 (6.1 TB/s); 46 us together before a head's blocks shared an XCD (and
// its L2 a record's lines) and the rows went past the L2.  In fp32, 152 MB: written in 29.1 us (5.2
// TB/s), read back in 52 (2.9 TB/s: each of a lane's two stores leaves every other 16 bytes to the other).
#include <algorithm>

#include "internal.hpp"
#include "kv4.hpp"

namespace cats {
namespace {

constexpr int kThreads = 256;

// Slot of a row: record and token, or false for one outside the cache.
struct Place {
  size_t rec;
  int t;
};
template <int D> __device__ __forceinline__ bool place(const KvRowsArgs& a, int row, int head, Place& p) {
  const int slot = a.slots[row];
  if (slot < 0 || slot >= a.tokens) return false;
  const uint32_t rec = (uint32_t)slot / kKvGroup, page = __umulhi(rec << 1, a.magic);
  p.rec = (((size_t)page * a.heads + head) * a.groups + (rec - page * a.groups)) * kv_record_bytes(D);
  p.t = slot % kKvGroup;
  return true;
}

// Byte of columns [8 c, 8 c + 8) of token t, values (two pieces 8 bytes apart where D is 64).
template <int D> __device__ __forceinline__ int value_at(int t, int c) {
  const int n = 8 * c / (D / 16), r = 8 * c % (D / 16);
  return 8 * D + (((t >> 2) * 16 + n) * 4 + (t & 3)) * (D / 32) + r / 2;
}
template <int D> __device__ __forceinline__ int scale_at(bool value, int t, int blk) {
  return 16 * D + (value ? D / 2 + ((t >> 2) * (D / 32) + blk) * 4 + (t & 3) : t * (D / 32) + blk);
}

// (rows are read once: non-temporal, which leaves the L2 to the records that fill up there)
template <bool BF16> __device__ __forceinline__ void load8(const void* src, size_t at, float* f) {
  if (BF16) {
    widen<wbf16>(__builtin_nontemporal_load(reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(src) + at)), f);
  } else {
    const u32x4* s = reinterpret_cast<const u32x4*>(static_cast<const float*>(src) + at);
    widen<wf32>(__builtin_nontemporal_load(s), f);
    widen<wf32>(__builtin_nontemporal_load(s + 1), f + 4);
  }
}

// Codes of a lane's 8 columns, with the scale of its four lanes' 32.
__device__ __forceinline__ uint32_t codes_of(const float* f, uint32_t& byte) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(f[i]) & 0x7fffffffu);
  top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0xb1, 0xf, 0xf, false));
  top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0x4e, 0xf, 0xf, false));
  byte = kv_scale_byte(top);
  const float s = kv_scale(byte);
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[0], f[1], s, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[2], f[3], s, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[4], f[5], s, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[6], f[7], s, 3);
  return byte == 255u ? 0u : w;  // (NaN by its scale; the codes of such a block are 0)
}

template <int D, bool BF16> __global__ __launch_bounds__(kThreads) void k_kv_write(KvRowsArgs a) {
  constexpr int L = D / 8;  // lanes of a row
  const uint32_t part = blockIdx.x / (uint32_t)a.heads;
  const int row = part * (kThreads / L) + threadIdx.x / L, head = blockIdx.x - part * a.heads, c = threadIdx.x % L;
  // (all four lanes of a scale have the same row)
  if (row >= a.rows) return;
  float k[8], v[8];
  load8<BF16>(a.k, (size_t)row * a.ldk + head * D + 8 * c, k);
  load8<BF16>(a.v, (size_t)row * a.ldv + head * D + 8 * c, v);
  Place p;
  if (!place<D>(a, row, head, p)) return;
  uint8_t* rec = a.cache + p.rec;
  uint32_t kb, vb;
  const uint32_t kw = codes_of(k, kb), vw = codes_of(v, vb);
  *reinterpret_cast<uint32_t*>(rec + p.t * (D / 2) + 4 * c) = kw;
  uint8_t* to = rec + value_at<D>(p.t, c);
  if (D == 64) {
    *reinterpret_cast<uint16_t*>(to) = (uint16_t)vw;
    *reinterpret_cast<uint16_t*>(to + 8) = (uint16_t)(vw >> 16);
  } else {
    *reinterpret_cast<uint32_t*>(to) = vw;
  }
  if (c % 4 == 0) {
    rec[scale_at<D>(false, p.t, c / 4)] = (uint8_t)kb;
    rec[scale_at<D>(true, p.t, c / 4)] = (uint8_t)vb;
  }
}

template <bool BF16> __device__ __forceinline__ void store8(void* dst, size_t at, uint32_t w, float s) {
  if (BF16) {
    u32x4 o;
    o.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 0));
    o.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 1));
    o.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 2));
    o.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 3));
    __builtin_nontemporal_store(o, reinterpret_cast<u32x4*>(static_cast<uint16_t*>(dst) + at));
  } else {
    const f32x2 v0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 0);
    const f32x2 v1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 1);
    const f32x2 v2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 2);
    const f32x2 v3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 3);
    f32x4* o = reinterpret_cast<f32x4*>(static_cast<float*>(dst) + at);
    __builtin_nontemporal_store(f32x4{v0[0], v0[1], v1[0], v1[1]}, o);
    __builtin_nontemporal_store(f32x4{v2[0], v2[1], v3[0], v3[1]}, o + 1);
  }
}

template <int D, bool BF16> __global__ __launch_bounds__(kThreads) void k_kv_read(KvRowsArgs a) {
  constexpr int L = D / 8;
  const uint32_t part = blockIdx.x / (uint32_t)a.heads;
  const int row = part * (kThreads / L) + threadIdx.x / L, head = blockIdx.x - part * a.heads, c = threadIdx.x % L;
  Place p;
  if (row >= a.rows || !place<D>(a, row, head, p)) return;
  const uint8_t* rec = a.cache + p.rec;
  const uint32_t kw = *reinterpret_cast<const uint32_t*>(rec + p.t * (D / 2) + 4 * c);
  const uint8_t* from = rec + value_at<D>(p.t, c);
  const uint32_t vw = D == 64 ? *reinterpret_cast<const uint16_t*>(from) |
                                    (uint32_t)*reinterpret_cast<const uint16_t*>(from + 8) << 16
                              : *reinterpret_cast<const uint32_t*>(from);
  const float ks = kv_scale(rec[scale_at<D>(false, p.t, c / 4)]), vs = kv_scale(rec[scale_at<D>(true, p.t, c / 4)]);
  const size_t at = ((size_t)row * a.heads + head) * D + 8 * c;
  store8<BF16>(a.k_out, at, kw, ks);
  store8<BF16>(a.v_out, at, vw, vs);
}

// A launch holds 2^31 threads; calls of more rows take several.
template <int D> hipError_t go(bool write, bool bf16, KvRowsArgs a, hipStream_t s) {
  constexpr int RB = kThreads / (D / 8);  // rows of a block
  const int all = a.rows, most = (int)std::min<int64_t>(all, (int64_t)((1u << 31) / kThreads / a.heads) * RB);
  const size_t elem = bf16 ? 2 : 4;
  for (int at = 0; at < all; at += most) {
    a.rows = std::min(most, all - at);
    const dim3 grid((uint32_t)((a.rows + RB - 1) / RB) * a.heads);
    KernelTimer tm(write ? "kv_write" : "kv_read", s);
#define CATS_GO(K) hipExtLaunchKernelGGL((K), grid, dim3(kThreads), 0, s, tm.start(), tm.stop(), 0, a)
    if (write) {
      if (bf16) CATS_GO((k_kv_write<D, true>));
      else CATS_GO((k_kv_write<D, false>));
    } else {
      if (bf16) CATS_GO((k_kv_read<D, true>));
      else CATS_GO((k_kv_read<D, false>));
    }
#undef CATS_GO
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    a.slots += a.rows;
    if (write) {
      a.k = static_cast<const uint8_t*>(a.k) + a.rows * a.ldk * elem;
      a.v = static_cast<const uint8_t*>(a.v) + a.rows * a.ldv * elem;
    } else {
      a.k_out = static_cast<uint8_t*>(a.k_out) + (size_t)a.rows * a.heads * D * elem;
      a.v_out = static_cast<uint8_t*>(a.v_out) + (size_t)a.rows * a.heads * D * elem;
    }
  }
  return hipSuccess;
}

}  // namespace

hipError_t launch_kv_rows(bool write, bool bf16, int d, const KvRowsArgs& a, hipStream_t s) {
  return d == 64 ? go<64>(write, bf16, a, s) : d == 128 ? go<128>(write, bf16, a, s) : go<256>(write, bf16, a, s);
}

}  // namespace cats
