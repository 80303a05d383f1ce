// C ABI of the operators around attention: argument checks on the host, then the launch.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdio>

#include "cats.h"
#include "internal.hpp"
#include "kv4.hpp"

namespace {

template <typename... A> cats_status fail(cats_status st, const char* fmt, A... a) {
  char buf[256];
  snprintf(buf, sizeof(buf), fmt, a...);
  return cats::report_error(st, buf);
}
cats_status fail(cats_status st, const char* msg) { return cats::report_error(st, msg); }

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

// A range of memory that a call reads or writes.
struct Range {
  const void* p;
  size_t n;
  const char* name;
};
bool overlap(const Range& a, const Range& b) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a.p), y = reinterpret_cast<uintptr_t>(b.p);
  return a.p && b.p && a.n && b.n && x < y + b.n && y < x + a.n;
}
// Every output against every other range.
template <size_t N> cats_status check_overlap(const Range (&r)[N], size_t outputs) {
  for (size_t i = 0; i < outputs; ++i)
    for (size_t j = i + 1; j < N; ++j)
      if (overlap(r[i], r[j])) return fail(CATS_ERR_RANGE, "%s must not overlap %s", r[i].name, r[j].name);
  return CATS_OK;
}

size_t elem_bytes(int32_t dtype) { return dtype == CATS_BF16 ? 2 : 4; }
bool dtype_ok(int32_t dtype) { return dtype == CATS_F32 || dtype == CATS_BF16; }

// Bytes of a [rows x cols] matrix of pitch ld.
size_t pitched(size_t rows, size_t cols, size_t ld, size_t elem) { return ((rows - 1) * ld + cols) * elem; }

cats_status launched(hipError_t e, void* stream, const char* what) {
  if (e != hipSuccess) return fail(CATS_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
  return cats::enqueued(stream, what);
}

bool heads_ok(int32_t h) { return h >= 1 && h <= CATS_MAX_KV_HEADS; }
bool rows_ok(int32_t n) { return n >= 1 && n <= CATS_MAX_KV_ROWS; }

bool cache_shape_ok(int32_t pages, int32_t page, int32_t heads, int32_t d) {
  return pages >= 1 && page >= 16 && page <= 256 && page % 16 == 0 && heads_ok(heads) &&
         (d == 64 || d == 128 || d == 256) && (int64_t)pages * page <= CATS_MAX_KV_TOKENS;
}
size_t cache_bytes(int32_t pages, int32_t page, int32_t heads, int32_t d) {
  return (size_t)pages * heads * (page / 16) * cats::kv_record_bytes(d);
}
cats_status check_cache(const cats_kv_cache* c) {
  if (!c || !c->data) return fail(CATS_ERR_NULL, "the cache or its data is NULL");
  if (!cache_shape_ok(c->pages, c->page, c->heads, c->d))
    return fail(CATS_ERR_SHAPE,
                "cache of %d pages of %d tokens, %d heads of %d: pages * page in [16, 2^30], page a multiple of 16 up to "
                "256, heads in [1, %d], d 64, 128 or 256",
                (int)c->pages, (int)c->page, (int)c->heads, (int)c->d, CATS_MAX_KV_HEADS);
  if (!aligned(c->data, 16)) return fail(CATS_ERR_ALIGN, "the cache must be 16-byte aligned");
  return CATS_OK;
}

// For the quotient of a record's number (below 2^26) by the records of a page (16 at most):
// rec / groups is the upper half of 2 rec ceil(2^31 / groups).  The factor is less than 16 / groups
// above 2^31 / groups, so the product is above the quotient by less than 2^26 * 16 / 2^31 of
// 1 / groups, and has its whole part.
uint32_t magic_of(int groups) { return (uint32_t)(((1ull << 31) + groups - 1) / groups); }

constexpr size_t kWsAlign = 256;

// Queries of a call: whether N rows for B sequences of hq heads on hkv are within the limits.
bool attention_shape_ok(int32_t N, int32_t B, int32_t hq, int32_t hkv, int32_t d) {
  return rows_ok(N) && rows_ok(B) && heads_ok(hkv) && heads_ok(hq) && hq % hkv == 0 && (d == 64 || d == 128 || d == 256);
}

}  // namespace

extern "C" {

cats_status cats_qk_norm_rope(const void* qkv, int32_t dtype, int64_t ld, int32_t N, int32_t hq, int32_t hkv, int32_t d,
                              int32_t norm, const float* gain_q, const float* gain_k, float eps, const int32_t* pos,
                              const float* freq, int32_t rot, int32_t interleaved, void* q, void* k, int32_t odtype,
                              void* stream) {
  if (!qkv || !q || !k) return fail(CATS_ERR_NULL, "qkv, q or k is NULL");
  if (!dtype_ok(dtype) || !dtype_ok(odtype)) return fail(CATS_ERR_DTYPE, "unknown dtype %d or %d", (int)dtype, (int)odtype);
  if (!rows_ok(N) || !heads_ok(hq) || !heads_ok(hkv) || d < 8 || d > 512 || d % 8)
    return fail(CATS_ERR_SHAPE, "N=%d, heads %d and %d of %d: N in [1, %d], heads in [1, %d], d a multiple of 8 up to 512",
                (int)N, (int)hq, (int)hkv, (int)d, CATS_MAX_KV_ROWS, CATS_MAX_KV_HEADS);
  if (rot < 0 || rot > d || rot % 8) return fail(CATS_ERR_SHAPE, "rot=%d must be a multiple of 8 in [0, %d]", (int)rot, (int)d);
  const int64_t cols = (int64_t)(hq + hkv) * d;
  if (ld < cols || ld % 8 || ld > CATS_MAX_KV_PITCH)
    return fail(CATS_ERR_SHAPE, "ld=%lld must be a multiple of 8 in [%lld, 2^30]", (long long)ld, (long long)cols);
  if (rot > 0 && (!pos || !freq)) return fail(CATS_ERR_NULL, "pos or freq is NULL");
  if (norm && (!std::isfinite(eps) || eps < 0.f)) return fail(CATS_ERR_RANGE, "eps must be finite and >= 0");
  if (!aligned(qkv, 16) || !aligned(q, 16) || !aligned(k, 16) || !aligned(gain_q, 16) || !aligned(gain_k, 16) ||
      !aligned(freq, 16) || !aligned(pos, 4))
    return fail(CATS_ERR_ALIGN, "qkv, gains, freq, q and k must be 16-byte aligned, pos 4-byte");
  const size_t o = elem_bytes(odtype);
  const Range r[] = {{q, (size_t)N * hq * d * o, "q"},
                     {k, (size_t)N * hkv * d * o, "k"},
                     {qkv, pitched(N, cols, ld, elem_bytes(dtype)), "qkv"},
                     {norm ? gain_q : nullptr, (size_t)d * 4, "gain_q"},
                     {norm ? gain_k : nullptr, (size_t)d * 4, "gain_k"},
                     {rot ? pos : nullptr, (size_t)N * 4, "pos"},
                     {rot ? freq : nullptr, (size_t)rot * 2, "freq"}};
  const cats_status st = check_overlap(r, 2);
  if (st != CATS_OK) return st;
  cats::QkRopeArgs a{};
  a.x = qkv;
  a.ld = (size_t)ld;
  a.pos = pos;
  a.freq = freq;
  a.gq = gain_q;
  a.gk = gain_k;
  a.q = q;
  a.k = k;
  a.N = N;
  a.hq = hq;
  a.hkv = hkv;
  a.d = d;
  a.rot = rot;
  a.norm = norm ? 1 : 0;
  a.interleaved = interleaved ? 1 : 0;
  a.eps = eps;
  return launched(cats::launch_qk_rope(a, dtype == CATS_BF16, odtype == CATS_BF16, static_cast<hipStream_t>(stream)), stream,
                  "cats_qk_norm_rope");
}

size_t cats_kv_cache_bytes(int32_t pages, int32_t page, int32_t heads, int32_t d) {
  return cache_shape_ok(pages, page, heads, d) ? cache_bytes(pages, page, heads, d) : 0;
}

cats_status cats_kv_write(const cats_kv_cache* cache, const void* k, int64_t ldk, const void* v, int64_t ldv, int32_t dtype,
                          const int32_t* slots, int32_t N, void* stream) {
  cats_status st = check_cache(cache);
  if (st != CATS_OK) return st;
  if (!k || !v || !slots) return fail(CATS_ERR_NULL, "k, v or slots is NULL");
  if (!dtype_ok(dtype)) return fail(CATS_ERR_DTYPE, "unknown dtype %d", (int)dtype);
  if (!rows_ok(N)) return fail(CATS_ERR_SHAPE, "N=%d outside [1, %d]", (int)N, CATS_MAX_KV_ROWS);
  const int64_t cols = (int64_t)cache->heads * cache->d;
  if (ldk < cols || ldv < cols || ldk % 8 || ldv % 8 || ldk > CATS_MAX_KV_PITCH || ldv > CATS_MAX_KV_PITCH)
    return fail(CATS_ERR_SHAPE, "ldk=%lld and ldv=%lld must be multiples of 8 in [%lld, 2^30]", (long long)ldk, (long long)ldv,
                (long long)cols);
  if (!aligned(k, 16) || !aligned(v, 16) || !aligned(slots, 4))
    return fail(CATS_ERR_ALIGN, "k and v must be 16-byte aligned, slots 4-byte");
  const Range r[] = {{cache->data, cache_bytes(cache->pages, cache->page, cache->heads, cache->d), "the cache"},
                     {k, pitched(N, cols, ldk, elem_bytes(dtype)), "k"},
                     {v, pitched(N, cols, ldv, elem_bytes(dtype)), "v"},
                     {slots, (size_t)N * 4, "slots"}};
  if ((st = check_overlap(r, 1)) != CATS_OK) return st;
  cats::KvRowsArgs a{};
  a.cache = static_cast<uint8_t*>(cache->data);
  a.slots = slots;
  a.tokens = cache->pages * cache->page;
  a.groups = cache->page / 16;
  a.magic = magic_of(a.groups);
  a.heads = cache->heads;
  a.rows = N;
  a.k = k;
  a.v = v;
  a.ldk = (size_t)ldk;
  a.ldv = (size_t)ldv;
  return launched(cats::launch_kv_rows(true, dtype == CATS_BF16, cache->d, a, static_cast<hipStream_t>(stream)), stream,
                  "cats_kv_write");
}

cats_status cats_kv_read(const cats_kv_cache* cache, const int32_t* slots, int32_t N, void* k, void* v, int32_t dtype,
                         void* stream) {
  cats_status st = check_cache(cache);
  if (st != CATS_OK) return st;
  if (!k || !v || !slots) return fail(CATS_ERR_NULL, "k, v or slots is NULL");
  if (!dtype_ok(dtype)) return fail(CATS_ERR_DTYPE, "unknown dtype %d", (int)dtype);
  if (!rows_ok(N)) return fail(CATS_ERR_SHAPE, "N=%d outside [1, %d]", (int)N, CATS_MAX_KV_ROWS);
  if (!aligned(k, 16) || !aligned(v, 16) || !aligned(slots, 4))
    return fail(CATS_ERR_ALIGN, "k and v must be 16-byte aligned, slots 4-byte");
  const size_t n = (size_t)N * cache->heads * cache->d * elem_bytes(dtype);
  const Range r[] = {{k, n, "k"},
                     {v, n, "v"},
                     {cache->data, cache_bytes(cache->pages, cache->page, cache->heads, cache->d), "the cache"},
                     {slots, (size_t)N * 4, "slots"}};
  if ((st = check_overlap(r, 2)) != CATS_OK) return st;
  cats::KvRowsArgs a{};
  a.cache = static_cast<uint8_t*>(cache->data);
  a.slots = slots;
  a.tokens = cache->pages * cache->page;
  a.groups = cache->page / 16;
  a.magic = magic_of(a.groups);
  a.heads = cache->heads;
  a.rows = N;
  a.k_out = k;
  a.v_out = v;
  return launched(cats::launch_kv_rows(false, dtype == CATS_BF16, cache->d, a, static_cast<hipStream_t>(stream)), stream,
                  "cats_kv_read");
}

size_t cats_kv_attention_workspace_bytes(int32_t N, int32_t B, int32_t hq, int32_t hkv, int32_t d) {
  if (!attention_shape_ok(N, B, hq, hkv, d)) return 0;
  return cats::kv_attention_most(N, B, hq, hkv, d);
}

cats_status cats_kv_attention(const void* q, int32_t dtype, int32_t N, int32_t hq, const cats_kv_cache* cache,
                              const int32_t* table, int32_t width, const int32_t* lens, const int32_t* q_start, int32_t B,
                              float scale, int32_t window, void* out, void* ws, size_t ws_bytes, void* stream) {
  cats_status st = check_cache(cache);
  if (st != CATS_OK) return st;
  if (!q || !table || !lens || !out) return fail(CATS_ERR_NULL, "q, table, lens or out is NULL");
  if (!dtype_ok(dtype)) return fail(CATS_ERR_DTYPE, "unknown dtype %d", (int)dtype);
  if (!attention_shape_ok(N, B, hq, cache->heads, cache->d))
    return fail(CATS_ERR_SHAPE, "N=%d, B=%d outside [1, %d], or %d query heads no multiple of %d up to %d", (int)N, (int)B,
                CATS_MAX_KV_ROWS, (int)hq, (int)cache->heads, CATS_MAX_KV_HEADS);
  if (!q_start && N != B) return fail(CATS_ERR_SHAPE, "without q_start N=%d must be B=%d", (int)N, (int)B);
  if (width < 1 || (int64_t)width * cache->page > CATS_MAX_KV_TOKENS)
    return fail(CATS_ERR_SHAPE, "width=%d pages of %d tokens must hold 1 to 2^30", (int)width, (int)cache->page);
  const float c = scale * 1.44269504088896340736f;
  if (!std::isfinite(c) || !(scale > 0.f)) return fail(CATS_ERR_RANGE, "scale must be finite (log2(e) times it too) and > 0");
  if (window < 0) return fail(CATS_ERR_RANGE, "window=%d must be >= 0", (int)window);
  if (!aligned(q, 16) || !aligned(out, 16) || !aligned(table, 4) || !aligned(lens, 4) || !aligned(q_start, 4))
    return fail(CATS_ERR_ALIGN, "q and out must be 16-byte aligned, table, lens and q_start 4-byte");
  const size_t need = cats::kv_attention_bytes(N, B, hq, cache->heads, cache->d, dtype == CATS_BF16, q_start != nullptr);
  if (!ws) return fail(CATS_ERR_WORKSPACE, "workspace is NULL");
  if (!aligned(ws, kWsAlign)) return fail(CATS_ERR_ALIGN, "workspace must be 256-byte aligned");
  if (ws_bytes < need) return fail(CATS_ERR_WORKSPACE, "workspace has %zu bytes, needs %zu", ws_bytes, need);
  const size_t rows = (size_t)N * hq * cache->d * elem_bytes(dtype);
  const Range r[] = {{out, rows, "out"},
                     {ws, need, "the workspace"},
                     {q, rows, "q"},
                     {cache->data, cache_bytes(cache->pages, cache->page, cache->heads, cache->d), "the cache"},
                     {table, (size_t)B * width * 4, "table"},
                     {lens, (size_t)B * 4, "lens"},
                     {q_start, (size_t)(B + 1) * 4, "q_start"}};
  if ((st = check_overlap(r, 2)) != CATS_OK) return st;
  cats::KvAttentionArgs a{};
  a.q = q;
  a.out = out;
  a.cache = static_cast<const uint8_t*>(cache->data);
  a.table = table;
  a.lens = lens;
  a.q_start = q_start;
  a.N = N;
  a.B = B;
  a.hq = hq;
  a.hkv = cache->heads;
  a.pages = cache->pages;
  a.width = width;
  a.groups = cache->page / 16;
  a.magic = magic_of(a.groups);
  a.limit = width * cache->page;
  a.c = c;
  a.window = window < a.limit ? window : 0;  // (one that holds every token is none)
  a.head = static_cast<int*>(ws);
  if (!cats::kv_attention_fits(a, cache->d, dtype == CATS_BF16))
    return fail(CATS_ERR_SHAPE, "%d rows of %d sequences over tables of %d tokens are too many for one call", (int)N, (int)B, a.limit);
  return launched(cats::launch_kv_attention(a, cache->d, dtype == CATS_BF16, static_cast<hipStream_t>(stream)), stream,
                  "cats_kv_attention");
}

}  // extern "C"
