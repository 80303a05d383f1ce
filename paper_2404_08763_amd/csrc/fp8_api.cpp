// C ABI of the 8-bit operators: argument checks on the host, then the launch.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdio>

#include "cats.h"
#include "fp8.hpp"
#include "internal.hpp"

namespace {

template <typename... A> cats_status fail(cats_status st, const char* fmt, A... a) {
  char buf[256];
  snprintf(buf, sizeof(buf), fmt, a...);
  return cats::report_error(st, buf);
}
cats_status fail(cats_status st, const char* msg) { return cats::report_error(st, msg); }

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

// Whether the two ranges share a byte.
bool overlap(const void* a, size_t na, const void* b, size_t nb) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y + nb && y < x + na;
}

size_t elem_bytes(int32_t dtype) { return dtype == CATS_BF16 ? 2 : 4; }
size_t scale_bytes(int32_t stype) { return stype == CATS_SCALE_E8M0 ? 1 : 4; }
size_t blocks_of(int32_t v) { return ((size_t)v + CATS_FP8_BLOCK - 1) / CATS_FP8_BLOCK; }

cats_status check_dtype(int32_t dtype) {
  if (dtype != CATS_F32 && dtype != CATS_BF16) return fail(CATS_ERR_DTYPE, "unknown dtype %d", (int)dtype);
  return CATS_OK;
}

// The common part of the calls that write 8-bit rows: sizes, types, the
// output and that it does not overlap the input.
cats_status check_quant(const void* x, size_t x_row, int32_t dtype, int32_t rows, int32_t cols, int32_t stype,
                        const void* q, const void* scale, int32_t block_rows) {
  if (!x || !q || !scale) return fail(CATS_ERR_NULL, "the input, q or scale is NULL");
  const cats_status st = check_dtype(dtype);
  if (st != CATS_OK) return st;
  if (stype != CATS_SCALE_F32 && stype != CATS_SCALE_E8M0)
    return fail(CATS_ERR_DTYPE, "unknown scale type %d", (int)stype);
  if (rows < 1 || rows > CATS_MAX_FP8_ROWS || cols < 1 || cols > CATS_MAX_FP8_COLS)
    return fail(CATS_ERR_SHAPE, "%d x %d outside [1, %d] x [1, %d]", (int)rows, (int)cols, CATS_MAX_FP8_ROWS, CATS_MAX_FP8_COLS);
  if (!aligned(x, elem_bytes(dtype))) return fail(CATS_ERR_ALIGN, "the input must be aligned to its elements");
  if (!aligned(q, 16) || !aligned(scale, scale_bytes(stype)))
    return fail(CATS_ERR_ALIGN, "q must be 16-byte aligned and scale to its elements");
  const size_t nx = (size_t)rows * x_row * elem_bytes(dtype), nq = (size_t)rows * blocks_of(cols) * CATS_FP8_BLOCK;
  const size_t ns = ((size_t)rows + block_rows - 1) / block_rows * blocks_of(cols) * scale_bytes(stype);
  if (overlap(x, nx, q, nq) || overlap(x, nx, scale, ns) || overlap(q, nq, scale, ns))
    return fail(CATS_ERR_RANGE, "the input, q and scale must not overlap");
  return CATS_OK;
}

cats::Fp8Out fp8_out(void* q, void* scale, int32_t cols, int32_t stype) {
  return cats::Fp8Out{static_cast<uint8_t*>(q), scale, cats::fp8_ld(cols), stype == CATS_SCALE_E8M0 ? 1 : 0};
}

cats_status launched(hipError_t e, void* stream, const char* what) {
  if (e != hipSuccess) return fail(CATS_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
  return cats::enqueued(stream, what);
}

constexpr size_t kWsAlign = 256;
size_t ws_size(size_t bytes) { return bytes < kWsAlign ? kWsAlign : (bytes + kWsAlign - 1) / kWsAlign * kWsAlign; }

bool linear_shape_ok(int32_t N, int32_t n, int32_t k) {
  return N >= 1 && N <= CATS_MAX_FP8_ROWS && n >= 1 && n <= CATS_MAX_FP8_ROWS && k >= 1 && k <= CATS_MAX_FP8_COLS;
}

}  // namespace

static_assert(CATS_FP8_BLOCK == cats::kFp8Block, "the header's block is the kernels'");

extern "C" {

int32_t cats_fp8_ld(int32_t cols) {
  return cols < 1 || cols > CATS_MAX_FP8_COLS ? 0 : cats::fp8_ld(cols);
}

cats_status cats_quantize_fp8(const void* x, int32_t dtype, int32_t rows, int32_t cols, int32_t block_rows,
                              int32_t stype, void* q, void* scale, void* stream) {
  if (block_rows != 1 && block_rows != CATS_FP8_BLOCK)
    return fail(CATS_ERR_RANGE, "block_rows=%d must be 1 or %d", (int)block_rows, CATS_FP8_BLOCK);
  const cats_status st = check_quant(x, cols, dtype, rows, cols, stype, q, scale, block_rows);
  if (st != CATS_OK) return st;
  return launched(cats::launch_quantize_fp8(x, dtype == CATS_BF16, rows, cols, block_rows, fp8_out(q, scale, cols, stype),
                                            static_cast<hipStream_t>(stream)),
                  stream, "cats_quantize_fp8");
}

cats_status cats_rmsnorm_fp8(const void* x, int32_t dtype, const float* residual, const float* gain, int32_t N,
                             int32_t d, float eps, int32_t stype, float* sum_out, void* q, void* scale, void* stream) {
  const cats_status st = check_quant(x, d, dtype, N, d, stype, q, scale, 1);
  if (st != CATS_OK) return st;
  if (!std::isfinite(eps) || eps < 0.f) return fail(CATS_ERR_RANGE, "eps must be finite and >= 0");
  if (!aligned(residual, 4) || !aligned(gain, 4) || !aligned(sum_out, 4))
    return fail(CATS_ERR_ALIGN, "residual, gain and sum_out must be 4-byte aligned");
  const size_t row4 = (size_t)N * d * 4, nx = (size_t)N * d * elem_bytes(dtype);
  const size_t nq = (size_t)N * blocks_of(d) * CATS_FP8_BLOCK, ns = (size_t)N * blocks_of(d) * scale_bytes(stype);
  if (residual && (overlap(residual, row4, q, nq) || overlap(residual, row4, scale, ns)))
    return fail(CATS_ERR_RANGE, "residual overlaps q or scale");
  if (gain && (overlap(gain, (size_t)d * 4, q, nq) || overlap(gain, (size_t)d * 4, scale, ns)))
    return fail(CATS_ERR_RANGE, "gain overlaps q or scale");
  if (sum_out) {
    if (overlap(sum_out, row4, q, nq) || overlap(sum_out, row4, scale, ns) ||
        (gain && overlap(sum_out, row4, gain, (size_t)d * 4)))
      return fail(CATS_ERR_RANGE, "sum_out overlaps gain, q or scale");
    const bool is_x = dtype == CATS_F32 && sum_out == x;
    if ((!is_x && overlap(sum_out, row4, x, nx)) || (residual && sum_out != residual && overlap(sum_out, row4, residual, row4)))
      return fail(CATS_ERR_RANGE, "sum_out may be x (fp32) or the residual, but not part of either");
  }
  cats::RmsnormFp8Args a;
  a.x = x;
  a.residual = residual;
  a.gain = gain;
  a.sum = sum_out;
  a.N = N;
  a.d = d;
  a.eps = eps;
  a.o = fp8_out(q, scale, d, stype);
  return launched(cats::launch_rmsnorm_fp8(a, dtype == CATS_BF16, static_cast<hipStream_t>(stream)), stream,
                  "cats_rmsnorm_fp8");
}

cats_status cats_silu_mul_fp8(const void* gate_up, int32_t dtype, int32_t N, int32_t m, float t, int32_t stype, void* q,
                              void* scale, void* stream) {
  const cats_status st = check_quant(gate_up, (size_t)2 * (m > 0 ? m : 0), dtype, N, m, stype, q, scale, 1);
  if (st != CATS_OK) return st;
  if (std::isnan(t) || t < 0.f) return fail(CATS_ERR_RANGE, "t must be >= 0 (got %g)", (double)t);
  return launched(cats::launch_silu_fp8(gate_up, dtype == CATS_BF16, N, m, t, fp8_out(q, scale, m, stype),
                                        static_cast<hipStream_t>(stream)),
                  stream, "cats_silu_mul_fp8");
}

size_t cats_linear_fp8_workspace_bytes(int32_t N, int32_t n, int32_t k) {
  if (!linear_shape_ok(N, n, k)) return 0;
  return ws_size(cats::linear_fp8_partial_most(N, n, (int)blocks_of(k)));
}

cats_status cats_linear_fp8(const void* xq, const void* xs, int32_t N, const void* wq, const void* wscale, int32_t n,
                            int32_t k, int32_t stype, const void* residual, void* y, int32_t ydtype, void* ws,
                            size_t ws_bytes, void* stream) {
  if (!xq || !xs || !wq || !wscale || !y) return fail(CATS_ERR_NULL, "xq, xs, wq, wscale or y is NULL");
  cats_status st = check_dtype(ydtype);
  if (st != CATS_OK) return st;
  if (stype != CATS_SCALE_F32 && stype != CATS_SCALE_E8M0)
    return fail(CATS_ERR_DTYPE, "unknown scale type %d", (int)stype);
  if (!linear_shape_ok(N, n, k))
    return fail(CATS_ERR_SHAPE, "N=%d, n=%d, k=%d outside [1, %d], [1, %d], [1, %d]", (int)N, (int)n, (int)k,
                CATS_MAX_FP8_ROWS, CATS_MAX_FP8_ROWS, CATS_MAX_FP8_COLS);
  if (!aligned(xq, 16) || !aligned(wq, 16)) return fail(CATS_ERR_ALIGN, "xq and wq must be 16-byte aligned");
  if (!aligned(xs, scale_bytes(stype)) || !aligned(wscale, scale_bytes(stype)))
    return fail(CATS_ERR_ALIGN, "the scales must be aligned to their elements");
  if (!aligned(y, 16) || !aligned(residual, 16)) return fail(CATS_ERR_ALIGN, "y and residual must be 16-byte aligned");
  const size_t ld = blocks_of(k) * CATS_FP8_BLOCK, ny = (size_t)N * n * elem_bytes(ydtype);
  if (overlap(y, ny, xq, (size_t)N * ld) || overlap(y, ny, wq, (size_t)n * ld) ||
      overlap(y, ny, xs, (size_t)N * blocks_of(k) * scale_bytes(stype)) ||
      overlap(y, ny, wscale, blocks_of(n) * blocks_of(k) * scale_bytes(stype)) ||
      (residual && residual != y && overlap(y, ny, residual, ny)))
    return fail(CATS_ERR_RANGE, "y may be the residual, but must not overlap any other input");
  const size_t need = ws_size(cats::linear_fp8_partial_bytes(N, n, (int)blocks_of(k), ydtype == CATS_BF16, stype == CATS_SCALE_E8M0));
  if (!ws) return fail(CATS_ERR_WORKSPACE, "workspace is NULL");
  if (!aligned(ws, kWsAlign)) return fail(CATS_ERR_ALIGN, "workspace must be 256-byte aligned");
  if (ws_bytes < need) return fail(CATS_ERR_WORKSPACE, "workspace has %zu bytes, needs %zu", ws_bytes, need);
  if (overlap(ws, need, xq, (size_t)N * ld) || overlap(ws, need, wq, (size_t)n * ld) || overlap(ws, need, y, ny) ||
      overlap(ws, need, xs, (size_t)N * blocks_of(k) * scale_bytes(stype)) ||
      overlap(ws, need, wscale, blocks_of(n) * blocks_of(k) * scale_bytes(stype)) ||
      (residual && overlap(ws, need, residual, ny)))
    return fail(CATS_ERR_RANGE, "the workspace must not overlap any operand");
  cats::LinearFp8Args a{};
  a.xq = static_cast<const uint8_t*>(xq);
  a.xs = xs;
  a.wq = static_cast<const uint8_t*>(wq);
  a.ws = wscale;
  a.residual = residual;
  a.y = y;
  a.N = N;
  a.n = n;
  a.ld = (int)ld;
  a.e8m0 = stype == CATS_SCALE_E8M0;
  a.ybf16 = ydtype == CATS_BF16;
  a.partial = static_cast<float*>(ws);
  return launched(cats::launch_linear_fp8(a, static_cast<hipStream_t>(stream)), stream, "cats_linear_fp8");
}

}  // extern "C"
