"""What the 8-bit operators refuse, on the CPU: nothing reaches the device.

Fake device addresses are passed where validation must fail first."""
import ctypes

import pytest
import torch

import paper_2404_08763_amd as P

OK, NULL, SHAPE, RANGE, DTYPE, ALIGN, WORKSPACE = 0, 1, 2, 3, 4, 5, 6
A = 0x100000  # aligned; the fake arrays below lie a gigabyte apart
G = 1 << 30


def _p(v):
    return ctypes.c_void_p(v) if v else None


def test_ld_and_workspace():
    L = P.raw()
    assert [L.cats_fp8_ld(c) for c in (0, -1, 1, 127, 128, 129, 65536, 65537)] == [0, 0, 128, 128, 128, 256, 65536, 0]
    assert [P.fp8_ld(c) for c in (1, 128, 129, 7001)] == [128, 128, 256, 7040]
    w = L.cats_linear_fp8_workspace_bytes
    assert w(1, 1, 1) > 0 and w(1 << 20, 1 << 20, 65536) > 0
    for bad in ((0, 1, 1), (1, 0, 1), (1, 1, 0), ((1 << 20) + 1, 1, 1), (1, (1 << 20) + 1, 1), (1, 1, 65537)):
        assert w(*bad) == 0


def _quant(x=A, dtype=0, rows=4, cols=256, up=1, stype=0, q=A + G, s=A + 2 * G):
    return P.raw().cats_quantize_fp8(_p(x), dtype, rows, cols, up, stype, _p(q), _p(s), None)


def _norm(x=A, dtype=0, res=None, gain=None, N=4, d=256, eps=1e-5, stype=0, total=None, q=A + G, s=A + 2 * G):
    return P.raw().cats_rmsnorm_fp8(_p(x), dtype, _p(res), _p(gain), N, d, eps, stype, _p(total), _p(q), _p(s), None)


def _gate(x=A, dtype=0, N=4, m=256, t=0.1, stype=0, q=A + G, s=A + 2 * G):
    return P.raw().cats_silu_mul_fp8(_p(x), dtype, N, m, t, stype, _p(q), _p(s), None)


@pytest.mark.parametrize("call,rows,cols", [(_quant, "rows", "cols"), (_norm, "N", "d"), (_gate, "N", "m")])
def test_quantising_calls(call, rows, cols):
    assert call(x=0) == NULL and call(q=0) == NULL and call(s=0) == NULL
    assert call(dtype=2) == DTYPE and call(stype=2) == DTYPE and call(stype=-1) == DTYPE
    for bad in (0, -1):
        assert call(**{rows: bad}) == SHAPE and call(**{cols: bad}) == SHAPE
    assert call(**{rows: (1 << 20) + 1}) == SHAPE and call(**{cols: 65537}) == SHAPE
    assert call(x=A + 2) == ALIGN and call(x=A + 1, dtype=1) == ALIGN
    assert call(q=A + G + 8) == ALIGN and call(s=A + 2 * G + 2) == ALIGN
    assert call(q=A) == RANGE and call(q=A + 4096 - 16) == RANGE  # (4 x 256 fp32 at A)
    assert call(s=A + 16) == RANGE and call(s=A + G) == RANGE
    assert b"overlap" in P.raw().cats_last_error()


def test_quantize_block_rows():
    assert _quant(up=0) == RANGE and _quant(up=64) == RANGE and _quant(up=-128) == RANGE


def test_rmsnorm_arguments():
    for eps in (-1.0, float("nan"), float("inf")):
        assert _norm(eps=eps) == RANGE
    far = A + 3 * G
    for name in ("res", "gain", "total"):
        assert _norm(**{name: far + 2}) == ALIGN
        assert _norm(**{name: A + G}) == RANGE and _norm(**{name: A + 2 * G}) == RANGE
    assert _norm(total=A + 64) == RANGE                  # part of x
    assert _norm(total=A, dtype=1) == RANGE              # bf16 x cannot be the sum
    assert _norm(res=far, total=far + 64) == RANGE       # part of the residual
    assert _norm(gain=far, total=far) == RANGE


def test_gate_arguments():
    assert _gate(t=-0.1) == RANGE and _gate(t=float("nan")) == RANGE
    assert _gate(q=A + 4 * 512 * 4 - 16) == RANGE  # (the up half counts)


def _linear(xq=A, xs=A + G, N=4, wq=A + 2 * G, ws=A + 3 * G, n=256, k=256, stype=0, res=None, y=A + 4 * G, ydtype=0,
            scratch=A + 5 * G, nbytes=None):
    if nbytes is None:
        nbytes = P.raw().cats_linear_fp8_workspace_bytes(N, n, k)
    return P.raw().cats_linear_fp8(_p(xq), _p(xs), N, _p(wq), _p(ws), n, k, stype, _p(res), _p(y), ydtype,
                                   _p(scratch), nbytes, None)


def test_linear_arguments():
    for name in ("xq", "xs", "wq", "ws", "y"):
        assert _linear(**{name: 0}) == NULL
    assert _linear(stype=2) == DTYPE and _linear(ydtype=2) == DTYPE
    for name in ("N", "n", "k"):
        assert _linear(**{name: 0}, nbytes=1 << 20) == SHAPE and _linear(**{name: -3}, nbytes=1 << 20) == SHAPE
    assert _linear(k=65537, nbytes=1 << 20) == SHAPE and _linear(n=(1 << 20) + 1, nbytes=1 << 20) == SHAPE
    assert _linear(xq=A + 8) == ALIGN and _linear(wq=A + 2 * G + 8) == ALIGN
    assert _linear(xs=A + G + 2) == ALIGN and _linear(ws=A + 3 * G + 1) == ALIGN
    assert _linear(y=A + 4 * G + 8) == ALIGN and _linear(res=A + 6 * G + 4) == ALIGN
    assert _linear(y=A) == RANGE and _linear(y=A + G) == RANGE and _linear(y=A + 2 * G + 4096) == RANGE
    assert _linear(y=A + 3 * G) == RANGE and _linear(res=A + 4 * G + 16) == RANGE
    assert _linear(scratch=0) == WORKSPACE and _linear(scratch=A + 5 * G + 64) == ALIGN
    for scratch in (A, A + G, A + 2 * G + 512, A + 3 * G, A + 4 * G + 256):  # an operand's
        assert _linear(scratch=scratch) == RANGE
    assert _linear(res=A + 5 * G) == RANGE
    for N in (1, 60, 400):
        assert _linear(N=N, nbytes=P.raw().cats_linear_fp8_workspace_bytes(N, 256, 256) - 1) == WORKSPACE


# ---- the binding: wrong tensors raise before the library is called -----------------

def _t(*shape, dtype=torch.float32):
    return torch.zeros(shape, dtype=dtype)


def test_binding_quantising_calls():
    for call in (P.quantize_fp8, P.rmsnorm_fp8, P.silu_mul_fp8):
        with pytest.raises(ValueError, match="two dimensions"):
            call(_t(4))
        with pytest.raises(ValueError, match="float32 or torch.bfloat16"):
            call(_t(4, 4, dtype=torch.float16))
        with pytest.raises(ValueError, match="scales are"):
            call(_t(4, 4), scale_dtype=torch.float16)
        with pytest.raises(ValueError, match="device tensor"):
            call(_t(4, 4))
    with pytest.raises(ValueError, match="block_rows"):
        P.quantize_fp8(_t(4, 4), block_rows=2)
    with pytest.raises(ValueError, match=r"\[N, 2 m\]"):
        P.silu_mul_fp8(_t(4, 5))
    q = _t(4, 128, dtype=torch.float8_e4m3fn)
    with pytest.raises(ValueError, match=r"q must be \[4, 256\]"):
        P.quantize_fp8(_t(4, 130), out=(q, _t(4, 2)))
    with pytest.raises(ValueError, match=r"scale must be \[4, 1\]"):
        P.quantize_fp8(_t(4, 100), out=(q, _t(4, 2)))
    with pytest.raises(ValueError, match=r"scale must be \[1, 1\]"):
        P.quantize_fp8(_t(4, 100), block_rows=128, out=(q, _t(4, 1)))
    with pytest.raises(ValueError, match="scales are"):
        P.quantize_fp8(_t(4, 100), out=(q, _t(4, 1, dtype=torch.uint8)))


def test_binding_linear():
    f8 = torch.float8_e4m3fn

    def call(xq=(4, 256), xs=(4, 2), wq=(300, 256), ws=(3, 2), **kw):
        return P.linear_fp8(_t(*xq, dtype=f8), _t(*xs), _t(*wq, dtype=f8), _t(*ws), **kw)

    with pytest.raises(ValueError, match="two dimensions"):
        call(xq=(256,))
    with pytest.raises(ValueError, match="same width"):
        call(wq=(300, 128))
    with pytest.raises(ValueError, match="multiple of 128"):
        call(xq=(4, 200), wq=(300, 200))
    with pytest.raises(ValueError, match=r"xs must be \[4, 2\]"):
        call(xs=(4, 1))
    with pytest.raises(ValueError, match=r"wscale must be \[3, 2\]"):
        call(ws=(2, 2))
    with pytest.raises(ValueError, match=r"out must be \[4, 300\]"):
        call(out=_t(4, 299))
    with pytest.raises(ValueError, match=r"residual must be \[4, 300\]"):
        call(residual=_t(4, 299))
    with pytest.raises(ValueError, match="unsupported weight dtype"):
        call(dtype=torch.float16)
    with pytest.raises(ValueError, match="device tensor"):
        call()
