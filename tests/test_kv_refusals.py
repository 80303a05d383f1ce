"""What the operators around attention refuse, on the CPU: nothing reaches the device.

Fake device addresses are passed where validation must fail first."""
import ctypes

import pytest
import torch

import paper_2404_08763_amd as P
from paper_2404_08763_amd import _lib

OK, NULL, SHAPE, RANGE, DTYPE, ALIGN, WORKSPACE = 0, 1, 2, 3, 4, 5, 6
A = 0x100000  # aligned; the fake arrays below lie far apart
G = 1 << 36


def _p(v):
    return ctypes.c_void_p(v) if v else None


def _cache(data=A, pages=10, page=64, heads=8, d=128):
    return _lib._KvCache(data, pages, page, heads, d)


# ---- norms and rotation ----------------------------------------------------------

def _rope(x=A, dtype=0, ld=4096, N=4, hq=16, hkv=4, d=128, norm=0, gq=None, gk=None, eps=1e-5, pos=A + G,
          freq=A + 2 * G, rot=128, inter=0, q=A + 3 * G, k=A + 4 * G, odtype=0):
    return P.raw().cats_qk_norm_rope(_p(x), dtype, ld, N, hq, hkv, d, norm, _p(gq), _p(gk), eps, _p(pos), _p(freq), rot,
                                     inter, _p(q), _p(k), odtype, None)


def test_norm_rope_arguments():
    assert _rope(x=0) == NULL and _rope(q=0) == NULL and _rope(k=0) == NULL
    assert _rope(pos=0) == NULL and _rope(freq=0) == NULL
    assert _rope(dtype=2) == DTYPE and _rope(odtype=-1) == DTYPE
    for bad in (dict(N=0), dict(N=(1 << 20) + 1), dict(hq=0), dict(hkv=0), dict(hq=1025), dict(d=0), dict(d=12), dict(d=520),
                dict(rot=-8), dict(rot=12), dict(rot=136), dict(ld=20 * 128 - 8), dict(ld=20 * 128 + 4), dict(ld=(1 << 30) + 8)):
        assert _rope(**bad) == SHAPE, bad
    for eps in (-1.0, float("nan"), float("inf")):
        assert _rope(norm=1, eps=eps) == RANGE
    for name, at in (("x", A), ("freq", A + 2 * G), ("q", A + 3 * G), ("k", A + 4 * G)):
        assert _rope(**{name: at + 8}) == ALIGN, name
    assert _rope(norm=1, gq=A + 5 * G + 4) == ALIGN and _rope(norm=1, gk=A + 5 * G + 4) == ALIGN
    assert _rope(pos=A + G + 2) == ALIGN


def test_norm_rope_overlaps():
    row = 4 * 16 * 128 * 4
    assert _rope(q=A) == RANGE and _rope(k=A + 4 * 4096 * 4 - 4096 * 4) == RANGE  # rows of qkv
    assert _rope(k=A + 3 * G + row - 16) == RANGE                                 # q and k
    assert b"q must not overlap k" in P.raw().cats_last_error()
    assert _rope(pos=A + 4 * G) == RANGE and _rope(freq=A + 3 * G) == RANGE
    assert _rope(norm=1, gq=A + 3 * G + 16) == RANGE and _rope(norm=1, gk=A + 4 * G) == RANGE


# ---- the cache --------------------------------------------------------------------

def test_cache_bytes():
    f = P.raw().cats_kv_cache_bytes
    assert f(1, 16, 1, 64) == 17 * 64 and f(10, 64, 8, 128) == 10 * 8 * 64 * 136
    assert f(1 << 22, 256, 8, 128) == (1 << 30) * 8 * 136
    for bad in ((0, 16, 1, 64), (1, 0, 1, 64), (1, 24, 1, 64), (1, 272, 1, 64), (1, 16, 0, 64), (1, 16, 1025, 64),
                (1, 16, 1, 32), (1, 16, 1, 96), ((1 << 22) + 1, 256, 1, 64), (-1, 16, 1, 64)):
        assert f(*bad) == 0, bad


BAD_CACHES = [(dict(data=0), NULL), (dict(data=A + 8), ALIGN), (dict(pages=0), SHAPE), (dict(page=8), SHAPE),
              (dict(page=40), SHAPE), (dict(page=512), SHAPE), (dict(heads=0), SHAPE), (dict(d=80), SHAPE),
              (dict(pages=1 << 29), SHAPE)]


def _write(c=None, k=A + G, ldk=1024, v=A + 2 * G, ldv=1024, dtype=0, slots=A + 3 * G, N=4):
    c = _cache() if c is None else c
    return P.raw().cats_kv_write(ctypes.byref(c), _p(k), ldk, _p(v), ldv, dtype, _p(slots), N, None)


def _read(c=None, slots=A + 3 * G, N=4, k=A + G, v=A + 2 * G, dtype=0):
    c = _cache() if c is None else c
    return P.raw().cats_kv_read(ctypes.byref(c), _p(slots), N, _p(k), _p(v), dtype, None)


@pytest.mark.parametrize("call", [_write, _read])
def test_rows_arguments(call):
    for kw, want in BAD_CACHES:
        assert call(_cache(**kw)) == want, kw
    assert call(k=0) == NULL and call(v=0) == NULL and call(slots=0) == NULL
    assert call(dtype=2) == DTYPE and call(N=0) == SHAPE and call(N=(1 << 20) + 1) == SHAPE
    assert call(k=A + G + 8) == ALIGN and call(v=A + 2 * G + 4) == ALIGN and call(slots=A + 3 * G + 2) == ALIGN
    assert call(k=A + 4096) == RANGE and call(v=A) == RANGE  # on the cache


def test_write_pitches_and_overlaps():
    assert _write(ldk=1016) == SHAPE and _write(ldv=1028) == SHAPE and _write(ldv=(1 << 30) + 8) == SHAPE
    assert _write(slots=A + 16) == RANGE
    L = P.raw()
    assert L.cats_kv_write(None, _p(A), 8, _p(A), 8, 0, _p(A), 1, None) == NULL


def test_read_overlaps():
    assert _read(v=A + G + 4 * 4096 - 16) == RANGE and _read(slots=A + G + 16) == RANGE and _read(slots=A + 2 * G) == RANGE


# ---- attention ----------------------------------------------------------------------

def _attn(q=A + G, dtype=1, N=4, hq=32, c=None, table=A + 2 * G, width=100, lens=A + 3 * G, start=None, B=4, scale=0.1,
          window=0, out=A + 4 * G, ws=A + 5 * G, nbytes=None):
    c = _cache() if c is None else c
    if nbytes is None:
        nbytes = 1 << 30
    return P.raw().cats_kv_attention(_p(q), dtype, N, hq, ctypes.byref(c), _p(table), width, _p(lens), _p(start), B, scale,
                                     window, _p(out), _p(ws), nbytes, None)


def test_attention_arguments():
    for kw, want in BAD_CACHES:
        assert _attn(c=_cache(**kw)) == want, kw
    for name in ("q", "table", "lens", "out"):
        assert _attn(**{name: 0}) == NULL, name
    assert _attn(dtype=2) == DTYPE
    for bad in (dict(N=0), dict(B=0), dict(N=5), dict(B=(1 << 20) + 1, N=(1 << 20) + 1), dict(hq=0), dict(hq=12),
                dict(hq=1032), dict(width=0), dict(width=(1 << 24) + 1)):
        assert _attn(**bad) == SHAPE, bad
    assert _attn(N=5, start=A + 6 * G, ws=0) == WORKSPACE  # (any N with q_start)
    for scale in (0.0, -1.0, float("nan"), float("inf"), 3e38):
        assert _attn(scale=scale) == RANGE
    assert _attn(window=-1) == RANGE
    for name, at in (("q", A + G), ("out", A + 4 * G)):
        assert _attn(**{name: at + 8}) == ALIGN, name
    for name, at in (("table", A + 2 * G), ("lens", A + 3 * G), ("start", A + 6 * G)):
        assert _attn(**{name: at + 2}) == ALIGN, name


def test_attention_workspace_and_overlaps():
    need = P.raw().cats_kv_attention_workspace_bytes(4, 4, 32, 8, 128)
    assert _attn(ws=0) == WORKSPACE and _attn(nbytes=1000) == WORKSPACE and _attn(ws=A + 5 * G + 16) == ALIGN
    assert need <= 64 << 20
    for at in (A, A + G, A + 2 * G, A + 3 * G):
        assert _attn(out=at) == RANGE, at
        assert _attn(ws=at, nbytes=need) == RANGE, at
    assert _attn(ws=A + 4 * G + 0x100, nbytes=need) == RANGE
    assert _attn(start=A + 6 * G, ws=A + 6 * G) == RANGE and _attn(start=A + 4 * G) == RANGE


def test_attention_work_beyond_32_bits():
    """512 tiles of 128 rows, of 2^24 units of 64 tokens each: 2^33."""
    kw = dict(N=1 << 16, B=1, hq=8, start=A + 6 * G, nbytes=1 << 35)
    assert _attn(width=1 << 24, **kw) == SHAPE
    assert b"too many for one call" in P.raw().cats_last_error()


@pytest.mark.parametrize("planned", [False, True])
@pytest.mark.parametrize("dtype", [0, 1])
def test_workspace_serves_smaller_calls(planned, dtype):
    """The largest call's workspace is enough for every call of fewer rows and sequences: its
    size is looked at before the overlap that refuses the call."""
    f = P.raw().cats_kv_attention_workspace_bytes
    for hq, hkv in ((8, 8), (32, 8), (40, 1)):
        for d in (64, 128, 256):
            most = f(4096, 64, hq, hkv, d)
            for N, B in ((1, 1), (2, 2), (64, 64), (4096, 64), (4096, 1), (100, 64), (17, 1)):
                if not planned and N != B:
                    continue
                assert f(N, B, hq, hkv, d) <= most
                start = A + 6 * G if planned else None
                assert _attn(c=_cache(heads=hkv, d=d), dtype=dtype, hq=hq, N=N, B=B, start=start, ws=A + G, nbytes=most) == RANGE
    for bad in ((0, 1, 8, 8, 64), (1, 0, 8, 8, 64), (1, 1, 9, 8, 64), (1, 1, 8, 8, 96), ((1 << 20) + 1, 1, 8, 8, 64)):
        assert f(*bad) == 0


# ---- the binding, on host tensors ---------------------------------------------------------

def _host(*shape, dtype=torch.float32):
    return torch.zeros(shape, dtype=dtype)


def _raises(match, fn, *a, **k):
    with pytest.raises(ValueError, match=match):
        fn(*a, **k)


def test_binding(monkeypatch):
    monkeypatch.setattr(_lib, "_device", lambda: 0)
    i32 = lambda *s: _host(*s, dtype=torch.int32)  # noqa: E731
    _raises("two dimensions", P.qk_norm_rope, _host(2, 3, 4), 2, 1, 64)
    _raises("192 columns or more", P.qk_norm_rope, _host(2, 128), 2, 1, 64)
    _raises("device tensor", P.qk_norm_rope, _host(2, 192), 2, 1, 64)
    cache = _host(3, 2, 4, 17 * 64, dtype=torch.uint8)
    _raises("17 d", P.kv_write, cache[0], _host(1, 2, 64), _host(1, 2, 64), i32(1))
    _raises("17 d", P.kv_read, cache[..., :-1], i32(1))
    for call in (lambda c: P.kv_write(c, _host(1, 2, 64), _host(1, 2, 64), i32(1)), lambda c: P.kv_read(c, i32(1)),
                 lambda c: P.kv_attention(_host(1, 2, 64), c, i32(1, 1), i32(1))):
        _raises("cache must be", call, cache)  # (on the host)
    # what is looked at behind the cache, with a stand-in for its check
    monkeypatch.setattr(_lib, "_kv", lambda c, dev: (None, 2, 64))
    monkeypatch.setattr(_lib, "_slots_of", lambda s, dev: s.shape[0])
    _raises("k must be", P.kv_write, cache, _host(1, 3, 64), _host(1, 2, 64), i32(1))
    _raises("v must be", P.kv_write, cache, _host(1, 2, 64), _host(2, 2, 64), i32(1))
    _raises("one type", P.kv_write, cache, _host(1, 2, 64), _host(1, 2, 64, dtype=torch.bfloat16), i32(1))
    _raises("k must be", P.kv_read, cache, i32(1), out=(_host(1, 64), _host(1, 2, 64)))
    _raises(r"\[N, heads, d\]", P.kv_attention, _host(2, 64), cache, i32(1, 1), i32(1))
    _raises("the cache's 64", P.kv_attention, _host(1, 2, 128), cache, i32(1, 1), i32(1))
    _raises("table must have two", P.kv_attention, _host(1, 2, 64), cache, i32(1), i32(1))
    _raises("lens must be", P.kv_attention, _host(1, 2, 64), cache, i32(1, 1), i32(2))
    _raises("q_start must be", P.kv_attention, _host(1, 2, 64), cache, i32(1, 1), i32(1), q_start=i32(1))
    _raises("a row for each", P.kv_attention, _host(2, 2, 64), cache, i32(1, 1), i32(1))
    _raises("device tensor", P.kv_attention, _host(1, 2, 64), cache, i32(1, 1), i32(1))
    for bad in ((0, 2, 64, 16), (1, 2, 96, 16), (1, 2, 64, 24)):
        _raises("supported range", P.kv_cache, *bad[:3], page=bad[3], device="cpu")
    _raises("supported range", P.kv_attention_workspace, 1, 1, 3, 2, 64)
