"""The linear layer's workspace: one sized for the largest call serves every smaller one."""
import ctypes
import random

import pytest
import torch

import paper_2404_08763_amd as P

RANGE, WORKSPACE = 3, 6
A, G = 0x100000, 1 << 36  # fake device addresses, far apart


def _p(v):
    return ctypes.c_void_p(v)


def _refused(N, n, k, nbytes, stype, ydtype):
    """The status of a call whose workspace lies on xq: RANGE if its size is enough,
    which is looked at first.  Nothing reaches the device."""
    return P.raw().cats_linear_fp8(_p(A), _p(A + G), N, _p(A + 2 * G), _p(A + 3 * G), n, k, stype, None,
                                   _p(A + 4 * G), ydtype, _p(A), nbytes, None)


def _size(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def test_size_grows_with_each_argument():
    w = P.raw().cats_linear_fp8_workspace_bytes
    rng = random.Random(1)
    for _ in range(20000):
        big = _size(rng, 1, 1 << 14), _size(rng, 1, 1 << 16), _size(rng, 1, 65536)
        small = tuple(_size(rng, 1, v) for v in big)
        assert w(*small) <= w(*big) <= 48 << 20, (small, big)
    for big, small in (((4096, 4096, 4096), (256, 4096, 4096)), ((300, 6144, 4096), (256, 6144, 4096))):
        assert w(*small) <= w(*big)


@pytest.mark.parametrize("stype", [0, 1], ids=["f32", "e8m0"])
@pytest.mark.parametrize("ydtype", [0, 1], ids=["y32", "y16"])
def test_a_larger_calls_workspace_is_enough(stype, ydtype):
    w = P.raw().cats_linear_fp8_workspace_bytes
    rng = random.Random(2)
    for _ in range(20000):
        big = _size(rng, 1, 1 << 14), _size(rng, 1, 1 << 16), _size(rng, 1, 65536)
        small = tuple(_size(rng, 1, v) for v in big)
        assert _refused(*small, w(*big), stype, ydtype) == RANGE, (small, big)
        assert _refused(*small, 255, stype, ydtype) == WORKSPACE


@pytest.mark.gpu
@pytest.mark.parametrize("stype", [torch.float32, torch.float8_e8m0fnu], ids=["f32", "e8m0"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["y32", "y16"])
def test_one_workspace_for_all_calls(dtype, stype):
    """The largest call's, its end guarded, gives each smaller call what its own gives it."""
    from gpu_util import say

    size = P.linear_fp8_workspace(600, 2048, 8320).numel()
    whole = torch.full((size + 4096,), 0x5a, dtype=torch.uint8, device="cuda")
    for k in (600, 8320):
        w = P.quantize_fp8(0.02 * torch.randn((2048, k), device="cuda"), 128, stype)
        x = P.quantize_fp8(torch.randn((600, k), device="cuda"), 1, stype)
        for n in (300, 2048):
            for N in (1, 20, 37, 64, 100, 300, 600):
                say("one workspace", N, n, k, dtype, stype)
                ops = x[0][:N], x[1][:N], w[0][:n], w[1][:(n + 127) // 128]
                y = P.linear_fp8(*ops, dtype=dtype, ws=whole[:size])
                assert torch.equal(y, P.linear_fp8(*ops, dtype=dtype))
    assert (whole[size:] == 0x5a).all()
