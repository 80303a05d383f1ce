"""The reference of the larger attention tests is the definition's."""
import math

import pytest
import torch

import paper_2404_08763_amd as P

import kv_paths
from kv_util import BF16, F32, attention, gen


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("window", [0, 5])
@pytest.mark.parametrize("counts", [None, [9, 1, 0, 12, 3]])
def test_same_as_the_definition(counts, window, dtype):
    lens, hq, hkv, d = [9, 30, 4, 7, 0], 4, 2, 16
    g = gen(1)
    ks, vs = ([torch.randn((n, hkv, d), generator=g, dtype=torch.float64) for n in lens] for _ in range(2))
    ks[1][27], vs[1][26, 1, 3:5] = math.nan, math.nan
    rows = len(lens) if counts is None else sum(counts)
    q = torch.randn((rows, hq, d), generator=g).to(dtype)
    start = None if counts is None else [sum(counts[:i]) for i in range(len(counts) + 1)]
    want, bound = attention(q, ks, vs, lens, start, window, 0.3)
    got, other = kv_paths.attention(q, ks, vs, lens, start, window, 0.3)
    # (a NaN that a row does not see reaches neither)
    assert torch.allclose(got, want, rtol=1e-12, atol=1e-14, equal_nan=True)
    fine = ~torch.isnan(want)
    assert torch.allclose(other[fine], bound[fine], rtol=1e-9, atol=1e-20)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("hq,hkv", [(1, 1), (32, 8), (40, 1), (1024, 1)])
def test_workspace_as_stated(hq, hkv, d):
    """64 MiB, and 12 bytes for each 16 rows of a key head and 16 for each sequence."""
    f = P.raw().cats_kv_attention_workspace_bytes
    for N, B in ((1, 1), (4096, 1), (4096, 64), (700, 700), (1 << 20, 1), (1 << 20, 1 << 20)):
        assert 0 < f(N, B, hq, hkv, d) <= (64 << 20) + 12 * -(-N * (hq // hkv) // 16) + 16 * B
