"""The rotation's sine and cosine: pairs (1, 0) become (cos a, sin a).

Each is off by the function's own error (4 units in the last place at most, 2^-21 of it), two roundings behind it
(2^-23 of it), and what the angle is off by: the product pos * freq and the one with 1 / pi in 64
bits, and 1 / pi itself, 3 2^-53 of the angle.  Nothing else: a sine near 0 keeps its digits."""
import pytest
import torch

import paper_2404_08763_amd as P

from gpu_util import say
from kv_util import F32, gen

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("inter", [False, True], ids=["halves", "neighbours"])
@pytest.mark.parametrize("far", [1, 50, 4096, 131072, 1 << 20, 1 << 28])
def test_sine_and_cosine(far, inter):
    say("qk angles", far, inter)
    N, d = 3000, 128
    g = gen(far)
    pos = torch.randint(-far, far + 1, (N,), generator=g).to(torch.int32)
    freq = (10000.0 ** -(torch.arange(0, d, 2, dtype=torch.float64) / d)).float()
    freq[:8] = torch.tensor([1.0, 0.5, 3.14159274, 1.57079637, 0.785398185, 1e-3, 2.0 ** -20, 0.0])
    x = torch.zeros(N, 2, d)
    one = slice(0, d, 2) if inter else slice(0, d // 2)
    two = slice(1, d, 2) if inter else slice(d // 2, d)
    x[..., one] = 1.0
    q, k = P.qk_norm_rope(x.view(N, -1).cuda(), 1, 1, d, pos.cuda(), freq.cuda(), interleaved=inter)
    a = pos.double()[:, None] * freq.double()
    for got in (q, k):
        assert got.dtype == F32
        for part, want in ((one, torch.cos(a)), (two, torch.sin(a))):
            err = (got[:, 0, part].cpu().double() - want).abs()
            bound = (2.0 ** -21 + 2.0 ** -23) * want.abs() + 3 * 2.0 ** -53 * a.abs()
            assert (err <= bound).all(), float((err / bound.clamp(min=1e-300)).max())
