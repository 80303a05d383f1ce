"""Norms of heads whose squares leave fp32 below, with an eps that does not cover them: the
definition's all the same, within the bound of test_gpu_qk_rope."""
import pytest
import torch

import paper_2404_08763_amd as P

from gpu_util import say
from kv_util import BF16, F32, HALF, gen, norm_rope

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("eps", [0.0, 1e-44, 1e-38, 1e-33, 1e-5])
@pytest.mark.parametrize("d,rot", [(64, 0), (128, 128), (80, 40), (512, 512)])
def test_small_heads(d, rot, eps, dtype):
    say("qk small heads", d, rot, eps, dtype)
    powers = [0, -20, -48, -52, -60, -66, -72, -75, -90, -110, -120]
    g = gen(d)
    N = len(powers)
    x = (torch.randn((N, 3, d), generator=g) * 2.0 ** torch.tensor(powers)[:, None, None]).to(dtype)
    x[:, 2] *= 2.0 ** -4  # (neighbours of other sizes)
    pos = torch.arange(N, dtype=torch.int32)
    freq = (10000.0 ** -(torch.arange(0, rot, 2, dtype=torch.float64) / max(rot, 1))).float() if rot else None
    gain = 1 + 0.2 * torch.randn(d, generator=g)
    eps32 = float(torch.tensor(eps, dtype=F32))
    q, k = P.qk_norm_rope(x.view(N, -1).cuda(), 2, 1, d, pos.cuda(), None if freq is None else freq.cuda(), norm=True,
                          gain_q=gain.cuda(), eps=eps, dtype=F32)
    for got, part, gn in ((q, x[:, :2], gain), (k, x[:, 2:], None)):
        want, mag = norm_rope(part, pos, freq, True, gn, eps32, False)
        err = (got.cpu().double() - want).abs()
        assert (err <= 24 * 2.0 ** -24 * mag + want.abs() * HALF[F32] * 1.001 + 1e-37).all(), float((err / (mag + 1e-300)).max())


def test_zeros():
    """0 / 0 with eps 0, else 0; beside other heads."""
    say("qk zero heads")
    x = torch.randn((2, 3, 64), generator=gen(3))
    x[0, 1] = 0.0
    for eps in (0.0, 1e-44, 1e-5):
        q, k = P.qk_norm_rope(x.view(2, -1).cuda(), 2, 1, 64, norm=True, eps=eps)
        assert torch.isnan(q[0, 1]).all() if eps == 0 else (q[0, 1] == 0).all()
        assert torch.isfinite(q[0, 0]).all() and torch.isfinite(q[1]).all() and torch.isfinite(k).all()
