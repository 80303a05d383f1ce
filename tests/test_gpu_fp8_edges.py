"""The 8-bit operators where a decision hangs on the last bits: gate values next to the
cutoff and far below zero, and quotients next to the middle of two e4m3 values."""
import pytest
import torch

import paper_2404_08763_amd as P

from fp8_util import BLOCK, E8M0, F32, gen
from gpu_util import say

pytestmark = pytest.mark.gpu

SCALES = [F32, E8M0]
IDS = ["f32", "e8m0"]
DEV = "cuda"


def _silu(z):
    z = z.double()
    return z / (1.0 + torch.exp(-z))


def _next_up(v: float) -> float:
    """The least fp32 number that is not below v."""
    f = torch.tensor(v, dtype=torch.float64).float()
    return float(f) if float(f) >= v else float(torch.nextafter(f, torch.tensor(float("inf"))))


def _nearest(quot):
    """e4m3 values nearest to float64 quotients, and which of these 64 bits decide
    (not within 2^-40 of the middle of two, and not below 2^-6)."""
    step = 2.0 ** (torch.frexp(quot)[1].double() - 4)
    steps = quot / step
    clear = (quot.abs() >= 2.0 ** -6) & (((steps - steps.floor()) - 0.5).abs() > 2.0 ** -40)
    return torch.round(steps) * step, clear


def _quotients(v, s, stype):
    """float64 v [N, whole blocks] over their scales: 448 / largest for fp32 ones, the stored power of two."""
    b = v.view(v.shape[0], -1, BLOCK)
    if stype == E8M0:
        return (b / s.float().double()[:, :, None]).view(v.shape)
    return (b * 448.0 / b.abs().amax(dim=2, keepdim=True)).view(v.shape)


# ---- the gate's cutoff --------------------------------------------------------------

@pytest.mark.parametrize("stype", SCALES, ids=IDS)
@pytest.mark.parametrize("lo,hi,u", [(-5.0, 5.0, 1.0), (-5.0, 5.0, 1e-35), (-8.0, -5.0, 1e-35), (-80.0, -5.0, 1.0)])
def test_cutoff_is_that_of_64_bits(lo, hi, u, stype):
    """t is the least fp32 number not below |SiLU(z)|, then its neighbour below: z is
    dropped in the first case and, where the two differ, kept in the second, however large
    its exponential's error in fp32 and however small the block's values are."""
    say("cutoff", lo, hi, u, stype)
    zs = (lo + (hi - lo) * torch.rand(150, generator=gen(5))).tolist()
    for z in zs:
        z = float(torch.tensor(z))
        v = abs(float(_silu(torch.tensor([z]))[0]))
        up = _next_up(v)
        gu = torch.tensor([[z, u]], device=DEV)
        for t in (up, float(torch.nextafter(torch.tensor(up), torch.tensor(0.0)))):
            if t == v:
                continue
            q, _ = P.silu_mul_fp8(gu, t=t, scale_dtype=stype)
            assert bool(q.float()[0, 0] != 0) == (v >= t), (z, t)


def test_cutoff_drops_whatever_up_is():
    """A value below the cutoff by less than fp32 tells is 0 beside an infinite or NaN up value."""
    say("cutoff, u not finite")
    for z in (1.0, -0.75, 3.25):
        v = abs(float(_silu(torch.tensor([z]))[0]))
        t = _next_up(v)
        assert t > v
        for u in (float("inf"), -float("inf"), float("nan")):
            gu = torch.tensor([[z, 4.0, u, 1.0]], device=DEV)
            q, _ = P.silu_mul_fp8(gu, t=t)
            kept = abs(float(_silu(torch.tensor([4.0]))[0])) >= t
            assert q.float()[0, :2].tolist() == [0.0, 448.0 if kept else 0.0], (z, u)


# ---- the nearest value ---------------------------------------------------------------

@pytest.mark.parametrize("stype", SCALES, ids=IDS)
def test_gate_values_far_below_zero_are_the_nearest(stype):
    """Blocks whose gate values lie about one number between -8 and -80, where fp32's
    e^-z is off by up to 60 steps."""
    say("gate far below zero", stype)
    N, nb = 1000, 16
    m = nb * BLOCK
    about = 8.0 + 72.0 * torch.rand((N, nb, 1), generator=gen(21))
    z = -(about + torch.rand((N, nb, BLOCK), generator=gen(22))).view(N, m)
    u = torch.randn((N, m), generator=gen(23)) * torch.exp(about).expand(N, nb, BLOCK).reshape(N, m)
    q, s = P.silu_mul_fp8(torch.cat([z, u], dim=1).to(DEV), scale_dtype=stype)
    v = _silu(z) * u.double()
    want, clear = _nearest(_quotients(v, s.cpu(), stype))
    wrong = clear & (q.cpu().float().double() != want)
    assert clear.double().mean() > 0.9
    assert not wrong.any(), int(wrong.sum())
