"""The 8-bit operators where a decision hangs on the last bits: gate values next to the cutoff."""
import pytest
import torch

import paper_2404_08763_amd as P

from fp8_util import E8M0, F32, gen
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


# ---- the gate's cutoff --------------------------------------------------------------

@pytest.mark.parametrize("stype", SCALES, ids=IDS)
@pytest.mark.parametrize("lo,hi,u", [(-5.0, 5.0, 1.0), (-5.0, 5.0, 1e-35), (-8.0, -5.0, 1e-35)])
def test_cutoff_is_that_of_64_bits(lo, hi, u, stype):
    """t is the least fp32 number not below |SiLU(z)|, then its neighbour below: z is
    dropped in the first case and, where the two differ, kept in the second, however small
    the block's values are."""
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
