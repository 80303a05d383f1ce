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


@pytest.mark.parametrize("res", [False, True])
def test_norm_values_next_to_a_middle_are_the_nearest(res):
    """Rows of two, f0 and f1 with sqrt(2) f1 / |f| next to (2 j + 1) / 16: which side of the
    middle q = 256 times that falls goes by the squares' roundings, and by what the residual's
    addition rounds off."""
    say("norm next to a middle", res)
    N = 1 << 16
    f0 = (1 + torch.rand(N, generator=gen(31))).double()
    T = (8.5 + torch.randint(0, 8, (N,), generator=gen(32)).double()) / 16
    x = torch.stack([f0.float(), (f0 * T / torch.sqrt(2 - T * T)).float()], 1)
    r = x * (2.0 ** -25 * (2 * torch.rand((N, 2), generator=gen(33)) - 1)) if res else None
    q, s = P.rmsnorm_fp8(x.to(DEV), residual=r.to(DEV) if res else None, eps=0.0, scale_dtype=E8M0)
    assert (s.float() == 2.0 ** -8).all()
    f = x.double() + (r.double() if res else 0.0)
    quot = f / torch.sqrt(f.square().mean(dim=1, keepdim=True)) * 256.0
    want, clear = _nearest(quot)
    wrong = clear & (q.cpu()[:, :2].float().double() != want)
    assert clear.double().mean() > 0.9
    assert not wrong.any(), int(wrong.sum())


@pytest.mark.parametrize("stype", SCALES, ids=IDS)
def test_norm_of_infinite_sums(stype):
    """An infinity in x or the residual, or an addition past fp32, makes NaN of its element and
    zeros of the row's others; the rows beside are what they are without it."""
    say("norm infinite sums", stype)
    x, r = torch.randn((5, 300), generator=gen(41)), torch.randn((5, 300), generator=gen(42))
    want = P.rmsnorm_fp8(x.to(DEV), residual=r.to(DEV), scale_dtype=stype)
    x[1, 7] = float("inf")
    r[2, 150] = -float("inf")
    x[3, 299] = r[3, 299] = 3e38
    q, s = P.rmsnorm_fp8(x.to(DEV), residual=r.to(DEV), scale_dtype=stype)
    qf = q.float().cpu()[:, :300]
    for row, c in ((1, 7), (2, 150), (3, 299)):
        bad = torch.zeros(300, dtype=torch.bool)
        bad[c] = True
        assert torch.equal(torch.isnan(qf[row]), bad) and (qf[row][~bad] == 0).all()
    for row in (0, 4):
        assert torch.equal(q[row].view(torch.uint8), want[0][row].view(torch.uint8))
        assert torch.equal(s[row].view(torch.uint8), want[1][row].view(torch.uint8))


# ---- rows as they are -------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["x32", "x16"])
def test_norm_of_bf16_numbers_alone(dtype):
    """Without residual and gain the row's factor drops out of f 448 / A, whose bf16
    operands 64 bits divide exactly wherever the quotient is the middle of two e4m3 values
    (and otherwise lie 2^-17 of it away): every value is the nearest, middles to even."""
    say("norm of bf16 numbers", dtype)
    N, d = 501, 4096
    x = torch.randn((N, d), generator=gen(51)).bfloat16().to(dtype)
    q, s = P.rmsnorm_fp8(x.to(DEV))
    f = x.double()
    b = f.view(N, -1, BLOCK)
    quot = (b * 448.0 / b.abs().amax(dim=2, keepdim=True)).view(N, d)
    step = 2.0 ** (torch.frexp(quot)[1].double() - 4).clamp(min=-9.0)
    assert torch.equal(q.cpu().float().double(), torch.round(quot / step) * step)
    y = f / torch.sqrt(f.square().mean(dim=1, keepdim=True) + 1e-5)
    top = y.view(N, -1, BLOCK).abs().amax(dim=2)
    assert ((s.cpu().double() - top / 448.0).abs() <= 4 * 2.0 ** -24 * top / 448.0).all()


def test_norm_of_bf16_numbers_alone_takes_no_longer_than_with_a_gain():
    """It reads less and computes less (0.92 of the time; 1.65 where most waves
    looked a second time at values on the middle of two)."""
    say("norm of bf16 numbers, time")
    x = [torch.randn((4096, 4096), device=DEV).bfloat16() for _ in range(6)]
    gain = 1 + 0.1 * torch.randn(4096, device=DEV)
    out = P.rmsnorm_fp8(x[0])

    def us(g):
        P.timer_reset()
        P.timer_enable(True)
        try:
            for v in x:
                P.rmsnorm_fp8(v, gain=g, out=out)
            torch.cuda.synchronize()
        finally:
            P.timer_enable(False)
        n, ms = P.timer_read()["rmsnorm_fp8"]
        return ms / n * 1e3

    both = [(us(None), us(gain)) for _ in range(8)]
    alone, gained = min(b[0] for b in both), min(b[1] for b in both)
    assert alone <= 1.3 * gained, (alone, gained)
