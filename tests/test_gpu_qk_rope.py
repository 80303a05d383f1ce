"""Norms and rotation of the heads against 64 bits.

A result is off by: the norm's factor (14 fp32 sums of squares, halved by the root, then
mean, root, quotient and two products: 12 half steps), sine and cosine (the angle's
rounding to fp32 after its reduction, below 2^-23, and two steps of the functions' own:
8 half steps), two products and their sum (3): 24 half steps of fp32 of |u| + |w| (24
2^-24), and its own rounding."""
import pytest
import torch

import paper_2404_08763_amd as P

from gpu_util import say
from kv_util import BF16, F32, HALF, gen, norm_rope

pytestmark = pytest.mark.gpu
IDS = {F32: "f32", BF16: "bf16"}


def _freq(rot):
    return (10000.0 ** -(torch.arange(0, rot, 2, dtype=torch.float64) / max(1, rot))).float()


def _check(got, want, mag, dtype):
    err = (got.cpu().double() - want).abs()
    bound = 24 * 2.0 ** -24 * mag + want.abs() * HALF[dtype] * 1.001 + 1e-37
    assert (err <= bound).all(), float((err / bound).max())


def _case(N, hq, hkv, d, rot, norm, gains, inter, x, y, extra=0, far=5000, seed=0):
    g = gen(seed)
    qkv = (torch.randn((N, (hq + hkv) * d + extra), generator=g) * torch.exp(torch.randn((N, 1), generator=g))).to(x)
    pos = torch.randint(0, far, (N,), generator=g).to(torch.int32)
    freq = _freq(rot) if rot else None
    gq, gk = (1 + 0.2 * torch.randn((2, d), generator=g)).unbind() if gains else (None, None)
    dev = lambda t: None if t is None else t.clone().cuda()  # noqa: E731
    q, k = P.qk_norm_rope(qkv.cuda(), hq, hkv, d, dev(pos), dev(freq), norm=norm, gain_q=dev(gq), gain_k=dev(gk),
                          eps=1e-5, interleaved=inter, dtype=y)
    assert q.dtype == k.dtype == y and q.shape == (N, hq, d) and k.shape == (N, hkv, d)
    heads = qkv[:, :(hq + hkv) * d].unflatten(1, (hq + hkv, d))
    _check(q, *norm_rope(heads[:, :hq], pos, freq, norm, gq, 1e-5, inter), y)
    _check(k, *norm_rope(heads[:, hq:], pos, freq, norm, gk, 1e-5, inter), y)


@pytest.mark.parametrize("x,y", [(F32, F32), (F32, BF16), (BF16, BF16), (BF16, F32)],
                         ids=["f32-f32", "f32-bf16", "bf16-bf16", "bf16-f32"])
@pytest.mark.parametrize("N,hq,hkv,d,rot,norm,gains,inter", [
    (1, 32, 32, 128, 128, False, False, False),
    (1, 1, 1, 8, 8, True, True, False),
    (3, 5, 1, 16, 8, True, False, True),
    (7, 3, 3, 40, 24, True, True, False),
    (33, 7, 1, 80, 40, True, True, True),
    (5, 8, 2, 256, 256, False, False, True),
    (9, 2, 2, 512, 512, True, True, False),
    (2, 4, 4, 64, 0, True, True, False),     # no rotation
    (13, 12, 4, 96, 96, True, True, False),
    (700, 32, 8, 128, 64, True, True, False),  # several heads to a wave
])
def test_against_64_bits(N, hq, hkv, d, rot, norm, gains, inter, x, y):
    say("qk rope", N, hq, hkv, d, rot, norm, gains, inter, x, y)
    _case(N, hq, hkv, d, rot, norm, gains, inter, x, y, seed=N + d)


@pytest.mark.parametrize("inter", [False, True], ids=["halves", "neighbours"])
def test_far_positions(inter):
    """Positions to 2^31 - 1: the angle's product in 64 bits is off by 2^-22 of a turn at most
    there, so up to 2^24 it costs nothing; negative ones turn back."""
    say("qk rope far", inter)
    _case(64, 2, 1, 128, 128, False, False, inter, F32, F32, far=1 << 24, seed=3)
    qkv = torch.randn((4, 3 * 64), generator=gen(4))
    pos = torch.tensor([-1, -4096, 1, 0], dtype=torch.int32)
    q, k = P.qk_norm_rope(qkv.cuda(), 2, 1, 64, pos.cuda(), _freq(64).cuda(), interleaved=inter)
    heads = qkv.unflatten(1, (3, 64))
    _check(q, *norm_rope(heads[:, :2], pos, _freq(64), False, None, 0, inter), F32)
    assert torch.equal(k[3].cpu(), heads[3, 2:])  # position 0: as it was


def test_strided_rows_and_untouched_neighbours():
    """A view of wider rows; nothing behind q and k is written."""
    say("qk rope strided")
    N, hq, hkv, d = 11, 6, 2, 64
    wide = torch.randn((N, 1000), generator=gen(5)).cuda()
    qkv = wide[:, 200:200 + (hq + 2 * hkv) * d]
    pos = torch.arange(N, dtype=torch.int32, device="cuda")
    q, k = P.qk_norm_rope(qkv, hq, hkv, d, pos, _freq(d).cuda(), norm=True)
    buf = torch.full((N * (hq + hkv) * d + 128,), 5.0, device="cuda")
    out = (buf[:N * hq * d].view(N, hq, d), buf[N * hq * d + 64:N * (hq + hkv) * d + 64].view(N, hkv, d))
    P.qk_norm_rope(qkv.contiguous(), hq, hkv, d, pos, _freq(d).cuda(), norm=True, out=out)
    assert torch.equal(out[0], q) and torch.equal(out[1], k)
    assert (buf[N * hq * d:N * hq * d + 64] == 5).all() and (buf[-64:] == 5).all()


def test_special_values():
    """NaN and infinities stay in their head; a head of zeros stays 0."""
    say("qk rope special")
    x = torch.randn((4, 4, 64), generator=gen(6))
    x[0, 1, 5], x[1, 2, 60], x[2, 0] = float("nan"), float("inf"), 0.0
    pos = torch.tensor([3, 4, 5, 6], dtype=torch.int32).cuda()
    for norm in (False, True):
        q, k = P.qk_norm_rope(x.view(4, -1).cuda(), 3, 1, 64, pos, _freq(64).cuda(), norm=norm)
        got = torch.cat([q, k], dim=1).cpu()
        bad = torch.zeros(4, 4, dtype=torch.bool)
        bad[0, 1] = bad[1, 2] = True
        assert torch.isfinite(got[~bad]).all() and not torch.isfinite(got[bad]).all(dim=-1).any()
        assert (got[2, 0] == 0).all()


def test_graph():
    say("qk rope graph")
    N, hq, hkv, d = 5, 4, 2, 128
    qkv = torch.zeros((N, (hq + hkv) * d), device="cuda", dtype=BF16)
    pos = torch.zeros(N, dtype=torch.int32, device="cuda")
    out = (torch.zeros((N, hq, d), device="cuda", dtype=BF16), torch.zeros((N, hkv, d), device="cuda", dtype=BF16))
    call = lambda o: P.qk_norm_rope(qkv, hq, hkv, d, pos, freq, norm=True, out=o)  # noqa: E731
    freq = _freq(d).cuda()
    call(out)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(out)
    for r in range(3):
        qkv.copy_(torch.randn(qkv.shape, generator=gen(r)))
        pos.copy_(torch.randint(0, 9999, (N,), generator=gen(r)))
        g.replay()
        torch.cuda.synchronize()
        want = call(tuple(torch.empty_like(t) for t in out))
        assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])
