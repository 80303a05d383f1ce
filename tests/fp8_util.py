"""64-bit definitions of the 8-bit operators, and their error bounds.

Roundings are counted in half steps: fp32 2^-24, bf16 2^-8, e4m3 2^-4 of a value
(half a step of the subnormals, 2^-10, below 2^-6)."""
from __future__ import annotations

import torch

BLOCK = 128
F32, E8M0 = torch.float32, torch.float8_e8m0fnu
U = 2.0 ** -24


def ld_of(cols: int) -> int:
    return (cols + BLOCK - 1) // BLOCK * BLOCK


def gen(seed: int, device="cpu") -> torch.Generator:
    return torch.Generator(device=device).manual_seed(seed)


def spread(scale: torch.Tensor, up: int, rows: int) -> torch.Tensor:
    """A scale array as a value for each element [rows, ld], float64."""
    s = scale.float().double()
    return s.repeat_interleave(up, 0)[:rows].repeat_interleave(BLOCK, 1)


def values(q: torch.Tensor, scale: torch.Tensor, up: int) -> torch.Tensor:
    return q.float().double() * spread(scale, up, q.shape[0])


def check_quantised(v: torch.Tensor, q: torch.Tensor, scale: torch.Tensor, up: int, delta: float, drop=None) -> None:
    """q, scale against the finite or non-finite float64 values v [rows, cols] that
    the device knows to a relative error of delta.  drop: elements that may
    be 0 instead (values at the cutoff); their blocks' scales are then not looked at."""
    v, q, scale = v.double().cpu(), q.cpu(), scale.cpu()
    rows, cols = v.shape
    ld = ld_of(cols)
    assert q.shape == (rows, ld) and q.dtype == torch.float8_e4m3fn
    nr, nb = (rows + up - 1) // up, ld // BLOCK
    assert scale.shape == (nr, nb)
    qf = q.float().double()
    assert (qf[:, cols:] == 0).all(), "padding"
    fin = torch.isfinite(v)
    assert (torch.isnan(qf[:, :cols]) == ~fin).all(), "NaN where, and only where, the element is not finite"

    full = torch.zeros((nr * up, ld), dtype=torch.float64)
    full[:rows, :cols] = torch.where(fin, v, torch.zeros_like(v)).abs()
    a = full.view(nr, up, nb, BLOCK).amax(dim=(1, 3))
    s = scale.float().double()
    look = torch.ones_like(a, dtype=torch.bool)
    if drop is not None:
        d = torch.zeros((nr * up, ld), dtype=torch.bool)
        d[:rows, :cols] = drop
        look = ~d.view(nr, up, nb, BLOCK).amax(dim=(1, 3))
    one = look & (a == 0)
    assert (s[one] == 1.0).all(), "the scale of zeros"
    look = look & (a > 0)
    if scale.dtype == F32:
        want = (a / 448.0).clamp(min=2.0 ** -126)
        # the quotient's rounding, and a's own error
        assert ((s - want).abs()[look] <= (want * (delta + U))[look] + 2.0 ** -150).all(), "fp32 scale"
    else:
        assert scale.dtype == E8M0
        assert (torch.log2(s) == torch.log2(s).round()).all()
        assert (a * (1 - delta) <= 448.0 * s)[look].all(), "a block's largest value fits"
        small = (a * (1 + delta) <= 224.0 * s) & (s > 2.0 ** -126)
        assert not small[look].any(), "no smaller power of two fits"

    x = torch.where(fin, v, torch.zeros_like(v)) / spread(scale, up, rows)[:, :cols]
    e = torch.frexp(x)[1].double() - 1
    half = torch.exp2(torch.clamp(e, min=-6.0) - 4)
    # the quotient: x times the rounded reciprocal of the scale, 1.5 fp32 steps
    tol = half + x.abs() * (delta + 4 * U)
    far = torch.where(fin, (qf[:, :cols] - x).abs(), torch.zeros_like(x))
    bad = far > tol
    if drop is not None:
        bad &= ~(drop & (qf[:, :cols] == 0))
    assert not bad.any(), (bad.nonzero()[0].tolist(), int(bad.sum()))


def quantised(v: torch.Tensor, up: int, stype: torch.dtype):
    """q, scale of fp32 values by torch operations (test inputs)."""
    rows, cols = v.shape
    ld, nr = ld_of(cols), (rows + up - 1) // up
    full = torch.zeros((nr * up, ld), device=v.device)
    full[:rows, :cols] = v
    b = full.view(nr, up, ld // BLOCK, BLOCK)
    a = b.abs().amax(dim=(1, 3))
    s = torch.where(a > 0, (a / 448.0).clamp(min=2.0 ** -126), torch.ones_like(a))
    if stype == E8M0:
        s = torch.exp2(torch.ceil(torch.log2(s.double()))).float().clamp(min=2.0 ** -126)
    q = (b / s[:, None, :, None]).to(torch.float8_e4m3fn).view(nr * up, ld)[:rows].contiguous()
    return q, s.to(stype)


def linear_ref(xq, xs, wq, ws, residual=None):
    """(y, sum of the terms' magnitudes) in float64 on the operands' device, by column blocks."""
    n = wq.shape[0]
    N, ld = xq.shape
    y = torch.zeros((N, n), dtype=torch.float64, device=xq.device)
    mag = torch.zeros_like(y)
    xv, wv = values(xq, xs, 1), values(wq, ws, BLOCK)
    for b in range(0, ld, 4096):
        y += xv[:, b:b + 4096] @ wv[:, b:b + 4096].t().contiguous()
        mag += xv[:, b:b + 4096].abs() @ wv[:, b:b + 4096].abs().t().contiguous()
    if residual is not None:
        y += residual.double()
        mag += residual.double().abs()
    return y, mag


def check_linear(y, ref, mag, ld: int) -> None:
    """fp32 sums of ld products in any order: at most ld roundings of partial sums
    below mag, and the scales' product and its use, 2 per block.  As independent
    roundings they add up to sqrt(ld) of them; twice that in the mean square.
    A bf16 output is rounded once more, and may come from the 8-bit matrix
    instructions: they cut each product at 2^-13 of the power of two in the largest
    of its group of eight (256 * 256 beside 2^2 gives 65536, beside 2^3 65544), so
    a group is off by at most 7 2^-13 of its largest product, all of them by 7 2^-13 mag."""
    err = (y.double() - ref).abs()
    out = 2.0 ** -8 * ref.abs() + 7 * 2.0 ** -13 * mag if y.dtype == torch.bfloat16 else 0.0
    over = err > (ld + 2 * (ld // BLOCK) + 8) * U * mag + out
    assert not over.any(), (over.nonzero()[0].tolist(), int(over.sum()), float(err.max()))
    if y.dtype != torch.bfloat16:
        assert float(err.square().mean().sqrt()) <= 2 * ld ** 0.5 * U * float(mag.square().mean().sqrt())
