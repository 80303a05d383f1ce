"""The 8-bit linear layer's bf16 outputs to their own rounding, and writes of every tile height."""
import pytest
import torch

import paper_2404_08763_amd as P

from fp8_util import BLOCK, E8M0, F32, check_linear, gen, ld_of, linear_ref, quantised
from gpu_util import kernels_of, say

pytestmark = pytest.mark.gpu

SCALES = [F32, E8M0]
IDS = ["f32", "e8m0"]
DEV = "cuda"


def _operands(N, n, k, stype):
    x = torch.randn((N, k), generator=gen(11))
    x[:, :: 97] *= 20.0
    w = 0.02 * torch.randn((n, k), generator=gen(13, DEV), device=DEV)
    return quantised(x.to(DEV), 1, stype) + quantised(w, BLOCK, stype)


# blocks of 32, 64 and 128 rows, whole and in parts of the columns
HEIGHTS = [(130, 259, 500), (40, 131, 3000), (700, 3001, 1000), (37, 11413, 1668), (300, 2048, 8320), (2000, 4100, 300), (1743, 852, 9346)]


@pytest.mark.parametrize("stype", SCALES, ids=IDS)
@pytest.mark.parametrize("N,n,k", [(1, 6144, 4096), (16, 257, 512), (32, 4097, 4096), (8, 300, 9000)] + HEIGHTS)
def test_bf16_output_is_the_fp32_one_rounded(N, n, k, stype):
    """Where the products are exact: the same sums, rounded once, after the residual."""
    say("bf16 is fp32 rounded", N, n, k, stype)
    ops = _operands(N, n, k, stype)
    r = torch.randn((N, n), generator=gen(9)).bfloat16().to(DEV)
    took = [kernels_of(lambda: P.linear_fp8(*ops, dtype=dt)) for dt in (torch.float32, torch.bfloat16)]
    if (N, n) == (2000, 4100):
        assert took == [{"linear_fp8_mid"}, {"linear_fp8_tile"}]  # (bf16: the test below)
        return
    assert took[0] == took[1] and "linear_fp8_tile" not in took[0]
    assert torch.equal(P.linear_fp8(*ops, dtype=torch.bfloat16), P.linear_fp8(*ops).bfloat16())
    assert torch.equal(P.linear_fp8(*ops, dtype=torch.bfloat16, residual=r), P.linear_fp8(*ops, residual=r.float()).bfloat16())


def _cut(xq, xs, wq, ws):
    """Root mean square, over 32 x 64 outputs spread over all of them, of what products lose
    that are cut at 2^-13 of the power of two in the largest of their group of eight columns."""
    rows = torch.linspace(0, xq.shape[0] - 1, 32, device=DEV).long()
    outs = torch.linspace(0, wq.shape[0] - 1, 64, device=DEV).long()
    x, w = xq[rows].float(), wq[outs].float()
    scale = xs.float()[rows][:, None] * ws.float()[outs // BLOCK][None]  # [32, 64, column blocks]
    lost = torch.zeros((32, 64), dtype=torch.float64, device=DEV)
    for b in range(scale.shape[2]):
        c = slice(b * BLOCK, (b + 1) * BLOCK)
        p = (x[:, None, c] * w[None, :, c]).view(32, 64, BLOCK // 8, 8)  # exact in fp32
        quantum = torch.exp2(torch.frexp(p.abs().amax(3, keepdim=True))[1].float() - 14)
        lost += ((p - torch.trunc(p / quantum) * quantum).sum((2, 3)) * scale[:, :, b]).double()
    return float(lost.square().mean().sqrt())


@pytest.mark.parametrize("N,n,k,stype", [(2000, 4100, 300, F32), (2000, 4100, 300, E8M0), (1537, 4097, 1153, E8M0), (1280, 4100, 4096, E8M0),
                                         (2048, 4100, 1153, F32), (2048, 4097, 4096, F32)])
def test_bf16_output_of_the_8_bit_instructions(N, n, k, stype):
    """The cut, of root mean square c by its definition, turns the bf16 rounding of the
    exact value into its neighbour for at most E|error| / step of the outputs, step a bf16 step at
    the output: at most c / step; twice that is allowed, and 2^-10 for fp32's sums."""
    say("bf16 of the 8-bit instructions", N, n, k, stype)
    ops = _operands(N, n, k, stype)
    assert kernels_of(lambda: P.linear_fp8(*ops, dtype=torch.bfloat16)) == {"linear_fp8_tile"}
    ref, mag = linear_ref(*ops)
    y = P.linear_fp8(*ops, dtype=torch.bfloat16)
    check_linear(y, ref, mag, ld_of(k))
    step = torch.exp2(torch.frexp(ref.abs().clamp(min=1e-30))[1].double() - 8)
    allowed = float((2 * _cut(*ops) / step).clamp(max=1.0).mean()) + 2.0 ** -10
    other = float((y != ref.bfloat16()).double().mean())
    print(f"other neighbour {other:.2e} of {allowed:.2e}")
    assert other <= allowed
    # and as root mean square: the rounding's own, and the cut's
    ideal = (ref.bfloat16().double() - ref).square().mean()
    assert float((y.double() - ref).square().mean()) <= float(ideal) * (1 + 2.0 ** -6) + 4 * _cut(*ops) ** 2


@pytest.mark.parametrize("stype", SCALES, ids=IDS)
@pytest.mark.parametrize("N,n,k", HEIGHTS)
def test_writes_stay_inside_at_every_height(N, n, k, stype):
    say("guards", N, n, k, stype)
    ops = _operands(N, n, k, stype)
    ref, mag = linear_ref(*ops)
    need = P.linear_fp8_workspace(N, n, ld_of(k)).numel()
    for dtype in (torch.float32, torch.bfloat16):
        size = N * n * (4 if dtype == torch.float32 else 2)
        whole = torch.full((size + 8192,), 0x5a, dtype=torch.uint8, device=DEV)
        scratch = torch.full((need + 8192,), 0x5a, dtype=torch.uint8, device=DEV)
        y = whole[4096:4096 + size].view(dtype).view(N, n)
        P.linear_fp8(*ops, out=y, ws=scratch[4096:4096 + need])
        for t, inner in ((whole, size), (scratch, need)):
            assert (t[:4096] == 0x5a).all() and (t[4096 + inner:] == 0x5a).all()
        check_linear(y, ref, mag, ld_of(k))
