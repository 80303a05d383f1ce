"""The cache's format as the tests' reference has it, by hand and by what must hold."""
import torch

from kv_util import garbage, gen, held, put, quantise, values


def test_codes_by_hand():
    x = torch.zeros(1, 64)
    x[0, :12] = torch.tensor([6.0, -6.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.1, 0.26, 4.9])
    x[0, 32:34] = torch.tensor([7.0, 3.0])  # above 6: the next scale
    codes, scales = quantise(x)
    assert codes[0, :12].tolist() == [7, 15, 0, 2, 2, 4, 4, 6, 6, 8, 1, 6]
    assert scales.tolist() == [[127, 128]]
    assert codes[0, 32:34].tolist() == [6, 3]  # 3.5 -> 4 (tie to even), 1.5
    assert values(codes, scales)[0, 32:34].tolist() == [8.0, 3.0]


def test_scales_and_special_values():
    x = torch.zeros(6, 32)
    x[1, 3], x[2, 5], x[3, 0], x[4, 1], x[5, 2] = 6 * 2.0 ** -130, 3e38, float("nan"), float("-inf"), 2.0 ** -127
    codes, scales = quantise(x)
    assert scales[:, 0].tolist() == [127, 2, 252, 255, 255, 2]
    got = values(codes, scales)
    assert got[2, 5] == 6 * 2.0 ** 125 and torch.isnan(got[3]).all() and torch.isnan(got[4]).all()
    assert got[5, 2] == 0  # 2^-127 is a quarter of 2^-125: to the even code


def test_no_value_is_nearer_and_pages_hold_what_is_put():
    x = torch.randn((40, 2, 64), generator=gen(3)) * torch.exp(2 * torch.randn((40, 2, 1), generator=gen(4)))
    h = held(x)
    codes, scales = quantise(x)
    step = torch.exp2(scales.double() - 127).repeat_interleave(32, dim=-1)
    for m in (-6, -4, -3, -2, -1.5, -1, -0.5, 0, 0.5, 1, 1.5, 2, 3, 4, 6):
        assert ((x.double() - h).abs() <= (x.double() - m * step).abs()).all()
    a, b = garbage(5, 2, 64, 32, 1), garbage(5, 2, 64, 32, 2)
    slots = torch.randperm(160, generator=gen(5))[:40]
    put(a, slots, x, -x)
    put(b, slots, x, -x)
    same = (a == b).sum(dim=-1)
    assert int(same.sum()) >= 40 * 2 * (64 + 4)  # every byte of the rows, whatever was there
