"""Attention over values up to the cache's largest, 6 * 2^125: a weighted mean of them is an
fp32 number, whatever the sums on the way to it come to.

The bound is attention()'s (kv_util), and for rows that see a value of 6 * 2^80 or more one term
besides.  Where their sums leave fp32 they are held 2^48 times smaller, and a product of a weight and a value that is
below fp32's least normal number, 2^-126, may be lost.  The largest weight is 2^7 or more
before that, 2^-41 after it, and l no less: each token's loss is 2^-126 / 2^-41 at most, and 2^-84 with
the rounding of what l is counted from.  Columns in which the large token's code is 0 come to as
little as that.  (Weights below 2^-85 of the largest are lost too, far less than the
bound's 2^-32 of it for each token.)"""
import pytest
import torch

import paper_2404_08763_amd as P

import kv_paths
from gpu_util import say
from kv_util import BF16, F32, Batch, attention, gen, held

pytestmark = pytest.mark.gpu
IDS = {F32: "f32", BF16: "bf16"}


def near(got, want, bound):
    got = got.cpu().double()
    assert bool((torch.isnan(got) == torch.isnan(want)).all()), "NaN elsewhere"
    err = (got - want).abs().nan_to_num(0)
    bad = ~(err <= bound.nan_to_num(0) + 1e-37)
    assert not bool(bad.any()), (int(bad.sum()), float((err / (bound.nan_to_num(1) + 1e-37)).max()))


def lost(b, window):
    """[N, hq, 1]: tokens * 2^-84 for the rows and heads that see a value of 6 * 2^80 or more."""
    out = torch.zeros((*b.q.shape[:2], 1), dtype=torch.float64)
    for s, n in enumerate(b.lens):
        rows = range(s, s + 1) if b.q_start is None else range(b.q_start[s], b.q_start[s + 1])
        for i, r in enumerate(rows):
            pos = n - len(rows) + i
            v = b.v[s][max(0, pos - window + 1) if window else 0:max(pos + 1, 0)]
            if len(v):
                out[r, :, 0] = ((v.abs() >= 6 * 2.0 ** 80).any(dim=0).any(dim=-1) * (len(v) * 2.0 ** -84)).repeat_interleave(
                    b.hq // b.hkv)
    return out


def check(b, window=0):
    q, cache, table, lens, start = b.device()
    got = P.kv_attention(q, cache, table, lens, q_start=start, window=window)
    want, bound = b.expect(window)
    near(got, want, bound + lost(b, window))


@pytest.mark.parametrize("dtype", [F32, BF16], ids=IDS.get)
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("far", [(81.0,), (113.0,), (121.0,), (124.0,), (124.0, 0.0), (124.0, -100.0), (90.0, 13.0, -17.0, -60.0)])
def test_values_up_to_the_largest(far, d, dtype):
    """Alone, beside ordinary and tiny ones, seen by some rows of a tile and not by others."""
    say("kv large values", far, d, dtype)
    check(Batch([1, 2, 31, 200], 4, 2, d, 16, dtype, seed=90, far=far))
    check(Batch([100, 31, 150], 4, 2, d, 16, dtype, counts=[60, 31, 150], seed=91, far=far))
    check(Batch([100, 31], 2, 2, d, 16, dtype, counts=[12, 3], seed=92, far=far), window=40)
    check(Batch([130, 90], 2, 2, d, 16, dtype, counts=[130, 70], seed=93, far=far), window=20)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=IDS.get)
@pytest.mark.parametrize("counts", [None, [60, 1]], ids=["rows", "ragged"])
def test_one_large_value(counts, dtype):
    """The last but few: rows in front of it and, with a window, behind it are what they are without."""
    say("kv one large value", counts, dtype)
    for window in (0, 9):
        b = Batch([60, 300], 4, 2, 128, 16, dtype, counts=counts, seed=94)
        plain = [v.clone() for v in b.v]
        for seq, tok in ((0, 40), (1, 297)):
            page, t = b.pages[seq][tok // 16], tok % 16
            v = torch.full((2, 128), 3.0 * 2.0 ** 125)
            v[:, ::2] *= -1
            rec = b.cache[page, :, 0]
            blk = torch.arange(4)
            rec[:, 16 * 128 + 64 + (t // 4 * 4 + blk) * 4 + t % 4] = 127 + 125
            c = torch.arange(128)
            n, r = c // 8, c % 8
            at = 8 * 128 + ((t // 4 * 16 + n) * 4 + t % 4) * 4 + r // 2
            rec[:, at[::2]] = 13 | 5 << 4  # -3, 3
            b.v[seq][tok] = v.double()
        q, cache, table, lens, start = b.device()
        got = P.kv_attention(q, cache, table, lens, q_start=start, window=window)
        want, bound = b.expect(window)
        near(got, want, bound + lost(b, window))
        if counts is not None:
            small, bound = attention(b.q, b.k, plain, b.lens, b.q_start, window, 128 ** -0.5)
            same = list(range(40)) + (list(range(49, 60)) if window else [])
            near(got[same], small[same], bound[same])


@pytest.mark.parametrize("dtype", [F32, BF16], ids=IDS.get)
@pytest.mark.parametrize("power", [80, 100, 118, 124])
@pytest.mark.parametrize("rows", [1, 40])
def test_weights_at_their_largest(rows, power, dtype):
    """Each wave's first tokens score 7.8 (in base 2) below all others, which is not enough for what the
    weights are counted from to move: they are near 2^15, for hundreds of tokens of every part."""
    say("kv large weights", rows, power, dtype)
    B, n, heads, d, page = (64, 600, 8, 64, 64) if rows == 1 else (8, 1400, 4, 64, 64)
    g = gen(power)
    k = torch.zeros(B, n, heads, d)
    k[..., 0] = 1.0
    k[:, :128, :, 0] = 0.0
    v = torch.randint(1, 3, (B, n, heads, d), generator=g) * 2.0 ** power
    v[..., ::3] *= -1
    need = -(-n // page)
    cache = P.kv_cache(B * need, heads, d, page=page)
    t = torch.arange(B * n)
    slots = (t // n * need * page + t % n).to(torch.int32).cuda()
    P.kv_write(cache, k.view(B * n, heads, d).cuda(), v.view(B * n, heads, d).cuda(), slots)
    table = torch.arange(B * need, dtype=torch.int32, device="cuda").view(B, need)
    lens = torch.full((B,), n, dtype=torch.int32, device="cuda")
    q = torch.zeros((B * rows, heads, d))
    q[..., 0] = 1.0
    starts = None if rows == 1 else [rows * b for b in range(B + 1)]
    at = None if rows == 1 else torch.tensor(starts, dtype=torch.int32, device="cuda")
    scale = 7.8125 / 1.4426950408889634
    got = P.kv_attention(q.to(dtype).cuda(), cache, table, lens, q_start=at, scale=scale)
    some = [0, B - 1]  # (sequences that are compared)
    ks, vs = ([held(x[b]) for b in some] for x in (k, v))
    pick = torch.cat([torch.arange(b * rows, (b + 1) * rows) for b in some])
    want, bound = attention(q[pick].to(dtype), ks, vs, [n, n], None if rows == 1 else [0, rows, 2 * rows], 0, scale)
    near(got[pick.cuda()], want, bound)
    assert torch.isfinite(got).all()


@pytest.mark.parametrize("dtype", [F32, BF16], ids=IDS.get)
@pytest.mark.parametrize("counts", [None, [2, 2, 2, 2, 90]], ids=["rows", "ragged"])
@pytest.mark.parametrize("power", [100, 123])
def test_maxima_next_to_integers(power, counts, dtype):
    """Maxima of a few steps of fp32 above and below integers (in base 2): one key column, equal scores."""
    say("kv maxima next to integers", power, counts, dtype)
    lens = [40, 100, 130, 2, 150]
    b = Batch(lens, 4, 2, 64, 16, dtype, counts=counts, seed=95, far=(float(power),))
    for s, n in enumerate(lens):
        k = torch.zeros(n, 2, 64)
        k[..., 0] = 1.0
        t = torch.arange(n)
        pages = torch.tensor(b.pages[s])
        cache = b.cache.cuda()
        slots = (pages[t // 16] * 16 + t % 16).to(torch.int32).cuda()
        _, v = P.kv_read(cache, slots, dtype=F32)
        P.kv_write(cache, k.cuda(), v, slots)
        b.cache = cache.cpu()
        b.k[s] = k.double()
    g = gen(96)
    whole = torch.randint(-9, 9, b.q.shape[:2], generator=g).float()
    steps = torch.randint(-3, 4, b.q.shape[:2], generator=g).float()
    b.q.zero_()
    b.q[..., 0] = (whole * (1 + steps * 2.0 ** -23)).to(dtype)
    scale = 0.6931471805599453  # its product with log2(e) is 1, or a step of fp32 beside it
    q, cache, table, ln, start = b.device()
    got = P.kv_attention(q, cache, table, ln, q_start=start, scale=scale)
    want, bound = b.expect(0, scale)
    near(got, want, bound + lost(b, 0))


@pytest.mark.parametrize("dtype", [F32, BF16], ids=IDS.get)
@pytest.mark.parametrize("hq,hkv,d", [(4, 1, 64), (20, 1, 64), (8, 2, 128), (4, 2, 256), (32, 1, 128)])
@pytest.mark.parametrize("far", [(100.0,), (124.0,), (124.0, 0.0)])
@pytest.mark.parametrize("rows", [None, [1, 4, 2]], ids=["rows", "ragged"])
def test_long_sequences_of_large_values(rows, far, hq, hkv, d, dtype):
    """Single tokens and few rows whose keys are shared by many blocks: parts with and without larger sums are
    joined, by the block that arrives last and by the joining kernel."""
    say("kv long large values", rows, far, hq, hkv, d, dtype)
    lens, page = [20000, 3, 7001], 64
    g = gen(97)
    need = [-(-n // page) for n in lens]
    cache = P.kv_cache(sum(need), hkv, d, page=page)
    table = torch.full((3, max(need)), -1, dtype=torch.int32)
    ks, vs = [], []
    for b, n in enumerate(lens):
        first = sum(need[:b])
        table[b, :need[b]] = torch.arange(need[b]) + first
        slots = torch.arange(n, dtype=torch.int32, device="cuda") + first * page
        k, v = (torch.randn((n, hkv, d), generator=g) for _ in range(2))
        # (one region of a sequence has them, or all of it)
        size = 2.0 ** torch.tensor(far)[(torch.arange(n) % 4096 > 2000).long() % len(far)]
        P.kv_write(cache, k.cuda(), (v * size[:, None, None]).cuda(), slots)
        k, v = P.kv_read(cache, slots, dtype=F32)
        ks.append(k.double())
        vs.append(v.double())
    counts = rows or [1, 1, 1]
    starts = [sum(counts[:i]) for i in range(4)]
    q = (torch.randn((sum(counts), hq, d), generator=g) * 2).to(dtype).cuda()
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    got = P.kv_attention(q, cache, table.cuda(), i32(lens), q_start=None if rows is None else i32(starts))
    want, bound = kv_paths.attention(q, ks, vs, lens, starts, 0, d ** -0.5)
    near(got, want.cpu(), bound.cpu() + max(lens) * 2.0 ** -84)
