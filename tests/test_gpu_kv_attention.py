"""Attention over the cache in 4 bits against 64 bits (kv_util.attention has the bound's terms)."""
import math

import pytest
import torch

import paper_2404_08763_amd as P

from gpu_util import say
from kv_util import BF16, F32, HALF, Batch, attention, garbage, gen

pytestmark = pytest.mark.gpu
IDS = {F32: "f32", BF16: "bf16"}


def _near(got, want, bound):
    got = got.cpu().double()
    assert bool((torch.isnan(got) == torch.isnan(want)).all()), "NaN elsewhere"
    err = (got - want).abs().nan_to_num(0)
    bad = err > bound.nan_to_num(0) + 1e-37
    assert not bool(bad.any()), (int(bad.sum()), float((err / (bound.nan_to_num(1) + 1e-37)).max()))


def _check(b, window=0, scale=None):
    q, cache, table, lens, start = b.device()
    got = P.kv_attention(q, cache, table, lens, q_start=start, window=window, scale=scale)
    assert got.dtype == b.q.dtype
    _near(got, *b.expect(window, scale))
    return got


LENS = [1, 0, 15, 16, 17, 31, 32, 33, 127, 128, 129, 300, 1000]


@pytest.mark.parametrize("dtype", [F32, BF16], ids=IDS.get)
@pytest.mark.parametrize("hq,hkv,d,page", [(1, 1, 64, 16), (4, 4, 128, 64), (32, 8, 128, 48), (5, 1, 256, 32),
                                           (16, 1, 128, 16), (17, 1, 64, 256), (40, 1, 128, 32), (20, 1, 256, 16)])
def test_one_row_for_each_sequence(hq, hkv, d, page, dtype):
    say("kv decode", hq, hkv, d, page, dtype)
    _check(Batch(LENS, hq, hkv, d, page, dtype, seed=hq + d, peak=1.5))


@pytest.mark.parametrize("dtype", [F32, BF16], ids=IDS.get)
@pytest.mark.parametrize("window", [0, 1, 30, 128, 500])
@pytest.mark.parametrize("hq,hkv,d,page,lens,counts", [
    (2, 2, 64, 16, [40], [40]),                                   # a whole prompt
    (8, 2, 128, 64, [1, 33, 300, 77, 0, 5], [1, 2, 130, 0, 0, 9]),  # the last: rows in front of its first token
    (3, 1, 256, 32, [200, 64, 17], [90, 64, 1]),
    (12, 4, 128, 48, [400, 399], [33, 70]),
])
def test_ragged_rows(hq, hkv, d, page, lens, counts, window, dtype):
    say("kv ragged", hq, hkv, d, page, lens, counts, window, dtype)
    _check(Batch(lens, hq, hkv, d, page, dtype, counts=counts, seed=sum(lens)), window=window)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=IDS.get)
@pytest.mark.parametrize("window", [1, 17, 100])
def test_window_of_single_rows(window, dtype):
    say("kv window", window, dtype)
    _check(Batch(LENS, 6, 2, 128, 32, dtype, seed=5), window=window)


@pytest.mark.parametrize("window", [79, 80, 81, 2 ** 30, 2 ** 31 - 1])
@pytest.mark.parametrize("counts", [[9, 80], [90, 70]])
def test_windows_around_and_beyond_the_table(counts, window):
    """Rows in front of a sequence's first token among them (positions down to -85)."""
    say("kv wide window", window, counts)
    _check(Batch([5, 80], 4, 2, 64, 16, BF16, counts=counts, seed=17), window=window)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=IDS.get)
def test_long_sequences_are_split_and_joined(dtype):
    """One sequence over every block, and a few of very different lengths."""
    say("kv long", dtype)
    _check(Batch([20001], 4, 1, 64, 256, dtype, seed=7))
    _check(Batch([5000, 3, 9000, 260], 6, 2, 128, 64, dtype, seed=8, peak=2.0))
    _check(Batch([6000, 100], 8, 1, 64, 64, dtype, counts=[21, 5], seed=9))


def test_many_sequences():
    """More sequences than a block has threads, empty ones among them."""
    say("kv many")
    lens = [(i * 37) % 50 for i in range(700)]
    _check(Batch(lens, 2, 1, 64, 16, BF16, seed=10))
    counts = [min(3, n) for n in lens]
    _check(Batch(lens, 2, 1, 64, 16, BF16, counts=counts, seed=11))


@pytest.mark.parametrize("dtype", [F32, BF16], ids=IDS.get)
def test_scale_and_peaks(dtype):
    """Scores of up to a few hundred: the maximum moves often, most weights vanish."""
    say("kv peaks", dtype)
    _check(Batch([700, 33], 4, 2, 128, 16, dtype, seed=12, peak=20.0))
    _check(Batch([700, 33], 4, 2, 128, 16, dtype, counts=[60, 33], seed=13), scale=1.5)
    b = Batch([500], 2, 1, 64, 32, dtype, seed=14)
    b.q *= 0  # equal weights
    _check(b)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=IDS.get)
@pytest.mark.parametrize("counts", [None, [1, 2, 130, 40, 3]])
@pytest.mark.parametrize("power", [18, 24, 25, 27, 31, 45, 90])
def test_scores_of_any_size(power, counts, dtype):
    """q has one column, so that the scores are exact, and so far apart that the largest ones
    alone count (a weight each): beyond 2^23, where half a step of a maximum is an exponent's error."""
    say("kv far scores", power, counts, dtype)
    lens = [1, 3, 200, 500, 5000]
    b = Batch(lens, 4, 2, 64, 16, dtype, counts=counts, seed=70 + power)
    g = gen(power)
    col = torch.randint(0, 64, b.q.shape[:2], generator=g)
    sign = torch.randint(0, 2, b.q.shape[:2], generator=g) * 2.0 - 1.0
    b.q = (torch.nn.functional.one_hot(col, 64) * sign[..., None] * 2.0 ** power).to(dtype)
    q, cache, table, start_lens, start = b.device()
    got = P.kv_attention(q, cache, table, start_lens, q_start=start, scale=1.0).cpu().double()
    want, _ = b.expect(scale=1.0)
    mag, _ = attention(b.q, b.k, [v.abs() for v in b.v], b.lens, b.q_start, 0, 1.0)
    # as attention()'s bound, without the scores' errors: equal scores have equal weights
    rel = (2.0 ** -11 if dtype is BF16 else 2.0 ** -22) + 2.0 ** -21 + 2 * 5064 * 2.0 ** -24
    _near(got, want, rel * mag + HALF[dtype] * want.abs())


@pytest.mark.parametrize("dtype", [F32, BF16], ids=IDS.get)
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("far", [(-19.0, 0.0), (14.0, -60.0), (-100.0, -17.0, 13.0, 100.0), (-30.0,)])
def test_values_of_any_size(far, d, dtype):
    """Scales inside, at the ends of and beyond f16's range, tokens of both sorts side by side."""
    say("kv far values", far, d, dtype)
    _check(Batch([200, 31, 64], 4, 2, d, 16, dtype, seed=50, far=far))
    _check(Batch([100, 31], 4, 2, d, 16, dtype, counts=[60, 31], seed=51, far=far))
    _check(Batch([100, 31], 2, 2, d, 16, dtype, counts=[12, 3], seed=52, far=far), window=40)


def _poison(b, seq, token, what):
    """Gives a token's keys or values the scale NaN (in cache and reference)."""
    d, page = b.d, b.page
    p, grp, t = b.pages[seq][token // page], token % page // 16, token % 16
    blk = torch.arange(d // 32)
    rec = b.cache[p, :, grp]
    if what == "k":
        rec[:, 16 * d + t * (d // 32) + blk] = 255
        b.k[seq][token] = math.nan
    else:
        rec[:, 16 * d + d // 2 + (t // 4 * (d // 32) + blk[1:]) * 4 + t % 4] = 255
        b.v[seq][token, :, 32:] = math.nan


@pytest.mark.parametrize("dtype", [F32, BF16], ids=IDS.get)
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("what", ["k", "v"])
def test_nan_reaches_the_rows_that_see_it_alone(what, d, dtype):
    """A NaN token in the middle of a step: rows in front of it and, with a window, far
    behind it have the results they have without it."""
    say("kv nan", what, d, dtype)
    for window in (0, 20):
        b = Batch([90, 50], 4, 2, d, 16, dtype, counts=[90, 7], seed=15)
        _poison(b, 0, 37, what)
        _poison(b, 1, 49, what)
        got = _check(b, window=window)
        assert torch.isnan(got[37:50]).any(dim=-1).all() and not torch.isnan(got[:37]).any()
        assert window == 0 or not torch.isnan(got[37 + 20:90]).any()
        assert not torch.isnan(got[90:96]).any() and torch.isnan(got[96]).any(dim=-1).all()


@pytest.mark.parametrize("dtype", [F32, BF16], ids=IDS.get)
def test_infinities_and_nan_in_q(dtype):
    say("kv q special", dtype)
    b = Batch([40, 41, 42, 43], 2, 1, 64, 16, dtype, seed=16)
    b.q[1, 0, 3], b.q[2, 1, 7] = math.nan, math.inf
    q, cache, table, lens, _ = b.device()
    got = P.kv_attention(q, cache, table, lens).cpu()
    want, bound = b.expect()
    ok = torch.ones(4, 2, dtype=torch.bool)
    ok[1, 0] = ok[2, 1] = False
    assert torch.isnan(got[1, 0]).all() and torch.isnan(got[2, 1]).all()
    _near(got[ok], want[ok], bound[ok])


def test_pages_outside_the_cache():
    """A row that sees a token of such a page becomes NaN; others are as they were; entries
    behind a sequence's length count for nothing."""
    say("kv bad pages")
    b = Batch([70, 70, 20], 4, 2, 128, 16, BF16, counts=[70, 1, 20], seed=17)
    q, cache, table, lens, start = b.device()
    good = P.kv_attention(q, cache, table, lens, q_start=start)
    table[0, 2], table[1, 4], table[2, 2:] = b.cache.shape[0], -7, 2 ** 31 - 1
    got = P.kv_attention(q, cache, table, lens, q_start=start)
    assert torch.equal(got[:32], good[:32]) and torch.isnan(got[32:71].float()).all()
    assert torch.equal(got[71:], good[71:])


def test_lengths_and_starts_outside_their_range():
    """Lengths below zero are none, those past the table are the table's; starts are cut to the rows."""
    say("kv bad lengths")
    b = Batch([64, 64, 64], 2, 1, 64, 16, F32, seed=18)
    q, cache, table, lens, _ = b.device()
    good = P.kv_attention(q, cache, table, lens)
    got = P.kv_attention(q, cache, table, torch.tensor([-5, 2 ** 31 - 1, 64], dtype=torch.int32).cuda())
    assert (got[0] == 0).all() and torch.equal(got[1:], good[1:])
    out = torch.full_like(q, 7.0)
    starts = torch.tensor([-3, 1, 2, 2 ** 31 - 1], dtype=torch.int32).cuda()
    P.kv_attention(q, cache, table, lens, q_start=starts, out=out)
    _near(out, *b.expect())
    out.fill_(7.0)
    P.kv_attention(q, cache, table, lens, q_start=torch.tensor([2, 1, 0, 0], dtype=torch.int32).cuda(), out=out)
    assert (out == 7).all()


def test_rows_of_no_sequence_are_left():
    say("kv rows behind")
    b = Batch([30, 20], 2, 2, 64, 16, BF16, counts=[4, 20], seed=19)
    q, cache, table, lens, start = b.device()
    want = P.kv_attention(q, cache, table, lens, q_start=start)
    wide = torch.cat([q[:2], q, q[:5]])
    out = torch.full_like(wide, 9.0)
    P.kv_attention(wide, cache, table, lens, q_start=start + 2, out=out)
    assert torch.equal(out[2:26], want) and (out[:2] == 9).all() and (out[26:] == 9).all()


def test_offsets_beyond_32_bits():
    """A sequence in the last pages of a cache of 4.6 GiB."""
    say("kv far pages")
    pages, heads, d, page = 17700, 8, 128, 256
    cache = P.kv_cache(pages, heads, d, page=page)
    g = gen(20)
    n = 300
    k, v = (torch.randn((n, heads, d), generator=g).cuda() for _ in range(2))
    table = torch.tensor([[pages - 1, pages - 2]], dtype=torch.int32).cuda()
    t = torch.arange(n, device="cuda")
    P.kv_write(cache, k, v, (table[0][t // page] * page + t % page).to(torch.int32))
    small = P.kv_cache(2, heads, d, page=page)
    P.kv_write(small, k, v, t.to(torch.int32))
    q = torch.randn((1, heads, d), generator=g).cuda().bfloat16()
    lens = torch.tensor([n], dtype=torch.int32).cuda()
    want = P.kv_attention(q, small, torch.tensor([[0, 1]], dtype=torch.int32).cuda(), lens)
    assert torch.equal(P.kv_attention(q, cache, table, lens), want)


@pytest.mark.parametrize("counts", [None, [100, 3, 1]], ids=["rows", "ragged"])
def test_same_bits_on_any_workspace(counts):
    say("kv determinism", counts)
    b = Batch([3000, 40, 900], 8, 2, 128, 16, BF16, counts=counts, seed=21)
    q, cache, table, lens, start = b.device()
    want = P.kv_attention(q, cache, table, lens, q_start=start)
    ws = P.kv_attention_workspace(200, 5, 8, 2, 128)
    for fill in (0, 255, 1, 127):
        ws.fill_(fill)
        assert torch.equal(P.kv_attention(q, cache, table, lens, q_start=start, ws=ws), want)


@pytest.mark.parametrize("counts", [None, [64, 3, 2]], ids=["rows", "ragged"])
def test_graph_serves_other_lengths_and_pages(counts):
    """Captured once, replayed on other rows, lengths, pages and starts, with an eager call
    on the same workspace and eager work between the replays."""
    say("kv graph", counts)
    sets = [Batch(lens, 4, 2, 64, 16, F32, counts=c, seed=22 + i, spare=2 + 8 * i) for i, (lens, c) in enumerate(
        ((([1500, 20, 7], counts)), ([70, 900, 33], counts and [9, 50, 10]), ([64, 3, 2], counts)))]
    pages, width = max(s.cache.shape[0] for s in sets), max(s.table.shape[1] for s in sets)
    rows = max(s.q.shape[0] for s in sets)
    cache = P.kv_cache(pages, 2, 64, page=16)
    q = torch.zeros((rows, 4, 64), device="cuda")
    out, table = torch.zeros_like(q), torch.full((3, width), -1, dtype=torch.int32, device="cuda")
    lens = torch.zeros(3, dtype=torch.int32, device="cuda")
    start = None if counts is None else torch.zeros(4, dtype=torch.int32, device="cuda")
    ws = P.kv_attention_workspace(rows, 3, 4, 2, 64)
    call = lambda o: P.kv_attention(q, cache, table, lens, q_start=start, out=o, ws=ws)  # noqa: E731
    call(out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out)
    for s in sets + sets[:1]:
        n, w = s.q.shape[0], s.table.shape[1]
        cache[:s.cache.shape[0]].copy_(s.cache)
        q[:n].copy_(s.q)
        table[:, :w].copy_(s.table)
        lens.copy_(torch.tensor(s.lens))
        if start is not None:
            start.copy_(torch.tensor(s.q_start))
        graph.replay()
        torch.cuda.synchronize()
        _near(out[:n], *s.expect())
        again = torch.empty_like(q)
        call(again)
        assert torch.equal(again[:n], out[:n])
        _ = (q * 2).sum()


def test_two_graphs_share_a_workspace():
    """Replayed in turn, one of single rows (whose parts are joined by tickets in the
    workspace) and one ragged, with eager calls of other sizes on it between them."""
    say("kv two graphs")
    a = Batch([1500, 20, 700], 4, 2, 64, 16, F32, seed=60)
    b = Batch([900, 300], 4, 2, 64, 16, F32, counts=[40, 300], seed=61)
    c = Batch([2000], 4, 2, 64, 16, F32, seed=62)
    ws = P.kv_attention_workspace(400, 3, 4, 2, 64)
    sets, graphs = [], []
    for x in (a, b, c):
        q, cache, table, lens, start = x.device()
        out = torch.zeros_like(q)
        call = lambda q=q, cache=cache, table=table, lens=lens, start=start, out=out: P.kv_attention(  # noqa: E731
            q, cache, table, lens, q_start=start, out=out, ws=ws)
        call()
        sets.append((call, out, x.expect()))
    torch.cuda.synchronize()
    for call, _, _ in sets[:2]:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call()
        graphs.append(g)
    for _ in range(3):
        for _, out, _ in sets:
            out.fill_(5.0)
        graphs[0].replay()
        graphs[1].replay()
        sets[2][0]()
        graphs[0].replay()
        torch.cuda.synchronize()
        for _, out, want in sets:
            _near(out, *want)


@pytest.mark.parametrize("n,hq,hkv,d,chunk", [(9000, 16, 1, 64, 2250), (6000, 24, 1, 128, 1500)])
def test_long_prompt_equals_its_chunks(n, hq, hkv, d, chunk):
    """More tiles than a block lists for itself: the same rows in chunks, which it does."""
    say("kv long prompt", n, hq, hkv, d)
    g = gen(63)
    page = 256
    cache = P.kv_cache(-(-n // page), hkv, d, page=page)
    k, v = (torch.randn((n, hkv, d), generator=g).cuda() for _ in range(2))
    q = torch.randn((n, hq, d), generator=g).cuda().bfloat16()
    P.kv_write(cache, k, v, torch.arange(n, dtype=torch.int32, device="cuda"))
    table = torch.arange(cache.shape[0], dtype=torch.int32, device="cuda")[None]
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    whole = P.kv_attention(q, cache, table, i32(n), q_start=i32(0, n)).float()
    for at in range(0, n, chunk):
        part = P.kv_attention(q[at:at + chunk], cache, table, i32(at + chunk), q_start=i32(0, chunk)).float()
        # each is within half a step of bf16 of its sum, and the sums within 2^-10 of the weighted
        # magnitudes (the weights' roundings to f16, half a step each), which are 1 or so
        bound = 2.0 ** -8 * (whole[at:at + chunk].abs() + part.abs()) + 2 * 2.0 ** -10
        assert bool(((whole[at:at + chunk] - part).abs() <= bound).all())


@pytest.mark.parametrize("dtype,d,n", [(BF16, 64, 200000), (F32, 64, 60001), (BF16, 128, 100000)])
def test_prompt_beside_a_long_sequence(dtype, d, n):
    """Tiles in one, two and, the long sequence's, in tens of parts, joined by the blocks that
    have them: as calls of each sequence alone, whose parts another kernel joins.  In a graph too,
    replayed with eager calls and rubbish on its workspace in between: the same bits."""
    say("kv skew", dtype, d, n)
    heads, rows, page = 16, [40, 4200], 256
    lens = [n, rows[1]]
    g = gen(64)
    need = [-(-x // page) for x in lens]
    cache = P.kv_cache(sum(need), heads, d, page=page)
    for b, x in enumerate(lens):
        k, v = (torch.randn((x, heads, d), generator=g).cuda() for _ in range(2))
        P.kv_write(cache, k, v, torch.arange(x, dtype=torch.int32, device="cuda") + sum(need[:b]) * page)
    table = torch.zeros((2, max(need)), dtype=torch.int32)
    table[0, :need[0]] = torch.arange(need[0])
    table[1, :need[1]] = torch.arange(need[1]) + need[0]
    table = table.cuda()
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    q = torch.randn((sum(rows), heads, d), generator=g).cuda().to(dtype)
    ws = P.kv_attention_workspace(sum(rows), 2, heads, heads, d)
    where, starts, out = i32(*lens), i32(0, rows[0], sum(rows)), torch.zeros_like(q)
    call = lambda: P.kv_attention(q, cache, table, where, q_start=starts, out=out, ws=ws)  # noqa: E731
    whole = call().clone()
    # the weights' roundings on both sides, 2^-11 or 2^-22 of their sum with |v|, which is 6 at most and
    # far less where there are many tokens; the sums of up to n terms; the output's rounding
    cut = 2 * (2.0 ** -11 if dtype is BF16 else 2.0 ** -22 + 4000 * 2.0 ** -24)
    for b, at in enumerate((0, rows[0])):
        step = 40 if b == 0 else 1050
        for i in range(0, rows[b], step):
            part = P.kv_attention(q[at + i:at + i + step], cache, table[b:b + 1], i32(lens[b] - rows[b] + i + step),
                                  q_start=i32(0, step), ws=ws).double()
            mine = whole[at + i:at + i + step].double()
            bound = HALF[dtype] * (mine.abs() + part.abs()) + 2 * cut
            assert bool(((mine - part).abs() <= bound).all()), (b, i)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for r in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, whole)
        P.kv_attention(q[:40], cache, table[:1], i32(5000), q_start=i32(0, 40), ws=ws)
        if r:
            ws.random_(0, 256)
        assert torch.equal(call(), whole)


def test_two_streams():
    """Two calls at once on streams and workspaces of their own."""
    say("kv streams")
    a, b = Batch([2000, 31], 4, 2, 128, 16, BF16, seed=30), Batch([900, 1500], 4, 2, 128, 16, BF16, seed=31)
    da, db = a.device(), b.device()
    sa, sb = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    outs = []
    for _ in range(3):
        for (q, cache, table, lens, _), s in ((da, sa), (db, sb)):
            with torch.cuda.stream(s):
                outs.append(P.kv_attention(q, cache, table, lens))
    torch.cuda.synchronize()
    for i in range(3):
        _near(outs[2 * i], *a.expect())
        _near(outs[2 * i + 1], *b.expect())


def test_prompt_and_single_tokens_agree():
    """Tokens written and answered one by one give what the whole prompt gives."""
    say("kv prompt and tokens")
    n, hq, hkv, d, page = 70, 8, 2, 128, 16
    g = gen(40)
    k, v = (torch.randn((n, hkv, d), generator=g).cuda() for _ in range(2))
    q = torch.randn((n, hq, d), generator=g).cuda().bfloat16()
    table = torch.tensor([[4, 0, 3, 1, 5]], dtype=torch.int32).cuda()
    t = torch.arange(n, device="cuda")
    slots = (table[0][t // page] * page + t % page).to(torch.int32)
    cache, step = garbage(6, hkv, d, page).cuda(), garbage(6, hkv, d, page, 5).cuda()
    P.kv_write(cache, k, v, slots)
    lens = torch.tensor([n], dtype=torch.int32).cuda()
    whole = P.kv_attention(q, cache, table, lens, q_start=torch.tensor([0, n], dtype=torch.int32).cuda())
    for i in range(n):
        P.kv_write(step, k[i:i + 1], v[i:i + 1], slots[i:i + 1])
        one = P.kv_attention(q[i:i + 1], step, table, lens * 0 + i + 1)
        # both within half a step of bf16 and 2^-14 of the weighted magnitudes of the same value
        assert (one[0].float() - whole[i].float()).abs().max() <= 2 * 2.0 ** -8 * float(whole[i].abs().max()) + 1e-3
