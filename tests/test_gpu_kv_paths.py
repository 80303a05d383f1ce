"""Attention's ways of sharing and joining work that need calls of some size: prompts whose parts
are joined by the blocks that have them, at every width and type and with masks, far and large values,
NaN and bad pages; notes for the joining kernel by block and by tile; more tiles and sequences than
a block lists for itself.  Against 64 bits (kv_paths.attention)."""
import math

import pytest
import torch

import paper_2404_08763_amd as P

import kv_paths
from gpu_util import say
from kv_util import BF16, F32, gen

pytestmark = pytest.mark.gpu
IDS = {F32: "f32", BF16: "bf16"}
WIDTHS = [(BF16, 64), (F32, 64), (BF16, 128), (F32, 128), (BF16, 256), (F32, 256)]


class Call:
    """Sequences in a cache, pages shuffled; `size` [tokens, heads, 1] multiplies the values."""

    def __init__(self, lens, counts, hq, hkv, d, page, dtype, seed, size=None):
        g = gen(seed)
        need = [-(-n // page) for n in lens]
        self.lens, self.counts, self.page, self.d = lens, counts, page, d
        self.cache = P.kv_cache(sum(need) + 1, hkv, d, page=page)
        self.cache.random_(0, 256)
        ids = torch.randperm(sum(need) + 1, generator=g).to(torch.int32)
        self.table = torch.full((len(lens), max(need)), -1, dtype=torch.int32)
        slots, at = [], 0
        for b, n in enumerate(need):
            self.table[b, :n] = ids[at:at + n]
            t = torch.arange(lens[b])
            slots.append((ids[at + t // page] * page + t % page).to(torch.int32))
            at += n
        slots = torch.cat(slots).cuda()
        k, v = (torch.randn((len(slots), hkv, d), generator=g).cuda() for _ in range(2))
        if size is not None:
            v *= size(len(slots), hkv, g).cuda()
        P.kv_write(self.cache, k, v, slots)
        k, v = P.kv_read(self.cache, slots, dtype=F32)  # exact
        self.k, self.v = ([x.double() for x in t.split(lens)] for t in (k, v))
        self.table = self.table.cuda()
        self.starts = [sum(counts[:i]) for i in range(len(counts) + 1)]
        self.q = torch.randn((sum(counts), hq, d), generator=g).to(dtype).cuda()

    def _place(self, seq, token):
        return int(self.table[seq, token // self.page]), token % self.page // 16, token % 16

    def poison(self, seq, token, keys):
        """The scales of a token's keys, or of its values' columns from 32 on, become NaN."""
        p, grp, t = self._place(seq, token)
        d, rec = self.d, self.cache[p, :, grp]
        blk = torch.arange(d // 32, device="cuda")
        if keys:
            rec[:, 16 * d + t * (d // 32) + blk] = 255
            self.k[seq][token] = math.nan
        else:
            rec[:, 16 * d + d // 2 + (t // 4 * (d // 32) + blk[1:]) * 4 + t % 4] = 255
            self.v[seq][token, :, 32:] = math.nan

    def lose_page(self, seq, page):
        self.table[seq, page] = self.cache.shape[0] + 5
        self.k[seq][page * self.page:(page + 1) * self.page] = math.nan

    def run(self, window=0, ws=None):
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
        out = torch.full_like(self.q, 7.0)
        P.kv_attention(self.q, self.cache, self.table, i32(self.lens), q_start=i32(self.starts), window=window, out=out, ws=ws)
        return out

    def check(self, window=0, lost=0.0):
        """lost: 2^-84 for each token where there are values near the largest (test_gpu_kv_large)."""
        got = self.run(window)
        want, bound = kv_paths.attention(self.q, self.k, self.v, self.lens, self.starts, window, self.d ** -0.5)
        x = got.double()
        assert bool((torch.isnan(x) == torch.isnan(want)).all()), "NaN elsewhere"
        err = (x - want).abs().nan_to_num(0)
        bad = ~(err <= bound.nan_to_num(0) + lost * max(self.lens) + 1e-37)
        assert not bool(bad.any()), (int(bad.sum()), bad.nonzero()[:4].tolist())
        return got


# A prompt, rows in front of a sequence's first token, and a few rows behind a long sequence, whose tiles
# are in tens of parts: with 16 heads on 8, 264 tiles of 128 rows or twice as many of 64.
LENS, COUNTS = [1500, 650, 20000], [1400, 700, 12]


@pytest.mark.parametrize("dtype,d", WIDTHS)
@pytest.mark.parametrize("window", [0, 100, 5000])
def test_parts_joined_by_their_blocks(window, dtype, d):
    say("kv ticketed prompt", window, dtype, d)
    c = Call(LENS, COUNTS, 16, 8, d, 64, dtype, seed=1)
    got = c.check(window)
    ws = P.kv_attention_workspace(sum(COUNTS), 3, 16, 8, d)
    for fill in (0, 255):
        ws.fill_(fill)
        assert torch.equal(c.run(window, ws), got)  # whoever joins


@pytest.mark.parametrize("dtype,d", WIDTHS)
def test_joined_parts_with_nan_and_bad_pages(dtype, d):
    """The long sequence's in the middle of its tiles' parts; beside them, and behind a window, rows as without."""
    say("kv ticketed prompt, nan", dtype, d)
    c = Call(LENS, COUNTS, 16, 8, d, 64, dtype, seed=2)
    c.poison(0, 700, True)
    c.poison(1, 300, False)
    c.poison(2, 19995, True)   # seen by the last rows alone
    c.lose_page(2, 100)
    for window in (0, 300):
        got = c.check(window)
        assert torch.isnan(got).any() and not torch.isnan(got[:600]).any()
    assert not torch.isnan(got[2100:2107]).any()  # (behind the lost page's window)


@pytest.mark.parametrize("dtype,d", WIDTHS)
@pytest.mark.parametrize("far", [(-30.0, 0.0), (14.0, -60.0), (121.0,), (124.0, 0.0)])
def test_joined_parts_of_far_and_large_values(far, dtype, d):
    say("kv ticketed prompt, far", far, dtype, d)
    size = lambda n, h, g: 2.0 ** torch.tensor(far)[torch.randint(0, len(far), (n, h, 1), generator=g)]  # noqa: E731
    c = Call(LENS, COUNTS, 16, 8, d, 64, dtype, seed=3, size=size)
    for window in (0, 100):
        c.check(window, lost=2.0 ** -84 if max(far) > 80 else 0.0)


def _many(n, most, rows, seed):
    g = gen(seed)
    lens = torch.randint(1, most, (n,), generator=g).tolist()
    counts = [min(int(r), m) for r, m in zip(torch.randint(rows[0], rows[1] + 1, (n,), generator=g), lens)]
    return lens, counts


@pytest.mark.parametrize("dtype,d", WIDTHS)
@pytest.mark.parametrize("n,hkv", [(700, 2), (250, 4)], ids=["listed in front", "listed by each block"])
def test_few_rows_of_many_sequences(n, hkv, dtype, d):
    """More tiles than blocks, of several units: the joining kernel's notes are by block."""
    say("kv many sequences", n, hkv, dtype, d)
    lens, counts = _many(n, 600, (1, 3), 4)
    Call(lens, counts, 2 * hkv, hkv, d, 32, dtype, seed=5).check()
    Call(lens, counts, 2 * hkv, hkv, d, 32, dtype, seed=6).check(window=150)


@pytest.mark.parametrize("dtype,d", WIDTHS)
@pytest.mark.parametrize("n,hkv,rows", [(200, 2, 40), (300, 2, 40), (300, 1, 45)],
                         ids=["listed by each block", "listed in front", "and few"])
def test_prompts_of_many_sequences(n, hkv, rows, dtype, d):
    """Prompts' tiles, joined by their blocks or by the kernel, with its notes by block or by tile."""
    say("kv many prompts", n, hkv, rows, dtype, d)
    lens, _ = _many(n, 600, (1, 1), 7)
    Call(lens, [rows] * n, hkv, hkv, d, 32, dtype, seed=8).check()
    Call(lens, [rows] * n, hkv, hkv, d, 32, dtype, seed=9).check(window=70)


@pytest.mark.parametrize("dtype,d", [(F32, 256), (BF16, 256), (F32, 64)])
def test_more_tiles_than_a_block_lists(dtype, d):
    say("kv many tiles", dtype, d)
    rows = 3000 if d == 256 else 6000
    Call([rows, 900], [rows, 400], 24, 1, d, 256, dtype, seed=10).check()
