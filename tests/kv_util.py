"""The operators around attention in 64 bits, on the CPU: heads' norms and rotation, the
cache's format from its byte addresses, attention over it."""
import math

import torch

F32, BF16 = torch.float32, torch.bfloat16
HALF = {F32: 2.0 ** -24, BF16: 2.0 ** -8}  # half a rounding step, relative

E2M1 = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)


def gen(seed):
    return torch.Generator().manual_seed(seed)


# ---- the format ------------------------------------------------------------------

def quantise(x):
    """x [.., d] -> (codes [.., d], scale bytes [.., d / 32]), uint8: the nearest of the
    eight magnitudes by comparing with all of them, ties to the even code."""
    b = x.double().unflatten(-1, (-1, 32))
    a = b.abs().amax(dim=-1)
    odd = ~torch.isfinite(b).all(dim=-1)
    a = torch.where(odd, torch.ones_like(a), a)
    e = torch.ceil(torch.log2(a.clamp(min=1e-300) / 6.0))
    e = e + (a > 6.0 * torch.exp2(e)).double() - (a <= 6.0 * torch.exp2(e - 1)).double()
    e = e.clamp(-125, 125)
    e = torch.where(a == 0, torch.zeros_like(e), e)
    u = torch.where(odd[..., None], torch.zeros_like(b), b) / torch.exp2(e)[..., None]
    gap = (u.abs()[..., None].clamp(max=6.0) - E2M1).abs()
    order = gap * 16 + torch.tensor([0.0, 1e-9, 0.0, 1e-9, 0.0, 1e-9, 0.0, 1e-9], dtype=torch.float64)
    code = order.argmin(dim=-1) + 8 * torch.signbit(u).long()
    code = torch.where(odd[..., None], torch.zeros_like(code), code)
    byte = torch.where(odd, torch.full_like(e, 255.0), e + 127)
    return code.flatten(-2).to(torch.uint8), byte.to(torch.uint8)


def values(codes, scales):
    """What codes [.., d] and scale bytes [.., d / 32] stand for, in 64 bits."""
    c = codes.long()
    v = E2M1[c % 8] * torch.where(c >= 8, -1.0, 1.0).double()
    s = torch.exp2(scales.double() - 127)
    s = torch.where(scales == 255, torch.full_like(s, math.nan), s)
    return (v.unflatten(-1, (-1, 32)) * s[..., None]).flatten(-2)


def held(x):
    """The values the cache has of x, in 64 bits."""
    return values(*quantise(x))


def put(cache, slots, k, v):
    """Writes rows k, v [N, heads, d] to a CPU cache [pages, heads, page / 16, 17 d]."""
    pages, heads, groups, rec = cache.shape
    d, page = rec // 17, 16 * groups
    c = torch.arange(d)
    (kc, ks), (vc, vs) = quantise(k), quantise(v)
    for r, s in enumerate(slots.tolist()):
        if not 0 <= s < pages * page:
            continue
        p, grp, t = s // page, s % page // 16, s % 16
        n, q = c // (d // 16), c % (d // 16)
        at_v = 8 * d + ((t // 4 * 16 + n) * 4 + t % 4) * (d // 32) + q // 2
        b = torch.arange(d // 32)
        for h in range(heads):
            to = cache[p, h, grp]
            to[t * d // 2 + c[::2] // 2] = kc[r, h, 0::2] | kc[r, h, 1::2] << 4
            to[at_v[::2]] = vc[r, h, 0::2] | vc[r, h, 1::2] << 4
            to[16 * d + t * (d // 32) + b] = ks[r, h]
            to[16 * d + d // 2 + (t // 4 * (d // 32) + b) * 4 + t % 4] = vs[r, h]


def garbage(pages, heads, d, page, seed=99):
    """A CPU cache full of leftovers, NaN scales among them."""
    c = torch.randint(0, 256, (pages, heads, page // 16, 17 * d), generator=gen(seed), dtype=torch.uint8)
    c[..., 16 * d:][torch.rand(c[..., 16 * d:].shape, generator=gen(seed + 1)) < 0.2] = 255
    return c


# ---- norms and rotation ------------------------------------------------------------

def norm_rope(x, pos, freq, norm, gain, eps, interleaved):
    """x [N, heads, d] -> (result, the magnitudes its error goes by), in 64 bits."""
    x = x.double()
    if norm:
        x = x / torch.sqrt((x * x).mean(dim=-1, keepdim=True) + eps)
        if gain is not None:
            x = x * gain.double()
    y, mag = x.clone(), x.abs().clone()
    if freq is not None:
        half = freq.shape[0]
        i = torch.arange(half)
        one, two = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        a = (pos.double()[:, None] * freq.double())[:, None]
        u, w = x[..., one], x[..., two]
        y[..., one] = u * torch.cos(a) - w * torch.sin(a)
        y[..., two] = w * torch.cos(a) + u * torch.sin(a)
        mag[..., one] = mag[..., two] = u.abs() + w.abs()
    return y, mag


# ---- attention ------------------------------------------------------------------------

def attention(q, ks, vs, lens, q_start, window, scale):
    """q [N, hq, d]; ks, vs: each sequence's held keys and values [tokens, heads, d] in 64
    bits -> (out, bound): bound is how far fp32 out may be off (rows of no sequence: NaN
    in both).  A weight p is off by the score's error (the fp32 sum of d products, its
    multiplication with the scale and the one with log2(e): |q| . |k| scale (d + 4) 2^-24 each way),
    the exponential's (2^-21), the sums' (tokens 2^-24 at most) and, as it enters the
    second product, its rounding to f16, half a step: 2^-11 for bf16 rows; for fp32 rows
    what that leaves is rounded again, 2^-22; all relative.  f16's steps are of one size
    below 2^-14: half of one is 2^-25, with weights that are counted from 2^-7 of the
    largest, so 2^-32 of that one's.  out is off by these times sum p |v|, the last by 2^-32
    of the largest weight times sum |v|, and by its own rounding."""
    N, hq, d = q.shape
    out = torch.full((N, hq, d), math.nan, dtype=torch.float64)
    bound = torch.full_like(out, math.nan)
    cut = 2.0 ** -11 if q.dtype is BF16 else 2.0 ** -22
    for b, n in enumerate(lens):
        rows = range(b, b + 1) if q_start is None else range(q_start[b], q_start[b + 1])
        G = hq // ks[b].shape[1] if len(ks[b]) else 1
        for i, r in enumerate(rows):
            pos = n - len(rows) + i
            lo = max(0, pos - window + 1) if window else 0
            if pos < 0:
                out[r] = bound[r] = 0.0
                continue
            k = ks[b][lo:pos + 1].repeat_interleave(G, dim=1)  # [tokens, hq, d]
            v = vs[b][lo:pos + 1].repeat_interleave(G, dim=1)
            z = (k * q[r].double()).sum(dim=-1) * scale        # [tokens, hq]
            p = torch.softmax(z, dim=0)
            out[r] = (p[..., None] * v).sum(dim=0)
            size = (k.abs() * q[r].double().abs()).sum(dim=-1).amax(dim=0) * scale
            rel = 2 * (d + 4) * 2.0 ** -24 * size + 2.0 ** -21 + 2 * (len(k) + 64) * 2.0 ** -24 + cut
            bound[r] = (p[..., None] * v.abs()).sum(dim=0) * rel[:, None] + out[r].abs() * HALF[q.dtype]
            bound[r] += 2.0 ** -32 * p.amax(dim=0)[:, None] * v.abs().sum(dim=0)
    return out, bound


class Batch:
    """Sequences in a cache: keys and values, pages in a shuffled order, queries."""

    def __init__(self, lens, hq, hkv, d, page, dtype, counts=None, seed=1, spare=2, peak=1.0, far=None):
        g = gen(seed)
        self.lens, self.counts, self.hq, self.hkv, self.d, self.page = lens, counts, hq, hkv, d, page
        need = [(n + page - 1) // page for n in lens]
        pages = sum(need) + spare
        ids = torch.randperm(pages, generator=g).tolist()
        self.table = torch.full((len(lens), max(1, max(need))), -1, dtype=torch.int32)
        self.cache = garbage(pages, hkv, d, page, seed)
        self.k, self.v, self.pages = [], [], []
        for b, n in enumerate(lens):
            mine, ids = ids[:need[b]], ids[need[b]:]
            self.table[b, :need[b]] = torch.tensor(mine, dtype=torch.int32)
            k, v = (torch.randn((n, hkv, d), generator=g) for _ in range(2))
            if far is not None:  # values of very different sizes
                v *= 2.0 ** torch.tensor(far)[torch.randint(0, len(far), (n, hkv, 1), generator=g)]
            t = torch.arange(n)
            slots = torch.tensor(mine + [0])[t // page] * page + t % page
            put(self.cache, slots, k, v)
            self.k.append(held(k) if n else torch.zeros((0, hkv, d), dtype=torch.float64))
            self.v.append(held(v) if n else torch.zeros((0, hkv, d), dtype=torch.float64))
            self.pages.append(mine)
        rows = len(lens) if counts is None else sum(counts)
        self.q = (torch.randn((rows, hq, d), generator=g) * peak).to(dtype)
        self.q_start = None
        if counts is not None:
            self.q_start = [sum(counts[:i]) for i in range(len(counts) + 1)]

    def device(self):
        """(q, cache, table, lens, q_start) on the GPU."""
        start = None if self.q_start is None else torch.tensor(self.q_start, dtype=torch.int32).cuda()
        return (self.q.cuda(), self.cache.cuda(), self.table.cuda(), torch.tensor(self.lens, dtype=torch.int32).cuda(),
                start)

    def expect(self, window=0, scale=None):
        return attention(self.q, self.k, self.v, self.lens, self.q_start, window, self.d ** -0.5 if scale is None else scale)
