"""Attention in 64 bits for larger calls than kv_util.attention's: the same definition and bound, a head of a
sequence at a time as products of matrices, on any device."""
import math

import torch

from kv_util import BF16, HALF


def attention(q, ks, vs, lens, q_start, window, scale):
    """q [N, hq, d]; ks, vs: each sequence's held keys and values [tokens, heads, d] in 64 bits, NaN
    where a token's are NaN -> (out, bound) as kv_util.attention (rows of no sequence: NaN in both)."""
    N, hq, d = q.shape
    out = torch.full((N, hq, d), math.nan, dtype=torch.float64, device=q.device)
    bound = torch.full_like(out, math.nan)
    cut = 2.0 ** -11 if q.dtype is BF16 else 2.0 ** -22
    for b, n in enumerate(lens):
        first, last = (b, b + 1) if q_start is None else (q_start[b], q_start[b + 1])
        if first == last:
            continue
        hkv = ks[b].shape[1]
        pos = torch.arange(n - (last - first), n, device=q.device)[:, None]
        j = torch.arange(n, device=q.device)[None]
        seen = j <= pos
        if window:
            seen &= j > pos - window
        some = seen.any(dim=1)
        for h in range(hq):
            x = q[first:last, h].double()
            k, v = ks[b][:, h // (hq // hkv)], vs[b][:, h // (hq // hkv)]
            odd = torch.isnan(v)
            v = v.masked_fill(odd, 0.0)
            z = (torch.mm(x, k.t().contiguous()) * scale).masked_fill(~seen, -math.inf)
            p = torch.softmax(z, dim=1)
            p[~some] = 0.0
            o = torch.mm(p, v)
            if bool(odd.any()):
                o = o.masked_fill(torch.mm(seen.double(), odd.double()) > 0, math.nan)
            size = torch.mm(x.abs(), k.abs().t().contiguous()).masked_fill(~seen, 0.0).amax(dim=1) * scale if n else o.new_zeros(len(o))
            count = seen.sum(dim=1)
            rel = 2 * (d + 4) * 2.0 ** -24 * size + 2.0 ** -21 + 2 * (count + 64) * 2.0 ** -24 + cut
            far = torch.mm(seen.double(), v.abs()) * (p.amax(dim=1) if n else o.new_zeros(len(o)))[:, None]
            e = torch.mm(p, v.abs()) * rel[:, None] + o.abs() * HALF[q.dtype] + 2.0 ** -32 * far
            e[~some] = 0.0
            out[first:last, h], bound[first:last, h] = o, e
    return out, bound
