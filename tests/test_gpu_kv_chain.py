"""The operators around attention as they are used: a block's attention half on 8-bit
projections (norm, Q/K/V, head norms and rotation, cache, attention, output projection
with the residual), a prompt and then single tokens, eager and as one graph."""
import torch
import pytest

import paper_2404_08763_amd as P

from gpu_util import say
from kv_util import BF16, F32, attention, gen, held, norm_rope

pytestmark = pytest.mark.gpu

D, HQ, HKV, DH, PAGE = 512, 8, 2, 64, 16
COLS = (HQ + 2 * HKV) * DH


@pytest.fixture(scope="module")
def model():
    g = gen(1)
    w = {"qkv": torch.randn((COLS, D), generator=g) * 0.05, "o": torch.randn((D, HQ * DH), generator=g) * 0.05}
    q = {n: P.quantize_fp8(t.cuda().contiguous(), block_rows=128) for n, t in w.items()}
    freq = (10000.0 ** -(torch.arange(0, DH, 2, dtype=torch.float64) / DH)).float().cuda()
    gains = (1 + 0.1 * torch.randn((2, DH), generator=g)).cuda()
    return q, freq, gains


def _half(model, x, pos, slots, cache, table, lens, start, ws, keep=None):
    """x [N, D] fp32 residual stream -> x + attention(x)."""
    w, freq, gains = model
    xq, xs = P.rmsnorm_fp8(x)
    qkv = P.linear_fp8(xq, xs, *w["qkv"], dtype=BF16, ws=ws[0])
    q, k = P.qk_norm_rope(qkv, HQ, HKV, DH, pos, freq, norm=True, gain_q=gains[0], gain_k=gains[1])
    v = qkv[:, (HQ + HKV) * DH:]
    P.kv_write(cache, k, v.unflatten(1, (HKV, DH)), slots)
    o = P.kv_attention(q, cache, table, lens, q_start=start, ws=ws[1])
    oq, os = P.quantize_fp8(o.view(o.shape[0], -1))
    if keep is not None:
        keep.append((qkv, q, k, v, o))
    return P.linear_fp8(oq, os, *w["o"], residual=x, ws=ws[0])


def _i32(*v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def test_prompt_then_tokens(model):
    say("kv chain")
    n, new = 45, 6
    x = torch.randn((n + new, D), generator=gen(2)).cuda()
    table = _i32(3, 1, 0, 4).view(1, 4)
    t = torch.arange(n + new, device="cuda")
    slots, pos = (table[0][t // PAGE] * PAGE + t % PAGE).to(torch.int32), t.to(torch.int32)
    ws = (P.linear_fp8_workspace(64, 4096, 4096), P.kv_attention_workspace(64, 1, HQ, HKV, DH))
    cache = P.kv_cache(5, HKV, DH, page=PAGE)
    keep = []
    _half(model, x[:n], pos[:n], slots[:n], cache, table, _i32(n), _i32(0, n), ws, keep)
    qkv, q, k, v, o = keep[0]
    # each operator on the tensors it got, against its formula in 64 bits
    cpu = qkv.cpu().unflatten(1, (HQ + 2 * HKV, DH))
    for got, part, gain in ((q, cpu[:, :HQ], model[2][0]), (k, cpu[:, HQ:HQ + HKV], model[2][1])):
        want, mag = norm_rope(part, pos[:n].cpu(), model[1].cpu(), True, gain.cpu(), 1e-5, False)
        assert ((got.cpu().double() - want).abs() <= 24 * 2.0 ** -24 * mag + 2.0 ** -8 * 1.001 * want.abs()).all()
    want, bound = attention(q.cpu(), [held(k.cpu())], [held(v.cpu().unflatten(1, (HKV, DH)))], [n], [0, n], 0, DH ** -0.5)
    assert ((o.cpu().double() - want).abs() <= bound).all()

    # single tokens: one graph, replayed with the next position, slot and length
    one, at, slot, length = x[n:n + 1].clone(), pos[n:n + 1].clone(), slots[n:n + 1].clone(), _i32(n + 1)
    mine = cache.clone()
    _half(model, one, at, slot, mine, table, length, None, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = _half(model, one, at, slot, mine, table, length, None, ws)
    for i in range(n, n + new):
        one.copy_(x[i:i + 1])
        at.copy_(pos[i:i + 1])
        slot.copy_(slots[i:i + 1])
        length.fill_(i + 1)
        graph.replay()
        torch.cuda.synchronize()
        want = _half(model, x[i:i + 1], pos[i:i + 1], slots[i:i + 1], cache, table, _i32(i + 1), None, ws)
        assert torch.equal(y, want)
    rk, rv = P.kv_read(cache, slots)
    mk, mv = P.kv_read(mine, slots)
    assert torch.equal(rk, mk) and torch.equal(rv, mv)


def test_fp32_rows_from_a_sparse_projection():
    """CATS on the attention's input: fp32 rows from cats_sparse_input_gemv through the cache
    and attention into the next sparse projection."""
    say("kv sparse chain")
    g = gen(3)
    B, n = 2, 33
    w = (torch.randn((D, COLS), generator=g) * 0.05).to(BF16).cuda()
    wo = (torch.randn((HQ * DH, D), generator=g) * 0.05).to(BF16).cuda()
    cache = P.kv_cache(6, HKV, DH, page=PAGE)
    table = _i32(0, 1, 2, 3, 4, 5).view(2, 3)
    freq = (10000.0 ** -(torch.arange(0, DH, 2, dtype=torch.float64) / DH)).float().cuda()
    ks, vs = [[], []], [[], []]
    for i in range(n):
        x = torch.randn((B, D), generator=g).cuda()
        qkv = P.sparse_input_gemv(w, x, 0.5)
        pos = _i32(i, i)
        q, k = P.qk_norm_rope(qkv, HQ, HKV, DH, pos, freq)
        v = qkv[:, (HQ + HKV) * DH:].unflatten(1, (HKV, DH))
        P.kv_write(cache, k, v, table[:, i // PAGE] * PAGE + i % PAGE)
        o = P.kv_attention(q, cache, table, pos + 1)
        y = P.sparse_input_gemv(wo, o.view(B, -1), 0.0, residual=x)
        assert o.dtype == F32 and torch.isfinite(y).all()
        for b in range(B):
            ks[b].append(held(k[b:b + 1].cpu()))
            vs[b].append(held(v[b:b + 1].cpu()))
    want, bound = attention(q.cpu(), [torch.cat(t) for t in ks], [torch.cat(t) for t in vs], [n, n], None, 0, DH ** -0.5)
    assert ((o.cpu().double() - want).abs() <= bound).all()
