"""Measured cases of the operators between the Q/K/V projection and the output
projection: norms and rotation of queries and keys, the cache in 4 bits as it is
written and read back, and attention over it.

Cache: uint8 [pages, heads, page / 16, 17 d], a record of 17 d bytes for 16
tokens of a head: keys (8 d bytes), values (8 d), the keys' scales (d / 2), the
values' scales (d / 2).  A value is an e2m1 code (sign, 0 .5 1 1.5 2 3 4 6) times
the scale 2^(e - 127) of its 32 columns.  Key (t, c) is in byte t d/2 + c/2, the
even column in the low half; value (t, c) in byte ((t/4 * 16 + n) * 4 + t%4) d/32 +
r/2 with n, r = divmod(c, d/16); key scale (t, c/32) at t d/32 + c/32, value scale at
(t/4 * d/32 + c/32) * 4 + t%4.

``run`` computes the plain form (elementary torch operations in fp32, angles in 64
bits), or the library's calls where ``own`` is set.  ``exact`` is the definition
in 64 bits.
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-5
_DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}


# ---- cases ---------------------------------------------------------------

def listed():
    return [
        # one token of a 7B-shaped decoder, no norm: latency
        dict(name="rope_token_7b", op="rope", rows=1, hq=32, hkv=32, d=128, rot=128, norm=False, interleaved=False,
             far=4096, x="f32", y="f32"),
        # partial rotation of neighbouring columns, few heads of an odd width, positions far out
        dict(name="rope_ragged", op="rope", rows=777, hq=7, hkv=1, d=80, rot=40, norm=True, interleaved=True,
             far=1000000, x="f32", y="bf16"),
        # a prompt of a Mistral-7B-shaped decoder, head norms
        dict(name="rope_prompt_mistral", op="rope", rows=4096, hq=32, hkv=8, d=128, rot=128, norm=True,
             interleaved=False, far=32768, x="bf16", y="bf16"),
        # 16 decoding sequences, each a token into its own page
        dict(name="cache_decode_16", op="cache", rows=16, heads=8, d=128, page=64, x="bf16"),
        # narrow heads, pages of 48, fp32 projections
        dict(name="cache_ragged", op="cache", rows=333, heads=3, d=64, page=48, x="f32"),
        # a 7B-shaped prompt
        dict(name="cache_prompt_7b", op="cache", rows=4096, heads=32, d=128, page=16, x="bf16"),
        # one token of one sequence: latency
        dict(name="attn_token_mistral", op="attn", B=1, nq=0, ctx=1000, ratio=1.0, hq=32, hkv=8, d=128, page=16,
             window=0, x="bf16"),
        # a batch of 7B-shaped sequences (a key head for every query head), lengths 200 to 4096
        dict(name="attn_decode_7b", op="attn", B=16, nq=0, ctx=4096, ratio=0.05, hq=32, hkv=32, d=128, page=64,
             window=0, x="bf16"),
        # a serving batch with long contexts
        dict(name="attn_decode_long", op="attn", B=32, nq=0, ctx=16384, ratio=0.25, hq=32, hkv=8, d=128, page=64,
             window=0, x="bf16"),
        # 20 heads on one key head, fp32 rows for a projection that takes those
        dict(name="attn_decode_shared", op="attn", B=3, nq=0, ctx=20001, ratio=0.3, hq=20, hkv=1, d=64, page=128,
             window=0, x="f32"),
        # chunks of prompts onto what is cached already, wide heads, a sliding window
        dict(name="attn_chunk_window", op="attn", B=5, nq=301, ctx=3001, ratio=0.1, hq=8, hkv=2, d=256, page=32,
             window=1024, x="f32"),
        # a whole prompt
        dict(name="attn_prompt_mistral", op="attn", B=1, nq=4096, ctx=0, ratio=1.0, hq=32, hkv=8, d=128, page=64,
             window=0, x="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    op = rng.choice(("rope", "cache", "attn", "attn"))
    x = rng.choice(("f32", "bf16"))
    if op == "rope":
        d = rng.choice((64, 72, 80, 96, 112, 128, 256))
        hkv = _log(rng, 1, 32)
        hq = hkv * rng.choice((1, 1, 3, 4, 7, 8)) if hkv <= 8 else hkv
        return dict(op=op, rows=_log(rng, 1, min(4096, 4096 * 5120 // ((hq + hkv) * d))), hq=hq, hkv=hkv, d=d,
                    rot=rng.choice((d, d, d // 16 * 8)), norm=rng.random() < 0.5, interleaved=rng.random() < 0.4,
                    far=rng.choice((4096, 131072, 1000000)), x=x, y=rng.choice(("f32", "bf16")))
    d, page = rng.choice((64, 128, 128, 256)), rng.choice((16, 32, 48, 64, 128, 256))
    if op == "cache":
        heads = _log(rng, 1, 40)
        return dict(op=op, rows=_log(rng, 1, min(4096, 2048 * 4096 // (heads * d))), heads=heads, d=d, page=page, x=x)
    hkv = _log(rng, 1, 40)
    hq = hkv * rng.choice((1, 2, 4, 5, 8, 20)) if hkv <= 8 else hkv
    ratio, window = rng.choice((1.0, 0.3, 0.05)), rng.choice((0, 0, 0, 100, 1024))
    B = _log(rng, 1, 64)
    if rng.random() < 0.6:  # one token for each sequence
        ctx = _log(rng, 1, min(32768, 32 * 16384 * 8 * 128 // 2 // (B * hkv * d)))
        return dict(op=op, B=B, nq=0, ctx=ctx, ratio=ratio, hq=hq, hkv=hkv, d=d, page=page, window=window, x=x)
    B = min(B, 16)
    nq = _log(rng, 2, min(2048, 4096 * 4096 // (B * hq * d)))
    ctx = _log(rng, 1, min(8192, 32 * 4096 * 2048 // (B * hq * nq))) - 1
    return dict(op=op, B=B, nq=nq, ctx=ctx, ratio=ratio, hq=hq, hkv=hkv, d=d, page=page, window=window, x=x)


def _lengths(case):
    """(queries, tokens) of each sequence, from the longest to the shortest: by the case alone."""
    B = case["B"]
    f = [case["ratio"] ** (i / max(1, B - 1)) for i in range(B)]
    nq = [max(1, round(case["nq"] * v)) for v in f]
    if case["nq"] == 0:
        return nq, [max(1, round(case["ctx"] * v)) for v in f]
    return nq, [round(case["ctx"] * v) + n for v, n in zip(f, nq)]


# ---- the format ------------------------------------------------------------

def _codes(x):
    """Plain form: fp32 x [..., d] -> (codes 0..15 of its values, scale bytes [..., d / 32])."""
    b = x.reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    a = b.abs().amax(dim=-1)
    f, e = torch.frexp(a)  # a = f 2^e, f in [0.5, 1): 6 = 0.75 * 2^3
    e = torch.where(a == 0, torch.zeros_like(e), (e - 3 + (f > 0.75).int()).clamp(-125, 125))
    v = torch.ldexp(b, -e[..., None])
    m = v.abs()
    # the borders between neighbouring values; a tie goes to the even code
    code = ((m > 0.25).int() + (m >= 0.75).int() + (m > 1.25).int() + (m >= 1.75).int() + (m > 2.5).int()
            + (m >= 3.5).int() + (m > 5.0).int())
    code = code + 8 * torch.signbit(v).int()
    return code.to(torch.uint8).view(x.shape), (e + 127).to(torch.uint8)


def _pack(codes):
    return codes[..., 0::2] | (codes[..., 1::2] << 4)


def _records(k, v):
    """fp32 keys and values [..., 16, d] -> records [..., 17 d]."""
    d, lead = k.shape[-1], k.shape[:-2]
    kc, ks = _codes(k)
    vc, vs = _codes(v)
    vb = _pack(vc).view(*lead, 4, 4, 16, d // 32).transpose(-3, -2)  # [.., t/4, n, t%4, bytes]
    vs = vs.view(*lead, 4, 4, d // 32).transpose(-2, -1)
    return torch.cat([_pack(kc).reshape(*lead, -1), vb.reshape(*lead, -1), ks.reshape(*lead, -1),
                      vs.reshape(*lead, -1)], dim=-1)


_E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _value(b, scales, shape):
    """Packed bytes [..., d / 2] and scale bytes [..., d / 32] -> fp32 [..., d]."""
    table = torch.tensor(_E2M1 + tuple(-t for t in _E2M1), device=b.device)
    code = torch.stack([b & 15, b >> 4], dim=-1).view(*shape[:-1], shape[-1] // 32, 32)
    s = torch.ldexp(torch.ones_like(scales, dtype=torch.float32), scales.int() - 127)
    return (table[code.long()] * s[..., None]).view(shape)


def _unpack(rec, d):
    """Records [..., 17 d] -> fp32 keys and values [..., 16, d]."""
    lead = rec.shape[:-1]
    kb, vb, ks, vs = rec.split([8 * d, 8 * d, d // 2, d // 2], dim=-1)
    vb = vb.reshape(*lead, 4, 16, 4, d // 32).transpose(-3, -2).reshape(*lead, 16, d // 2)
    vs = vs.reshape(*lead, 4, d // 32, 4).transpose(-2, -1).reshape(*lead, 16, d // 32)
    shape = (*lead, 16, d)
    return (_value(kb.reshape(*lead, 16, d // 2), ks.reshape(*lead, 16, d // 32), shape), _value(vb, vs, shape))


# ---- inputs ------------------------------------------------------------------

def _heads(g, shape):
    """Keys or values: normal, one column in 16 four times as large."""
    x = torch.randn(shape, generator=g, device="cuda")
    d = shape[-1]
    x[..., torch.randperm(d, generator=g, device="cuda")[: d // 16]] *= 4.0
    return x


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    s = dict(case)
    d, dt = case["d"], _DTYPE[case["x"]]
    if case["op"] == "rope":
        rows, hq, hkv = case["rows"], case["hq"], case["hkv"]
        s["qkv"] = _heads(g, (rows, hq + 2 * hkv, d)).to(dt).view(rows, -1)
        first = int(torch.randint(0, case["far"], (1,), generator=g, device="cuda"))
        s["pos"] = (first + torch.arange(rows, device="cuda")).to(torch.int32)
        r = torch.arange(0, case["rot"], 2, device="cuda", dtype=torch.float64) / max(1, case["rot"])
        s["freq"] = (10000.0 ** -r).float()
        gains = 1.0 + 0.1 * torch.randn((2, d), generator=g, device="cuda")
        s["gq"], s["gk"] = (gains[0].clone(), gains[1].clone()) if case["norm"] else (None, None)
        s["q"] = torch.empty((rows, hq, d), dtype=_DTYPE[case["y"]], device="cuda")
        s["k"] = torch.empty((rows, hkv, d), dtype=_DTYPE[case["y"]], device="cuda")
        return s
    page = case["page"]
    if case["op"] == "cache":
        rows, heads = case["rows"], case["heads"]
        s["k"], s["v"] = (_heads(g, (rows, heads, d)).to(dt) for _ in range(2))
        pages = 2 * ((rows + page - 1) // page) + 1
        s["cache"] = torch.zeros((pages, heads, page // 16, 17 * d), dtype=torch.uint8, device="cuda")
        # a prompt's consecutive tokens in scattered pages, or (few rows) one token each in pages of its own
        at = torch.randperm(pages, generator=g, device="cuda")
        t = torch.arange(rows, device="cuda") + int(torch.randint(0, page, (1,), generator=g, device="cuda"))
        s["slots"] = (at[t // page] * page + t % page).to(torch.int32)
        s["rk"], s["rv"] = (torch.empty((rows, heads, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        return s
    B, hq, hkv = case["B"], case["hq"], case["hkv"]
    nq, lens = _lengths(case)
    order = torch.randperm(B, generator=g, device="cuda").tolist()
    nq, lens = [nq[i] for i in order], [lens[i] for i in order]
    width = (max(lens) + page - 1) // page
    need = [(n + page - 1) // page for n in lens]
    pages = sum(need) + 3
    ids = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    s["table"] = torch.full((B, width), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b in range(B):
        s["table"][b, : need[b]] = ids[at : at + need[b]]
        at += need[b]
    shape = (pages, hkv, page // 16, 16, d)
    s["cache"] = _records(_heads(g, shape), _heads(g, shape))
    rows = sum(nq)
    s["qrows"] = (1.5 * torch.randn((rows, hq, d), generator=g, device="cuda")).to(dt)
    s["lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
    starts = [sum(nq[:b]) for b in range(B + 1)]
    s["q_start"] = torch.tensor(starts, dtype=torch.int32, device="cuda") if case["nq"] else None
    s["most"] = max(nq)
    s["out"] = torch.empty((rows, hq, d), dtype=dt, device="cuda")
    s["scratch"] = torch.zeros(64 << 20, dtype=torch.uint8, device="cuda")  # held once for all calls
    return s


# ---- one pass ------------------------------------------------------------------

def _run_own(s):
    import paper_2404_08763_amd as P

    if s["op"] == "rope":
        return list(P.qk_norm_rope(s["qkv"], s["hq"], s["hkv"], s["d"], s["pos"], s["freq"], norm=s["norm"],
                                   gain_q=s["gq"], gain_k=s["gk"], eps=EPS, interleaved=s["interleaved"],
                                   out=(s["q"], s["k"])))
    if s["op"] == "cache":
        P.kv_write(s["cache"], s["k"], s["v"], s["slots"])
        return list(P.kv_read(s["cache"], s["slots"], out=(s["rk"], s["rv"])))
    return P.kv_attention(s["qrows"], s["cache"], s["table"], s["lens"], q_start=s["q_start"], window=s["window"],
                          out=s["out"], ws=s["scratch"])


def _rotate(x, s, gain):
    """x [rows, heads, d] fp32."""
    if s["norm"]:
        x = x / torch.sqrt((x * x).mean(dim=-1, keepdim=True) + EPS) * gain
    rot = s["rot"]
    if rot == 0:
        return x
    a = s["pos"].double()[:, None] * s["freq"].double()
    c, w = torch.cos(a).float()[:, None], torch.sin(a).float()[:, None]
    if s["interleaved"]:
        lo, hi = x[..., 0:rot:2], x[..., 1:rot:2]
        y = torch.stack([lo * c - hi * w, hi * c + lo * w], dim=-1).flatten(-2)
    else:
        lo, hi = x[..., : rot // 2], x[..., rot // 2 : rot]
        y = torch.cat([lo * c - hi * w, hi * c + lo * w], dim=-1)
    return torch.cat([y, x[..., rot:]], dim=-1)


def run(s):
    if own:
        return _run_own(s)
    d = s["d"]
    if s["op"] == "rope":
        x = s["qkv"].float().view(s["rows"], -1, d)
        hq, hkv, dt = s["hq"], s["hkv"], _DTYPE[s["y"]]
        return [_rotate(x[:, :hq], s, s["gq"]).to(dt), _rotate(x[:, hq : hq + hkv], s, s["gk"]).to(dt)]
    if s["op"] == "cache":
        rows, heads, page = s["rows"], s["heads"], s["page"]
        slot = s["slots"].long()
        p, grp, t = slot // page, slot % page // 16, slot % 16
        kc, ks = _codes(s["k"].float())
        vc, vs = _codes(s["v"].float())
        # the bytes of a row in its record: as in _records
        rec = s["cache"]
        n, m = d // 2, d // 32
        c = torch.arange(n, device=rec.device)
        e = torch.arange(m, device=rec.device)
        kat, vat = t[:, None] * n + c, ((t[:, None] // 4 * 16 + c // m) * 4 + t[:, None] % 4) * m + c % m + 8 * d
        ksat, vsat = t[:, None] * m + e + 16 * d, (t[:, None] // 4 * m + e) * 4 + t[:, None] % 4 + 16 * d + n
        at = torch.cat([kat, vat, ksat, vsat], dim=1)[:, None]
        h = torch.arange(heads, device=rec.device)[None, :, None]
        here = (p[:, None, None], h, grp[:, None, None], at)
        rec[here] = torch.cat([_pack(kc), _pack(vc), ks, vs], dim=-1)
        kb, vb, ks, vs = rec[here].split([n, n, m, m], dim=-1)
        shape = (rows, heads, d)
        return [_value(kb, ks, shape).to(torch.bfloat16), _value(vb, vs, shape).to(torch.bfloat16)]
    B, hq, hkv, most = s["B"], s["hq"], s["hkv"], s["most"]
    rec = s["cache"][s["table"].clamp(min=0).long()]  # [B, pages, heads, page / 16, 17 d]
    rec = rec.transpose(1, 2).reshape(B * hkv, -1, 17 * d)
    k, v = (t.view(B * hkv, -1, d) for t in _unpack(rec, d))
    L, G = k.shape[1], hq // hkv
    lens = s["lens"].long()
    ar = torch.arange(B, device=lens.device)
    start = s["q_start"].long() if s["q_start"] is not None else torch.arange(B + 1, device=lens.device)
    nq = start[1:] - start[:-1]
    i = torch.arange(most, device=lens.device)
    at = (start[:-1, None] + i).clamp(max=s["qrows"].shape[0] - 1)
    q = s["qrows"].float()[at].view(B, most, hkv, G, d).transpose(1, 2).reshape(B * hkv, most * G, d)
    z = torch.bmm(q, k.transpose(1, 2).contiguous()).mul_(1.0 / math.sqrt(d)).view(B, hkv, most, G, L)
    pos = (lens - nq)[:, None] + i  # [B, most]
    j = torch.arange(L, device=lens.device)
    seen = j <= pos[..., None]
    if s["window"]:
        seen = seen & (j > pos[..., None] - s["window"])
    z.masked_fill_(~seen[:, None, :, None], -math.inf)
    z = z.sub_(z.amax(dim=-1, keepdim=True)).exp_()
    z = z.div_(z.sum(dim=-1, keepdim=True))
    o = torch.bmm(z.view(B * hkv, most * G, L), v).view(B, hkv, most, G, d).transpose(1, 2).reshape(B, most, hq, d)
    b = torch.repeat_interleave(ar, nq, output_size=s["qrows"].shape[0])
    r = torch.arange(s["qrows"].shape[0], device=lens.device) - start[b]
    return o[b, r].to(_DTYPE[s["x"]])


# ---- what a pass cannot do without -----------------------------------------------

def work(case):
    d, xb = case["d"], 4 if case["x"] == "f32" else 2
    if case["op"] == "rope":
        n = case["rows"] * (case["hq"] + case["hkv"]) * d
        yb = 4 if case["y"] == "f32" else 2
        return {"bytes": n * (xb + yb) + 4 * case["rows"] + 2 * case["rot"], "flops": n * (7 if case["norm"] else 3)}
    if case["op"] == "cache":
        n = case["rows"] * case["heads"] * 2
        held = n * (d // 2 + d // 32)
        return {"bytes": n * d * xb + 2 * held + n * d * 2 + 8 * case["rows"], "flops": 4 * n * d}
    nq, lens = _lengths(case)
    keys = pairs = 0
    w = case["window"] or 1 << 30
    for n, length in zip(nq, lens):
        keys += length - max(0, length - n + 1 - w)
        pairs += sum(min(length - n + i + 1, w) for i in range(n))
    rows = sum(nq)
    held = keys * case["hkv"] * (d + d // 16)
    return {"bytes": held + 2 * rows * case["hq"] * d * xb + 4 * sum((t + case["page"] - 1) // case["page"] for t in lens),
            "flops": 4 * d * case["hq"] * pairs}


# ---- the definition in 64 bits -----------------------------------------------------

def _nearest(x):
    """The values that 4 bits hold of x [.., d], in 64 bits."""
    b = x.double().unflatten(-1, (-1, 32))
    top = b.abs().max(dim=-1, keepdim=True).values
    e = torch.ceil(torch.log2(torch.clamp(top, min=1e-300) / 6.0)).clamp(-125, 125)
    u = b / torch.exp2(e)
    # steps of 0.5 below 2, of 1 below 4, of 2 up to 6; round takes ties to the even one
    step = torch.where(u.abs() < 2, 0.5, torch.where(u.abs() < 4, 1.0, 2.0)).double()
    return (torch.clamp(torch.round(u / step) * step, -6, 6) * torch.exp2(e)).flatten(-2)


def _held(cache, d, head, ids):
    """Keys and values [tokens, d] in 64 bits of a head in the pages `ids`."""
    rec = cache[ids, head].reshape(-1, 17 * d)
    tok = torch.arange(rec.shape[0] * 16, device=rec.device)[:, None]
    rows, t = tok // 16, tok % 16
    c = torch.arange(d, device=rec.device)[None]
    got = []
    for at, scale in ((t * (d // 2) + c // 2, 16 * d + t * (d // 32) + c // 32),
                      (8 * d + ((t // 4 * 16 + c // (d // 16)) * 4 + t % 4) * (d // 32) + c % (d // 16) // 2,
                       16 * d + d // 2 + (t // 4 * (d // 32) + c // 32) * 4 + t % 4)):
        code = (rec[rows, at].int() >> (4 * (c % 2))) & 15
        ex, man = (code >> 1) & 3, (code & 1).double()
        mag = torch.where(ex == 0, 0.5 * man, (1 + 0.5 * man) * torch.exp2(ex.double() - 1))
        got.append(mag * (1.0 - 2.0 * (code >> 3).double()) * torch.exp2(rec[rows, scale].double() - 127))
    return got


def exact(case, seed):
    s = prepare(case, seed)
    d = case["d"]
    if case["op"] == "cache":
        return [_nearest(s["k"]), _nearest(s["v"])]
    if case["op"] == "rope":
        x = s["qkv"].double().unflatten(1, (-1, d))
        half = case["rot"] // 2
        turn = torch.polar(torch.ones(1, dtype=torch.float64, device="cuda"), s["pos"].double()[:, None] * s["freq"].double())
        got = []
        for part, gain in ((x[:, : case["hq"]], s["gq"]), (x[:, case["hq"] : case["hq"] + case["hkv"]], s["gk"])):
            y = part.clone()
            if case["norm"]:
                y = y * torch.rsqrt(y.square().sum(dim=-1, keepdim=True) / d + EPS) * gain.double()
            i = torch.arange(half, device="cuda")
            one, two = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + half)
            z = torch.complex(y[..., one], y[..., two]) * turn[:, None]
            y[..., one], y[..., two] = z.real, z.imag
            got.append(y)
        return got
    G = case["hq"] // case["hkv"]
    lens = s["lens"].tolist()
    start = s["q_start"].tolist() if s["q_start"] is not None else list(range(case["B"] + 1))
    out = torch.empty(s["qrows"].shape, dtype=torch.float64, device="cuda")
    for b, n in enumerate(lens):
        ids = s["table"][b, : (n + case["page"] - 1) // case["page"]].long()
        rows = slice(start[b], start[b + 1])
        count = start[b + 1] - start[b]
        pos = torch.arange(n - count, n, device="cuda")[:, None]
        j = torch.arange(n, device="cuda")[None]
        hidden = (j > pos) if not case["window"] else (j > pos) | (pos - j >= case["window"])
        for h in range(case["hkv"]):
            k, v = (t[:n] for t in _held(s["cache"], d, h, ids))
            kt = k.t().contiguous()
            for one in range(h * G, h * G + G):
                z = torch.mm(s["qrows"][rows, one].double(), kt) * d ** -0.5
                out[rows, one] = torch.mm(torch.softmax(z.masked_fill(hidden, -math.inf), dim=1), v)
    return out
