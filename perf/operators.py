"""The 8-bit operators' measured cases: RMSNorm with the residual's addition
and an 8-bit output, the SiLU gate with the CATS cutoff and an 8-bit output,
quantisation of weights and rows, and the linear layer on 8-bit operands with
a scale for each block of 128.

Format: e4m3 values q [rows, ld] with ld = the columns rounded up to 128 (zeros
behind them) and a scale for each 1 or 128 rows by 128 columns, fp32 ("f32") or a
power of two ("e8m0").  A block's scale is its largest magnitude over 448 (f32)
or the smallest power of two that brings it to 448 or less (e8m0), 1 for
a block of zeros; a value is q times its scale.

``run`` computes the plain form (elementary torch operations in fp32), or the
library's calls where ``own`` is set.  ``exact`` is the definition in 64 bits.
"""
from __future__ import annotations

import math

import torch

own = False

BLOCK = 128
TOP = 448.0
EPS = 1e-5


# ---- cases ---------------------------------------------------------------

def listed():
    return [
        # one token entering a block of a 7B-shaped decoder: latency
        dict(name="norm_decode_7b", op="norm", rows=1, d=4096, x="f32", residual=True, gain=True, scale="f32"),
        # the calibration tests' ragged width, no addition, unit gain
        dict(name="norm_ragged", op="norm", rows=777, d=2856, x="f32", residual=False, gain=False, scale="e8m0"),
        # a prompt of 4096 tokens, the projection's output in bf16 on an fp32 residual stream
        dict(name="norm_prompt_7b", op="norm", rows=4096, d=4096, x="bf16", residual=True, gain=True, scale="f32"),
        # one token's gate and up values of a 7B-shaped block, cutoff at about half of them
        dict(name="gate_decode_7b", op="gate", rows=1, m=11008, x="f32", t=0.15, scale="e8m0"),
        # a prompt's gate and up values of a Mistral-7B-shaped block
        dict(name="gate_prompt_mistral", op="gate", rows=2048, m=14336, x="bf16", t=0.15, scale="f32"),
        # rows of an odd width that no norm precedes (a projection's input)
        dict(name="quant_rows_ragged", op="quant", rows=333, cols=7001, block_rows=1, x="f32", scale="f32"),
        # a 7B-shaped block's weight, once per model
        dict(name="quant_weights_7b", op="quant", rows=11008, cols=4096, block_rows=128, x="bf16", scale="e8m0"),
        # Mistral-7B-shaped Q/K/V projection of one token
        dict(name="linear_qkv_1", op="linear", rows=1, k=4096, n=6144, residual=False, y="f32", scale="f32"),
        # 13B-shaped gate and up projection of 16 decoding rows
        dict(name="linear_gateup_16", op="linear", rows=16, k=5120, n=27648, residual=False, y="f32", scale="e8m0"),
        # a ragged block's down-projection (7001 neurons, padded to 7040) of a short prompt
        dict(name="linear_ragged_101", op="linear", rows=101, k=7001, n=2857, residual=True, y="f32", scale="f32"),
        # 7B-shaped gate and up projection of a prompt
        dict(name="linear_gateup_prompt", op="linear", rows=2048, k=4096, n=22016, residual=False, y="bf16", scale="f32"),
        # Mistral-7B-shaped down-projection of a long prompt into the residual stream
        dict(name="linear_down_prompt", op="linear", rows=4096, k=14336, n=4096, residual=True, y="f32", scale="e8m0"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A width over [lo, hi]: any, a multiple of 8 or a multiple of 128."""
    w = _log(rng, lo, hi)
    step = rng.choice((1, 8, 128))
    return max(step, w // step * step)


def draw(rng):
    op = rng.choice(("norm", "gate", "quant", "linear", "linear"))
    scale = rng.choice(("f32", "e8m0"))
    x = rng.choice(("f32", "bf16"))
    if op == "norm":
        d = _width(rng, 256, 8192)
        return dict(op=op, rows=_log(rng, 1, min(4096, 4096 * 4096 // d)), d=d, x=x, residual=rng.random() < 0.5,
                    gain=rng.random() < 0.5, scale=scale)
    if op == "gate":
        m = _width(rng, 256, 28672)
        return dict(op=op, rows=_log(rng, 1, min(4096, 1024 * 14336 // m)), m=m, x=x, t=rng.choice((0.0, 0.05, 0.15)),
                    scale=scale)
    if op == "quant":
        cols = _width(rng, 256, 14336)
        return dict(op=op, rows=_log(rng, 1, min(11008, 5504 * 4096 // cols)), cols=cols,
                    block_rows=rng.choice((1, 128)), x=x, scale=scale)
    k, n = _width(rng, 256, 14336), _width(rng, 256, 28672)
    most = 4096 * 4096 * 14336 // 2 // (k * n)  # half of the largest listed product
    return dict(op=op, rows=_log(rng, 1, max(1, min(4096, most))), k=k, n=n, residual=rng.random() < 0.5,
                y=rng.choice(("f32", "bf16")), scale=scale)


# ---- the format ------------------------------------------------------------

def _ld(cols):
    return (cols + BLOCK - 1) // BLOCK * BLOCK


_DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
_SCALE = {"f32": torch.float32, "e8m0": torch.float8_e8m0fnu}


def _blocks(x, block_rows):
    """x [rows, cols] with zeros up to whole blocks, as [row blocks, block_rows, column blocks, 128]."""
    rows, cols = x.shape
    up = (rows + block_rows - 1) // block_rows * block_rows
    x = torch.nn.functional.pad(x, (0, _ld(cols) - cols, 0, up - rows))
    return x.view(up // block_rows, block_rows, _ld(cols) // BLOCK, BLOCK)


def _quantise(x, block_rows, scale):
    """Plain form: fp32 x -> (q e4m3 [rows, ld], scale [row blocks, ld / 128])."""
    rows, cols = x.shape
    b = _blocks(x, block_rows)
    a = b.abs().amax(dim=(1, 3))
    if scale == "f32":
        s = torch.where(a == 0, torch.ones_like(a), (a / TOP).clamp(min=2.0 ** -126))
        stored = s
    else:
        f, e = torch.frexp(a)  # a = f 2^e, f in [0.5, 1): 448 = 0.875 * 2^9
        e = torch.where(a == 0, torch.zeros_like(e), (e - 9 + (f > 0.875).int()).clamp(min=-126))
        s = torch.ldexp(torch.ones_like(a), e)
        stored = (e + 127).to(torch.uint8).view(torch.float8_e8m0fnu)
    q = (b / s[:, None, :, None]).to(torch.float8_e4m3fn)
    return q.view(-1, _ld(cols))[:rows], stored


# ---- inputs ------------------------------------------------------------------

def _activations(g, rows, d):
    """Hidden vectors: normal, 1% of the channels 20 times as large."""
    x = torch.randn((rows, d), generator=g, device="cuda")
    x[:, torch.randperm(d, generator=g, device="cuda")[: max(1, d // 100)]] *= 20.0
    return x


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    op, rows = case["op"], case["rows"]
    s = dict(case)
    if op == "linear":
        k, n, stype = case["k"], case["n"], case["scale"]
        s["xq"], s["xs"] = _quantise(_activations(g, rows, k), 1, stype)
        s["wq"], s["ws"] = _quantise(torch.randn((n, k), generator=g, device="cuda") * 0.02, BLOCK, stype)
        s["r"] = torch.randn((rows, n), generator=g, device="cuda").to(_DTYPE[case["y"]]) if case["residual"] else None
        s["out"] = torch.empty((rows, n), dtype=_DTYPE[case["y"]], device="cuda")
        # scratch memory that a serving program holds once for all its calls
        s["scratch"] = torch.zeros(128 << 20, dtype=torch.uint8, device="cuda")
        return s
    if op == "norm":
        cols = case["d"]
        s["in"] = _activations(g, rows, cols).to(_DTYPE[case["x"]])
        s["r"] = torch.randn((rows, cols), generator=g, device="cuda") if case["residual"] else None
        s["g"] = 1.0 + 0.1 * torch.randn(cols, generator=g, device="cuda") if case["gain"] else None
        s["sum"] = torch.empty((rows, cols), device="cuda") if case["residual"] else None
        up = 1
    elif op == "gate":
        cols, up = case["m"], 1
        s["in"] = (1.3 * torch.randn((rows, 2 * cols), generator=g, device="cuda")).to(_DTYPE[case["x"]])
    else:
        cols, up = case["cols"], case["block_rows"]
        v = _activations(g, rows, cols) if up == 1 else 0.02 * torch.randn((rows, cols), generator=g, device="cuda")
        s["in"] = v.to(_DTYPE[case["x"]])
    s["q"] = torch.empty((rows, _ld(cols)), dtype=torch.float8_e4m3fn, device="cuda")
    s["s"] = torch.empty(((rows + up - 1) // up, _ld(cols) // BLOCK), dtype=_SCALE[case["scale"]], device="cuda")
    return s


# ---- one pass ------------------------------------------------------------------

def _run_own(s):
    import paper_2404_08763_amd as P

    if s["op"] == "linear":
        return P.linear_fp8(s["xq"], s["xs"], s["wq"], s["ws"], residual=s["r"], out=s["out"], ws=s["scratch"])
    out = (s["q"], s["s"])
    if s["op"] == "norm":
        P.rmsnorm_fp8(s["in"], residual=s["r"], gain=s["g"], eps=EPS, out=out, sum_out=s["sum"])
        return list(out) + ([s["sum"]] if s["sum"] is not None else [])
    if s["op"] == "gate":
        P.silu_mul_fp8(s["in"], t=s["t"], out=out)
    else:
        P.quantize_fp8(s["in"], block_rows=s["block_rows"], out=out)
    return list(out)


def run(s):
    if own:
        return _run_own(s)
    if s["op"] == "linear":
        rows, ld = s["xq"].shape
        n = s["wq"].shape[0]
        x = s["xq"].float().view(rows, -1, BLOCK) * s["xs"].float()[:, :, None]
        w = s["wq"].float().view(n, -1, BLOCK) * s["ws"].float().repeat_interleave(BLOCK, dim=0)[:n, :, None]
        y = x.view(rows, ld) @ w.view(n, ld).t()
        if s["r"] is not None:
            y = y + s["r"].float()
        return y.to(_DTYPE[s["y"]])
    x = s["in"].float()
    if s["op"] == "norm":
        if s["r"] is not None:
            x = x + s["r"]
        y = x / torch.sqrt((x * x).mean(dim=1, keepdim=True) + EPS)
        if s["g"] is not None:
            y = y * s["g"]
        return list(_quantise(y, 1, s["scale"])) + ([x] if s["r"] is not None else [])
    if s["op"] == "gate":
        m = s["m"]
        z = x[:, :m].double()  # (in 64 bits: values next to the cutoff)
        v = z / (1.0 + torch.exp(-z))
        h = torch.where(v.abs() < s["t"], torch.zeros_like(v), v).float() * x[:, m:]
        return list(_quantise(h, 1, s["scale"]))
    return list(_quantise(x, s["block_rows"], s["scale"]))


# ---- what a pass cannot do without -----------------------------------------------

def work(case):
    rows, sb = case["rows"], 4 if case["scale"] == "f32" else 1
    if case["op"] == "linear":
        k, n, yb = _ld(case["k"]), case["n"], 4 if case["y"] == "f32" else 2
        scales = (rows + (n + BLOCK - 1) // BLOCK) * (k // BLOCK) * sb
        return {"bytes": rows * k + n * k + scales + rows * n * yb * (2 if case["residual"] else 1),
                "flops": 2 * rows * n * case["k"]}
    xb = 4 if case["x"] == "f32" else 2
    if case["op"] == "norm":
        d = case["d"]
        moved = rows * d * (xb + (8 if case["residual"] else 0)) + (4 * d if case["gain"] else 0)
        return {"bytes": moved + rows * _ld(d) + rows * _ld(d) // BLOCK * sb, "flops": 6 * rows * d}
    if case["op"] == "gate":
        m = case["m"]
        return {"bytes": 2 * rows * m * xb + rows * _ld(m) + rows * _ld(m) // BLOCK * sb, "flops": 8 * rows * m}
    c, up = case["cols"], case["block_rows"]
    return {"bytes": rows * c * xb + rows * _ld(c) + (rows + up - 1) // up * _ld(c) // BLOCK * sb,
            "flops": 3 * rows * c}


# ---- the definition in 64 bits -----------------------------------------------------

def _e4m3(v):
    """Nearest e4m3 value (ties to even) of finite v, |v| <= 448, in float64."""
    e = (torch.frexp(v)[1] - 1).clamp(min=-6)
    step = torch.ldexp(torch.ones_like(v), e - 3)
    return torch.round(v / step) * step


def _exact_quantised(v, up, scale):
    rows, cols = v.shape
    nr, nc = (rows + up - 1) // up, _ld(cols) // BLOCK
    full = torch.zeros((nr * up, nc * BLOCK), dtype=torch.float64, device=v.device)
    full[:rows, :cols] = v
    tiles = full.reshape(nr, up, nc, BLOCK).transpose(1, 2)  # [nr, nc, up, 128]
    top = tiles.abs().flatten(2).max(dim=2).values
    if scale == "f32":
        s = torch.clamp(top / TOP, min=2.0 ** -126)
    else:
        s = torch.exp2(torch.clamp(torch.ceil(torch.log2(top / TOP)), min=-126.0))
    s = torch.where(top > 0, s, torch.ones_like(s))
    q = _e4m3(tiles / s[:, :, None, None]).transpose(1, 2).reshape(nr * up, nc * BLOCK)
    return [q[:rows], s]


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "linear":
        rows, n = case["rows"], case["n"]
        y = torch.zeros((rows, n), dtype=torch.float64, device="cuda")
        xs, ws = s["xs"].float().double(), s["ws"].float().double()
        of = torch.arange(n, device="cuda") // BLOCK
        for b in range(xs.shape[1]):
            part = slice(b * BLOCK, (b + 1) * BLOCK)
            xb = s["xq"][:, part].float().double() * xs[:, b:b + 1]
            wb = s["wq"][:, part].float().double() * ws[of, b][:, None]
            y += torch.mm(xb, wb.t())
        return y if s["r"] is None else y + s["r"].double()
    x = s["in"].double()
    if case["op"] == "norm":
        total = x if s["r"] is None else x + s["r"].double()
        y = total * torch.rsqrt(torch.linalg.vector_norm(total, dim=1, keepdim=True).square() / case["d"] + EPS)
        if s["g"] is not None:
            y = y * s["g"].double()
        return _exact_quantised(y, 1, case["scale"]) + ([] if s["r"] is None else [total])
    if case["op"] == "gate":
        gate, u = x.split(case["m"], dim=1)
        v = gate * torch.sigmoid(gate)
        return _exact_quantised(v * (v.abs() >= case["t"]) * u, 1, case["scale"])
    return _exact_quantised(x, case["block_rows"], case["scale"])
