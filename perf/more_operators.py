"""Performance cases of 8-bit rows: the norm and the activation that make them, and the product of 8-bit integers
that takes them (projections of prompts and of decode steps with weights and activations in 8 bits).

Each case is one pass through one operator.  Fields of a case:
  op       "norm"     residual addition and root-mean-square norm of rows; out "q8": the normed rows as 8-bit codes
                      with a scale a row, "16": in the rows' own type, "both"
           "quant"    rows as 8-bit codes with a scale a row: of x itself, or of act(gate) * up, the two halves of
                      rows as a fused projection leaves them
           "linear"   8-bit rows [rows][k] times 8-bit weights [n][k] with a scale a row and a scale an output
  norm:    rows, d, add (a residual is added and handed on), gain, out
  quant:   rows, d, act ("none", "silu", "gelu")
  linear:  rows, n, k, bias
8-bit outputs are returned as the values that they stand for, in 32 bits, which a pass reads back.
"""
from __future__ import annotations

import math

import torch

own = False

_DT = {"bf16": torch.bfloat16, "f16": torch.float16}
_EPS = 1e-6


def _norm(name, rows, d, **kw):
    return {"name": name, "op": "norm", "rows": rows, "d": d, "add": True, "gain": True, "out": "q8", "dtype": "bf16", **kw}


def _quant(name, rows, d, act, **kw):
    return {"name": name, "op": "quant", "rows": rows, "d": d, "act": act, "dtype": "bf16", **kw}


def _linear(name, rows, n, k, **kw):
    return {"name": name, "op": "linear", "rows": rows, "n": n, "k": k, "bias": False, "dtype": "bf16", **kw}


def listed():
    return [
        # Smallest: one token of a small model before its projections; launch and latency.
        _norm("norm_1x1024", 1, 1024),
        # Batched decode, 4096 wide, before the sparse FFN: that takes 16-bit rows.
        _norm("norm_16x4096_out16", 16, 4096, out="16"),
        # Ragged: a prompt of 777 tokens, a width that fills no vector, fp16, both outputs, nothing added (a first layer).
        _norm("norm_777x3457_both_f16", 777, 3457, add=False, out="both", dtype="f16"),
        # Prompts of 2048 tokens, 8192 wide.
        _norm("norm_2048x8192", 2048, 8192),
        # Attention's output of a few decoding sequences, before the output projection.
        _quant("quant_7x4096", 7, 4096, "none"),
        # A GeGLU of odd width over a ragged prompt, fp16.
        _quant("quant_1111x9973_gelu_f16", 1111, 9973, "gelu", dtype="f16"),
        # Prompts of 2048 tokens through the widest SwiGLU.
        _quant("quant_2048x28672_silu", 2048, 28672, "silu"),
        # Smallest: a key/value projection of a small model, single stream.
        _linear("linear_1x512x1024", 1, 512, 1024),
        # Batched decode on the widest projection: the weights' bytes count.
        _linear("linear_16x28672x8192", 16, 28672, 8192),
        # A chunk of a prompt through the fused q, k, v projection of a 4096-wide layer.
        _linear("linear_512x6144x4096", 512, 6144, 4096),
        # Ragged: rows, outputs and inputs that fill no tile, fp16, a bias.
        _linear("linear_700x9973x3457_f16", 700, 9973, 3457, bias=True, dtype="f16"),
        # Largest: prompts of 4096 tokens through the widest projection.
        _linear("linear_4096x28672x8192", 4096, 28672, 8192),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A width: a multiple of 128 or 256 half of the time, else any number."""
    d, m = _log(rng, lo, hi), rng.choice([0, 0, 128, 256])
    return max(m, d // m * m) if m else d


def draw(rng):
    op = rng.choice(["norm", "norm", "quant", "quant", "linear", "linear", "linear"])
    c = {"op": op, "rows": rng.choice([_log(rng, 1, 64), _log(rng, 1, 4096)]), "dtype": rng.choice(["bf16", "bf16", "f16"])}
    if op == "norm":
        c.update(d=_width(rng, 64, 16384), add=rng.random() < 0.8, gain=rng.random() < 0.9, out=rng.choice(["q8", "q8", "16", "both"]))
        while c["rows"] * c["d"] > 2048 * 8192:
            c["rows"] = c["rows"] * 2 // 3
    elif op == "quant":
        c.update(d=_width(rng, 64, 28672), act=rng.choice(["none", "silu", "silu", "gelu"]))
        while c["rows"] * c["d"] > 2048 * 28672:
            c["rows"] = c["rows"] * 2 // 3
    else:
        c.update(n=_width(rng, 200, 28672), k=_width(rng, 128, 28672), bias=rng.random() < 0.3)
        while c["n"] * c["k"] > 28672 * 8192:
            c["n"] = c["n"] * 2 // 3
    return c


# ---------------------------------------------------------------------------
# Inputs, from the seed alone
# ---------------------------------------------------------------------------

def _gen(seed, stream):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 16 + stream)


def _randn(shape, seed, stream):
    return torch.randn(shape, generator=_gen(seed, stream), device="cuda")


def _hidden(rows, d, seed, stream, dt):
    """Rows of a residual stream: a few channels stand out, and some tokens are louder than others."""
    x = _randn((rows, d), seed, stream) * (0.5 + torch.rand((rows, 1), generator=_gen(seed, stream + 1), device="cuda"))
    x[:, torch.randperm(d, generator=_gen(seed, 15), device="cuda")[:max(1, d // 256)]] *= 20.0
    return x.to(dt)


def _weights(c, seed):
    out = torch.empty((c["n"], c["k"]), dtype=_DT[c["dtype"]], device="cuda")
    g = _gen(seed, 0)
    for r in range(0, c["n"], 4096):   # fp32 draws a chunk of rows at a time
        m = min(4096, c["n"] - r)
        out[r:r + m] = torch.randn((m, c["k"]), generator=g, device="cuda") * 0.02
    return out


def _codes(p, factor=1.0):
    """Codes and scales of rows p (64 bits): c = 127 p / max|p| rounded half to even, sigma = max|p| factor / 127."""
    top = p.abs().amax(-1, keepdim=True)
    return torch.round(p * 127 / top.clamp(min=1e-300)).to(torch.int8), (top * factor / 127).float().squeeze(-1)


def prepare(c, seed):
    dt, st = _DT[c["dtype"]], {"case": c}
    if own:
        from paper_2607_27591_amd import prox
    if c["op"] == "linear":
        st["x"], st["sx"] = _codes(_hidden(c["rows"], c["k"], seed, 1, dt).double())
        st["bias"] = _randn((c["n"],), seed, 3).to(dt) if c["bias"] else None
        w = _weights(c, seed)
        if own:
            st["w"] = prox.pack_linear_w8(w)
            st["q"] = prox.new_rows_q8(c["rows"], c["k"])
            st["q"].codes.copy_(st["x"])
            st["q"].scales.copy_(st["sx"])
            st["y"] = torch.empty((c["rows"], c["n"]), dtype=dt, device="cuda")
        else:
            st["w"], st["sw"] = torch.empty((c["n"], c["k"]), dtype=torch.int8, device="cuda"), torch.empty(c["n"], device="cuda")
            for r in range(0, c["n"], 4096):
                st["w"][r:r + 4096], st["sw"][r:r + 4096] = _codes(w[r:r + 4096].double())
        return st
    rows, d = c["rows"], c["d"]
    if c["op"] == "norm":
        st["x"] = _hidden(rows, d, seed, 4, dt)
        st["y"] = _randn((rows, d), seed, 6).to(dt) if c["add"] else None
        st["gain"] = (1 + 0.3 * _randn((d,), seed, 7)).to(dt) if c["gain"] else None
    else:
        wide = d if c["act"] == "none" else 2 * d
        st["x"] = (1.5 * _randn((rows, wide), seed, 8)).to(dt)
    if own:
        st["q"] = prox.new_rows_q8(rows, d)
        st["values"] = torch.empty((rows, d), device="cuda")
        if c["op"] == "norm":
            st["r"] = torch.empty_like(st["x"]) if c["add"] else None
            st["out"] = torch.empty_like(st["x"])
    return st


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------

def _run_own(st, c):
    from paper_2607_27591_amd import prox
    if c["op"] == "linear":
        return {"y": prox.linear_w8(st["w"], st["q"], bias=st["bias"], y=st["y"])}
    res = {}
    if c["op"] == "norm":
        if c["add"]:
            res["r"] = st["r"]
        if c["out"] != "q8":
            res["out"] = st["out"]
        if c["out"] == "16":
            prox.rmsnorm(st["x"], st["y"], gain=st["gain"], eps=_EPS, residual=st["r"], out=st["out"])
            return res
        prox.rmsnorm_q8(st["x"], st["y"], gain=st["gain"], eps=_EPS, residual=st["r"], out=res.get("out"), q=st["q"])
    elif c["act"] == "none":
        prox.quant_q8(st["x"], q=st["q"])
    else:
        d = c["d"]
        prox.quant_q8(st["x"][:, :d], up=st["x"][:, d:], act=prox.SILU if c["act"] == "silu" else prox.GELU, q=st["q"])
    res["values"], res["scales"] = prox.read_q8(st["q"], out=st["values"]), st["q"].scales
    return res


def run(st):
    c = st["case"]
    if own:
        return _run_own(st, c)
    if c["op"] == "linear":
        y = torch.matmul(st["x"].float(), st["w"].float().t()) * st["sw"] * st["sx"][:, None]
        return {"y": (y if st["bias"] is None else y + st["bias"].float()).to(_DT[c["dtype"]])}
    x, res, factor = st["x"], {}, 1.0
    if c["op"] == "norm":
        if c["add"]:
            x = res["r"] = (x.float() + st["y"].float()).to(x.dtype)
        # In 64 bits: a code next to the border between two goes by the last bits of its row.
        p = x.double()
        factor = 1 / torch.sqrt(p.square().mean(-1, keepdim=True) + _EPS)
        if c["gain"]:
            p = p * st["gain"].double()
        if c["out"] != "q8":
            res["out"] = (p.float() * factor.float()).to(x.dtype)
        if c["out"] == "16":
            return res
    elif c["act"] == "none":
        p = x.double()
    else:
        g, u = x.double().split(c["d"], -1)
        p = u * (g / (1 + torch.exp(-g)) if c["act"] == "silu" else 0.5 * g * torch.erfc(-g * math.sqrt(0.5)))
        p = p.float().double()    # the activation, held in 32 bits, is what is quantised
    codes, scales = _codes(p, factor)
    res["values"], res["scales"] = codes.float() * scales[:, None], scales
    return res


# ---------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------

def work(c):
    if c["op"] == "linear":
        n, k, rows = c["n"], c["k"], c["rows"]
        return {"bytes": n * k + 4 * n + rows * (k + 4 + 2 * n) + (2 * n if c["bias"] else 0), "flops": 2.0 * rows * n * k}
    size = c["rows"] * c["d"]
    codes = size + 4 * c["rows"]
    back = codes + codes + 4 * size    # codes and scales written and read back, the values written
    if c["op"] == "quant":
        gated = c["act"] != "none"
        return {"bytes": (4 if gated else 2) * size + back, "flops": (9.0 if gated else 3.0) * size}
    bytes_ = 2 * size + (4 * size if c["add"] else 0) + (2 * c["d"] if c["gain"] else 0)
    bytes_ += (2 * size if c["out"] != "q8" else 0) + (back if c["out"] != "16" else 0)
    return {"bytes": bytes_, "flops": 7.0 * size}


# ---------------------------------------------------------------------------
# The same in 64 bits, from the definitions
# ---------------------------------------------------------------------------

def _exact_codes(p):
    """The integer nearest to 127 p / max|p| in each row, the even one of two, as fp64; and max|p|."""
    top = torch.maximum(p.max(1, keepdim=True).values, -p.min(1, keepdim=True).values)
    t = 127 * p / torch.where(top > 0, top, 1.0)
    low = torch.floor(t)
    up = (t - low > 0.5) | ((t - low == 0.5) & (torch.remainder(low, 2) == 1))
    return low + up.double(), top


def exact(c, seed):
    dt = _DT[c["dtype"]]
    if c["op"] == "linear":
        x, tx = _exact_codes(_hidden(c["rows"], c["k"], seed, 1, dt).double())
        tx = (tx / 127).float().double()
        w, y = _weights(c, seed), []
        for r in range(0, c["n"], 4096):
            q, tw = _exact_codes(w[r:r + 4096].double())
            y.append(torch.mm(x, q.t().contiguous()) * tx * (tw / 127).float().double().t())
        y = torch.cat(y, 1)
        if c["bias"]:
            y += _randn((c["n"],), seed, 3).to(dt).double()
        return {"y": y}
    rows, d, res = c["rows"], c["d"], {}
    if c["op"] == "norm":
        r = _hidden(rows, d, seed, 4, dt)
        if c["add"]:
            res["r"] = r.double() + _randn((rows, d), seed, 6).to(dt).double()
            r = res["r"].float().to(dt)       # what the norm is of: the residual as it is kept
        size = torch.linalg.vector_norm(r.double(), dim=1, keepdim=True)
        length = torch.hypot(size / math.sqrt(d), torch.full_like(size, math.sqrt(_EPS)))
        p = r.double()
        if c["gain"]:
            p = p * (1 + 0.3 * _randn((d,), seed, 7)).to(dt).double()
        if c["out"] != "q8":
            res["out"] = p / length
        if c["out"] == "16":
            return res
    else:
        length = 1.0
        x = (1.5 * _randn((rows, d if c["act"] == "none" else 2 * d), seed, 8)).to(dt).double()
        p = x[:, :d]
        if c["act"] == "silu":
            p = p * torch.sigmoid(p) * x[:, d:]
        elif c["act"] == "gelu":
            p = p * torch.special.ndtr(p) * x[:, d:]
        p = p.float().double()    # what is quantised: 32 bits
    codes, top = _exact_codes(p)
    scale = top / length / 127
    res["values"], res["scales"] = codes * scale, scale[:, 0]
    return res
