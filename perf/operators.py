"""Performance cases of the attention half of a decoder layer at decode time: projections on INT4 weights,
the 4-bit paged key/value cache, and attention over it.

Each case is one pass through one operator.  Fields of a case:
  op       "linear"   x [batch][k] times INT4 weights [n][k] with group scales, plus a bias
           "append"   rotation of q and k, keys and values quantised into the paged cache, then the cached
                      values of the new tokens read back
           "attn"     attention of the new tokens over the paged cache
  linear:  n, k, batch, group, bias
  append, attn: seqs, new (new tokens of the longest sequence), ragged (the sequences have fewer: new tokens and
           lengths spread evenly), len (tokens of the longest sequence, the new ones included), q_heads, kv_heads,
           head_dim, group, page; append: rope ("half": channels i and i + dim / 2 turn together, "pairs": 2 i
           and 2 i + 1), rope_dim; attn: window (0: none)
"""
from __future__ import annotations

import math

import torch

own = False

_DT = {"bf16": torch.bfloat16, "f16": torch.float16}


def _linear(name, n, k, batch, **kw):
    return {"name": name, "op": "linear", "n": n, "k": k, "batch": batch, "group": 128, "bias": False,
            "dtype": "bf16", **kw}


def _kv(name, op, seqs, new, length, **kw):
    c = {"name": name, "op": op, "seqs": seqs, "new": new, "ragged": False, "len": length, "q_heads": 32,
         "kv_heads": 8, "head_dim": 128, "group": 64, "page": 64, "dtype": "bf16"}
    c.update({"rope": "half", "rope_dim": kw.get("head_dim", 128)} if op == "append" else {"window": 0})
    c.update(kw)
    return c


def listed():
    return [
        # Smallest: a key/value projection of a small model, single stream; launch and latency.
        _linear("linear_512x1024_b1", 512, 1024, 1),
        # The fused q, k, v projection (32 + 8 + 8 heads of 128) of a 4096-wide layer, single stream.
        _linear("linear_6144x4096_b1", 6144, 4096, 1),
        # The output projection of an 8192-wide layer, batched decode on a full matrix-core tile.
        _linear("linear_8192x8192_b16", 8192, 8192, 16),
        # Ragged: rows, inputs and batch that fill no tile, finer groups, fp16, a bias.
        _linear("linear_9973x3456_b7_f16", 9973, 3456, 7, group=64, bias=True, dtype="f16"),
        # Largest: the widest projection of the headline model at the largest batch of a call.
        _linear("linear_28672x8192_b64", 28672, 8192, 64),
        # Batched decode: one new token in each of 16 sequences.
        _kv("append_16x1", "append", 16, 1, 2050),
        # Prompts of unequal length entering the cache, fp16, half of each head's channels rotated in pairs.
        _kv("append_prompts_6x700_f16", "append", 6, 700, 700, ragged=True, q_heads=28, kv_heads=4, dtype="f16",
            rope="pairs", rope_dim=64, group=32, page=32),
        # Single-stream decode, ordinary context: latency.
        _kv("attn_1x1_ctx2000", "attn", 1, 1, 2000),
        # Single-stream decode over the longest context.
        _kv("attn_1x1_ctx131072", "attn", 1, 1, 131072, page=256),
        # Batched decode of 32 sequences of unequal length.
        _kv("attn_32x1_ctx8192", "attn", 32, 1, 8192, ragged=True),
        # Drafted tokens checked together: five queries a sequence, odd sizes, fp16, narrow heads, a window.
        _kv("attn_7x5_ctx4001_f16", "attn", 7, 5, 4001, ragged=True, q_heads=14, kv_heads=2, head_dim=64, group=32,
            page=32, window=1000, dtype="f16"),
        # A chunk of two prompts over their cached prefix.
        _kv("attn_2x512_ctx4096", "attn", 2, 512, 4096, group=128),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["linear", "linear", "append", "attn", "attn", "attn"])
    dtype = rng.choice(["bf16", "bf16", "f16"])
    if op == "linear":
        group = rng.choice([32, 64, 128, 128, 128, 256])
        n, k = _log(rng, 200, 28672), max(group, _log(rng, 512, 28672) // group * group)
        if rng.random() < 0.5:
            n = max(256, n // 256 * 256)
        while n * k > 8192 * 28672:
            n = int(n * 0.7)
        batch = 1 if rng.random() < 0.35 else _log(rng, 1, 64)
        return {"op": op, "n": n, "k": k, "batch": batch, "group": group, "bias": rng.random() < 0.3, "dtype": dtype}
    head_dim = rng.choice([64, 128, 128, 128, 256])
    group = rng.choice([g for g in (32, 64, 64, 128) if g <= head_dim])
    kv_heads = rng.choice([1, 2, 4, 8, 8])
    ratio = rng.choice([1, 2, 3, 4, 4, 5, 7, 8, 16])
    c = {"op": op, "q_heads": kv_heads * ratio, "kv_heads": kv_heads, "head_dim": head_dim, "group": group,
         "page": rng.choice([32, 64, 64, 128, 256, 96]), "dtype": dtype, "ragged": rng.random() < 0.6}
    if op == "append":
        if rng.random() < 0.5:
            c.update(seqs=_log(rng, 1, 64), new=_log(rng, 1, 6), len=_log(rng, 64, 8192))
        else:
            c.update(seqs=_log(rng, 1, 8), new=_log(rng, 16, 1024))
            c.update(len=c["new"] + rng.choice([0, _log(rng, 1, 4096)]))
        c.update(rope=rng.choice(["half", "half", "pairs"]), rope_dim=rng.choice([head_dim, head_dim, head_dim // 2]))
        while c["seqs"] * c["new"] * c["q_heads"] * head_dim > 4096 * 4096:
            c["seqs"] = (c["seqs"] + 1) // 2 if c["seqs"] > 1 else 1
            c["new"] = c["new"] * 2 // 3
    else:
        kind = rng.random()
        if kind < 0.6:     # single new tokens
            c.update(seqs=_log(rng, 1, 64), new=1, len=_log(rng, 1, 65536))
        elif kind < 0.8:   # drafted tokens
            c.update(seqs=_log(rng, 1, 16), new=_log(rng, 2, 16), len=_log(rng, 64, 16384))
        else:              # prompt chunks
            c.update(seqs=_log(rng, 1, 4), new=_log(rng, 64, 512), len=_log(rng, 512, 4096))
        c["window"] = rng.choice([0, 0, 0, _log(rng, 16, 4096)])
        while c["seqs"] * c["len"] * kv_heads * head_dim > 131072 * 8 * 128 and c["seqs"] > 1:
            c["seqs"] = c["seqs"] * 2 // 3
        while c["seqs"] * c["new"] * c["len"] * c["q_heads"] * head_dim > 2 * 512 * 4096 * 32 * 128:
            c["len"] = c["len"] * 2 // 3
    c["len"] = max(c["len"], c["new"])
    return c


# ---------------------------------------------------------------------------
# Inputs, from the seed alone
# ---------------------------------------------------------------------------

def _gen(seed, stream):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 16 + stream)


def _randn(shape, seed, stream, dtype):
    return torch.randn(shape, generator=_gen(seed, stream), device="cuda").to(dtype)


def _news(c):
    """New tokens of each sequence, and its tokens in the cache with them."""
    S, new, length = c["seqs"], c["new"], c["len"]
    if not c["ragged"] or S == 1:
        return [new] * S, [length] * S
    news = [max(1, new - s * new // S) for s in range(S)]
    return news, [max(news[s], length - s * (length - new) // S) for s in range(S)]


def _weights(c, seed):
    out = torch.empty((c["n"], c["k"]), dtype=_DT[c["dtype"]], device="cuda")
    g = _gen(seed, 0)
    for r in range(0, c["n"], 4096):   # fp32 draws a chunk of rows at a time
        m = min(4096, c["n"] - r)
        out[r:r + m] = torch.randn((m, c["k"]), generator=g, device="cuda") * 0.02
    return out


def _x(c, seed):
    # Inputs after a norm: a few channels stand out.
    x = torch.randn((c["batch"], c["k"]), generator=_gen(seed, 1), device="cuda")
    x[:, torch.randperm(c["k"], generator=_gen(seed, 2), device="cuda")[:max(1, c["k"] // 256)]] *= 20.0
    return x.to(_DT[c["dtype"]])


def _keys(shape, c, seed, stream):
    """Keys: some channels of each head carry larger values, alike in every token."""
    k = torch.randn(shape, generator=_gen(seed, stream), device="cuda")
    boost = 1 + 3 * (torch.rand(shape[1:], generator=_gen(seed, 15), device="cuda") < 0.04).float()
    return (k * boost).to(_DT[c["dtype"]])


def _rope_table(c, n_pos):
    """fp32 [n_pos][dim]: cosines of dim / 2 frequencies, then their sines; angles in 64 bits."""
    d = c["rope_dim"]
    f = 1e6 ** (-torch.arange(0, d, 2, dtype=torch.float64, device="cuda") / d)
    a = torch.arange(n_pos, dtype=torch.float64, device="cuda")[:, None] * f
    return torch.cat([a.cos(), a.sin()], 1).float().contiguous()


def _quantise(v, group):
    """The symmetric 4-bit quantiser: codes int8 and fp16 scales per group of the last axis."""
    v = v.double().unflatten(-1, (-1, group))
    s = (v.abs().amax(-1) / 7).float().clamp(max=65504).half()
    q = torch.round(v / s.double().clamp(min=1e-30)[..., None]).clamp(-7, 7)
    return torch.where(s[..., None] > 0, q, 0.0).to(torch.int8).flatten(-2), s


def _values(codes, scales):
    """What codes and scales stand for, in 32 bits (exact)."""
    v = codes.float().unflatten(-1, (scales.shape[-1], -1)) * scales.float()[..., None]
    return v.flatten(-2)


def _paging(c, seed):
    """(page table [seqs][pages a sequence], pages): every sequence's pages stand anywhere in the cache."""
    per = -(-c["len"] // c["page"])
    n = c["seqs"] * per + 3
    order = torch.randperm(n, generator=_gen(seed, 14), device="cuda")[:c["seqs"] * per]
    return order.to(torch.int32).view(c["seqs"], per).contiguous(), n


def prepare(c, seed):
    dt = _DT[c["dtype"]]
    st = {"case": c}
    if c["op"] == "linear":
        w = _weights(c, seed)
        st["x"] = _x(c, seed)
        st["bias"] = _randn((c["n"],), seed, 3, dt) if c["bias"] else None
        if own:
            from paper_2607_27591_amd import prox
            st["w4"] = prox.pack_linear_w4(w, c["group"])
            st["y"] = torch.empty((c["batch"], c["n"]), dtype=dt, device="cuda")
        else:
            st["codes"] = torch.empty((c["n"], c["k"]), dtype=torch.int8, device="cuda")
            st["scales"] = torch.empty((c["n"], c["k"] // c["group"]), dtype=torch.float16, device="cuda")
            for r in range(0, c["n"], 4096):
                st["codes"][r:r + 4096], st["scales"][r:r + 4096] = _quantise(w[r:r + 4096], c["group"])
        return st
    news, lens = _news(c)
    H, D, T = c["kv_heads"], c["head_dim"], sum(news)
    st["table"], n_pages = _paging(c, seed)
    st["kv_len"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
    st["cu_new"] = torch.tensor([sum(news[:s]) for s in range(c["seqs"] + 1)], dtype=torch.int32, device="cuda")
    st["q"] = _randn((T, c["q_heads"], D), seed, 4, dt)
    slots = n_pages * c["page"]
    if own:
        from paper_2607_27591_amd import prox
        st["cache"] = prox.new_kv_cache(n_pages, c["page"], H, D, dt, group=c["group"])
        st["seqs"] = prox.KVSeqs(st["kv_len"], st["table"], max_new=c["new"],
                                 cu_new=st["cu_new"] if c["ragged"] else None, max_kv=c["len"])
        st["out"] = torch.empty_like(st["q"])
    if c["op"] == "append":
        st["k"], st["v"] = _keys((T, H, D), c, seed, 5), _randn((T, H, D), seed, 6, dt)
        st["rope"] = _rope_table(c, c["len"])
        if own:
            st["rope"] = prox.Rope(st["rope"], interleaved=c["rope"] == "pairs")
            st["kv"] = [torch.empty((T, H, D), dtype=torch.float32, device="cuda") for _ in range(2)]
        else:
            st["pages"] = [torch.zeros((slots, H, n), dtype=t, device="cuda") for n, t in
                           ((D, torch.int8), (D // c["group"], torch.float16)) * 2]
        return st
    # A cache that holds every sequence's keys and values.
    k, v = _cached(c, seed)
    if own:
        every = prox.KVSeqs(st["kv_len"], st["table"], max_new=c["len"], cu_new=_starts(lens), max_kv=c["len"])
        prox.kv_append(st["cache"], every, k, v)
        st["ws"] = prox.new_kv_attn_workspace(D)
    else:
        seq, pos = _places(_starts(lens), st["kv_len"], sum(lens))
        at = _slots(st["table"], seq, pos, c["page"])
        st["pages"] = [torch.zeros((slots, H, n), dtype=t, device="cuda") for n, t in
                       ((D, torch.int8), (D // c["group"], torch.float16)) * 2]
        for i, x in enumerate(_quantise(k, c["group"]) + _quantise(v, c["group"])):
            st["pages"][i][at] = x
    return st


def _cached(c, seed):
    n = sum(_news(c)[1])
    return (_keys((n, c["kv_heads"], c["head_dim"]), c, seed, 7),
            _randn((n, c["kv_heads"], c["head_dim"]), seed, 8, _DT[c["dtype"]]))


def _starts(lens):
    return torch.tensor([sum(lens[:s]) for s in range(len(lens) + 1)], dtype=torch.int32, device="cuda")


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------

def _places(cu, kv_len, T):
    """(sequence, position) of each of the T rows."""
    t = torch.arange(T, device="cuda")
    seq = torch.bucketize(t, cu[1:].long(), right=True)
    return seq, (kv_len.long() - cu[1:].long())[seq] + t


def _slots(table, seq, pos, page):
    return table.long()[seq, pos // page] * page + pos % page


def _rotated(x, table, pos, kind):
    """Rotation by the table's rows at pos: products in 64 bits, rounded to 32 bits, then to the type."""
    half = table.shape[1] // 2
    cos, sin = table[pos].double()[:, None].split(half, -1)
    r = x[..., :2 * half].double()
    a, b = (r[..., :half], r[..., half:]) if kind == "half" else (r[..., 0::2], r[..., 1::2])
    a, b = a * cos - b * sin, a * sin + b * cos
    r = torch.cat([a, b], -1) if kind == "half" else torch.stack([a, b], -1).flatten(-2)
    return torch.cat([r.float().to(x.dtype), x[..., 2 * half:]], -1)


def _attend(st):
    c = st["case"]
    S, N, L, H, D = c["seqs"], c["new"], c["len"], c["kv_heads"], c["head_dim"]
    T, G = st["q"].shape[0], c["q_heads"] // H
    seq, qpos = _places(st["cu_new"], st["kv_len"], T)
    row = torch.arange(T, device="cuda") - st["cu_new"].long()[seq]
    pos = torch.arange(L, device="cuda")
    at = _slots(st["table"], torch.arange(S, device="cuda")[:, None], pos[None], c["page"]).flatten()
    kc, ks, vc, vs = (p[at].view(S, L, H, -1).transpose(1, 2) for p in st["pages"])
    q = torch.zeros((S, N, c["q_heads"], D), device="cuda")
    q[seq, row] = st["q"].float()
    where = torch.full((S, N), -1, dtype=torch.long, device="cuda")
    where[seq, row] = qpos
    q = q.view(S, N, H, G, D).permute(0, 2, 3, 1, 4).reshape(S, H, G * N, D)
    s = torch.matmul(q, _values(kc, ks).transpose(2, 3).contiguous()) / math.sqrt(D)
    seen = pos[None, None] <= where[..., None]
    if c["window"]:
        seen &= pos[None, None] > where[..., None] - c["window"]
    s = s.view(S, H, G, N, L).masked_fill(~seen[:, None, None], -math.inf)
    m = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(m > -math.inf, m, 0.0))
    o = torch.matmul(p.view(S, H, G * N, L), _values(vc, vs)).view(S, H, G, N, D)
    total = p.sum(-1)[..., None]
    o = torch.where(total > 0, o / total, 0.0)
    return o.permute(0, 3, 1, 2, 4).reshape(S, N, c["q_heads"], D)[seq, row].to(st["q"].dtype)


def run(st):
    c = st["case"]
    if own:
        from paper_2607_27591_amd import prox
        if c["op"] == "linear":
            return {"y": prox.linear_w4(st["w4"], st["x"], bias=st["bias"], y=st["y"])}
        if c["op"] == "append":
            prox.kv_append(st["cache"], st["seqs"], st["k"], st["v"], q=st["q"], q_out=st["out"], rope=st["rope"])
            k, v = prox.kv_read(st["cache"], st["seqs"], k=st["kv"][0], v=st["kv"][1])
            return {"q": st["out"], "k": k, "v": v}
        return {"out": prox.kv_attn(st["cache"], st["seqs"], st["q"], window=c["window"], out=st["out"], ws=st["ws"])}
    if c["op"] == "linear":
        y = torch.matmul(st["x"].float(), _values(st["codes"], st["scales"]).t())
        return {"y": (y if st["bias"] is None else y + st["bias"].float()).to(st["x"].dtype)}
    if c["op"] == "append":
        seq, pos = _places(st["cu_new"], st["kv_len"], st["q"].shape[0])
        q, k = (_rotated(x, st["rope"], pos, c["rope"]) for x in (st["q"], st["k"]))
        at = _slots(st["table"], seq, pos, c["page"])
        kc, ks, vc, vs = st["pages"]
        kc[at], ks[at] = _quantise(k, c["group"])
        vc[at], vs[at] = _quantise(st["v"], c["group"])
        return {"q": q, "k": _values(kc[at], ks[at]), "v": _values(vc[at], vs[at])}
    return {"out": _attend(st)}


# ---------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------

def work(c):
    if c["op"] == "linear":
        n, k, B = c["n"], c["k"], c["batch"]
        return {"bytes": n * k / 2 + 2 * n * (k // c["group"]) + 2 * B * (n + k) + (2 * n if c["bias"] else 0),
                "flops": 2.0 * B * n * k}
    news, lens = _news(c)
    H, D, T = c["kv_heads"], c["head_dim"], sum(news)
    token = H * (D + 4 * (D // c["group"]))   # of the cache, keys and values
    if c["op"] == "append":
        # q, k, v and a table row in; q, the cache and the values read back out
        return {"bytes": T * (4 * c["q_heads"] * D + 4 * H * D + 4 * c["rope_dim"] + token + 8 * H * D),
                "flops": 3.0 * T * c["rope_dim"] * (c["q_heads"] + H)}
    bytes_, pairs = 4 * T * c["q_heads"] * D, 0
    for n, l in zip(news, lens):
        first = max(0, l - n - c["window"] + 1) if c["window"] else 0
        bytes_ += (l - first) * token
        pairs += sum(min(p + 1, c["window"] or p + 1) for p in range(l - n, l))
    return {"bytes": bytes_, "flops": 4.0 * D * c["q_heads"] * pairs}


# ---------------------------------------------------------------------------
# The same in 64 bits, from the definitions
# ---------------------------------------------------------------------------

def _exact_values(x, group):
    """fp64 values that the cache or the weights hold for the 16-bit x [...][m group]."""
    shape = x.shape
    x = x.double().reshape(-1, group)
    sigma = torch.clamp((x.abs().max(1, keepdim=True).values / 7).float(), max=65504.0).half().double()
    n = torch.round(x / torch.where(sigma > 0, sigma, 1.0))
    return (torch.clamp(n, -7, 7) * sigma).reshape(shape)


def exact(c, seed):
    dt = _DT[c["dtype"]]
    if c["op"] == "linear":
        w, x = _weights(c, seed), _x(c, seed).double()
        y = torch.cat([x @ _exact_values(w[r:r + 4096], c["group"]).t().contiguous()
                       for r in range(0, c["n"], 4096)], 1)
        if c["bias"]:
            y += _randn((c["n"],), seed, 3, dt).double()
        return {"y": y}
    news, lens = _news(c)
    H, D, T = c["kv_heads"], c["head_dim"], sum(news)
    q = _randn((T, c["q_heads"], D), seed, 4, dt)
    if c["op"] == "append":
        pos = torch.cat([torch.arange(l - n, l, device="cuda") for n, l in zip(news, lens)])
        table = _rope_table(c, c["len"]).double()[pos]
        half = c["rope_dim"] // 2
        i = torch.arange(half, device="cuda")
        at = (i, i + half) if c["rope"] == "half" else (2 * i, 2 * i + 1)

        def turn(x):
            z = torch.complex(x[..., at[0]].double(), x[..., at[1]].double())
            z = z * torch.complex(table[:, None, :half], table[:, None, half:])
            y = x.double()
            y[..., at[0]], y[..., at[1]] = z.real, z.imag
            return y

        k = turn(_keys((T, H, D), c, seed, 5)).float().to(dt)   # the type that is quantised
        return {"q": turn(q), "k": _exact_values(k, c["group"]),
                "v": _exact_values(_randn((T, H, D), seed, 6, dt), c["group"])}
    k, v = _cached(c, seed)
    out = torch.empty((T, c["q_heads"], D), dtype=torch.float64, device="cuda")
    t = a = 0
    for n, l in zip(news, lens):
        pos = torch.arange(l, device="cuda")
        at = torch.arange(l - n, l, device="cuda")[:, None]
        hidden = (pos > at) | ((pos <= at - c["window"]) if c["window"] else (pos < 0))
        for h in range(H):
            keys, vals = (_exact_values(x[a:a + l, h], c["group"]) for x in (k, v))
            for e in range(h * (c["q_heads"] // H), (h + 1) * (c["q_heads"] // H)):
                s = (q[t:t + n, e].double() @ keys.t().contiguous()) * D ** -0.5
                out[t:t + n, e] = torch.softmax(s.masked_fill(hidden, -math.inf), 1) @ vals
        t, a = t + n, a + l
    return {"out": out}
