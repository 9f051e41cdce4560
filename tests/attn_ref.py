"""Inputs of attention whose answers show a lost, doubled or misplaced token, and checks tight
enough to see it: the 64-bit formula with mistakes planted in it is in test_attn_bounds_cpu.py, the
kernels are run in test_gpu_attn_sharp.py.  numpy and torch on the CPU."""
import math

import numpy as np
import torch

import layer_ref as R

BF16, F16 = torch.bfloat16, torch.float16

SHAPES = [  # heads, ratio, dim, group, page, dtype, lengths, new tokens, window
    (8, 1, 128, 64, 64, F16, [20000, 3], [1, 1], 0),
    (2, 4, 128, 64, 256, BF16, [9001, 5000], [1, 1], 0),
    (2, 8, 64, 32, 96, F16, [2049, 999], [1, 1], 0),
    (1, 16, 256, 64, 32, BF16, [2049, 700], [1, 1], 300),
    (4, 2, 128, 32, 32, F16, [3001], [2], 500),
    (2, 4, 128, 128, 64, BF16, [1500, 700], [20, 33], 0),
    (4, 4, 64, 64, 32, F16, [1300], [40], 129),
    (2, 7, 128, 64, 128, F16, [2500, 65], [5, 3], 1000),
    (1, 4, 256, 128, 64, F16, [4097], [3], 0),
    (2, 1, 256, 32, 64, BF16, [600, 33], [5, 2], 64),
]
MORE = [(8, 4, 128, 64, 64, BF16, [520, 520], [300, 300], 0), (4, 4, 64, 64, 32, F16, [1300], [300], 129)]   # two tiles a workgroup

KINDS = ["random", "flat", "planted"]


def randn(shape, seed, scale=1.0):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64) * scale


class Inputs:
    """q, k, v of a shape, 16-bit on the CPU, what the cache holds of k and v, and each row's place."""

    def __init__(self, heads, ratio, dim, group, page, dtype, lens, news, window, kind):
        self.heads, self.ratio, self.dim, self.group, self.page, self.dtype = heads, ratio, dim, group, page, dtype
        self.lens, self.news, self.window, self.kind = lens, news, window, kind
        n, T = sum(lens), sum(news)
        self.k, self.v = randn((n, heads, dim), 1), randn((n, heads, dim), 2)
        self.q = randn((T, heads * ratio, dim), 3)
        self.scale = dim ** -0.5
        if kind == "flat":
            # All weights alike, token t of a sequence a 1 in channel t % dim: an output is the share of the
            # tokens seen that stand on its channel.
            self.scale = 0.0
            self.v = torch.zeros_like(self.v)
            t = torch.cat([torch.arange(l) for l in lens])
            self.v[torch.arange(n), :, t % dim] = 1.0
        elif kind == "planted":
            # Row j looks along an axis of its own, on which one token stands out: its own, the one before, the
            # first, one behind it, the window's first, the one before that; it takes all where it is seen, and
            # leaves an average of the others where it is not.
            self.k, self.q = self.k * 0.01, torch.zeros_like(self.q)
            a = row = 0
            for l, m in zip(lens, news):
                for i in range(m):
                    p = l - m + i
                    first = max(p - window + 1, 0) if window else 0
                    for g in range(ratio):
                        axis = (row * ratio + g) % dim
                        t = [p, max(p - 1, 0), first, min(p + 1, l - 1), max(first - 1, 0), p // 2, p // 32 * 32, first // 32 * 32 + 31][(i + g) % 8]
                        self.q[row, g::ratio, axis] = 60.0 / self.scale
                        self.k[a + min(t, l - 1), :, axis] = 1.0
                    row += 1
                a += l
        self.k, self.v, self.q = (x.to(dtype) for x in (self.k, self.v, self.q))
        self.kw, self.vw = (R.values(*R.quantise(R.f64(x), group, 65504.0)) for x in (self.k, self.v))

    def rows(self):
        """(row, first token of its sequence, length, position) of each."""
        a = row = 0
        for l, m in zip(self.lens, self.news):
            for i in range(m):
                yield row, a, l, l - m + i
                row += 1
            a += l

    def attention(self, mistakes=()):
        """(out, bound) in 64 bits, and the outputs with each of the mistakes; the bound on what the kernels'
        arithmetic may be off before the rounding of the output: weights times scales to 2^-16 each (two
        bf16 terms keep 2^-18; scores of s are off by 2^-22 (1 + |s|) at most where sums keep within 4 of
        their size), which add up in squares, and 2^-19 of sum p |v| for the sums.
        mistake(seen, pos, first): weights of the tokens, instead of those of seen."""
        q, T = R.f64(self.q), sum(self.news)
        outs = np.zeros((1 + len(mistakes), T, self.heads * self.ratio, self.dim))
        bound = np.zeros(outs.shape[1:])
        for row, a, l, p in self.rows():
            if p < 0:
                continue
            t = np.arange(l)
            first = max(p - self.window + 1, 0) if self.window else 0
            seen = ((t <= p) & (t >= first)).astype(np.float64)
            every = [seen] + [m(seen, p, first) for m in mistakes]
            for h in range(self.heads):
                r = slice(h * self.ratio, (h + 1) * self.ratio)
                s = self.scale * (q[row, r] @ self.kw[a:a + l, h].T)
                e = np.exp(s - s[:, seen > 0].max(-1, keepdims=True))
                v = self.vw[a:a + l, h]
                for i, m in enumerate(every):
                    if i > 0 and np.array_equal(m, seen):
                        outs[i, row, r] = outs[0, row, r]
                        continue
                    w = e * m
                    w /= np.maximum(w.sum(-1, keepdims=True), 1e-300)
                    outs[i, row, r] = w @ v
                    if i == 0:
                        top = np.abs(s[:, seen > 0]).max(-1, keepdims=True)
                        each = np.sqrt((w ** 2) @ (v ** 2)) * (2.0 ** -16 + 2.0 ** -22 * (1 + top))
                        bound[row, r] = 4 * each + 2.0 ** -19 * (w @ np.abs(v).max(-1, keepdims=True))
        return outs[0], bound, outs[1:]


def violations(got, ref, bound, dtype):
    """What of a result is off: (share of values past half a step and the bound, error of the whole in the
    2-norm over what uniform rounding leaves of it)."""
    got = got if isinstance(got, np.ndarray) else R.f64(got)
    tol = R.HALF_STEP[dtype] * (np.abs(ref) + bound) + bound + R.TINY[dtype]
    # A rounding is off by half a step at most, uniformly: 1 / sqrt 3 of it; 2 % more as steps vary.
    whole = math.sqrt(np.square(R.HALF_STEP[dtype] * ref).sum() / 3) * 1.02 + math.sqrt(np.square(bound).sum()) + R.TINY[dtype] * math.sqrt(ref.size)
    return float((np.abs(got - ref) > tol).mean()), float(np.linalg.norm(got - ref) / whole)


def lose(tokens):
    def f(seen, p, first):
        s = seen.copy()
        s[tokens(p, first)] = 0
        return s
    return f


def double(tokens):
    def f(seen, p, first):
        s = seen.copy()
        s[tokens(p, first)] *= 2
        return s
    return f


def add(token):
    def f(seen, p, first):
        s = seen.copy()
        t = token(p, first)
        if 0 <= t < len(s):
            s[t] = 1
        return s
    return f


def none(p, first):
    return slice(0, 0)


# Mistakes of a kernel: the tokens of a split, of a block of 32, of a page's last block lost or taken twice, a mask off
# by one.  (Only rows that see more than a few tokens lose some.)
MISTAKES = {
    "first split lost": lose(lambda p, first: slice(first // 32 * 32, first // 32 * 32 + 128) if p - first > 300 else none(p, first)),
    "a block lost": lose(lambda p, first: slice((p + first) // 64 * 32, (p + first) // 64 * 32 + 32) if p - first > 100 else none(p, first)),
    "a block twice": double(lambda p, first: slice((p + first) // 64 * 32, (p + first) // 64 * 32 + 32) if p - first > 100 else none(p, first)),
    "own token lost": lose(lambda p, first: slice(p, p + 1) if p > first else none(p, first)),
    "first token lost": lose(lambda p, first: slice(first, first + 1) if p > first else none(p, first)),
    "next token seen": add(lambda p, first: p + 1),
    "token before the window seen": add(lambda p, first: first - 1),
}
