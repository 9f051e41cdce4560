"""Plain 64-bit implementations of the attention half of a decoder layer (INT4 projections,
4-bit cache, attention) for the tests, and their error bounds.  numpy only."""
import numpy as np
import torch

U32 = 2.0 ** -24
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}   # of a rounded result, relative
TINY = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}      # half the smallest subnormal
# A code q enters a matrix product as M + q with M at most 72 (an exponent's worth of
# offset), so partial sums stay within (72 + 7) sum |x|.
OFFSET = 80.0


def f64(t):
    return t.detach().cpu().double().numpy()


def quantise(x, group, limit=np.inf):
    """(codes, fp16 scales) of x [..., m group], fp64: sigma = fp16(amax / 7), at most limit;
    codes round half to even."""
    g = x.reshape(x.shape[:-1] + (x.shape[-1] // group, group))
    with np.errstate(over="ignore"):
        s = np.minimum((np.abs(g).max(-1) / 7).astype(np.float16).astype(np.float64), limit)
    q = np.clip(np.rint(g / np.where(s > 0, s, 1.0)[..., None]), -7, 7) * (s > 0)[..., None]
    return q.reshape(x.shape).astype(np.int8), s.astype(np.float16)


def values(codes, scales):
    g = codes.astype(np.float64).reshape(scales.shape + (codes.shape[-1] // scales.shape[-1],))
    return (g * scales.astype(np.float64)[..., None]).reshape(codes.shape)


def linear(x, codes, scales, bias=None):
    """(y, bound on |fp32 accumulation - y|): per group at most `group` additions of partial
    sums below OFFSET sigma sum |x|, then one addition per group and wave."""
    w = values(codes, scales)
    y = x @ w.T
    group = codes.shape[1] // scales.shape[1]
    xs = np.abs(x).reshape(x.shape[0], -1, group).sum(-1) @ scales.astype(np.float64).T   # sum |x| sigma
    bound = U32 * (group * OFFSET + 7 * (scales.shape[1] + 16)) * xs
    if bias is not None:
        y = y + bias
        bound = bound + U32 * np.abs(y)
    return y, bound


def rotate(x, table, pos, interleaved):
    """x [T][heads][D] (fp64 of 16-bit values), rotated: fp64, rounded to fp32."""
    dim = table.shape[1]
    h = dim // 2
    cos, sin = table[pos, :h][:, None], table[pos, h:][:, None]
    a = np.arange(0, dim, 2) if interleaved else np.arange(h)
    b = a + 1 if interleaved else a + h
    y = x.copy()
    y[..., a] = (x[..., a] * cos - x[..., b] * sin).astype(np.float32)
    y[..., b] = (x[..., a] * sin + x[..., b] * cos).astype(np.float32)
    return y


def to_type(x, dtype):
    """fp64 of fp32 values -> the nearest values of the 16-bit type, as fp64."""
    return torch.from_numpy(x.astype(np.float32)).to(dtype).double().numpy()


def attention(q, k, v, pos, scale, window=0, hidden=None, chunk=64):
    """q [n][Hq][D] at positions pos [n], over k, v [len][H][D] (fp64).  Returns (out, bound):
    the bound on the fp32 result's error before its rounding.
      score    d_s = scale * sum over groups of at most 128 products of partial sums below OFFSET
               sum |q| sigma <= OFFSET 128 U32 scale sum_i |q_i| max_p |k_pi| (|k| / 7 <= sigma <= |k|max),
               plus 16 U32 |s|;
      weight   relative d_s of this score and of the largest, exp and the running rescalings
               (at most one per block) within (8 + len / 32) U32, probability times scale
               split in two bf16 terms: 2^-16;
      sums     over len terms in blocks: (64 + len / 32) OFFSET U32 of sum p |v|max.
    """
    n, Hq, D = q.shape
    H = k.shape[1]
    out = np.zeros((n, Hq, D))
    bound = np.zeros((n, Hq, D))
    L = k.shape[0]
    for i in range(n):
        see = np.arange(L) <= pos[i]
        if window:
            see &= np.arange(L) > pos[i] - window
        if hidden is not None:
            see &= ~hidden
        if pos[i] < 0 or not see.any():
            continue
        ks, vs = k[see], v[see]
        for h in range(H):
            r = slice(h * (Hq // H), (h + 1) * (Hq // H))
            s = scale * (q[i, r] @ ks[:, h].T)
            kmax = np.abs(ks[:, h]).max(-1)   # [p]
            ds = U32 * (OFFSET * 128 * abs(scale) * np.abs(q[i, r]).sum(-1)[:, None] * kmax[None] / 7 + 16 * np.abs(s))
            p = np.exp(s - s.max(-1, keepdims=True))
            p /= p.sum(-1, keepdims=True)
            out[i, r] = p @ vs[:, h]
            rel = 2 * ds.max(-1, keepdims=True) + (8 + L / 32) * U32 + 2.0 ** -16
            vmax = np.abs(vs[:, h]).max(0)
            bound[i, r] = 2 * rel * (p @ np.abs(vs[:, h])) + U32 * OFFSET / 7 * (64 + L / 32) * \
                (p @ np.abs(vs[:, h]).max(-1, keepdims=True))
            bound[i, r] = np.minimum(bound[i, r], 2 * vmax)
    return out, bound


def check(got, ref, bound, dtype, tag=""):
    """|got - ref| <= half a step of the type on ref, plus the bound of the fp32 sums."""
    got = f64(got)
    assert got.shape == ref.shape, (got.shape, ref.shape)
    assert np.isfinite(got).all(), f"{tag}: not finite"
    tol = HALF_STEP[dtype] * (np.abs(ref) + bound) + bound + TINY[dtype]
    bad = np.abs(got - ref) > tol
    worst = (np.abs(got - ref) / tol).max() if ref.size else 0.0
    print(f"    {tag}: worst error {worst:.3f} of its bound", flush=True)
    assert not bad.any(), f"{tag}: {bad.sum()} of {bad.size} values off, worst {worst} of the bound"
