"""How much of 32 bits the sums of the attention half keep: results that are small beside what
they are summed from, so that a 16-bit output shows the sums' own rounding.

The codes enter the products as q + 24 and q - 23 in turn (fp16: q + 72, q - 71).  Tolerances count
roundings: a product of 32 terms adds them in at most 8 steps of 4, each rounded once to a
step of 2^-23 of the partial sum at that place, uniformly (rms step / sqrt 12).  With
offsets of one sign the partial sums grow to many times the size, and so do the errors."""
import math

import numpy as np
import pytest
import torch

import layer_ref as R
from paper_2607_27591_amd import prox
from test_gpu_kv_cache import i32, poisoned, randn, table_of, want_kv

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16


def step(v):
    """Distance of fp32 numbers at v."""
    return 2.0 ** (math.floor(math.log2(v)) - 23)


def rms(x):
    return float(np.sqrt(np.mean(np.square(x))))


@pytest.mark.parametrize("group,batch,n", [(128, 1, 500), (64, 9, 500), (32, 24, 500), (128, 40, 9000), (256, 64, 16400)])
def test_projection_of_inputs_with_a_mean(group, batch, n):
    # x = 1000 and a little, weights whose codes come in pairs q, -q: y is what the little makes of it.
    k, mean = 1024, 1000.0
    g = torch.Generator().manual_seed(1)
    code = torch.randint(-7, 8, (n, k // 2), generator=g).double()
    code[:, ::group // 2] = 7.0                         # sigma is 2^-3 in every group
    w = torch.stack([code, -code], -1).flatten(1) * 0.125
    x = mean + torch.randint(-2, 3, (batch, k), generator=g).double() * 0.5
    q = prox.pack_linear_w4(w.to(F16).cuda(), group)
    y = R.f64(prox.linear_w4(q, x.to(F16).cuda()))
    ref = x.numpy() @ w.numpy().T
    # Partial sums of 128 inputs or fewer: a mean left by every pair, and four terms of (72 + 7) mean.
    # 4 products of 32 inputs for the codes and as many for the offset.
    one = step(64 * mean + 4 * 79 * mean) / math.sqrt(12)
    sums = 0.125 * one * math.sqrt(8 * 8 * k / 128)
    tol = math.sqrt(rms(ref) ** 2 * R.HALF_STEP[F16] ** 2 / 3 + (2 * sums) ** 2)
    print(f"    rms error {rms(y - ref):.3g}, {rms(y - ref) / tol:.3f} of its bound; y {rms(ref):.3g}", flush=True)
    assert rms(y - ref) <= tol


def cancelling(dtype, tokens, group, dim, heads, ratio, news, k, v, seed=3):
    """Attention of `news` queries over k, v, and its rows whose tokens are whole pairs of blocks."""
    page = 64
    per = tokens // page
    c = poisoned(per, page, heads, dim, dtype, group=group)
    table = table_of(1, per, per)
    prox.kv_append(c, prox.KVSeqs(i32([tokens]), table, max_new=tokens), k, v)
    kw, vw = want_kv(k, v, None, c)
    q = randn((news, heads * ratio, dim), seed, dtype)
    rows = [i for i in range(news) if (tokens - news + i) % 64 == 63]
    return c, prox.KVSeqs(i32([tokens]), table, max_new=news), q, rows, kw, vw


def block_sums(codes, scales):
    """fp32 sums of flat weights times the values q + 24 (the first half of a block of 32 tokens) and q - 23,
    less the offset, as four waves form them over 8 blocks at a time, one rounding for each product of 32
    terms: codes [tokens][dim], scales [tokens]."""
    f, off = np.float32, np.where(np.arange(32) < 16, 24.0, -23.0)
    total = np.zeros(codes.shape[1])
    for wave in range(4):
        acc, base = np.zeros(codes.shape[1], f), f(0)
        for n, b in enumerate(range(32 * wave, len(scales), 128)):
            w = scales[b:b + 32]
            hi = torch.from_numpy(w).bfloat16().double().numpy()
            for t in (hi, w - hi):
                acc = (acc + t @ (codes[b:b + 32] + off[:, None])).astype(f)
                base = f(base - t @ off)
            if n % 8 == 7:
                acc, base = (acc + base).astype(f), f(0)
        total += (acc + base).astype(f)
    return total


ROWS = [(1, 1), (4, 1), (8, 1), (16, 1), (4, 64), (1, 300)]


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("ratio,news", ROWS)
@pytest.mark.parametrize("tokens", [2048, 4096])
def test_offsets_of_codes_leave_the_sums(dtype, ratio, news, tokens):
    # Flat weights over values of many sizes: block 2 j + 1 holds those of block 2 j with the other sign, so that
    # outputs are 0 but for the roundings of the sums.
    heads, dim, group = 2, 128, 64
    g = torch.Generator().manual_seed(5)
    size = 2.0 ** (torch.rand((tokens // 64, 32, heads, 1), generator=g).double() * 8 - 1)
    code = torch.randint(-7, 8, (tokens // 64, 32, heads, dim), generator=g).double()
    code[..., ::group] = 7.0
    v = (code * size).to(dtype)
    v = torch.stack([v, -v], 1).reshape(tokens, heads, dim).cuda()
    c, seqs, q, rows, _, _ = cancelling(dtype, tokens, group, dim, heads, ratio, news, torch.zeros_like(v), v)
    got = R.f64(prox.kv_attn(c, seqs, q, scale=0.0))[rows]
    codes, scales = R.quantise(R.f64(v), group)
    sums = [block_sums(codes[:, h, :group].astype(np.float64), scales[:, h, 0].astype(np.float64)) for h in range(heads)]
    tol = 4 * rms(np.stack(sums)) / (tokens - news) + R.TINY[dtype]   # 8 roundings a product instead of 1: sqrt 8
    print(f"    rms of what is left {rms(got):.3g}, {rms(got) / tol:.3f} of its bound", flush=True)
    assert rms(got) <= tol


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("ratio,news", ROWS)
def test_weights_keep_16_bits(dtype, ratio, news):
    # Block 2 j + 1 has the keys of block 2 j, and a third of its values' codes at three times the scale, with the
    # other sign: outputs are 0 but for the rounding of weights times scales, under 2^-16 of each.
    heads, dim, group, tokens = 2, 128, 64, 2048
    g = torch.Generator().manual_seed(5)
    code = torch.randint(-2, 3, (tokens // 64, 32, heads, dim), generator=g).double() * 3
    code[..., ::group] = 7.0
    other = -code
    other[..., ::group] = 21.0
    v = torch.stack([code, other], 1).reshape(tokens, heads, dim).to(dtype).cuda()
    k = randn((tokens // 64, 1, 32, heads, dim), 1, dtype).expand(-1, 2, -1, -1, -1).reshape(tokens, heads, dim).contiguous()
    c, seqs, q, rows, kw, vw = cancelling(dtype, tokens, group, dim, heads, ratio, news, k, v)
    got = R.f64(prox.kv_attn(c, seqs, q))[rows]
    sq = tol2 = n = 0.0
    keep = np.arange(dim) % group != 0
    for i, row in enumerate(rows):
        p = tokens - news + row
        for h in range(heads * ratio):
            s = (R.f64(q)[row, h] @ kw[:p + 1, h // ratio].T) * dim ** -0.5
            w = np.exp(s - s.max())
            ref = (w / w.sum()) @ vw[:p + 1, h // ratio]
            assert np.abs(ref[keep]).max() < 1e-12
            sq += np.square(got[i, h, keep]).sum()
            tol2 += ((2.0 ** -16 * w[:, None] * vw[:p + 1, h // ratio][:, keep]) ** 2).sum() / w.sum() ** 2 + keep.sum() * R.TINY[dtype] ** 2
            n += keep.sum()
    print(f"    rms of what is left {math.sqrt(sq / n):.3g}, {math.sqrt(sq / tol2):.3f} of its bound", flush=True)
    assert sq <= tol2


@pytest.mark.parametrize("ratio,news", [(1, 1), (4, 1), (8, 1), (16, 1), (4, 40)])
@pytest.mark.parametrize("dim,group", [(64, 32), (128, 64), (256, 128)])
def test_weights_keep_more_than_one_16_bit_term(dim, group, ratio, news):
    # fp16 outputs: the rounding of an output is uniform and at most half a step, rms 2^-11 / sqrt 3, beside 2^-16
    # of the weights and sums.  Weights of one bf16 term would give 1.6e-3.
    heads, tokens, page = 2, 700, 64
    per = -(-tokens // page)
    c = poisoned(2 * per, page, heads, dim, F16, group=group)
    table = table_of(2, per, 2 * per)
    k, v = (randn((2 * tokens, heads, dim), i, F16) for i in (1, 2))
    prox.kv_append(c, prox.KVSeqs(i32([tokens] * 2), table, max_new=tokens), k, v)
    kw, vw = want_kv(k, v, None, c)
    q = randn((2 * news, heads * ratio, dim), 3, F16)
    got = R.f64(prox.kv_attn(c, prox.KVSeqs(i32([tokens] * 2), table, max_new=news), q))
    ref = np.concatenate([R.attention(R.f64(q)[s * news:(s + 1) * news], kw[s * tokens:(s + 1) * tokens], vw[s * tokens:(s + 1) * tokens],
                                      np.arange(tokens - news, tokens), dim ** -0.5)[0] for s in (0, 1)])
    off, tol = rms(got - ref) / rms(ref), R.HALF_STEP[F16] / math.sqrt(3) + 2.0 ** -16
    print(f"    relative error {off:.3g}, {off / tol:.3f} of its bound", flush=True)
    assert off <= tol
