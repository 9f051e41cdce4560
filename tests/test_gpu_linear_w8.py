"""Projections on 8-bit integers against the formula on the quantiser's codes; a layer's run of them."""
import pickle

import numpy as np
import pytest
import torch

import rows8_ref as R
from layer_ref import f64
from paper_2607_27591_amd import prox

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16


def randn(shape, seed, dtype, scale=1.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * scale).to(dtype).cuda()


def rows8(rows, k, seed, pad=0):
    """Rows of any int8, marks behind them."""
    gen = torch.Generator().manual_seed(seed)
    codes = torch.full((rows, (k + 15) // 16 * 16 + pad), 101, dtype=torch.int8, device="cuda")
    codes[:, :k] = torch.randint(-128, 128, (rows, k), generator=gen, dtype=torch.int8)
    return prox.RowsQ8(codes[:, :k], (0.5 + torch.rand(rows, generator=gen)).cuda() / 100)


def weights(n, k, dtype, seed=0):
    w = randn((n, k), seed, dtype, 0.02)
    return prox.pack_linear_w8(w), *R.codes(f64(w))


def check(w, q, sw, x, bias=None, tag="", y=None):
    got = prox.linear_w8(w, x, bias=bias, y=y)
    want, bound = R.linear(x.codes.cpu().numpy(), f64(x.scales), q, sw.astype(np.float32), None if bias is None else f64(bias))
    R.check(got, want, bound, w.dtype, tag)
    return got


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("n,k", [(1, 1), (16, 64), (37, 97), (64, 128), (65, 129), (129, 640), (1000, 1030), (70, 8192)])
def test_packing_is_exact(n, k, dtype):
    w = randn((n, k), 5, dtype, 0.02)
    w[0] = 0
    w[n // 2] *= 1e-4 if dtype == F16 else 1e-37
    if n > 20:
        w[3, k // 2], w[5, k - 1], w[7, 0] = float("nan"), float("inf"), 127 / 64.0   # ties with the rest
        w[7, 1:] = (torch.arange(k - 1) % 127 + 0.5) / 64
    q = prox.pack_linear_w8(w)
    codes, scales = prox.unpack_linear_w8(q)
    c, s = R.codes(f64(w))
    R.check_codes(codes, c)
    R.check_scales(scales, s)


# Rows, outputs and inputs around every size at which a call takes another variant or a tile ends.
ROWS = [1, 2, 4, 5, 8, 9, 15, 16, 17, 31, 32, 33, 48, 63, 64, 65, 100, 127, 128, 129, 192, 255, 256, 257, 300, 384, 511, 513, 700, 1025]


@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("n,k,dtype,bias", [(1, 1, BF16, True), (65, 300, F16, True), (256, 1024, BF16, False), (515, 1111, BF16, True),
                                            (1024, 130, F16, False), (2050, 640, BF16, False)])
def test_parity(rows, n, k, dtype, bias):
    w, q, sw = weights(n, k, dtype)
    x = rows8(rows, k, rows)
    b = randn((n,), 2, dtype) if bias else None
    y = check(w, q, sw, x, b, f"{rows}x{n}x{k}")
    assert torch.equal(y, prox.linear_w8(w, x, bias=b))


@pytest.mark.parametrize("k", [1, 15, 16, 17, 63, 64, 65, 127, 128, 129, 191, 192, 193, 255, 256, 257, 383, 512, 1000, 1024, 2047, 4224])
@pytest.mark.parametrize("rows,n", [(1, 70), (16, 200), (40, 300), (200, 400), (600, 260)])
def test_inputs(k, rows, n):
    w, q, sw = weights(n, k, BF16, seed=k)
    check(w, q, sw, rows8(rows, k, k), None, f"{rows}x{n}x{k}")


@pytest.mark.parametrize("n", [1, 3, 15, 16, 17, 63, 64, 65, 127, 129, 255, 257, 4000, 4097, 8200, 16385, 28672])
@pytest.mark.parametrize("rows", [1, 7, 16, 33, 64, 150, 520])
def test_outputs(n, rows):
    w, q, sw = weights(n, 200, F16, seed=n)
    check(w, q, sw, rows8(rows, 200, n), randn((n,), 1, F16), f"{rows}x{n}")


@pytest.mark.parametrize("rows", [1, 16, 64, 300])
def test_the_largest_sums_are_exact(rows):
    # 65536 products of 127 and -128: sums of 1.07e9, told apart by one unit in the inputs' last place.
    k, n = 65536, 130
    w = torch.full((n, k), 0.5, dtype=BF16, device="cuda")
    w[1::2] *= -1
    q = prox.pack_linear_w8(w)
    x = prox.new_rows_q8(rows, k)
    x.codes.fill_(-128)
    x.scales.fill_(1.0)
    want = 65536 * 127 * 128
    scale = float(np.float32(0.5 / 127))
    y = prox.linear_w8(q, x)
    assert torch.equal(y[:, 1::2], torch.full_like(y[:, 1::2], want * scale)) and torch.equal(y[:, ::2], -y[:, 1::2])
    # Sums that all but cancel keep their last units.
    x.codes[:, 1::2] = 127
    x.codes[:, 5] = 126
    y = prox.linear_w8(q, x)
    total = (-128 + 127) * 127 * 32768 - 127
    assert torch.allclose(y[:, 0].double(), torch.tensor(total * scale, dtype=torch.float64, device="cuda"), rtol=2.0 ** -8, atol=0)
    x.codes.fill_(0)
    x.codes[:, 65535] = 1
    assert torch.equal(prox.linear_w8(q, x)[:, 0], torch.full((rows,), 127 * scale, device="cuda").to(BF16))


@pytest.mark.parametrize("rows", [1, 5, 33, 130, 300])
def test_every_input_by_itself(rows):
    # One code a row and distinct weights: each product alone, to the last bit.
    k, n = 400, 128
    codes = torch.randint(-127, 128, (n, k), generator=torch.Generator().manual_seed(1)).to(torch.int8)
    codes[:, 0] = 127
    w = (codes.float() / 128).to(BF16).cuda()        # 127 / 128 at most: the scale is 2^-7
    q = prox.pack_linear_w8(w)
    got, s = prox.unpack_linear_w8(q)
    assert torch.equal(got.cpu(), codes) and (s == 2.0 ** -7).all()
    for start in range(0, k, rows):
        m = min(rows, k - start)
        x = prox.new_rows_q8(rows, k)
        x.codes.zero_()
        x.scales.fill_(2.0)
        for i in range(m):
            x.codes[i, start + i] = 1
        y = prox.linear_w8(q, x)
        assert torch.equal(y[:m].float().cpu(), codes[:, start:start + m].t().float() * 2 / 128), start
        assert (y[m:] == 0).all()


@pytest.mark.parametrize("rows,n,k", [(1, 300, 500), (9, 300, 500), (70, 1000, 300), (300, 515, 300), (520, 300, 640)])
def test_rows_apart_and_marks(rows, n, k):
    # Rows of codes and of y inside wider ones: what stands behind them is not read as inputs and not written.
    w, q, sw = weights(n, k, BF16)
    x = rows8(rows, k, 3, pad=48)
    wide = torch.full((rows + 2, n + 9), 7.0, dtype=BF16, device="cuda")
    y = wide[1:rows + 1, 3:3 + n]
    check(w, q, sw, x, None, "wide", y=y)
    assert torch.equal(y, prox.linear_w8(w, prox.RowsQ8(x.codes, x.scales)))
    assert (wide[0] == 7).all() and (wide[-1] == 7).all() and (wide[:, :3] == 7).all() and (wide[:, 3 + n:] == 7).all()
    if rows > 8:     # some of the rows, by themselves
        part = prox.RowsQ8(x.codes[4:9], x.scales[4:9])
        assert torch.equal(prox.linear_w8(w, part), y[4:9])


@pytest.mark.parametrize("rows", [2, 16, 70, 300])
def test_rows_that_are_not_finite(rows):
    x = randn((rows, 700), 1, BF16)
    x[rows // 2, 3] = float("nan")
    w = randn((200, 700), 2, BF16)
    want = prox.linear_w8(prox.pack_linear_w8(w), prox.quant_q8(x))
    w[11, 5] = float("inf")
    y = prox.linear_w8(prox.pack_linear_w8(w), prox.quant_q8(x))
    assert torch.isnan(y[rows // 2]).all() and torch.isnan(y[:, 11]).all()
    keep = [b for b in range(rows) if b != rows // 2]
    rest = [j for j in range(200) if j != 11]
    assert torch.equal(y[keep][:, rest], want[keep][:, rest]) and torch.isfinite(y[keep][:, rest]).all()


@pytest.mark.parametrize("rows", [1, 20, 300])
def test_scales_at_the_ends_of_the_range(rows):
    w = randn((100, 256), 2, BF16)
    q = prox.pack_linear_w8(w)
    x = rows8(rows, 256, 1)
    for f in (0.0, 2.0 ** -100, 2.0 ** 90):
        y = prox.linear_w8(q, prox.RowsQ8(x.codes, x.scales * f))
        assert torch.equal(y.double(), prox.linear_w8(q, x).double() * f)


@pytest.mark.parametrize("rows,n,k", [(1, 512, 1024), (16, 4096, 1024), (64, 4096, 512), (300, 1500, 777), (1024, 4096, 256)])
def test_capture_and_streams(rows, n, k):
    w = prox.pack_linear_w8(randn((n, k), 1, BF16, 0.02))
    x, y = rows8(rows, k, 1), torch.empty((rows, n), dtype=BF16, device="cuda")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):   # the first call of the shape
        prox.linear_w8(w, x, y=y)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for seed in range(3):
        x.codes.copy_(rows8(rows, k, 5 + seed).codes)
        y.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        got = []
        for s in streams:
            with torch.cuda.stream(s):
                got.append(prox.linear_w8(w, x))
        torch.cuda.synchronize()
        assert torch.equal(y, got[0]) and torch.equal(y, got[1])


@pytest.mark.parametrize("n,k,rows", [(1 << 20, 64, 5), (1 << 20, 100, 130), (300, 65536, 70), (300, 65535, 3)])
def test_largest_projections(n, k, rows):
    few = min(n, 4096)
    w = randn((few, k), 1, BF16, 0.02)
    q = prox.pack_linear_w8(w.repeat(n // few, 1))
    x = rows8(rows, k, 2)
    y = prox.linear_w8(q, x)
    want, bound = R.linear(x.codes.cpu().numpy(), f64(x.scales), *((lambda c, s: (c, s.astype(np.float32)))(*R.codes(f64(w)))))
    R.check(y[:, :few], want, bound, BF16, "first outputs")
    assert torch.equal(y, y[:, :few].repeat(1, n // few))


def test_many_rows():
    # y past 2^32 bytes, rows of codes far apart.
    n, k, rows = 8192, 64, 300000
    w, q, sw = weights(n, k, BF16)
    x = rows8(1000, k, 1)
    big = prox.RowsQ8(x.codes.repeat(rows // 1000, 1)[:, :k], x.scales.repeat(rows // 1000))
    y = prox.linear_w8(w, big)
    few = check(w, q, sw, x)
    for a in range(0, rows, 50000):
        assert torch.equal(y[a:a + 1000], few), a
    assert torch.equal(y[-1000:], few)
    far = torch.empty_strided((1030, k), (prox.MAX_Q8_PITCH, 1), dtype=torch.int8, device="cuda")
    far.copy_(big.codes[:1030])
    assert torch.equal(prox.linear_w8(w, prox.RowsQ8(far, big.scales[:1030])), y[:1030])


def test_refusals_and_copies():
    w, q, sw = weights(100, 64, BF16)
    x = rows8(4, 64, 1)
    assert torch.equal(prox.linear_w8(pickle.loads(pickle.dumps(w)), x), prox.linear_w8(w, x))
    assert prox.linear_w8(w, prox.new_rows_q8(0, 64)).shape == (0, 100)
    with pytest.raises(ValueError):
        prox.linear_w8(w, rows8(4, 65, 1))
    with pytest.raises(ValueError):
        prox.linear_w8(w, x, y=torch.empty((3, 100), dtype=BF16, device="cuda"))
    with pytest.raises(ValueError):
        prox.linear_w8(w, x, y=torch.empty((4, 100), dtype=F16, device="cuda"))
    with pytest.raises(ValueError):
        prox.linear_w8(w, x, bias=torch.empty(99, dtype=BF16, device="cuda"))
    with pytest.raises(ValueError):
        prox.linear_w8(w, prox.RowsQ8(x.codes.cpu(), x.scales))
    with pytest.raises(prox.ProxError):
        prox.linear_w8(w, prox.RowsQ8(x.codes[:1].expand(4, 64), x.scales))
    with pytest.raises(prox.ProxError):
        prox.linear_w8(prox.LinearW8(w.blob[:-256], BF16, 100, 64), x)
    with pytest.raises(prox.ProxError):
        prox.pack_linear_w8(torch.empty((1, 65537), dtype=BF16, device="cuda"))


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("tokens", [1, 7, 130])
def test_a_layer(tokens, dtype):
    """A decoder layer in 8 bits around the 4-bit cache: norm, q/k/v, rotation and append, attention, output, norm,
    gate and up, activation, down, each step against 64 bits on what the steps before it gave."""
    d, heads, kv, hd, f = 512, 8, 2, 64, 1408
    lin = {n: weights(o, i, dtype, seed=s) for s, (n, o, i) in enumerate(
        [("qkv", (heads + 2 * kv) * hd, d), ("o", d, heads * hd), ("up", 2 * f, d), ("down", d, f)])}
    g1, g2 = ((1 + randn((d,), s, torch.float32, 0.2)).to(dtype) for s in (11, 12))
    x, y0 = randn((tokens, d), 13, dtype, 3.0), randn((tokens, d), 14, dtype)
    res = torch.empty_like(x)

    def norm(a, b, gain):
        q = prox.rmsnorm_q8(a, b, gain, residual=res)
        r, _, c, s = R.norm(f64(a) if a is not res else before, f64(b), f64(gain), 1e-6, dtype)
        assert np.array_equal(f64(res), r)
        R.check_codes(q.codes, c)
        R.check_scales(q.scales, s)
        return q

    before = f64(x)
    qkv = check(*lin["qkv"], norm(x, y0, g1)).view(tokens, heads + 2 * kv, hd)
    c = prox.new_kv_cache(8, 64, kv, hd, dtype)
    s = prox.KVSeqs(torch.tensor([tokens], dtype=torch.int32, device="cuda"), torch.arange(8, dtype=torch.int32, device="cuda")[None], max_new=tokens)
    ang = torch.arange(512)[:, None] * 1e4 ** (-torch.arange(0, hd, 2) / hd)
    q = prox.kv_append(c, s, qkv[:, heads:heads + kv], qkv[:, heads + kv:], q=qkv[:, :heads].contiguous(),
                       rope=prox.Rope(torch.cat([ang.cos(), ang.sin()], 1).float().cuda()))
    a = prox.kv_attn(c, s, q).view(tokens, heads * hd)
    a8 = prox.quant_q8(a)
    cw, sw = R.codes(f64(a))
    R.check_codes(a8.codes, cw)
    R.check_scales(a8.scales, sw)
    o = check(*lin["o"], a8)
    before = f64(res)
    gu = check(*lin["up"], norm(res, o, g2))
    s8 = prox.quant_q8(gu[:, :f], gu[:, f:], prox.SILU)
    cw, sw = R.codes(R.act(f64(gu[:, :f]), f64(gu[:, f:]), 0))
    R.check_codes(s8.codes, cw)
    R.check_scales(s8.scales, sw)
    check(*lin["down"], s8)


# A shape for each kind of tile, and calls that are cut in two launches.
TILES = [(2717, 2918, 928), (2433, 1563, 917), (1229, 1585, 900), (1425, 1413, 908), (1236, 782, 909), (822, 582, 919), (897, 1025, 905),
         (618, 390, 903), (305, 385, 1060), (311, 388, 928), (193, 312, 900), (60, 70, 900), (2967, 6729, 902), (2362, 7175, 927),
         (3104, 5250, 913), (633, 28477, 1112), (347, 23276, 1243), (3334, 2405, 1234), (2476, 3142, 901), (3227, 2314, 902)]


@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("rows,n,k", TILES)
def test_every_tile(rows, n, k, bias):
    for more in (0, 130, 260) if bias else (0, 515):       # steps of 128 inputs, in turns of 1 to 3, over up to 8 waves
        kk = k + more
        w = prox.pack_linear_w8(randn((n, kk), 1, BF16, 0.02))
        q, sw = prox.unpack_linear_w8(w)
        x = rows8(rows, kk, more, pad=16)
        b = randn((n,), 2, BF16) if bias else None
        wide = torch.full((rows + 1, n + 5), 7.0, dtype=BF16, device="cuda")
        y = prox.linear_w8(w, x, bias=b, y=wide[:rows, :n])
        a = torch.mm(x.codes.double(), q.double().t().contiguous())          # whole numbers below 2^53: exact
        a = a * sw.double() * x.scales.double()[:, None]
        want = a if b is None else a + b.double()
        # three roundings of the product, one of the sum, half a step of the type
        room = 3.01 * 2.0 ** -24 * a.abs() + 2.0 ** -24 * want.abs()
        room = room + 2.0 ** -8 * (want.abs() + room) + 2.0 ** -134
        far = (y.double() - want).abs()
        assert (far <= room).all(), f"{rows}x{n}x{kk}: {(far / room).max().item()}"
        assert (wide[rows] == 7).all() and (wide[:, n:] == 7).all()
