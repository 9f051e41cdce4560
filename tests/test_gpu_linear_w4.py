"""Projections on INT4 weights against the 64-bit formula on the quantiser's codes."""
import numpy as np
import pytest
import torch

import layer_ref as R
from paper_2607_27591_amd import prox

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16


def _randn(shape, seed, dtype, scale=1.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * scale).to(dtype).cuda()


def _case(n, k, group, dtype, seed=0, w=None):
    w = _randn((n, k), seed, dtype, 0.02) if w is None else w
    q = prox.pack_linear_w4(w, group)
    codes, scales = R.quantise(R.f64(w), group)
    return q, codes, scales


def _check(q, codes, scales, x, bias=None, tag=""):
    y = prox.linear_w4(q, x, bias=bias)
    ref, bound = R.linear(R.f64(x), codes, scales, None if bias is None else R.f64(bias))
    R.check(y, ref, bound, q.dtype, tag)
    return y


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("n,k,group", [(1, 32, 32), (16, 128, 128), (37, 96, 32), (50, 192, 64), (129, 640, 128),
                                       (17, 768, 256), (33, 1152, 384), (1000, 4096, 128)])
def test_packing_is_exact(n, k, group, dtype):
    w = _randn((n, k), 5, dtype, 0.02)
    w[0, :group] = 0                                  # a group of zeros
    w[n // 2, -group:] *= 1e-4 if dtype == F16 else 1e-7   # subnormal and vanishing scales
    w[n - 1, 0] = 7 * w[n - 1, 0].abs() + 1           # ties and a large entry
    q, codes, scales = _case(n, k, group, dtype, w=w)
    c, s = prox.unpack_linear_w4(q)
    assert np.array_equal(c.cpu().numpy(), codes)
    assert np.array_equal(s.cpu().numpy().view(np.uint16), scales.view(np.uint16))


@pytest.mark.parametrize("n,k,group,batch,dtype,bias", [
    (1, 32, 32, 1, BF16, True), (16, 128, 128, 1, F16, False), (15, 96, 32, 2, BF16, False),
    (37, 160, 32, 3, F16, True), (64, 192, 64, 16, BF16, True), (512, 1024, 128, 1, BF16, False),
    (1000, 3456, 64, 7, F16, True), (999, 4096, 128, 1, BF16, True), (777, 4096, 128, 17, BF16, False),
    (250, 28672, 128, 1, BF16, False), (130, 8192, 256, 33, F16, True), (100, 1152, 384, 48, BF16, False),
    (515, 2048, 32, 64, BF16, True), (515, 2048, 64, 64, F16, False), (70, 65536, 128, 5, BF16, False),
    (6144, 4096, 128, 16, BF16, False), (4100, 1024, 32, 2, F16, False), (3000, 512, 512, 31, BF16, False),
])
def test_parity(n, k, group, batch, dtype, bias):
    q, codes, scales = _case(n, k, group, dtype)
    x = _randn((batch, k), 1, dtype)
    b = _randn((n,), 2, dtype) if bias else None
    y = _check(q, codes, scales, x, b, f"{n}x{k} g{group} b{batch}")
    assert torch.equal(y, prox.linear_w4(q, x, bias=b))   # the same bits every time


# Outputs and rows on both sides of every size at which a call takes another variant.
EDGES = [(n, b) for n in (1024, 1025, 2048, 4096, 4097, 8192, 8193, 12288, 12290, 16384, 16390) for b in (1, 8, 16, 17, 32, 33, 64)]


@pytest.mark.parametrize("n,batch", EDGES)
def test_variants(n, batch):
    group, k, dtype = [(32, 224, BF16), (64, 320, F16), (128, 384, BF16), (128, 256, F16)][(n + batch) % 4]
    q, codes, scales = _case(n, k, group, dtype, seed=n)
    _check(q, codes, scales, _randn((batch, k), 1, dtype), _randn((n,), 2, dtype), f"{n}x{k} g{group} b{batch}")


@pytest.mark.parametrize("group,k,dtype", [(32, 1120, BF16), (32, 1280, F16), (64, 1088, F16), (64, 768, BF16), (128, 1152, F16), (384, 1536, BF16)])
@pytest.mark.parametrize("n,batch", [(16400, 64), (16400, 37), (8200, 64), (16400, 20)])
def test_many_rows_of_many_outputs(n, batch, group, k, dtype):
    # Variants whose waves share the rows, over several blocks a wave, with groups inside a block and a last block in part.
    q, codes, scales = _case(n, k, group, dtype, seed=n)
    x = _randn((batch, k), 1, dtype)
    _check(q, codes, scales, x, None, f"{n}x{k} g{group} b{batch}")
    y = prox.linear_w4(q, x)
    z = x.clone()
    z[batch - 2] = float("nan")
    keep = [b for b in range(batch) if b != batch - 2]
    y2 = prox.linear_w4(q, z)
    assert torch.equal(y[keep], y2[keep]) and torch.isnan(y2[batch - 2]).all()


@pytest.mark.parametrize("dtype,lo,hi", [(BF16, 1e-30, 1e30), (F16, 6e-8, 6e4)])
@pytest.mark.parametrize("batch", [1, 5, 40])
def test_inputs_of_any_size(dtype, lo, hi, batch):
    # Each row of x at another exponent: a row's result does not see the others'.
    n, k = 48, 512
    q, codes, scales = _case(n, k, 128, dtype, w=_randn((n, k), 0, dtype, 2.0 ** -9))
    size = torch.logspace(np.log10(lo), np.log10(hi / 8), batch, dtype=torch.float64)
    x = (torch.randn((batch, k), generator=torch.Generator().manual_seed(3)).double().clamp(-4, 4) * size[:, None])
    x = x.to(dtype).cuda()
    ref, bound = R.linear(R.f64(x), codes, scales)
    top = 3e38 if dtype == BF16 else 6e4
    keep = np.abs(ref).max(1) < top
    y = prox.linear_w4(q, x)
    R.check(y[torch.from_numpy(keep).cuda()], ref[keep], bound[keep], dtype, f"b{batch}")


def test_rows_do_not_meet():
    q, _, _ = _case(300, 1024, 128, BF16)
    x = _randn((20, 1024), 1, BF16)
    y = prox.linear_w4(q, x)
    z = x.clone()
    z[3] = float("nan")
    z[11] = float("inf")
    y2 = prox.linear_w4(q, z)
    keep = [b for b in range(20) if b not in (3, 11)]
    assert torch.equal(y[keep], y2[keep])
    assert torch.isnan(y2[3]).all()


@pytest.mark.parametrize("batch", [1, 3, 21, 64])
def test_strides_and_neighbours(batch):
    n, k = 77, 256
    q, codes, scales = _case(n, k, 64, BF16)
    wide = _randn((batch, 3 * k), 1, BF16)
    x = wide[:, k:2 * k]
    out = torch.full((batch, n + 40), 7.0, dtype=BF16, device="cuda")
    y = prox.linear_w4(q, x, y=out[:, 13:13 + n])
    ref, bound = R.linear(R.f64(x), codes, scales)
    R.check(y, ref, bound, BF16, "strided")
    assert (out[:, :13] == 7).all() and (out[:, 13 + n:] == 7).all()
    assert torch.equal(y.contiguous(), prox.linear_w4(q, x.contiguous()))


def test_one_vector_and_refusals():
    q, codes, scales = _case(40, 128, 32, F16)
    x = _randn((128,), 1, F16)
    y = prox.linear_w4(q, x)
    assert y.shape == (40,)
    ref, bound = R.linear(R.f64(x)[None], codes, scales)
    R.check(y[None], ref, bound, F16, "vector")
    for bad in [x[:64], x.float(), x.cpu(), x.to(BF16), torch.zeros((2, 256), dtype=F16, device="cuda")[:, ::2],
                torch.zeros((65, 128), dtype=F16, device="cuda")]:
        with pytest.raises((ValueError, prox.ProxError)):
            prox.linear_w4(q, bad)
    with pytest.raises(ValueError):
        prox.linear_w4(q, x, bias=torch.zeros(39, dtype=F16, device="cuda"))
    with pytest.raises(prox.ProxError):
        prox.pack_linear_w4(torch.zeros((4, 96), dtype=F16, device="cuda"), 64)
    with pytest.raises(ValueError):
        prox.pack_linear_w4(torch.zeros((4, 96), device="cuda"), 32)


def test_streams_and_graph():
    q, codes, scales = _case(900, 2048, 128, BF16)
    x = _randn((9, 2048), 1, BF16)
    want = prox.linear_w4(q, x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y = prox.linear_w4(q, x)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(y, want)
    out = torch.empty_like(want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        prox.linear_w4(q, x, y=out)
    for seed in range(4):
        x.copy_(_randn((9, 2048), 10 + seed, BF16))
        out.zero_()
        g.replay()
        assert torch.equal(out, prox.linear_w4(q, x))
        torch.cuda.synchronize()
