"""What keys, values and weights that are not finite become: the cache holds finite numbers, and nothing
outside the groups that they stand in changes."""
import math

import numpy as np
import pytest
import torch

import layer_ref as R
from paper_2607_27591_amd import prox
from test_gpu_kv_cache import i32, poisoned, randn, want_kv

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("dim,group", [(64, 32), (128, 128), (256, 64)])
def test_cache_stays_finite(dim, group, dtype):
    T = 40
    c = poisoned(2, 32, 2, dim, dtype, group=group)
    s = prox.KVSeqs(i32([T]), i32([[1, 0]]), max_new=T)
    k, v = (randn((T, 2, dim), i, dtype) for i in (1, 2))
    want = want_kv(k, v, None, c)
    for x, w in zip((k, v), want):
        x[3, 1, 5] = math.nan
        x[7, 0, group - 1] = math.inf
        x[8, 0, 0] = -math.inf
        x[35, 1, :group] = math.nan
        f = R.f64(x)
        g = f[3, 1, :group].copy()
        g[5] = 0                                   # left out of the maximum
        codes, scales = R.quantise(g, group, 65504.0)
        codes[5] = -7
        w[3, 1, :group] = R.values(codes, scales)
        for t, h, e in ((7, 0, group - 1), (8, 0, 0)):
            g = f[t, h, :group].copy()
            w[t, h, :group] = 65504.0 * np.rint(np.where(np.isfinite(g), g, 0) / 65504.0)
            w[t, h, e] = np.copysign(7 * 65504.0, g[e])
        w[35, 1, :group] = 0                       # no finite entry: sigma 0
    prox.kv_append(c, s, k, v)
    for got, w in zip(prox.kv_read(c, s), want):
        assert np.array_equal(R.f64(got), w)


def test_rows_that_see_none_of_them_keep_their_results():
    # Two sequences on pages of their own, one of them with keys and values that are not finite, and rows of the
    # same sequence before them.
    T, heads, dim = 90, 2, 128
    c = poisoned(8, 32, heads, dim, BF16, group=64)
    s = prox.KVSeqs(i32([T, T]), i32([[1, 0, 4], [7, 5, 3]]), max_new=T)
    k, v = (randn((2 * T, heads, dim), i, BF16) for i in (1, 2))
    q = randn((2 * T, 2 * heads, dim), 3, BF16)
    prox.kv_append(c, s, k, v)
    want = prox.kv_attn(c, s, q)
    k[T + 50:, :, 3] = math.nan
    v[T + 50:, :, 70] = math.inf
    prox.kv_append(c, s, k, v)
    got = prox.kv_attn(c, s, q)
    assert torch.equal(got[:T + 50], want[:T + 50]) and torch.isfinite(got).all()


def test_weights():
    # A NaN weight has code -7 of its group; an infinite one spoils the outputs of its row only.
    w = randn((48, 256), 1, BF16)
    codes, scales = R.quantise(R.f64(w), 128)
    w[5, 7] = math.nan
    w[20, 130] = math.inf
    c, sc = prox.unpack_linear_w4(prox.pack_linear_w4(w))
    g = R.f64(w)[5, :128].copy()
    g[7] = 0
    codes[5, :128], scales[5, :1] = R.quantise(g, 128)
    codes[5, 7] = -7
    rest = np.arange(48) != 20
    assert np.array_equal(c.cpu().numpy()[rest], codes[rest])
    assert np.array_equal(sc.cpu().numpy().view(np.uint16)[rest], scales.view(np.uint16)[rest])
    x = randn((9, 256), 2, BF16)
    y = prox.linear_w4(prox.pack_linear_w4(w), x)
    ref, bound = R.linear(R.f64(x), codes, scales)
    R.check(y[:, torch.from_numpy(rest).cuda()], ref[:, rest], bound[:, rest], BF16, "other rows")
    assert not torch.isfinite(y[:, 20]).any()
