"""Rows in 8 bits where a value of the row decides about the others: against the definition in 64 bits."""
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


def norm(x, y, gain, eps, dtype):
    """(r, n, codes, scales): n = r gain / sqrt(mean(r^2) + eps), a row of zeros zeros for any eps."""
    with np.errstate(all="ignore"):
        r = x if y is None else R.to_type(x + y, dtype)
        p = r if gain is None else r * gain
        rms = np.sqrt((r * r).mean(-1) + float(np.float32(eps)))
        n = np.where(rms[:, None] == 0, p, p / rms[:, None])    # p is 0 there, or 0 times a gain that is not finite
        fine = np.isfinite(r).all(-1)
        c, s = R.codes(np.where(fine[:, None], p, np.nan), np.where(rms == 0, 0.0, 1 / rms))
    return r, n, c, s


def check_norm(x, y, gain, eps, tag):
    res, out = torch.full_like(x, 3.0), torch.full_like(x, 3.0)
    q = prox.rmsnorm_q8(x, y, gain, eps, residual=res, out=out)
    r, n, c, s = norm(f64(x), None if y is None else f64(y), None if gain is None else f64(gain), eps, x.dtype)
    assert np.array_equal(f64(res), r, equal_nan=True), f"{tag}: residual"
    R.check_codes(q.codes, c, tag)
    R.check_scales(q.scales, s, tag)
    R.check_out(out, n, x.dtype, tag)
    alone = prox.rmsnorm(x, y, gain, eps)
    assert torch.equal(alone.view(torch.int16), out.view(torch.int16)), tag
    return out


# One for every way in which a row is cut among threads.
WIDTHS = [8, 96, 511, 512, 1500, 4000, 8192, 9000, 20000, 40001]


@pytest.mark.parametrize("eps", [0.0, 1e-6])
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("d", WIDTHS)
def test_norm_of_rows_that_are_not_finite(d, dtype, eps):
    x, y, gain = randn((9, d), 1, dtype), randn((9, d), 2, dtype), randn((d,), 3, dtype)
    nan, inf, big = float("nan"), float("inf"), torch.finfo(dtype).max
    x[1, 5], y[2, d - 1], x[3, 0], x[4, 7], y[4, 7] = nan, nan, inf, inf, -inf
    x[5, 3], y[5, 3] = big, big              # the residual overflows
    x[6], y[6] = 0, 0
    x[7], y[7] = nan, nan
    for g in (gain, None):
        out = check_norm(x, y, g, eps, f"{d}")
        # A NaN spoils its row; behind an infinite one the others are 0, and it is NaN.
        assert torch.isnan(out[[1, 2, 4, 7]]).all() and (out[6] == 0).all()
        assert torch.isnan(out[3, 0]) and torch.isnan(out[5, 3]) and (out[3, 1:] == 0).all() and (out[5, 4:] == 0).all()
        assert torch.isfinite(out[[0, 8]]).all()
    check_norm(x, None, gain, eps, f"{d}, nothing added")
    gain[2] = inf
    check_norm(x, y, gain, eps, f"{d}, gain")
    gain[2] = nan
    check_norm(x, y, gain, eps, f"{d}, gain NaN")


@pytest.mark.parametrize("swap", [False, True])
def test_lanes_of_a_row_agree_on_its_mean(swap):
    # A row of one wave whose 64-bit sum of squares, 2^119 and little more, goes to one of two neighbours by the order in which
    # its lanes' parts are added: the quads of lanes that hold 4 and 2 squares of 2^62 each lose them, or not.  The mean is then at
    # 2^110 or above, where the kernel turns to 64 bits: lanes that take different ways do not see each other's largest.
    r = torch.zeros((4, 4, 4, 8))                    # rows of 16 lanes, quads of 4, elements of a lane
    r[:, int(swap)::2, :, :2] = 2.0 ** 56            # every quad's squares: 2^115
    r[:, 1 - int(swap)::2, :2, :1] = 2.0 ** 57
    r[:, 0, :, 4] = 2.0 ** 31
    r[:, 3, :2, 4] = 2.0 ** 31
    x = r.reshape(1, 512).to(BF16).cuda()
    check_norm(x.expand(5, 512).contiguous(), None, None, 0.0, "rows")
    check_norm(x.expand(5, 512).contiguous(), None, torch.linspace(1, 2, 512).to(BF16).cuda(), 0.0, "gain")


@pytest.mark.parametrize("d", [64, 500, 1000, 3000, 9000])
def test_norm_of_small_products(d):
    # Products r gain below 32 bits' normal range, and a 1 / rms that brings them back into it: eps 0 and a row of 2^-40 to 2^-49.
    gen = torch.Generator().manual_seed(d)
    for small in (40, 45, 49):
        x = torch.randn((6, d), generator=gen) * 2.0 ** -105
        x[:, d // 2] = 2.0 ** -small * (1 + torch.arange(6) / 8)
        gain = 2.0 ** -torch.randint(20, 46, (d,), generator=gen).float() * (1 + torch.rand(d, generator=gen))
        gain[d // 2] = 2.0 ** -9
        check_norm(x.to(BF16).cuda(), None, gain.to(BF16).cuda(), 0.0, f"{d}, {small}")


def just_above(act, far):
    """(g, u, far u): an activation of the gate `far` that is larger than that of g by 5e-5 to 1.1e-4 of it."""
    us = (1 + np.arange(128) / 128) * 2.0 ** 127
    tops = R.act(np.full(128, far), us, act)
    gates = f64((2 + torch.arange(512) / 512).to(BF16))
    gates = np.unique(gates)
    scale = 2.0 ** np.floor(np.log2(np.abs(tops).max()))
    ups = (1 + np.arange(128) / 128) * scale / 4
    v = R.act(gates[:, None], ups[None, :], act)
    ratio = np.abs(tops)[:, None, None] / v[None]
    a, b, c = np.argwhere((ratio > 1 + 5e-5) & (ratio < 1 + 1.1e-4))[0]
    return gates[b], ups[c], us[a], v[b, c]


@pytest.mark.parametrize("far", [-88.5, -90.0])
@pytest.mark.parametrize("d", [100, 3000, 9000, 20000])
def test_a_silu_gate_that_32_bits_lose_makes_the_largest(d, far):
    check_far(prox.SILU, d, far)


@pytest.mark.parametrize("far", [-13.375, -13.5])
@pytest.mark.parametrize("d", [100, 3000, 9000, 20000])
def test_a_gelu_gate_that_32_bits_lose_makes_the_largest(d, far):
    check_far(prox.GELU, d, far)


def check_far(act, d, far):
    # By so little that the codes are all but those of the largest of the others, and only those near a border differ.
    g0, u0, u1, top = just_above(act, far)
    g, u = randn((5, d), 1, BF16), randn((5, d), 2, BF16)
    size = np.abs(R.act(f64(g), f64(u), act)).max()
    u = (u.float() * (0.9 * top / size)).to(BF16)
    u[3:] = (torch.linspace(0.2, 0.99, d) * u0).to(BF16).cuda()      # rows of codes that are far from 0
    g[3:] = float(g0)
    g[:, d // 3], u[:, d // 3] = float(g0), float(u0)
    g[:, d // 2], u[:, d // 2] = far, float(u1)
    x, up = f64(g), f64(u)
    v = np.abs(R.act(x, up, act))
    assert (v.argmax(-1) == d // 2).all() and (v[:, d // 2] < 1.00012 * np.sort(v, -1)[:, -2]).all()
    q = prox.quant_q8(g, u, act)
    c, s = R.codes(R.act(x, up, act))
    R.check_codes(q.codes, c, f"{d}")
    R.check_scales(q.scales, s, f"{d}")
