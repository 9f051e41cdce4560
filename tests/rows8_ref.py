"""Plain 64-bit implementations of rows and weights in 8 bits for the tests, and their error bounds.  numpy only."""
import numpy as np
import torch
from scipy.special import erfc

from layer_ref import HALF_STEP, TINY, f64

U32 = 2.0 ** -24
BF16, F16 = torch.bfloat16, torch.float16


def to_type(x, dtype):
    """fp64 rounded to fp32 and then to the dtype, as fp64."""
    with np.errstate(over="ignore"):
        return torch.from_numpy(np.asarray(x, dtype=np.float64)).float().to(dtype).double().numpy()


def codes(p, factor=1.0):
    """(codes, scales as fp64 not rounded) of rows p (few bits, so that 127 p is exact): half to even; rows that
    are not finite: 0 and NaN."""
    p = np.asarray(p, dtype=np.float64)
    fine = np.isfinite(p).all(-1) & np.isfinite(np.broadcast_to(factor, p.shape[:-1]))
    q = np.where(fine[..., None], p, 0.0)
    top = np.abs(q).max(-1)
    c = np.rint(q * 127 / np.where(top > 0, top, 1.0)[..., None]).astype(np.int8)
    return c, np.where(fine, top * np.where(fine, factor, 0.0) / 127, np.nan)


def norm(x, y, gain, eps, dtype):
    """(r, n as fp64, codes, scales) of fp64 copies of 16-bit values."""
    with np.errstate(all="ignore"):
        r = x if y is None else to_type(x + y, dtype)
        p = r if gain is None else r * gain
        mean = (r * r).mean(-1) + float(np.float32(eps))
        inv = np.where(mean > 0, 1 / np.sqrt(mean), 0.0)
        n = p * inv[:, None]
    fine = np.isfinite(r).all(-1)
    c, s = codes(np.where(fine[:, None], p, np.nan), inv)
    return r, n, c, s


def act(g, u, kind):
    """act(g) u, fp64 rounded to fp32."""
    with np.errstate(all="ignore"):
        h = g / (1 + np.exp(-g)) if kind == 0 else 0.5 * g * erfc(-g * np.sqrt(0.5))
        return (h * u).astype(np.float32).astype(np.float64)


def check_scales(got, want, tag=""):
    """Rounded once to fp32, after a few roundings in 64 bits."""
    got = f64(got)
    assert np.array_equal(np.isnan(got), np.isnan(want)), f"{tag}: NaN"
    fine = ~np.isnan(want)
    far = np.abs(got[fine] - want[fine])
    bound = (U32 + 2.0 ** -48) * np.abs(want[fine]) + 2.0 ** -150
    assert (far <= bound).all(), f"{tag}: scale off by {np.max(far / np.maximum(np.abs(want[fine]), 1e-300))}"


def check_codes(got, want, tag=""):
    got = got.cpu().numpy().astype(int)
    bad = np.argwhere(got != want)
    assert len(bad) == 0, f"{tag}: {len(bad)} codes differ, first at {bad[0]}: {got[tuple(bad[0])]} for {want[tuple(bad[0])]}"


def check(got, want, bound, dtype, tag=""):
    """got: a 16-bit tensor; bound: error before the last rounding."""
    got = f64(got)
    assert np.array_equal(np.isnan(got), np.isnan(want)), f"{tag}: NaN"
    fine = np.isfinite(want)
    far = np.abs(got[fine] - want[fine])
    bound = np.broadcast_to(bound, want.shape)
    room = bound[fine] + HALF_STEP[dtype] * (np.abs(want[fine]) + bound[fine]) + TINY[dtype]
    assert (far <= room).all(), f"{tag}: off by {np.max(far / room):.3f} of the bound"


def check_out(got, n, dtype, tag=""):
    """The norm in its own type: 1 / rms rounded to fp32, times an exact product."""
    check(got, n, 2 * U32 * (1 + U32) * np.abs(np.where(np.isfinite(n), n, 0)), dtype, tag)


def linear(c, sx, q, sw, bias=None):
    """(y, bound on the fp32 part): the sum in whole numbers, rounded, two products, one addition."""
    with np.errstate(all="ignore"):
        a = (c.astype(np.float64) @ q.astype(np.float64).T) * sw.astype(np.float64) * sx.astype(np.float64)[:, None]
        y = a if bias is None else a + bias
        return y, 3 * U32 * (1 + 4 * U32) * np.abs(a) + U32 * np.abs(y)
