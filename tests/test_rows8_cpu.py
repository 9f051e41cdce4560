"""Host-side checks of the calls on rows in 8 bits: sizes, and refusals before any HIP call (the pointers are never
dereferenced), of the library and of its binding."""
import ctypes
import re

import pytest
import torch

from paper_2607_27591_amd import build as B
from paper_2607_27591_amd import prox

OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3
FAKE = 0x100000
BIG = 1 << 45
F = ctypes.c_float


def _lin(dtype=prox.BF16, n=1000, k=1000, blob=FAKE, nbytes=BIG):
    return prox._W8Linear(dtype, n, k, blob, nbytes)


def _run(q=None, codes=FAKE, ldc=1008, scales=FAKE, rows=3, bias=None, y=FAKE, ldy=1000):
    return prox.lib().prox_linear_w8(ctypes.byref(q or _lin()), codes, ldc, scales, rows, bias, y, ldy, None)


def _norm(x=FAKE, ldx=100, y=2 * FAKE, ldy=100, gain=FAKE, rows=3, d=100, dtype=prox.BF16, eps=1e-6, r=3 * FAKE, ldr=100, out=4 * FAKE,
          ldo=100, codes=FAKE, ldc=112, scales=FAKE):
    return prox.lib().prox_rmsnorm_q8(x, ldx, y, ldy, gain, rows, d, dtype, F(eps), r, ldr, out, ldo, codes, ldc, scales, None)


def _quant(x=FAKE, ldx=100, up=FAKE, ldu=100, act=0, rows=3, d=100, dtype=prox.F16, codes=FAKE, ldc=112, scales=FAKE):
    return prox.lib().prox_quant_q8(x, ldx, up, ldu, act, rows, d, dtype, codes, ldc, scales, None)


def _read(codes=FAKE, ldc=112, scales=FAKE, rows=3, d=100, out=FAKE):
    return prox.lib().prox_read_q8(codes, ldc, scales, rows, d, out, None)


def test_linear_sizes():
    assert prox.linear_w8_bytes(1, 1) >= 64 * 128 + 64 * 4
    assert prox.linear_w8_bytes(1000, 1000) >= 1024 * 1024 + 4000
    assert prox.linear_w8_bytes(1 << 20, 65536) > 1 << 36        # past 32 bits
    for bad in [(0, 1), (1, 0), (-1, 5), (1, 65537), ((1 << 20) + 1, 1), (2 ** 32 + 5, 64), (5, 2 ** 32 + 64)]:
        assert prox.linear_w8_bytes(*bad) == 0, bad
    with pytest.raises(TypeError):
        prox.linear_w8_bytes(10.0, 10)


def test_linear_refusals():
    L = prox.lib()
    assert L.prox_linear_w8(None, FAKE, 1008, FAKE, 1, None, FAKE, 1000, None) == INVALID
    for q, want in [(_lin(blob=None), INVALID), (_lin(blob=FAKE + 16), INVALID), (_lin(dtype=2), INVALID), (_lin(n=0), INVALID),
                    (_lin(k=-1), INVALID), (_lin(k=65537), UNSUPPORTED), (_lin(n=(1 << 20) + 1), UNSUPPORTED),
                    (_lin(nbytes=prox.linear_w8_bytes(1000, 1000) - 1), WORKSPACE)]:
        assert _run(q) == want
        assert L.prox_pack_linear_w8(FAKE, ctypes.byref(q), None) == want
        assert L.prox_unpack_linear_w8(ctypes.byref(q), FAKE, FAKE, None) == want
    assert _run(codes=None) == INVALID and _run(scales=None) == INVALID and _run(y=None) == INVALID
    assert _run(codes=FAKE + 8) == INVALID and _run(scales=FAKE + 2) == INVALID and _run(y=FAKE + 1) == INVALID
    assert _run(bias=FAKE + 1) == INVALID and _run(rows=-1) == INVALID
    assert _run(ldc=1000) == INVALID and _run(ldc=992) == INVALID and _run(ldy=999) == INVALID
    assert _run(ldc=prox.MAX_Q8_PITCH + 16) == UNSUPPORTED and _run(rows=prox.MAX_Q8_ROWS + 1) == UNSUPPORTED
    assert _run(q=_lin(n=1 << 20, k=16), rows=1 << 22, ldc=16, ldy=1 << 20) == UNSUPPORTED      # grid
    assert _run(rows=0, codes=None, y=None) == OK                                            # nothing is enqueued
    assert L.prox_pack_linear_w8(None, ctypes.byref(_lin()), None) == INVALID
    assert L.prox_pack_linear_w8(FAKE + 1, ctypes.byref(_lin()), None) == INVALID
    assert L.prox_unpack_linear_w8(ctypes.byref(_lin()), None, FAKE, None) == INVALID
    assert L.prox_unpack_linear_w8(ctypes.byref(_lin()), FAKE, FAKE + 2, None) == INVALID


@pytest.mark.parametrize("call", [_norm, _quant, _read])
def test_rows_refusals(call):
    assert call(rows=-1) == INVALID and call(d=0) == INVALID and call(d=-5) == INVALID
    assert call(rows=prox.MAX_Q8_ROWS + 1) == UNSUPPORTED and call(d=65537) == UNSUPPORTED
    assert call(rows=0) == OK
    assert call(codes=None) == INVALID and call(scales=None) == INVALID
    assert call(codes=FAKE + 8) == INVALID and call(scales=FAKE + 2) == INVALID
    assert call(ldc=96) == INVALID and call(ldc=104) == INVALID and call(ldc=-112) == INVALID


def test_norm_refusals():
    for name in ("x", "y", "r", "out", "gain"):
        assert _norm(**{name: FAKE + 1}) == INVALID, name
    for name in ("ldx", "ldy", "ldr", "ldo"):
        assert _norm(**{name: 99}) == INVALID and _norm(**{name: -100}) == INVALID and _norm(**{name: 0}) == INVALID, name
    assert _norm(x=None) == INVALID and _norm(dtype=2) == INVALID and _norm(dtype=-1) == INVALID
    for eps in (-1e-6, float("nan"), float("inf")):
        assert _norm(eps=eps) == INVALID
    assert _norm(codes=None, scales=None, out=None) == INVALID              # nothing to compute
    assert _norm(out=3 * FAKE) == INVALID                                   # r and out the same
    assert _norm(r=FAKE, ldr=104) == INVALID and _norm(out=2 * FAKE, ldo=104) == INVALID   # in place, another stride


def test_quant_refusals():
    assert _quant(x=None) == INVALID and _quant(x=FAKE + 1) == INVALID and _quant(up=FAKE + 1) == INVALID
    assert _quant(ldx=99) == INVALID and _quant(ldu=99) == INVALID and _quant(dtype=3) == INVALID
    assert _quant(act=2) == INVALID and _quant(act=-1) == INVALID
    assert _read(out=None) == INVALID and _read(out=FAKE + 2) == INVALID


def test_limits_match_the_header():
    text = open(f"{B.INCLUDE}/prox.h").read()
    for name, value in (("ROWS", prox.MAX_Q8_ROWS), ("PITCH", prox.MAX_Q8_PITCH)):
        a, b = re.search(rf"#define PROX_MAX_Q8_{name} \((\d+) << (\d+)\)", text).groups()
        assert int(a) << int(b) == value


def test_binding_refuses_host_tensors_and_other_types():
    x = torch.zeros((2, 32), dtype=torch.bfloat16)
    for f in (prox.rmsnorm, prox.rmsnorm_q8, prox.quant_q8):
        with pytest.raises(ValueError):
            f(x)
        with pytest.raises(ValueError):
            f(x.float())
    q = prox.new_rows_q8(2, 30, device="cpu")
    assert q.codes.shape == (2, 30) and q.codes.stride(0) == 32
    with pytest.raises(ValueError):
        prox.read_q8(q)
    with pytest.raises(ValueError):
        prox.pack_linear_w8(x.float())
    with pytest.raises(TypeError):
        prox.new_rows_q8(2.0, 30, device="cpu")


@pytest.mark.parametrize("far", [2 ** 32, -2 ** 32, 2 ** 64])
def test_structs_keep_no_lower_bits(far, monkeypatch):
    monkeypatch.setattr(prox, "_dev_tensor", lambda t, *a: t)
    w = prox.LinearW8(torch.zeros(256, dtype=torch.uint8), torch.bfloat16, 100 + far, 1024 + far).struct()
    end = 2 ** 31 - 1 if far > 0 else -2 ** 31
    assert [w.n, w.k] == [end] * 2
