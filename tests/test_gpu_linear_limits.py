"""Projections at the ends of their sizes: what is served, and what is refused."""
import pytest
import torch

import rows8_ref as R
from layer_ref import f64
from paper_2607_27591_amd import prox

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def randn(shape, seed, dtype, scale=1.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * scale).to(dtype).cuda()


def test_linear_w4_refuses_batches_past_32_bits():
    """They do not lose their upper bits: one row is not taken for all."""
    w = prox.pack_linear_w4(randn((32, 128), 1, BF16))
    x, y = randn((1, 128), 2, BF16), torch.zeros((1, 32), dtype=BF16, device="cuda")
    for rows in (2 ** 32 + 1, 2 ** 32 + 2, 2 ** 31):
        with pytest.raises(prox.ProxError) as e:
            prox.linear_w4(w, x.expand(rows, 128), y=y.expand(rows, 32))
        assert e.value.status == 1
    assert (y == 0).all()


def test_linear_w8_of_the_most_rows():
    # 2^22 rows of 8200 outputs: y of 69 GB.
    rows, n, k, few = prox.MAX_Q8_ROWS, 8200, 16, 4096
    codes = torch.randint(-128, 128, (few, k), generator=torch.Generator().manual_seed(1)).to(torch.int8).cuda()
    scales = torch.linspace(0.01, 0.02, few, device="cuda")
    w = randn((n, k), 2, BF16, 0.02)
    p = prox.pack_linear_w8(w)
    one = prox.linear_w8(p, prox.RowsQ8(codes, scales))
    want, bound = R.linear(codes.cpu().numpy(), f64(scales), *(lambda c, s: (c, s.astype("float32")))(*R.codes(f64(w))))
    R.check(one, want, bound, BF16)
    y = torch.full((rows, n), 7.0, dtype=BF16, device="cuda")
    prox.linear_w8(p, prox.RowsQ8(codes.repeat(rows // few, 1), scales.repeat(rows // few)), y=y)
    for a in range(0, rows, few):
        assert torch.equal(y[a:a + few], one), a
