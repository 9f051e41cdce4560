"""Projections on INT4 weights of rows with a single input: each output is that input's weight,
sigma q, to the last bit, so that an input lost, doubled or misplaced shows."""
import pytest
import torch

import layer_ref as R
from paper_2607_27591_amd import prox

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16


@pytest.mark.parametrize("n,k,group,dtype", [(33, 1120, 32, BF16), (500, 1088, 64, F16), (1025, 640, 128, BF16), (4100, 768, 384, F16),
                                             (8200, 480, 32, F16), (9000, 576, 64, BF16), (12300, 512, 128, F16), (16400, 352, 32, BF16)])
@pytest.mark.parametrize("batch", [1, 5, 16, 23, 40, 64])
def test_single_inputs(n, k, group, dtype, batch):
    g = torch.Generator().manual_seed(n)
    w = (torch.randn((n, k), generator=g) * 0.02).to(dtype)
    q = prox.pack_linear_w4(w.cuda(), group)
    want = torch.from_numpy(R.values(*R.quantise(R.f64(w), group))).to(dtype).cuda()   # fp64 of 15 bits, rounded once
    step = 7 if batch == 1 else 1
    order = torch.randperm(k, generator=g)[::step]
    for i in range(0, len(order), batch):
        at = order[i:i + batch]
        at = torch.cat([at, order[:batch - len(at)]])
        x = torch.zeros((batch, k), dtype=dtype)
        x[torch.arange(batch), at] = 1.0
        y = prox.linear_w4(q, x.cuda())
        assert torch.equal(y, want[:, at.cuda()].t()), f"inputs {at.tolist()}"
