"""A decoder layer's decode steps on INT4 weights and the 4-bit cache, as a serving loop runs
them: projection, append with rotation, attention, output projection, residual and norm, sparse
FFN, residual and norm.  Each operator against its 64-bit formula on its own input, and the
whole step captured once and replayed."""
import numpy as np
import pytest
import torch

import layer_ref as R
from paper_2607_27591_amd import prox
from test_gpu_kv_cache import i32, poisoned, randn, rope_table, starts, table_of

pytestmark = pytest.mark.gpu


class Layer:
    def __init__(self, dtype, batch, d=512, f=700, hq=8, hkv=2, dim=64, group=32):
        self.dtype, self.hq, self.hkv, self.dim, self.batch = dtype, hq, hkv, dim, batch
        self.w_qkv = randn(((hq + 2 * hkv) * dim, d), 1, dtype, 0.05)
        self.w_o = randn((d, hq * dim), 2, dtype, 0.05)
        ffn = prox.Weights(*(randn((f, d), 3 + i, dtype, 0.02) for i in range(3)))
        self.qkv, self.o = prox.pack_linear_w4(self.w_qkv), prox.pack_linear_w4(self.w_o)
        self.ffn, self.proxy = prox.pack_w4(ffn), prox.pack_proxy(ffn)
        self.cache = poisoned(4 * batch, 32, hkv, dim, dtype, group=group)
        self.table = table_of(batch, 4, 4 * batch)
        self.rope = prox.Rope(rope_table(128, dim))
        self.kv_len = i32([0] * batch)
        self.ws, self.aws = prox.new_workspace(d, f, batch, w4=True), prox.new_kv_attn_workspace(dim)
        self.d, self.f = d, f

    def parts(self, qkv):
        return (p.view(qkv.shape[0], -1, self.dim) for p in
                qkv.split([self.hq * self.dim, self.hkv * self.dim, self.hkv * self.dim], 1))

    def step(self, x):
        seqs = prox.KVSeqs(self.kv_len, self.table)
        self.kv_len.add_(1)
        qkv = prox.linear_w4(self.qkv, x)
        raw = qkv.clone()
        q, k, v = self.parts(qkv)
        prox.kv_append(self.cache, seqs, k, v, q=q, q_out=q, rope=self.rope)
        a = prox.kv_attn(self.cache, seqs, q, ws=self.aws)
        o = prox.linear_w4(self.o, a.view(self.batch, -1))
        h = prox.add_rmsnorm(x, o)
        y, _ = prox.ffn_sparse_w4(self.ffn, self.proxy, h, self.d // 2, self.f // 2, ws=self.ws)
        return raw, q, a, o, h, prox.add_rmsnorm(h, y)


@pytest.mark.parametrize("dtype,batch", [(torch.bfloat16, 1), (torch.float16, 5)])
def test_decode_steps(dtype, batch):
    L = Layer(dtype, batch)
    codes = [R.quantise(R.f64(w), 128) for w in (L.w_qkv, L.w_o)]
    ks, vs = [[] for _ in range(batch)], [[] for _ in range(batch)]
    x = randn((batch, L.d), 9, dtype)
    for step in range(40):   # over a block and a page of 32
        raw, q, a, o, h, x_next = L.step(x)
        ref, bound = R.linear(R.f64(x), *codes[0])
        R.check(raw, ref, bound, dtype, f"step {step} qkv")
        qr, kr, vr = (R.f64(p) for p in L.parts(raw))
        pos, table = np.full(batch, step), R.f64(L.rope.table)
        assert np.array_equal(R.f64(q), R.to_type(R.rotate(qr, table, pos, False), dtype))
        kr = R.to_type(R.rotate(kr, table, pos, False), dtype)
        want = [np.zeros((0,))] * 2
        for b in range(batch):
            ks[b].append(R.values(*R.quantise(kr[b], 32)))
            vs[b].append(R.values(*R.quantise(vr[b], 32)))
            want = R.attention(R.f64(q)[b:b + 1], np.stack(ks[b]), np.stack(vs[b]), [step], L.dim ** -0.5)
            R.check(a[b:b + 1], *want, dtype, f"step {step} attention {b}")
        ref, bound = R.linear(R.f64(a.view(batch, -1)), *codes[1])
        R.check(o, ref, bound, dtype, f"step {step} out")
        assert torch.isfinite(x_next).all()
        x = x_next


def test_prompt_then_captured_steps():
    # A prompt of unequal lengths enters the cache, then decode steps run eagerly in one layer
    # and as replays of one captured step in another.
    dtype, batch, lens = torch.bfloat16, 3, [50, 1, 33]
    eager, graph = Layer(dtype, batch), Layer(dtype, batch)
    T = sum(lens)
    for L in (eager, graph):
        L.kv_len.copy_(i32(lens))
        seqs = prox.KVSeqs(L.kv_len, L.table, max_new=50, cu_new=starts(lens))
        q, k, v = L.parts(torch.cat([prox.linear_w4(L.qkv, randn((T, L.d), 7, dtype)[i:i + 64]) for i in range(0, T, 64)]))
        prox.kv_append(L.cache, seqs, k, v, q=q, q_out=q, rope=L.rope)
        L.prompt = prox.kv_attn(L.cache, seqs, q, ws=L.aws)
    assert torch.equal(eager.prompt, graph.prompt)
    x = randn((batch, eager.d), 9, dtype)
    graph.step(x)                        # warm-up, taken back
    graph.kv_len.copy_(i32(lens))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = graph.step(x)
    graph.kv_len.copy_(i32(lens))
    for step in range(5):
        x.copy_(randn((batch, eager.d), 30 + step, dtype))
        g.replay()
        want = eager.step(x)
        for i, (p, w) in enumerate(zip(out, want)):
            assert torch.equal(p, w), f"step {step}, output {i}"
        torch.cuda.synchronize()
