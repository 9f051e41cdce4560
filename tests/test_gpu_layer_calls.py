"""Calls of the attention half that stand apart: the largest sizes, capture of every kind of variant, calls on two
streams at once, prompts attended in place, handles shared by calls of several sizes."""
import pickle

import numpy as np
import pytest
import torch

import layer_ref as R
from paper_2607_27591_amd import prox
from test_gpu_attn import Case
from test_gpu_kv_cache import i32, poisoned, randn, rope_table, starts, want_kv

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16


@pytest.mark.parametrize("n,k,group,batch", [(1 << 20, 128, 128, 3), (1 << 20, 64, 32, 64), (40, 65536, 65536, 1), (40, 65536, 65536, 64), (17, 65504, 32, 9)])
def test_largest_projections(n, k, group, batch):
    w = randn((n, k), 1, BF16, 0.02) if n < 1000 else randn((4096, k), 1, BF16, 0.02).repeat(n // 4096, 1)
    q = prox.pack_linear_w4(w, group)
    x = randn((batch, k), 2, BF16)
    y = prox.linear_w4(q, x)
    few = min(n, 4096)
    ref, bound = R.linear(R.f64(x), *R.quantise(R.f64(w[:few]), group))
    R.check(y[:, :few], ref, bound, BF16, "first outputs")
    assert torch.equal(y, y[:, :few].repeat(1, n // few))


@pytest.mark.parametrize("n,k,batch", [(28672, 256, 64), (9000, 384, 30), (9000, 384, 7), (300, 1024, 1)])
def test_captured_projections(n, k, batch):
    q = prox.pack_linear_w4(randn((n, k), 1, BF16, 0.02))
    x, y = randn((batch, k), 2, BF16), torch.empty((batch, n), dtype=BF16, device="cuda")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):   # the first call of the shape
        prox.linear_w4(q, x, y=y)
    for seed in range(3):
        x.copy_(randn((batch, k), 5 + seed, BF16))
        y.fill_(float("nan"))
        g.replay()
        assert torch.equal(y, prox.linear_w4(q, x))
        torch.cuda.synchronize()


@pytest.mark.parametrize("ratio,lens,news,window", [(4, [900, 33, 700], [5, 3, 1], 0), (8, [3000, 40], [1, 1], 0), (2, [300, 200], [300, 120], 100),
                                                    (4, [700] * 8, [300] * 8, 0)])
def test_prompts_in_place(ratio, lens, news, window):
    case = Case(2, ratio, 128, 64, 64, BF16, lens, news)
    want = prox.kv_attn(case.c, case.seqs(), case.q, window=window)
    q = case.q.clone()
    assert prox.kv_attn(case.c, case.seqs(), q, window=window, out=q) is q
    assert torch.equal(q, want)


def test_two_streams_at_once():
    # Calls on two streams, each with a workspace of its own, over one cache; the second appends to pages of its own.
    case = Case(2, 4, 128, 64, 64, BF16, [5000, 300], [1, 1], slack=2)
    want = prox.kv_attn(case.c, case.seqs(), case.q)
    k, v = (randn((40, 2, 128), i, BF16) for i in (7, 8))
    free = sorted(set(range(case.c.n_pages)) - set(case.table.flatten().tolist()))
    other = prox.KVSeqs(i32([40]), i32([[free[0]]]), max_new=40)
    q2 = randn((40, 8, 128), 9, BF16)
    prox.kv_append(case.c, other, k, v)
    want2 = prox.kv_attn(case.c, other, q2)
    ws = [prox.new_kv_attn_workspace(128) for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(10):
        with torch.cuda.stream(streams[0]):
            got[0].append(prox.kv_attn(case.c, case.seqs(), case.q, ws=ws[0]))
        with torch.cuda.stream(streams[1]):
            prox.kv_append(case.c, other, k, v)
            got[1].append(prox.kv_attn(case.c, other, q2, ws=ws[1]))
    torch.cuda.synchronize()
    assert all(torch.equal(g, want) for g in got[0]) and all(torch.equal(g, want2) for g in got[1])


def test_a_handle_serves_calls_of_several_sizes():
    case = Case(1, 2, 64, 32, 32, F16, [70, 33], [1, 1])
    s = prox.KVSeqs(case.kv_len, case.table, max_new=4, cu_new=starts([1, 1]))
    want = prox.kv_attn(case.c, s, case.q)
    for rows in (5, 2, 9, 2):   # rows behind the last sequence
        q = torch.cat([case.q, randn((rows, 2, 64), rows, F16)])[:max(rows, 2)]
        out = torch.full_like(q, 3.0)
        prox.kv_attn(case.c, s, q, out=out)
        assert torch.equal(out[:2], want) and (out[2:] == 3).all()
    c, t = pickle.loads(pickle.dumps((case.c, s)))
    assert torch.equal(prox.kv_attn(c, t, case.q), want)


@pytest.mark.parametrize("heads,ratio,dim,group,page", [(256, 1, 64, 64, 32), (1, 4096, 64, 32, 32768), (2, 300, 128, 128, 4096)])
def test_most_heads_and_largest_pages(heads, ratio, dim, group, page):
    lens = [40, 3]
    c = poisoned(3, page, heads, dim, BF16, group=group)
    table = i32([[2], [0]]) if page > 32 else i32([[2, 1], [0, 0]])
    n = sum(lens)
    k, v = (randn((n, heads, dim), i, BF16) for i in (1, 2))
    rope = prox.Rope(rope_table(2 * page, dim))
    s = prox.KVSeqs(i32(lens), table, max_new=40, cu_new=starts(lens))
    q = randn((n, heads * ratio, dim), 3, BF16)
    qr = prox.kv_append(c, s, k, v, q=q, rope=rope)
    pos = np.concatenate([np.arange(l) for l in lens])
    assert np.array_equal(R.f64(qr), R.to_type(R.rotate(R.f64(q), R.f64(rope.table), pos, False), BF16))
    kw, vw = want_kv(k, v, pos, c, rope)
    last = torch.tensor([39, 42], device="cuda")
    got = prox.kv_attn(c, prox.KVSeqs(i32(lens), table), qr[last].contiguous())
    for i, (a, l) in enumerate(((0, 40), (40, 3))):
        ref, bound = R.attention(R.f64(qr[last[i:i + 1]]), kw[a:a + l], vw[a:a + l], np.array([l - 1]), dim ** -0.5)
        R.check(got[i:i + 1], ref, bound, BF16, f"sequence {i}")


def test_a_page_table_of_the_most_positions():
    # 2^30 positions of room, 1000 of them taken: grids and splits follow the room, the work the lengths.
    page, n = 32768, 1000
    c = poisoned(2, page, 1, 64, BF16, group=64)
    table = torch.full((1, 2 ** 30 // page), -1, dtype=torch.int32, device="cuda")
    table[0, 0] = 1
    k, v, q = (randn((n, h, 64), i, BF16) for i, h in ((1, 1), (2, 1), (3, 4)))
    s = prox.KVSeqs(i32([n]), table, max_new=n)
    prox.kv_append(c, s, k, v)
    kw, vw = want_kv(k, v, None, c)
    for new in (1, 70):
        got = prox.kv_attn(c, prox.KVSeqs(i32([n]), table, max_new=new), q[:new], window=0 if new == 1 else 2 ** 30 - 1)
        ref, bound = R.attention(R.f64(q[:new]), kw, vw, np.arange(n - new, n), 0.125)
        R.check(got, ref, bound, BF16, f"{new} new")
