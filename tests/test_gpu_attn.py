"""Attention over the 4-bit paged cache against the 64-bit formula on what the cache holds."""
import copy
import sys

import numpy as np
import pytest
import torch

import layer_ref as R
from paper_2607_27591_amd import prox
from test_gpu_kv_cache import i32, poisoned, randn, starts, table_of, want_kv

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16


class Case:
    """A cache that holds `lens` tokens of each sequence, and `news` queries of each."""

    def __init__(self, heads, ratio, dim, group, page, dtype, lens, news, seed=0, spread=1.0, slack=0):
        self.lens, self.news, self.ratio = lens, news, ratio
        S, per = len(lens), -(-max(max(lens), 1) // page) + slack
        self.c = poisoned(S * per + 2, page, heads, dim, dtype, group=group)
        self.table = table_of(S, per, self.c.n_pages, seed)
        n = sum(lens)
        self.k, self.v = randn((n, heads, dim), seed + 1, dtype), randn((n, heads, dim), seed + 2, dtype)
        self.q = randn((sum(news), heads * ratio, dim), seed + 3, dtype, spread)
        self.kv_len = i32(lens)
        if n:
            prox.kv_append(self.c, prox.KVSeqs(self.kv_len, self.table, max_new=max(lens), cu_new=starts(lens)), self.k, self.v)
        self.kw, self.vw = want_kv(self.k, self.v, None, self.c) if n else (R.f64(self.k), R.f64(self.v))

    def seqs(self, **kw):
        uniform = len(set(self.news)) == 1
        return prox.KVSeqs(self.kv_len, self.table, max_new=max(max(self.news), 1),
                           cu_new=None if uniform else starts(self.news), **kw)

    def want(self, scale, window=0, q=None):
        q = R.f64(self.q if q is None else q)
        out, bound, t, a = [], [], 0, 0
        for n, l in zip(self.news, self.lens):
            o, b = R.attention(q[t:t + n], self.kw[a:a + l], self.vw[a:a + l], np.arange(l - n, l), scale, window)
            out.append(o)
            bound.append(b)
            t, a = t + n, a + l
        return np.concatenate(out), np.concatenate(bound)

    def check(self, window=0, scale=None, tag="", **kw):
        scale = self.c.head_dim ** -0.5 if scale is None else scale
        got = prox.kv_attn(self.c, self.seqs(**kw), self.q, scale=scale, window=window)
        ref, bound = self.want(scale, window)
        R.check(got, ref, bound, self.c.dtype, tag)
        return got


SHAPES = [  # heads, ratio, dim, group, page, dtype, lengths, new tokens, window
    (1, 1, 64, 32, 32, BF16, [1], [1], 0),
    (1, 1, 64, 64, 32, F16, [1, 2, 31, 32, 33, 0], [1] * 6, 0),
    (8, 4, 128, 64, 64, BF16, [100, 1, 64, 999], [1] * 4, 0),
    (2, 7, 128, 32, 96, F16, [500, 97], [1] * 2, 0),
    (8, 8, 128, 128, 64, BF16, [2049], [1], 0),
    (1, 16, 256, 64, 256, F16, [300, 1024], [1] * 2, 100),
    (1, 17, 64, 32, 32, BF16, [130], [1], 0),
    (2, 5, 256, 128, 32, BF16, [333, 40], [3, 3], 0),
    (2, 7, 64, 32, 32, F16, [401, 5, 64, 33], [5, 1, 2, 4], 33),
    (4, 4, 128, 64, 128, BF16, [200, 150, 70], [70, 33, 70], 0),
    (1, 3, 128, 128, 32, F16, [513], [513], 0),
    (2, 2, 256, 32, 64, F16, [95, 180], [95, 20], 17),
    (3, 1, 64, 64, 32, BF16, [260], [260], 1),
    (1, 32, 128, 64, 64, BF16, [700], [3], 0),
    (1, 64, 64, 32, 64, BF16, [100, 63], [2, 1], 0),
    (2, 4, 128, 64, 64, F16, [20000], [1], 0),
    (1, 8, 128, 32, 256, BF16, [9001, 3, 5000], [2, 1, 1], 0),
    # up to 4 and up to 8 rows of a kv head, at every head_dim and group
    (2, 2, 256, 32, 32, BF16, [700, 40, 33], [1] * 3, 0),
    (2, 1, 256, 64, 64, F16, [1, 95, 600], [4, 2, 3], 20),
    (1, 4, 256, 128, 32, BF16, [45], [1], 0),
    (1, 8, 256, 32, 64, F16, [650, 32], [1] * 2, 0),
    (2, 3, 256, 64, 32, BF16, [77, 2], [2, 1], 31),
    (1, 7, 256, 128, 32, F16, [300], [1], 0),
    (3, 2, 64, 32, 32, F16, [64, 700], [2, 1], 0),
    (2, 6, 64, 64, 96, BF16, [95, 1, 640], [1] * 3, 40),
    (2, 3, 64, 32, 32, BF16, [0, 90], [2, 2], 1),
    (2, 3, 128, 32, 32, BF16, [600, 31], [1] * 2, 0),
    (4, 1, 128, 128, 64, F16, [100, 3], [3, 4], 0),
    (2, 2, 128, 32, 32, F16, [700, 4], [3, 4], 64),
    (1, 5, 128, 128, 32, BF16, [520, 9], [1] * 2, 0),
    # many rows of many heads: the cache is not split
    (8, 1, 128, 64, 64, BF16, [300] * 16, [70] * 16, 0),
    (16, 2, 64, 32, 32, F16, [150, 90, 400, 33, 70, 64, 100, 65], [90, 90, 130, 1, 70, 64, 3, 65], 0),
    (16, 3, 64, 64, 96, BF16, [260, 130, 95, 30], [200, 128, 95, 40], 50),
    (32, 4, 128, 128, 128, F16, [100, 64], [100, 64], 0),
    (32, 1, 128, 32, 32, BF16, [333, 200], [200, 140], 33),
]


@pytest.mark.parametrize("heads,ratio,dim,group,page,dtype,lens,news,window", SHAPES)
def test_parity(heads, ratio, dim, group, page, dtype, lens, news, window):
    case = Case(heads, ratio, dim, group, page, dtype, lens, news)
    a = case.check(window, tag="parity")
    b = prox.kv_attn(case.c, case.seqs(), case.q, window=window)
    assert torch.equal(a, b)                               # the same bits every time
    case.check(window, tag="tight max_kv", max_kv=max(lens) or 1)


PAIRS = [  # as SHAPES, and pages past the longest sequence: rows and room for two tiles a workgroup
    (2, 7, 128, 32, 256, BF16, [700, 5], [5, 5], 0, 128),
    (2, 8, 128, 128, 256, F16, [300, 64, 33], [5, 1, 4], 0, 128),
    (8, 4, 128, 64, 256, BF16, [900, 0, 340, 600], [300, 2, 299, 40], 150, 0),
    (4, 7, 64, 32, 256, F16, [401, 5, 300, 333], [300, 1, 200, 133], 133, 0),
    (4, 5, 64, 64, 256, BF16, [2, 95], [4, 4], 0, 128),
    (1, 20, 128, 64, 256, F16, [1100] * 9, [1] * 9, 0, 128),
    # not split
    (8, 4, 128, 64, 64, BF16, [520] * 4, [300] * 4, 0, 0),
    (2, 8, 128, 128, 64, F16, [700, 650, 600], [512, 300, 200], 0, 0),
    (8, 4, 128, 32, 32, BF16, [500, 480, 470, 490], [300, 1, 299, 300], 160, 0),
    (8, 4, 64, 64, 64, F16, [520] * 4, [300, 299, 1, 300], 0, 0),
]


@pytest.mark.parametrize("heads,ratio,dim,group,page,dtype,lens,news,window,slack", PAIRS)
def test_two_tiles(heads, ratio, dim, group, page, dtype, lens, news, window, slack):
    Case(heads, ratio, dim, group, page, dtype, lens, news, slack=slack).check(window, tag="room")


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("news", [[1, 1], [20, 20]])
def test_peaked_and_flat_scores(dtype, news):
    # Scores far apart (one position takes all) and all alike.
    case = Case(2, 4, 128, 64, 64, dtype, [900, 450], news, spread=12.0)
    case.check(tag="peaked")
    case.check(scale=0.0, tag="flat")
    case.check(scale=-0.05, tag="negative")


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_values_of_any_size(dtype):
    # Values (and their scales) over the type's range from token to token, weights that
    # bring them together: each keeps its precision.
    case = Case(1, 2, 64, 32, 32, dtype, [96], [1])
    size = torch.logspace(-4, 3 if dtype == F16 else 4, 96, dtype=torch.float64)[torch.randperm(96, generator=torch.Generator().manual_seed(3))]
    v = (torch.randn((96, 1, 64), generator=torch.Generator().manual_seed(4)).double() * size[:, None, None]).to(dtype).cuda()
    case.v = v
    prox.kv_append(case.c, prox.KVSeqs(case.kv_len, case.table, max_new=96), case.k, v)
    case.kw, case.vw = want_kv(case.k, v, None, case.c)
    case.check(tag="values", scale=0.6)


def test_empty_rows_are_zero_whatever_the_query_holds():
    # A sequence of length 0, a padded one (fewer tokens than rows), and rows behind the last
    # sequence, which stay as they are.
    case = Case(2, 2, 128, 64, 32, BF16, [0, 2, 40], [3, 4, 2])
    q = torch.cat([case.q, randn((2, 4, 128), 9, BF16)])
    q[:5] = float("nan")
    out = torch.full_like(q, 5.0)
    prox.kv_attn(case.c, case.seqs(), q, out=out)
    assert (out[:5] == 0).all() and (out[9:] == 5).all()
    case.q = q[:9]
    case.q[:5] = 0
    ref, bound = case.want(128 ** -0.5)
    R.check(out[:9], ref, bound, BF16, "padded")


@pytest.mark.parametrize("ratio,news", [(4, 1), (3, 1), (4, 2), (7, 1), (16, 1), (4, 8)])
@pytest.mark.parametrize("value", ["nan", "inf"])
def test_a_row_spoils_no_other(ratio, news, value):
    # One head's query of one token is NaN or infinite, over whole and split caches.
    case = Case(2, ratio, 128, 64, 64, BF16, [40, 900], [news, news])
    want, bound = case.want(128 ** -0.5)
    q = case.q.clone()
    q[news - 1, 1] = q[2 * news - 1, ratio] = float(value)
    got = prox.kv_attn(case.c, case.seqs(), q)
    keep = torch.ones(q.shape[:2], dtype=torch.bool)
    keep[news - 1, 1] = keep[2 * news - 1, ratio] = False
    R.check(got[keep.cuda()], want[keep.numpy()], bound[keep.numpy()], BF16, "other rows")
    if value == "nan":
        assert torch.isnan(got[~keep.cuda()]).all()


def test_rows_past_max_new_and_bad_pages():
    case = Case(1, 2, 64, 32, 32, BF16, [200, 100], [4, 2])
    case.table[0, 2] = -5            # positions 64 .. 95 and 128 .. 159 of sequence 0 are hidden
    case.table[0, 4] = case.c.n_pages
    case.table[1] = 1 << 30          # all of sequence 1
    out = torch.full_like(case.q, 5.0)
    s = prox.KVSeqs(case.kv_len, case.table, max_new=3, cu_new=starts(case.news))
    prox.kv_attn(case.c, s, case.q, out=out)
    hidden = np.zeros(200, bool)
    hidden[64:96] = hidden[128:160] = True
    ref, bound = R.attention(R.f64(case.q[:3]), case.kw[:200], case.vw[:200], np.arange(196, 199), 0.125, hidden=hidden)
    R.check(out[:3], ref, bound, BF16, "hidden pages")
    assert (out[3] == 5).all() and (out[4:6] == 0).all()


def test_in_place_strides_and_shared_pages():
    # Queries as part of a fused projection, the output over the queries, and two sequences
    # that read the same pages.
    case = Case(2, 3, 128, 64, 64, BF16, [300, 300], [1, 1])
    case.table[1] = case.table[0]
    case.kw[300:], case.vw[300:] = case.kw[:300], case.vw[:300]
    want, bound = case.want(128 ** -0.5)
    wide = torch.zeros((2, 10 * 128), dtype=BF16, device="cuda")
    q = wide[:, 128:7 * 128].view(2, 6, 128)
    q.copy_(case.q)
    R.check(prox.kv_attn(case.c, case.seqs(), q), want, bound, BF16, "strided")
    prox.kv_attn(case.c, case.seqs(), q, out=q)
    R.check(q, want, bound, BF16, "in place")
    assert (wide[:, :128] == 0).all() and (wide[:, 7 * 128:] == 0).all()


@pytest.mark.parametrize("dtype,lens,news", [(BF16, [5000, 1, 70], [1, 1, 1]), (F16, [600, 64, 300], [40, 3, 17])])
def test_workspace_streams_and_graph(dtype, lens, news):
    # A workspace full of NaNs, another stream, and a captured call that follows lengths and
    # queries on replays, with eager work on the same workspace between them.
    case = Case(2, 4, 128, 64, 64, dtype, lens, news)
    ws = prox.new_kv_attn_workspace(128)
    ws.fill_(0xFF)
    want = case.check(tag="own workspace")
    assert torch.equal(want, prox.kv_attn(case.c, case.seqs(), case.q, ws=ws))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = prox.kv_attn(case.c, case.seqs(), case.q, ws=ws)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)
    out, full, seqs = torch.empty_like(want), case.kv_len.clone(), case.seqs()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        prox.kv_attn(case.c, seqs, case.q, out=out, ws=ws)
    for step in range(4):
        case.kv_len.copy_((full - step * 7).clamp(min=1))
        case.q.copy_(randn(case.q.shape, 20 + step, dtype))
        out.fill_(float("nan"))
        g.replay()
        assert torch.equal(out, prox.kv_attn(case.c, case.seqs(), case.q, ws=ws))
        torch.cuda.synchronize()


@pytest.mark.parametrize("news", [1, 40])
def test_pages_past_32_bits(news):
    # A cache of 5 GiB whose sequences stand on its first and last pages.
    heads, dim, page = 8, 128, 128
    per = prox.kv_bytes(heads, dim, 64, page, 1)
    c = prox.new_kv_cache(5 * 2 ** 30 // per, page, heads, dim, BF16)
    table = i32([[c.n_pages - 1, 0, c.n_pages - 2], [c.n_pages // 2, c.n_pages - 3, 1]])
    lens = [300, 257]
    k, v = (randn((sum(lens), heads, dim), i, BF16) for i in (1, 2))
    prox.kv_append(c, prox.KVSeqs(i32(lens), table, max_new=300, cu_new=starts(lens)), k, v)
    kw, vw = want_kv(k, v, None, c)
    q = randn((2 * news, heads, dim), 3, BF16)
    got = prox.kv_attn(c, prox.KVSeqs(i32(lens), table, max_new=news), q)
    for s, a in ((0, 0), (1, 300)):
        r = slice(s * news, (s + 1) * news)
        ref, bound = R.attention(R.f64(q[r]), kw[a:a + lens[s]], vw[a:a + lens[s]], np.arange(lens[s] - news, lens[s]), dim ** -0.5)
        R.check(got[r], ref, bound, BF16, f"sequence {s}")


def test_long_prompt_of_many_heads():
    # 9e6 rows of queries in one call.
    n, heads, window = 70000, 128, 40
    c = poisoned(n // 128 + 1, 128, 1, 64, BF16, group=64)
    s = prox.KVSeqs(i32([n]), i32([range(c.n_pages)]), max_new=n)
    k, v = (randn((n, 1, 64), i, BF16) for i in (1, 2))
    prox.kv_append(c, s, k, v)
    kw, vw = want_kv(k, v, None, c)
    q = randn((500, heads, 64), 3, BF16).repeat(n // 500, 1, 1)
    got = prox.kv_attn(c, s, q, window=window)
    for i in (0, 1, 39, 40, 35001, n - 1):
        a = max(i - window + 1, 0)
        ref, bound = R.attention(R.f64(q[i:i + 1]), kw[a:i + 1], vw[a:i + 1], np.array([i - a]), 64 ** -0.5)
        R.check(got[i:i + 1], ref, bound, BF16, f"row {i}")


@pytest.mark.parametrize("window", [40, 2 ** 31 - 1, 2 ** 32 + 5, sys.maxsize])
def test_window_past_the_cache(window):
    case = Case(2, 2, 64, 32, 32, BF16, [40, 3], [2, 2])
    assert torch.equal(prox.kv_attn(case.c, case.seqs(), case.q, window=window), prox.kv_attn(case.c, case.seqs(), case.q))


def test_copies_of_handles():
    case = Case(2, 2, 64, 32, 32, BF16, [40, 3], [1, 1])
    want = prox.kv_attn(case.c, case.seqs(), case.q)
    s = case.seqs()
    prox.kv_attn(case.c, s, case.q)
    c2, s2 = copy.deepcopy((case.c, s))
    assert torch.equal(prox.kv_attn(c2, s2, case.q), want)
    case.kv_len.zero_()                                  # the copy has lengths of its own
    assert torch.equal(prox.kv_attn(c2, s2, case.q), want)
    assert (prox.kv_attn(case.c, s, case.q) == 0).all()


def test_refusals():
    case = Case(2, 2, 64, 32, 32, BF16, [40], [1])
    s = case.seqs()
    for bad in [dict(q=case.q[:, :3]), dict(q=case.q.half()), dict(q=case.q.cpu()), dict(q=case.q[0]), dict(out=case.q[:, :2]),
                dict(ws=torch.empty(1024, dtype=torch.uint8, device="cuda")), dict(window=-1), dict(scale=float("nan")),
                dict(out=torch.empty((2, 4, 64), dtype=BF16, device="cuda"))]:
        with pytest.raises((ValueError, prox.ProxError)):
            prox.kv_attn(case.c, s, **{**dict(q=case.q), **bad})
