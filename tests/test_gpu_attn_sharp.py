"""Attention over the 4-bit paged cache on inputs whose answers show a lost, doubled or misplaced token
(attn_ref.py; test_attn_bounds_cpu.py shows which mistakes these checks see)."""
import numpy as np
import pytest

import attn_ref as A
import layer_ref as R
from paper_2607_27591_amd import prox
from test_gpu_kv_cache import i32, poisoned, starts, table_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shape", A.SHAPES + A.MORE, ids=lambda s: "-".join(map(str, s[:5])))
@pytest.mark.parametrize("kind", A.KINDS)
def test_sharp_answers(shape, kind):
    x = A.Inputs(*shape, kind)
    S, per = len(x.lens), -(-max(x.lens) // x.page)
    c = poisoned(S * per + 2, x.page, x.heads, x.dim, x.dtype, group=x.group)
    table = table_of(S, per, c.n_pages, 7)
    every = prox.KVSeqs(i32(x.lens), table, max_new=max(x.lens), cu_new=starts(x.lens))
    prox.kv_append(c, every, x.k.cuda(), x.v.cuda())
    ref, bound, _ = x.attention()
    for max_kv in (0, max(x.lens)):   # splits for the room in the pages, and for the longest sequence
        s = prox.KVSeqs(every.kv_len, table, max_new=max(x.news), cu_new=starts(x.news), max_kv=max_kv)
        got = R.f64(prox.kv_attn(c, s, x.q.cuda(), scale=x.scale, window=x.window))
        share, whole = A.violations(got, ref, bound, x.dtype)
        print(f"    {kind}: {share:.4f} of the values past the bound, the whole {whole:.3f}", flush=True)
        assert np.isfinite(got).all() and share == 0 and whole <= 1
