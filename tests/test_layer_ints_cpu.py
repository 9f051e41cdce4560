"""Sizes past 32 bits are refused by the binding of the attention half's calls, not cut to their lower bits."""
import pytest
import torch

from paper_2607_27591_amd import prox

FAR = [2 ** 32, -2 ** 32, 2 ** 64]


@pytest.mark.parametrize("far", FAR)
def test_sizes(far):
    good = (8, 128, 64, 64, 100)
    assert prox.kv_bytes(*good) > 0 and prox.linear_w4_bytes(100, 1024, 128) > 0
    for i in range(5):
        assert prox.kv_bytes(*(v + far * (i == j) for j, v in enumerate(good))) == 0
    for i in range(3):
        assert prox.linear_w4_bytes(*(v + far * (i == j) for j, v in enumerate((100, 1024, 128)))) == 0
    assert prox.kv_attn_workspace_bytes(128 + far) == 0
    with pytest.raises(prox.ProxError):
        prox.new_kv_cache(100 + far, 64, 8, 128, torch.bfloat16, device="cpu")


@pytest.mark.parametrize("far", FAR)
def test_structs_keep_no_lower_bits(far, monkeypatch):
    monkeypatch.setattr(prox, "_dev_tensor", lambda t, *a: t)
    blob = torch.zeros(256, dtype=torch.uint8)
    end = 2 ** 31 - 1 if far > 0 else -2 ** 31
    c = prox.KVCache(blob, torch.bfloat16, 8 + far, 128 + far, 64 + far, 64 + far, 100 + far).struct()
    assert [c.kv_heads, c.head_dim, c.group, c.page_size, c.n_pages] == [end] * 5
    q = prox.LinearW4(blob, torch.bfloat16, 100 + far, 1024 + far, 128 + far).struct()
    assert [q.n, q.k, q.group] == [end] * 3
    lens, table = torch.zeros(2, dtype=torch.int32), torch.zeros((2, 3), dtype=torch.int32)
    s = prox.KVSeqs(lens, table, max_new=1 + far, max_kv=5 + far).struct(2)
    assert [s.n_seq, s.max_new, s.n_tokens, s.max_kv, s.max_pages] == [2, end, 2, end, 3]


def test_numbers_that_are_not_whole_are_refused(monkeypatch):
    monkeypatch.setattr(prox, "_dev_tensor", lambda t, *a: t)
    lens, table = torch.zeros(2, dtype=torch.int32), torch.zeros((2, 3), dtype=torch.int32)
    for kw in (dict(max_new=1.5), dict(max_new=1.0), dict(max_kv=5.0), dict(max_kv="5")):
        with pytest.raises(TypeError):
            prox.KVSeqs(lens, table, **kw).struct(2)
    for bad in ((8.0, 128, 64, 64, 100), (8, 128, 64, 64.5, 100)):
        with pytest.raises(TypeError):
            prox.kv_bytes(*bad)
    assert prox.KVSeqs(lens, table, max_new=torch.tensor(3)).struct(2).max_new == 3


def test_append_grid_past_64_bits():
    # n_seq * max_new * q_heads * head_dim / 8 = 2^63 (nothing is dereferenced or launched).
    import ctypes
    at = 0x100000
    c = prox._KVCache(prox.BF16, 1, 256, 64, 32768, 1, at, 1 << 45)
    for new in (1 << 30, (1 << 30) - 1, 1 << 29):
        s = prox._KVSeqs(65536, new, 10, 0, 32768, at, at, at)
        assert prox.lib().prox_kv_append(ctypes.byref(c), ctypes.byref(s), at, 256, at, 256, at, 4096, 1 << 20, at, 1 << 20,
                                         None, None) == 2
