"""Host-side checks of the attention half's entry points: sizes, and refusals before any
HIP call (the pointers are never dereferenced), and where a row's token stands for odd
lengths, offsets and pages, compiled for the host."""
import ctypes
import re
import shutil
import subprocess

import pytest

from paper_2607_27591_amd import build as B
from paper_2607_27591_amd import prox

OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3
FAKE = 0x100000
BIG = 1 << 45


def _lin(dtype=prox.BF16, n=1000, k=1024, group=128, blob=FAKE, nbytes=BIG):
    return prox._W4Linear(dtype, n, k, group, blob, nbytes)


def test_linear_sizes():
    assert prox.linear_w4_bytes(1000, 1024, 128) >= 1000 * 512 + 1000 * 8 * 2
    assert prox.linear_w4_bytes(1, 32, 32) > 0
    assert prox.linear_w4_bytes(1 << 20, 65536, 128) > 1 << 34        # past 32 bits
    for bad in [(0, 128, 128), (1, 0, 128), (1, 130, 128), (1, 96, 96), (1, 128, 16), (1, 128, 0),
                (1, 128, -128), (1, 65536 + 128, 128), ((1 << 20) + 1, 128, 128), (1, 128, 256)]:
        assert prox.linear_w4_bytes(*bad) == 0, bad
    assert prox.linear_w4_bytes(10, 96, 32) > 0 and prox.linear_w4_bytes(10, 384, 384) > 0


def test_linear_refusals():
    L = prox.lib()

    def run(q=None, x=FAKE, ldx=1024, batch=1, bias=None, y=FAKE, ldy=1000):
        return L.prox_linear_w4(ctypes.byref(q or _lin()), x, ldx, batch, bias, y, ldy, None)

    assert L.prox_linear_w4(None, FAKE, 1024, 1, None, FAKE, 1000, None) == INVALID
    for q, want in [(_lin(blob=None), INVALID), (_lin(blob=FAKE + 16), INVALID), (_lin(dtype=2), INVALID),
                    (_lin(n=0), INVALID), (_lin(k=-32), INVALID), (_lin(k=1000), UNSUPPORTED),
                    (_lin(group=96), UNSUPPORTED), (_lin(nbytes=1000), WORKSPACE)]:
        assert run(q) == want
        assert L.prox_pack_linear_w4(FAKE, ctypes.byref(q), None) == want
        assert L.prox_unpack_linear_w4(ctypes.byref(q), FAKE, FAKE, None) == want
    assert run(x=None) == INVALID and run(y=None) == INVALID
    assert run(x=FAKE + 2) == INVALID and run(y=FAKE + 1) == INVALID and run(bias=FAKE + 1) == INVALID
    assert run(batch=0) == INVALID and run(batch=prox.MAX_BATCH + 1) == INVALID
    assert run(batch=2, ldx=1020) == INVALID and run(batch=2, ldx=1028) == INVALID
    assert run(batch=2, ldx=512) == INVALID and run(batch=2, ldy=999) == INVALID
    assert L.prox_pack_linear_w4(None, ctypes.byref(_lin()), None) == INVALID
    assert L.prox_pack_linear_w4(FAKE + 8, ctypes.byref(_lin()), None) == INVALID
    assert L.prox_unpack_linear_w4(ctypes.byref(_lin()), None, FAKE, None) == INVALID
    assert L.prox_unpack_linear_w4(ctypes.byref(_lin()), FAKE, FAKE + 1, None) == INVALID


def _cache(dtype=prox.BF16, heads=8, dim=128, group=64, page=64, pages=100, blob=FAKE, nbytes=BIG):
    return prox._KVCache(dtype, heads, dim, group, page, pages, blob, nbytes)


def _seqs(n=3, new=2, tokens=6, max_kv=0, pages=10, cu=None, kv_len=FAKE, table=FAKE):
    return prox._KVSeqs(n, new, tokens, max_kv, pages, cu, kv_len, table)


BAD_CACHES = [(dict(blob=None), INVALID), (dict(blob=FAKE + 64), INVALID), (dict(dtype=5), INVALID),
              (dict(heads=0), UNSUPPORTED), (dict(heads=257), UNSUPPORTED), (dict(dim=96), UNSUPPORTED),
              (dict(group=16), UNSUPPORTED), (dict(dim=64, group=128), UNSUPPORTED), (dict(page=16), UNSUPPORTED),
              (dict(page=80), UNSUPPORTED), (dict(page=65536), UNSUPPORTED), (dict(pages=0), UNSUPPORTED),
              (dict(pages=(1 << 24) + 1), UNSUPPORTED), (dict(nbytes=1000), WORKSPACE)]
BAD_SEQS = [(dict(n=0), INVALID), (dict(new=0), INVALID), (dict(tokens=-1, cu=FAKE), INVALID), (dict(tokens=5), INVALID),
            (dict(pages=0), INVALID), (dict(kv_len=None), INVALID), (dict(table=None), INVALID),
            (dict(max_kv=641), INVALID), (dict(max_kv=-1), INVALID), (dict(kv_len=FAKE + 2), INVALID),
            (dict(table=FAKE + 1), INVALID), (dict(cu=FAKE + 2), INVALID),
            (dict(n=65537, new=1, tokens=65537), UNSUPPORTED), (dict(pages=1 << 25), UNSUPPORTED)]


def test_kv_sizes():
    # codes and scales: head_dim + 4 head_dim / group bytes per token and head
    assert prox.kv_bytes(8, 128, 64, 64, 10) == 10 * 64 * 8 * (128 + 8)
    assert prox.kv_bytes(1, 64, 32, 32, 1) == 32 * (64 + 8)
    assert prox.kv_bytes(8, 256, 128, 96, 1 << 24) == (1 << 24) * 96 * 8 * (256 + 8)   # past 32 bits
    for kw, _ in BAD_CACHES[3:-1]:
        a = dict(heads=8, dim=128, group=64, page=64, pages=100, **{}) | kw
        assert prox.kv_bytes(a["heads"], a["dim"], a["group"], a["page"], a["pages"]) == 0, kw
    assert [prox.kv_attn_workspace_bytes(d) > 0 for d in (64, 128, 256, 96, 0)] == [True] * 3 + [False] * 2


def _append(c=None, s=None, k=FAKE, ldk=1024, v=FAKE, ldv=1024, q=FAKE, heads=32, ldq=4096, qo=FAKE, ldo=4096, rope=None):
    c, s = c or _cache(), s or _seqs()
    return prox.lib().prox_kv_append(ctypes.byref(c), ctypes.byref(s), k, ldk, v, ldv, q, heads, ldq, qo, ldo,
                                     None if rope is None else ctypes.byref(rope), None)


def _attn(c=None, s=None, q=FAKE, heads=32, ldq=4096, scale=0.1, window=0, out=FAKE, ldo=4096, ws=FAKE, nbytes=BIG):
    c, s = c or _cache(), s or _seqs()
    return prox.lib().prox_kv_attn(ctypes.byref(c), ctypes.byref(s), q, heads, ldq, scale, window, out, ldo, ws, nbytes, None)


def _read(c=None, s=None, k=FAKE, v=FAKE):
    c, s = c or _cache(), s or _seqs()
    return prox.lib().prox_kv_read(ctypes.byref(c), ctypes.byref(s), k, v, None)


@pytest.mark.parametrize("call", [_append, _attn, _read])
def test_kv_refuses_bad_caches_and_sequences(call):
    for kw, want in BAD_CACHES:
        assert call(c=_cache(**kw)) == want, kw
    for kw, want in BAD_SEQS:
        assert call(s=_seqs(**kw)) == want, kw


@pytest.mark.parametrize("call", [_append, _attn, _read])
def test_no_tokens_is_no_work(call):
    assert call(s=_seqs(tokens=0, cu=FAKE)) == OK   # nothing is enqueued


def test_append_refusals():
    assert _append(k=None) == INVALID and _append(v=None) == INVALID
    assert _append(k=FAKE + 2) == INVALID and _append(ldk=1016) == INVALID and _append(ldv=1028) == INVALID
    assert _append(q=None) == INVALID and _append(qo=None) == INVALID      # one without the other
    assert _append(heads=0) == INVALID and _append(heads=4097, ldq=1 << 20, ldo=1 << 20) == INVALID
    assert _append(ldq=4088) == INVALID and _append(ldo=4100) == INVALID
    assert _append(ldq=4104) == INVALID                                    # in place, another stride
    R = prox._Rope
    for r, want in [(R(None, 640, 128, 0), INVALID), (R(FAKE + 8, 640, 128, 0), INVALID), (R(FAKE, 639, 128, 0), INVALID),
                    (R(FAKE, 640, 0, 0), INVALID), (R(FAKE, 640, 24, 0), UNSUPPORTED), (R(FAKE, 640, 144, 0), UNSUPPORTED)]:
        assert _append(rope=r) == want
    assert _append(s=_seqs(n=65536, new=100000, tokens=10, cu=FAKE)) == UNSUPPORTED   # grid


def test_attention_refusals():
    assert _attn(heads=0) == INVALID and _attn(heads=12) == INVALID and _attn(heads=-8) == INVALID
    assert _attn(window=-1) == INVALID
    assert _attn(scale=float("nan")) == INVALID and _attn(scale=float("inf")) == INVALID
    assert _attn(scale=3e38) == INVALID and _attn(scale=-3e38) == INVALID   # finite, but not in powers of 2
    assert _attn(q=None) == INVALID and _attn(out=None) == INVALID and _attn(ws=None) == INVALID
    assert _attn(q=FAKE + 8) == INVALID and _attn(ws=FAKE + 16) == INVALID
    assert _attn(ldq=4088) == INVALID and _attn(ldo=4100) == INVALID and _attn(ldo=8192) == INVALID
    assert _attn(nbytes=prox.kv_attn_workspace_bytes(128) - 1) == WORKSPACE
    assert _attn(s=_seqs(n=65536, new=100000, tokens=10, cu=FAKE)) == UNSUPPORTED
    assert _read(k=None) == INVALID and _read(v=FAKE + 4) == INVALID


def test_limits_match_the_header():
    text = open(f"{B.INCLUDE}/prox.h").read()
    assert int(re.search(r"#define PROX_MAX_LINEAR_K\s+(\d+)", text).group(1)) == 65536


PLACES = r"""
#define __host__
#define __device__
#include "layout.hpp"
#include <cstdio>
#include <cstdlib>
#include <vector>
using namespace prox;
static void need(bool ok, const char *what) { if (!ok) { std::printf("%s\n", what); std::exit(1); } }
int main() {
    // Every (half block, lane, word, nibble) of keys and values is one (token, channel), and back.
    for (int D : {64, 128, 256}) {
        std::vector<int> k(32 * D), v(32 * D);
        for (int t = 0; t < 32; ++t)
            for (int c = 0; c < D; ++c) {
                const int ch = c / 8, e = c % 8;
                ++k.at(kv_k_word(D, t, ch) * 8 + nibble_of(e));
                const int lane = ((t % 16) / 4) * 16 + c % 16;
                ++v.at(kv_v_word(lane, c / 16) * 8 + t % 4 + 4 * (t / 16));
            }
        for (int i = 0; i < 32 * D; ++i) need(k[i] == 1 && v[i] == 1, "codes");
    }
    std::vector<int> slot(32);
    for (int t = 0; t < 32; ++t) ++slot.at(kv_slot(t));
    for (int t = 0; t < 32; ++t) need(slot[t] == 1, "slots");
    // Rows, positions and records stay inside their arrays whatever the device arrays hold.
    const int odd[] = {-2147483647 - 1, -7, -1, 0, 1, 5, 31, 32, 33, 63, 64, 95, 96, 1000, 2147483647};
    long n = 0;
    std::vector<uint8_t> blob(1);
    for (int a : odd) for (int b : odd) for (int len : odd) for (int id : odd) for (int max_new : {1, 3, 64, 200}) {
        const int cu[3] = {a, b, 5}, lens[2] = {len, 7}, table[6] = {id, id, id, 0, 1, 2};
        for (bool with : {true, false}) {
            KvSeqs q{with ? cu : nullptr, lens, table, 2, max_new, with ? 64 : 2 * max_new, 90, 3};
            KvCache c{nullptr, 2, 64, 32, 32, 4, 2 * KvLayout(64, 32).record};
            for (int s = 0; s < 2; ++s) {
                const SeqTokens t = seq_tokens(q, s);
                need(t.n >= 0 && t.n <= max_new && t.t0 >= 0 && t.t0 + t.n <= q.n_tokens, "rows");
                need(t.len >= 0 && t.len <= 90 && t.pos0 + t.n <= t.len, "positions");
                for (int blk = 0; 32 * blk < t.len; ++blk) {
                    const uint8_t *r = kv_record(c, q, KvLayout(64, 32).record, s, 1, blk);
                    const size_t o = (size_t)(r - (const uint8_t *)nullptr);
                    need(!r || o + KvLayout(64, 32).record <= 4 * c.page_bytes, "record");
                    if (s == 0) need((r != nullptr) == (id >= 0 && id < 4), "page");
                    ++n;
                }
            }
        }
    }
    // Offsets past 32 bits.
    KvSeqs q{nullptr, nullptr, nullptr, 1, 1, 1, 1 << 20, 1};
    const int table[1] = {(1 << 24) - 1};
    q.table = table;
    const KvLayout L(256, 32);
    KvCache c{nullptr, 256, 256, 32, 32768, 1 << 24, (size_t)256 * 1024 * L.record};
    const uint8_t *r = kv_record(c, q, L.record, 0, 255, 1023);
    need((size_t)(r - (const uint8_t *)nullptr) == ((size_t)(1 << 24) * 256 * 1024 - 1) * L.record, "far record");
    std::printf("%ld\n", n);
    return 0;
}
"""


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_places_of_tokens(tmp_path):
    src, exe = tmp_path / "places.cpp", tmp_path / "places"
    src.write_text(PLACES)
    subprocess.run(["g++", "-std=c++17", "-O1", "-include", "initializer_list", "-I", B.CSRC, str(src),
                    "-o", str(exe)], check=True, capture_output=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout
    assert int(r.stdout) > 10000
