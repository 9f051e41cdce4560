"""Blocks of the cache that a tile of query rows sees, compiled for the host and compared with
64-bit arithmetic: padded sequences, windows up to the largest, splits."""
import shutil
import subprocess

import pytest

from paper_2607_27591_amd import build as B

SPANS = r"""
#define __host__
#define __device__
#include "layout.hpp"
#include <cstdio>
#include <cstdlib>
using namespace prox;
static void need(bool ok, const char *what, long a, long b, long c) {
    if (!ok) { std::printf("%s %ld %ld %ld\n", what, a, b, c); std::exit(1); }
}
int main() {
    const int top = 2147483647;
    long n = 0;
    for (int pos0 : {-top, -top + 1, -1000000, -100, -33, -5, -3, -2, -1, 0, 1, 31, 32, 700, 65536, (1 << 30) - 300})
        for (int window : {0, 1, 2, 31, 32, 33, 500, 65536, 1 << 30, top - 1, top}) {
            for (int pos : {pos0, pos0 + 2, pos0 + 40}) {
                const long first = window > 0 && (long)pos - window + 1 > 0 ? (long)pos - window + 1 : 0;
                need(attn_first(pos, window) == first, "first", pos, window, attn_first(pos, window));
            }
            for (int ratio : {1, 3, 8}) for (int r0 : {0, 16, 96}) for (int rows : {1, 16, 32}) for (int splits : {1, 2, 7, 1024}) {
                const int r1 = r0 + rows - 1;
                const AttnSpan s = attn_span(SeqTokens{0, 300, pos0, pos0 + 300}, ratio, window, splits, r0, r1);
                const long hi = (long)pos0 + r1 / ratio, at = (long)pos0 + r0 / ratio;
                if (hi < 0) {
                    need(s.eff == 0 && s.b0 == s.b1, "nothing seen", pos0, window, r0);
                } else {
                    const long lo = window > 0 && at - window + 1 > 0 ? at - window + 1 : 0;
                    need(s.b0 == lo / 32 && s.b1 == hi / 32 + 1, "blocks", pos0, window, s.b0);
                    need(s.per >= 1 && s.eff >= 1 && s.eff <= splits, "splits", s.per, s.eff, splits);
                    need((long)s.b0 + (long)s.eff * s.per >= s.b1 && (long)s.b0 + (long)(s.eff - 1) * s.per < s.b1, "cover", s.per, s.eff, splits);
                }
                ++n;
            }
        }
    std::printf("%ld\n", n);
    return 0;
}
"""


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_spans_of_padded_sequences_and_large_windows(tmp_path):
    src, exe = tmp_path / "spans.cpp", tmp_path / "spans"
    src.write_text(SPANS)
    subprocess.run(["g++", "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-include",
                    "initializer_list", "-I", B.CSRC, str(src), "-o", str(exe)], check=True, capture_output=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr
    assert int(r.stdout) > 10000
