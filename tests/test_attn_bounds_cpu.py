"""The checks of attn_ref.py pass the rounded 64-bit result and reject it with a mistake planted."""
import numpy as np
import pytest
import torch

import attn_ref as A
import layer_ref as R


@pytest.mark.parametrize("shape", A.SHAPES, ids=lambda s: "-".join(map(str, s[:5])))
def test_mistakes_are_seen(shape):
    seen = {name: [] for name in A.MISTAKES}
    for kind in A.KINDS:
        x = A.Inputs(*shape, kind)
        ref, bound, outs = x.attention(list(A.MISTAKES.values()))
        share, whole = A.violations(R.f64(torch.from_numpy(ref).to(x.dtype)), ref, bound, x.dtype)
        assert share == 0 and whole <= 1, (kind, share, whole)
        for name, out in zip(A.MISTAKES, outs):
            if np.array_equal(out, ref):
                seen[name].append("-")
                continue
            share, whole = A.violations(R.f64(torch.from_numpy(out).to(x.dtype)), ref, bound, x.dtype)
            seen[name].append("yes" if share > 0 or whole > 1 else "no")
            print(f"    {kind}, {name}: {share:.4f} of the values past the bound, the whole {whole:.2f}", flush=True)
    print(seen)
    for name, kinds in seen.items():
        # Rows at the end of a sequence see no token behind it, those without a window none before it.
        assert "yes" in kinds or set(kinds) == {"-"}, (name, kinds)


@pytest.mark.parametrize("shape", [s for s in A.SHAPES if s[5] == A.F16][:4], ids=lambda s: "-".join(map(str, s[:5])))
def test_weights_of_one_term_are_seen(shape):
    # fp16 outputs from weights rounded to one bf16 term.
    x = A.Inputs(*shape, "random")
    ref, bound, _ = x.attention()
    v = x.vw
    out = np.zeros_like(ref)
    q = R.f64(x.q)
    for row, a, l, p in x.rows():
        first = max(p - x.window + 1, 0) if x.window else 0
        for h in range(x.heads):
            r = slice(h * x.ratio, (h + 1) * x.ratio)
            s = x.scale * (q[row, r] @ x.kw[a + first:a + p + 1, h].T)
            w = np.exp(s - s.max(-1, keepdims=True))
            w1 = torch.from_numpy(w).float().bfloat16().double().numpy()
            out[row, r] = w1 @ v[a + first:a + p + 1, h] / w.sum(-1, keepdims=True)
    share, whole = A.violations(R.f64(torch.from_numpy(out).to(x.dtype)), ref, bound, x.dtype)
    assert share > 0 and whole > 1, (share, whole)
