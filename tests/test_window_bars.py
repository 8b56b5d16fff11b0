"""The bars of the window attention tests (CPU): their values are the oracle's, and
they are narrow enough to see lower precision in each product."""
import numpy as np
import pytest

from oracle import tokens as T
from oracle.numerics import round_bf16
from paper_2609_30379_amd import synth

from . import window_bars as W

NAMES = ("q", "k", "v", "do")


def operands(n, m, H, K, d, dtype, seed=0):
    rows = dict(q=(sum(n), H), k=(sum(m), K), v=(sum(m), K), do=(sum(n), H))
    return {a: np.asarray(synth.normal(seed, "w." + a, (r, h * d), 1.0, dtype), np.float64) for a, (r, h) in rows.items()}


@pytest.mark.parametrize("left,right,sinks", [(-1, 0, 0), (5, 0, 2), (4, 3, 1), (-1, -1, 0)])
def test_values_are_the_oracles(left, right, sinks):
    n, m, H, K, d = [7, 0, 30, 3], [9, 4, 30, 1], 4, 2, 16
    x, kw = operands(n, m, H, K, d, "f32"), dict(left=left, right=right, sinks=sinks)
    f = W.forward(x, n, m, H, K, d, "f32", **kw)
    o, lse, _ = T.window_attention(x["q"], x["k"], x["v"], n, m, H, K, d, **kw)
    assert np.allclose(f["o"][0], o, rtol=0, atol=1e-13)
    assert np.array_equal(np.isneginf(f["lse"][0]), np.isneginf(lse))
    some = np.isfinite(lse)
    assert np.allclose(f["lse"][0][some], lse[some], rtol=0, atol=1e-13)
    ref, _ = T.window_attention_backward(x["q"], x["k"], x["v"], o, lse, x["do"], n, m, H, K, d, **kw)
    b = W.backward(x, o, lse, n, m, H, K, d, "f32", **kw)
    for a, r in zip(("dq", "dk", "dv"), ref):
        assert np.allclose(b[a][0], r, rtol=0, atol=1e-12)


def low_precision(x, n, H, d, what):
    """Causal attention and its gradients in float64 but for `what`, which goes through bf16."""
    r = lambda name, y: round_bf16(y).astype(np.float64) if name == what else y   # noqa: E731
    y = {a: r(a, x[a]) for a in NAMES}
    out = {a: np.zeros_like(x["q"]) for a in ("o", "dq", "dk", "dv")}
    seen = T.visible(n, n, -1, 0, 0)
    for h in range(H):
        c = slice(h * d, h * d + d)
        s = np.where(seen, y["q"][:, c] @ y["k"][:, c].T / np.sqrt(d), -np.inf)
        P = np.exp(s - s.max(1, keepdims=True))
        P /= P.sum(1, keepdims=True)
        o = r("P", P) @ y["v"][:, c]
        dS = P * (y["do"][:, c] @ y["v"][:, c].T - (y["do"][:, c] * o).sum(1, keepdims=True))
        out["o"][:, c], out["dv"][:, c] = o, r("P", P).T @ y["do"][:, c]
        out["dq"][:, c] = r("dS", dS) @ y["k"][:, c] / np.sqrt(d)
        out["dk"][:, c] = r("dS", dS).T @ y["q"][:, c] / np.sqrt(d)
    return out


@pytest.mark.parametrize("d", [32, 72, 96, 128])
@pytest.mark.parametrize("what,seen_in", [("q", ("o", "dq", "dk", "dv")), ("k", ("o", "dq", "dk", "dv")), ("v", ("o", "dq", "dk")),
                                          ("do", ("dq", "dk", "dv")), ("P", ("o", "dv")), ("dS", ("dq", "dk"))])
def test_fp32_bars_see_a_bf16_rounding_anywhere(d, what, seen_in):
    n, H = 130, 2
    x = operands([n], [n], H, H, d, "f32")
    f = W.forward(x, [n], [n], H, H, d, "f32")
    b = W.backward(x, f["o"][0], f["lse"][0], [n], [n], H, H, d, "f32")
    exact, rounded = low_precision(x, n, H, d, None), low_precision(x, n, H, d, what)
    for a in ("o", "dq", "dk", "dv"):
        ref, bar = f[a] if a == "o" else b[a]
        assert W.worst(exact[a], ref, bar) < 1e-3
        if a in seen_in:
            assert W.worst(rounded[a], ref, bar) > 1.0, (a, W.worst(rounded[a], ref, bar))


@pytest.mark.parametrize("what", ["o", "dq", "dk", "dv"])
def test_bars_see_a_misplaced_window(what):
    """One key more or fewer on the left, or one sink fewer, in bf16."""
    n, H, d = 200, 2, 64
    x, kw = operands([n], [n], H, H, d, "bf16"), dict(left=20, right=0, sinks=2)
    f = W.forward(x, [n], [n], H, H, d, "bf16", **kw)
    b = W.backward(x, f["o"][0], f["lse"][0], [n], [n], H, H, d, "bf16", **kw)
    ref, bar = f["o"] if what == "o" else b[what]
    for bad in (dict(left=21), dict(left=19), dict(sinks=1), dict(right=1)):
        g = W.forward(x, [n], [n], H, H, d, "bf16", **{**kw, **bad})
        got = g["o"][0] if what == "o" else W.backward(x, g["o"][0], g["lse"][0], [n], [n], H, H, d, "bf16", **{**kw, **bad})[what][0]
        assert W.worst(got, ref, bar) > 2.0, bad
