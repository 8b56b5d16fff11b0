"""The float64 oracle of the token operators against closed forms, dense
attention and finite differences (CPU)."""
import numpy as np
import pytest

from oracle import tokens as T

RNG = np.random.default_rng


def test_visible_closed_forms():
    assert T.visible(3, 3, -1, 0, 0).tolist() == np.tril(np.ones((3, 3), bool)).tolist()
    assert T.visible(2, 5, -1, 0, 0).tolist() == [[True] * 4 + [False], [True] * 5]
    assert T.visible(1, 6, 1, 0, 2).tolist() == [[True, True, False, False, True, True]]
    assert T.visible(3, 1, -1, 0, 0).tolist() == [[False], [False], [True]]      # more queries than keys
    assert T.visible(4, 4, 1, 1, 0).tolist() == [[abs(a - b) <= 1 for b in range(4)] for a in range(4)]
    assert T.visible(3, 3, 0, 0, 1).tolist() == [[True, False, False], [True, True, False], [True, False, True]]
    assert T.visible(2, 0, -1, -1, 3).shape == (2, 0)


def test_all_visible_is_softmax_attention():
    rng = RNG(0)
    q, k, v = (rng.standard_normal((5, 8)) for _ in range(3))
    o, lse, _ = T.window_attention(q, k, v, [5], [5], 2, 2, 4, right=-1)
    for h in range(2):
        s = q[:, 4 * h:4 * h + 4] @ k[:, 4 * h:4 * h + 4].T / 2.0
        e = np.exp(s)
        assert np.allclose(o[:, 4 * h:4 * h + 4], e / e.sum(1, keepdims=True) @ v[:, 4 * h:4 * h + 4], atol=1e-14)
        assert np.allclose(lse[h], np.log(e.sum(1)), atol=1e-14)


def test_masked_values_do_not_enter():
    rng = RNG(1)
    q, k, v = (rng.standard_normal((4, 8)) for _ in range(3))
    want = T.window_attention(q[:2], k, v, [2], [3], 1, 1, 8, slots=[4])[0]
    k[3], v[3] = np.nan, np.inf                                                  # a slot not in use
    o, lse, _ = T.window_attention(q[:2], k, v, [2], [3], 1, 1, 8, slots=[4])
    assert np.array_equal(o, want) and np.isfinite(lse).all()


def test_nothing_visible_is_zero():
    q, k, v = RNG(2).standard_normal((3, 3, 8))
    o, lse, _ = T.window_attention(q, k[:1], v[:1], [3], [1], 1, 1, 8)
    assert not o[:2].any() and np.isneginf(lse[0, :2]).all() and np.allclose(o[2], v[0])


@pytest.mark.parametrize("n,m,left,right,sinks", [([4, 0, 3], [4, 2, 5], -1, 0, 0), ([5, 2], [5, 1], 1, 0, 1),
                                                  ([4, 1], [4, 3], 2, 1, 0), ([3], [3], -1, -1, 0)])
def test_gradients_by_differences(n, m, left, right, sinks):
    rng, H, K, d = RNG(3), 4, 2, 8
    q, w = rng.standard_normal((2, sum(n), H * d))
    k, v = rng.standard_normal((2, sum(m), K * d))
    kw = dict(left=left, right=right, sinks=sinks, scale=0.4)
    f = lambda q, k, v: (T.window_attention(q, k, v, n, m, H, K, d, **kw)[0] * w).sum()   # noqa: E731
    o, lse, _ = T.window_attention(q, k, v, n, m, H, K, d, **kw)
    grads, _ = T.window_attention_backward(q, k, v, o, lse, w, n, m, H, K, d, **kw)
    xs = [q, k, v]
    for a, g in enumerate(grads):
        for _ in range(12):
            at = tuple(rng.integers(s) for s in xs[a].shape)
            step = np.zeros_like(xs[a])
            step[at] = 1e-5
            up, down = list(xs), list(xs)
            up[a], down[a] = xs[a] + step, xs[a] - step
            assert abs((f(*up) - f(*down)) / 2e-5 - g[at]) < 1e-8


def test_embedding_and_gradient():
    rng = RNG(4)
    table, ids = rng.standard_normal((5, 8)), np.array([3, -1, 0, 3, 5, 4])
    y = T.embedding(table, ids, 2.0)
    assert np.array_equal(y[[0, 2, 3, 5]], 2.0 * table[[3, 0, 3, 4]]) and not y[[1, 4]].any()
    w = rng.standard_normal((6, 8))
    g, mag, count = T.embedding_backward(ids, w, 5, 2.0)
    assert count.tolist() == [1, 0, 0, 2, 1] and not g[1:3].any()
    for _ in range(10):
        at = (rng.integers(5), rng.integers(8))
        step = np.zeros_like(table)
        step[at] = 0.5                                                           # linear in the table
        diff = ((T.embedding(table + step, ids, 2.0) - T.embedding(table - step, ids, 2.0)) * w).sum()
        assert abs(diff - g[at]) < 1e-12 and mag[at] >= abs(g[at])


@pytest.mark.parametrize("left,right,sinks", [(-1, 0, 0), (2, 0, 1), (1, 2, 2), (-1, -1, 0)])
def test_gradients_against_autograd(left, right, sinks):
    """Dense float64 autograd of the definition, shared heads and fewer keys than queries included."""
    torch = pytest.importorskip("torch")
    n, m, H, K, d, rng = [6, 0, 9, 4], [6, 3, 14, 2], 6, 2, 8, RNG(5)
    q, k, v, w = (rng.standard_normal((r, h * d)) for r, h in ((sum(n), H), (sum(m), K), (sum(m), K), (sum(n), H)))
    Q, Kt, V = (torch.tensor(x, dtype=torch.float64, requires_grad=True) for x in (q, k, v))
    a = b = 0
    total = torch.zeros((), dtype=torch.float64)
    for i in range(len(n)):
        for t in range(n[i]):
            p = m[i] - n[i] + t
            js = [j for j in range(m[i]) if (right < 0 or j <= p + right) and (left < 0 or j >= p - left or j < sinks)]
            for h in range(H):
                if not js:
                    continue
                c, r = slice(h * d, h * d + d), slice(h // (H // K) * d, h // (H // K) * d + d)
                rows = [b + j for j in js]
                weight = torch.softmax(0.3 * (Kt[rows, r] @ Q[a + t, c]), 0)
                total = total + (weight @ V[rows, r]) @ torch.tensor(w[a + t, c])
        a, b = a + n[i], b + m[i]
    total.backward()
    kw = dict(left=left, right=right, sinks=sinks, scale=0.3)
    o, lse, _ = T.window_attention(q, k, v, n, m, H, K, d, **kw)
    assert abs((o * w).sum() - float(total)) < 1e-11
    grads, _ = T.window_attention_backward(q, k, v, o, lse, w, n, m, H, K, d, **kw)
    for g, x in zip(grads, (Q, Kt, V)):
        assert np.allclose(g, x.grad.numpy(), rtol=0, atol=1e-11)
