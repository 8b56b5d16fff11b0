"""float64 oracle of the token operators: sliding-window attention with first
keys that stay visible and shared key/value heads, the embedding lookup, and
their gradients.  Plain loops over samples and heads; nothing is shared with the
GPU path.
"""
from __future__ import annotations

import numpy as np


def visible(n: int, m: int, left: int, right: int, sinks: int) -> np.ndarray:
    """[n, m] truth values: query t, the position m - n + t of m keys, sees key j."""
    p = (m - n + np.arange(n))[:, None]
    j = np.arange(m)[None, :]
    seen = np.ones((n, m), bool)
    if right >= 0:
        seen &= j <= p + right
    if left >= 0:
        seen &= (j >= p - left) | (j < sinks)
    return seen


def _samples(n, m, slots):
    a = b = 0
    for i in range(len(n)):
        yield i, slice(a, a + n[i]), slice(b, b + m[i])
        a += n[i]
        b += slots[i]


def _weights(q, k, seen, scale):
    """(P, lse) of one head; rows that see nothing have P = 0, lse = -inf."""
    s = scale * np.where(seen, q @ k.T, 0.0)
    s = np.where(seen, s, -np.inf)
    lse = np.full(q.shape[0], -np.inf)
    some = seen.any(1)
    if some.any():
        top = s[some].max(1)
        lse[some] = top + np.log(np.exp(s[some] - top[:, None]).sum(1))
    P = np.zeros_like(s)
    P[some] = np.exp(s[some] - lse[some][:, None])
    return P, lse


def _mix(P, v):
    """P @ v over the keys with weight: values that no row gives weight do not enter."""
    used = (P != 0).any(0)
    return P[:, used] @ v[used]


def window_attention(q, k, v, n, m, heads, kv_heads, d, left=-1, right=0, sinks=0, scale=None, slots=None):
    """q [sum N, heads*d], k, v [sum slots, kv_heads*d]; m keys in use of `slots`
    (default m) per sample.  Returns (o, lse [heads, sum N], A) with
    A = sum_j P_j |v_j|, the scale of o's rounding errors."""
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    scale = 1.0 / np.sqrt(d) if scale is None else scale
    G = heads // kv_heads
    o, A = np.zeros_like(q), np.zeros_like(q)
    lse = np.full((heads, q.shape[0]), -np.inf)
    for i, rq, rk in _samples(n, m, m if slots is None else slots):
        seen = visible(n[i], m[i], left, right, sinks)
        for h in range(heads):
            cq, ck = slice(h * d, h * d + d), slice(h // G * d, h // G * d + d)
            P, lse[h, rq] = _weights(q[rq, cq], k[rk, ck], seen, scale)
            o[rq, cq] = _mix(P, v[rk, ck])
            A[rq, cq] = _mix(P, np.abs(v[rk, ck]))
    return o, lse, A


def window_attention_backward(q, k, v, o, lse, dout, n, m, heads, kv_heads, d, left=-1, right=0, sinks=0, scale=None,
                              ds_rel=0.0, p_rel=0.0, fp_rel=0.0):
    """(dq, dk, dv) from the forward's operands and its stored o and lse, and how
    far they may be off where P is off by p_rel + fp_rel of itself, and dS by
    ds_rel of itself + fp_rel P (|dout| . |v| + |dout| . |o|)."""
    q, k, v, o, lse, dout = (np.asarray(x, np.float64) for x in (q, k, v, o, lse, dout))
    scale = 1.0 / np.sqrt(d) if scale is None else scale
    G = heads // kv_heads
    g = [np.zeros_like(x) for x in (q, k, v)]
    e = [np.zeros_like(x) for x in (q, k, v)]
    for i, rq, rk in _samples(n, m, m):
        seen = visible(n[i], m[i], left, right, sinks)
        for h in range(heads):
            cq, ck = slice(h * d, h * d + d), slice(h // G * d, h // G * d + d)
            Q, K, V, D = q[rq, cq], k[rk, ck], v[rk, ck], dout[rq, cq]
            L = lse[h, rq][:, None]
            P = np.where(seen, np.exp(np.where(seen, scale * (Q @ K.T) - np.where(np.isfinite(L), L, 0.0), 0.0)), 0.0)
            delta = (D * o[rq, cq]).sum(1, keepdims=True)
            dS = P * (D @ V.T - delta)
            g[0][rq, cq] += scale * dS @ K
            g[1][rk, ck] += scale * dS.T @ Q
            g[2][rk, ck] += P.T @ D
            eP = P * (p_rel + fp_rel)
            eS = ds_rel * np.abs(dS) + fp_rel * P * (np.abs(D) @ np.abs(V).T + (np.abs(D) * np.abs(o[rq, cq])).sum(1, keepdims=True))
            e[0][rq, cq] += abs(scale) * eS @ np.abs(K)
            e[1][rk, ck] += abs(scale) * eS.T @ np.abs(Q)
            e[2][rk, ck] += eP.T @ np.abs(D)
    return g, e


def embedding(table, ids, scale=1.0):
    table, ids = np.asarray(table, np.float64), np.asarray(ids, np.int64)
    y = np.zeros((len(ids), table.shape[1]))
    ok = (ids >= 0) & (ids < table.shape[0])
    y[ok] = scale * table[ids[ok]]
    return y


def embedding_backward(ids, dy, vocab, scale=1.0, start=None):
    """(gradient, sum of |dy| per table row, number of tokens per table row)."""
    dy, ids = np.asarray(dy, np.float64), np.asarray(ids, np.int64)
    g = np.zeros((vocab, dy.shape[1])) if start is None else np.array(start, np.float64)
    mag, count = np.zeros((vocab, dy.shape[1])), np.zeros(vocab, np.int64)
    for r, v in enumerate(ids):
        if 0 <= v < vocab:
            g[v] += scale * dy[r]
            mag[v] += abs(scale) * np.abs(dy[r])
            count[v] += 1
    return g, mag, count
