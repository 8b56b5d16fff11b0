"""Values and error bars of a window attention call, both in float64, for tests.

With u = finfo(type).eps / 2 (bf16 2^-8; 2^-24 for fp32) and e = 2^-24 for fp32
operands, 2^-23 for bf16 ones (matrix instructions may cut the sum of a product
instead of rounding it), per query row i and key j:

  t_ij = |scale| sum_c |q_c k_c|, T_i = max over the visible j, L_i = |lse_i|
  a score is a chain of d products, then multiplied by log2(e) and subtracted
  from the maximum or lse, whose own roundings are relative to T_i + L_i:
    |d s_ij| <= e ((d + 8) T_i + 4 (T_i + L_i))
  the exponential adds two units of its own: a weight is off by w_i of itself,
    w_i = e ((d + 8) T_i + 4 (T_i + L_i)) + 2^-22
  o = sum P v / sum P: both sums are off by w_i + e (M_i + 8) of their terms'
  sizes; bf16 rounds P for the first sum and o at the end:
    |d o| <= (2 w_i + 2 e (M_i + 8) + u [bf16]) A_i + u |o|, A = sum_j P_j |v_j|
  lse: the sum's relative error, and the rounding of its logarithm:
    |d lse| <= w_i + e (M_i + 8) + 2^-22 (1 + L_i)
  backward, from the stored o and lse: with B_ij = |dO|.|V| + |dO|.|o|,
    |d dS_ij| <= (w_i + 2^-23 + u [bf16]) |dS_ij| + P_ij e (d + 8) B_ij
  and each gradient sums such terms over M_i keys, or over all rows of the
  query heads that share the key, with e per addition, then rounds once.
Products of two of these errors are covered by a factor of 1.01."""
import numpy as np

from oracle import tokens as T

U = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
E = {"bf16": 2.0 ** -23, "f32": 2.0 ** -24}


def _samples(n, slots):
    a = b = 0
    for i, (x, s) in enumerate(zip(n, slots)):
        yield i, slice(a, a + x), b
        a, b = a + x, b + s


def _head(q, k, seen, scale, d, e, lse=None):
    """(P, lse, w) of one head of one sample, w as a column."""
    s = np.where(seen, scale * (q @ k.T), -np.inf)
    t = np.where(seen, abs(scale) * (np.abs(q) @ np.abs(k).T), 0.0).max(1, initial=0.0)
    if lse is None:
        top = s.max(1, initial=-np.inf)
        safe = np.where(np.isfinite(top), top, 0.0)
        with np.errstate(divide="ignore"):
            lse = safe + np.log(np.exp(s - safe[:, None]).sum(1))
    fin = np.where(np.isfinite(lse), lse, 0.0)
    P = np.where(seen, np.exp(s - fin[:, None]), 0.0)
    w = e * ((d + 8) * t + 4 * (t + np.abs(fin))) + 2.0 ** -22
    return P, lse, w[:, None]


def forward(x, n, m, H, K, d, dtype, left=-1, right=0, sinks=0, scale=None, slots=None):
    """{"o": (values, bars), "lse": (values, bars)} of q, k, v in x."""
    q, k, v = (np.asarray(x[a], np.float64) for a in ("q", "k", "v"))
    scale, G, u, e = 1.0 / np.sqrt(d) if scale is None else scale, H // K, U[dtype], E[dtype]
    o, bo = np.zeros_like(q), np.zeros_like(q)
    lse, bl = np.full((H, q.shape[0]), -np.inf), np.zeros((H, q.shape[0]))
    for i, rq, b in _samples(n, m if slots is None else slots):
        rk, seen = slice(b, b + m[i]), T.visible(n[i], m[i], left, right, sinks)
        count = seen.sum(1)[:, None]
        for h in range(H):
            cq, ck = slice(h * d, h * d + d), slice(h // G * d, h // G * d + d)
            P, lse[h, rq], w = _head(q[rq, cq], k[rk, ck], seen, scale, d, e)
            o[rq, cq] = P @ v[rk, ck]
            sums = w + e * (count + 8)
            bo[rq, cq] = 1.01 * (2 * sums + (u if dtype == "bf16" else 0.0)) * (P @ np.abs(v[rk, ck])) + u * np.abs(o[rq, cq])
            L = np.where(np.isfinite(lse[h, rq]), np.abs(lse[h, rq]), 0.0)
            bl[h, rq] = 1.01 * sums[:, 0] + 2.0 ** -22 * (1 + L)
    return {"o": (o, bo), "lse": (lse, bl)}


def backward(x, o, lse, n, m, H, K, d, dtype, left=-1, right=0, sinks=0, scale=None):
    """{"dq": (values, bars), ...} of q, k, v, do in x and the stored o and lse."""
    q, k, v, do = (np.asarray(x[a], np.float64) for a in ("q", "k", "v", "do"))
    o, lse = np.asarray(o, np.float64), np.asarray(lse, np.float64)
    scale, G, u, e = 1.0 / np.sqrt(d) if scale is None else scale, H // K, U[dtype], E[dtype]
    low = u if dtype == "bf16" else 0.0
    g = {a: np.zeros_like(y) for a, y in (("dq", q), ("dk", k), ("dv", v))}
    bar = {a: np.zeros_like(y) for a, y in g.items()}
    for i, rq, b in _samples(n, m):
        rk, seen = slice(b, b + m[i]), T.visible(n[i], m[i], left, right, sinks)
        keys, rows = seen.sum(1)[:, None], G * seen.sum(0)[:, None]
        for h in range(H):
            cq, ck = slice(h * d, h * d + d), slice(h // G * d, h // G * d + d)
            Q, Kh, V, D, O = q[rq, cq], k[rk, ck], v[rk, ck], do[rq, cq], o[rq, cq]
            P, _, w = _head(Q, Kh, seen, scale, d, e, lse[h, rq])
            dS = P * (D @ V.T - (D * O).sum(1, keepdims=True))
            B = np.abs(D) @ np.abs(V).T + (np.abs(D) * np.abs(O)).sum(1, keepdims=True)
            eS = (w + 2.0 ** -23 + low) * np.abs(dS) + e * (d + 8) * P * B
            sc = abs(scale)
            g["dq"][rq, cq] += scale * dS @ Kh
            g["dk"][rk, ck] += scale * dS.T @ Q
            g["dv"][rk, ck] += P.T @ D
            bar["dq"][rq, cq] += sc * (eS + e * (keys + 8) * np.abs(dS)) @ np.abs(Kh)
            bar["dk"][rk, ck] += sc * (eS.T + e * (rows + 8) * np.abs(dS).T) @ np.abs(Q)
            bar["dv"][rk, ck] += ((P * (w + low)).T + e * (rows + 8) * P.T) @ np.abs(D)
    return {a: (g[a], 1.01 * bar[a] + (u + 2.0 ** -23) * np.abs(g[a])) for a in g}


def worst(got, ref, bar):
    """Largest error in units of its bar."""
    got, ref = np.asarray(got, np.float64), np.asarray(ref, np.float64)
    assert got.shape == ref.shape and np.isfinite(got).all()
    return float((np.abs(got - ref) / np.maximum(bar, 1e-30)).max(initial=0.0))
