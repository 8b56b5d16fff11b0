"""The token operators of the packed library as measurable cases.

Two operators, forward and backward:

  window attention   attention over the packed tokens of each sample with a
                     sliding window, a few first keys (sinks) that stay
                     visible, and key/value heads shared by groups of query
                     heads; the queries are the last N_i positions of M_i keys
                     (prompts, chunks over a cache, single tokens)
  embedding          rows of a table by token id, times a scale, and the
                     table's gradient, summed over equal ids

With `own` false, run() computes them in their plain form with elementary torch
operations in fp32; with `own` true it calls the library's entry points.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ------------------------------------------------------------------ the cases
def _window(**kw):
    c = dict(kind="window", batch=1, lo=1, hi=1, median=0.0, past_lo=0, past_hi=0, heads=1, kv_heads=1, d=64,
             left=-1, right=0, sinks=0, dtype="bf16", train=False, length_seed=0)
    c.update(kw)
    return c


def _embed(**kw):
    c = dict(kind="embed", rows=1, vocab=1000, c=64, dtype="bf16", ids="int64", scale=1.0, outside=0.0, train=False)
    c.update(kw)
    return c


def listed():
    return [
        # The small fp32 model's few short samples, two-sided window: only
        # latency counts.
        _window(name="window_f32_b4_n4_16", batch=4, lo=4, hi=16, heads=2, kv_heads=2, d=8, left=3, right=3, sinks=1,
                dtype="f32"),
        # The token encoder's batch and heads with a local window and one
        # sample token that all see.
        _window(name="window_encoder_b64", batch=64, lo=16, hi=512, median=230.0, heads=12, kv_heads=12, d=64, left=64,
                right=64, sinks=1),
        # Long prompts, causal window, shared key/value heads.
        _window(name="window_causal_b4_to_8192", batch=4, lo=3000, hi=8192, heads=16, kv_heads=4, d=128, left=1023,
                sinks=4, length_seed=1),
        # A chunk of new tokens over what is in the cache already, no window.
        _window(name="chunk_b2_over_30000", batch=2, lo=300, hi=700, past_lo=8000, past_hi=30000, heads=16, kv_heads=4,
                d=64, length_seed=2),
        # One request's next token, windowed cache: latency.
        _window(name="token_b1_over_4099", batch=1, past_lo=4099, past_hi=4099, heads=12, kv_heads=12, d=64, left=1023,
                sinks=4),
        # The next token of many requests of very different length, all keys
        # visible: the cache's bandwidth.
        _window(name="token_b64_to_32000", batch=64, past_lo=500, past_hi=32000, heads=32, kv_heads=8, d=128,
                length_seed=3),
        # Training in fp32 on short ragged samples, every key visible.
        _window(name="train_f32_b8_n66_317", batch=8, lo=66, hi=317, heads=4, kv_heads=4, d=32, right=-1, dtype="f32",
                train=True, length_seed=2),
        # Training on mid-size samples, causal window.
        _window(name="train_b16_n200_1024", batch=16, lo=200, hi=1024, heads=8, kv_heads=2, d=64, left=255, sinks=4,
                train=True, length_seed=4),
        # Training on long samples: the largest.
        _window(name="train_b2_to_8192", batch=2, lo=4000, hi=8192, heads=16, kv_heads=4, d=128, left=2047, sinks=4,
                train=True, length_seed=5),
        # The rows of a few short requests, fp32: latency.
        _embed(name="embed_f32_r48", rows=48, vocab=1000, c=32, dtype="f32", scale=math.sqrt(32.0)),
        # A training step's tokens at the encoder's width, some of them padding.
        _embed(name="embed_train_r14999_c768", rows=14999, vocab=30011, c=768, scale=math.sqrt(768.0), outside=0.02,
               train=True),
        # A large step on a large table: what writing its gradient costs.
        _embed(name="embed_train_r131072_c2048", rows=131072, vocab=128011, c=2048, train=True, ids="int32"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["prompt", "prompt", "chunk", "token", "token", "train", "train", "embed", "embed_train"])
    if kind.startswith("embed"):
        c = rng.choice([32, 64, 200, 384, 768, 1024, 2048])
        return _embed(rows=_log(rng, 1, min(131072, 200_000_000 // c)), vocab=_log(rng, 50, min(128000, 200_000_000 // c)),
                      c=c, dtype=rng.choice(["bf16", "bf16", "f32"]), ids=rng.choice(["int32", "int64"]),
                      scale=rng.choice([1.0, math.sqrt(c)]), outside=rng.choice([0.0, 0.0, 0.1]),
                      train=kind == "embed_train")
    d = rng.choice([32, 64, 64, 80, 96, 128, 128])
    group = rng.choice([1, 1, 2, 3, 4, 8])
    kv_heads = rng.choice([1, 2, 4, 8, 12] if group == 1 else [1, 2, 4])
    w = _window(heads=group * kv_heads, kv_heads=kv_heads, d=d, sinks=rng.choice([0, 1, 4, 16, 70]),
                dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]), length_seed=rng.randrange(1 << 20))
    cells = 800_000_000 // w["heads"]            # padded query-key pairs of one head that the batch may have
    if kind == "token":
        w["past_hi"] = _log(rng, 16, 32000)
        w["past_lo"] = rng.choice([w["past_hi"], w["past_hi"] // 2, 0])
        w["left"] = rng.choice([-1, -1, _log(rng, 8, 4096)])
        most = 1_000_000_000 // (w["past_hi"] * kv_heads * d)
        w["batch"] = max(1, min(_log(rng, 1, 128), most))
        return w
    w["hi"] = _log(rng, 8, 4096 if kind == "train" else 8192)
    if kind == "chunk":
        w["hi"] = _log(rng, 2, 700)
        w["past_hi"] = _log(rng, 16, 24000)
        w["past_lo"] = rng.choice([w["past_hi"], w["past_hi"] // 3, 0])
    w["lo"] = rng.choice([w["hi"], max(1, w["hi"] // 2), max(1, w["hi"] // 8), 1])
    w["batch"] = max(1, min(_log(rng, 1, 64), cells // (w["hi"] * (w["hi"] + w["past_hi"]))))
    w["left"] = rng.choice([-1, _log(rng, 4, 2048), _log(rng, 4, 2048)])
    w["right"] = rng.choice([0, 0, w["left"], -1]) if kind != "chunk" else 0
    w["train"] = kind == "train"
    return w


def _lengths(c):
    """New tokens and keys of every sample: (N_i, M_i)."""
    rng = random.Random(c["length_seed"])
    n = []
    for _ in range(c["batch"]):
        x = rng.lognormvariate(math.log(c["median"]), 0.5) if c["median"] else rng.uniform(c["lo"], c["hi"])
        n.append(min(c["hi"], max(c["lo"], round(x))))
    return n, [x + rng.randint(c["past_lo"], c["past_hi"]) for x in n]


# ------------------------------------------------------------------ the inputs
def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    t = TYPES[case["dtype"]]
    normal = lambda *shape: torch.randn(shape, generator=g, device="cuda").to(t)   # noqa: E731
    s = dict(case=case)
    if case["kind"] == "embed":
        rows, vocab = case["rows"], case["vocab"]
        s["table"] = normal(vocab, case["c"])
        # frequent and rare tokens: the k-th most frequent id has weight 1 / k,
        # and the frequent ones lie anywhere in the table
        u = torch.rand((rows,), generator=g, device="cuda", dtype=torch.float64)
        rank = torch.clamp(torch.exp(u * math.log(vocab + 1.0)).to(torch.int64), 1, vocab) - 1
        ids = torch.randperm(vocab, generator=g, device="cuda")[rank]
        out = torch.rand((rows,), generator=g, device="cuda") < case["outside"]
        s["ids"] = torch.where(out, -1, ids).to(getattr(torch, case["ids"]))
        if case["train"]:
            s["dy"] = normal(rows, case["c"])
        if own:
            from paper_2609_30379_amd import binding as B
            s["y"] = torch.empty((rows, case["c"]), dtype=t, device="cuda")
            if case["train"]:
                s["dtable"] = torch.empty((vocab, case["c"]), dtype=torch.float32, device="cuda")
                s["ws"] = B.workspace_tensor(B.embedding_backward_workspace_bytes(rows, vocab, case["c"]))
        return s
    n, m = _lengths(case)
    # keys and values stand in slots of the cache: for tokens over a cache each
    # sample's slots are more than it uses so far, and the rest holds leftovers
    cached = case["past_hi"] > 0
    slots = [-(-x // 256) * 256 for x in m] if cached else m
    s["n"] = torch.tensor(n, device="cuda", dtype=torch.int32)
    s["m"] = torch.tensor(m, device="cuda", dtype=torch.int32)
    s["slots"] = torch.tensor(slots, device="cuda", dtype=torch.int32)
    H, K, d = case["heads"], case["kv_heads"], case["d"]
    s["q"] = normal(sum(n), H * d)
    s["k"], s["v"] = normal(sum(slots), K * d), normal(sum(slots), K * d)
    if case["train"]:
        s["do"] = normal(sum(n), H * d)
    if own:
        from paper_2609_30379_amd import binding as B
        s["layout"] = B.NestedLayout(n, cols=[1] * len(n))
        s["kv_layout"] = B.NestedLayout(slots, cols=[1] * len(n)) if cached else None
        s["o"] = torch.empty_like(s["q"])
        shape = dict(kv_layout=s["kv_layout"], kv_heads=K, left=case["left"], right=case["right"], sinks=case["sinks"])
        s["shape"] = shape
        s["ws"] = B.workspace_tensor(B.window_attention_workspace_bytes(s["layout"], H, d, dtype=case["dtype"], **shape))
        if case["train"]:
            s["lse"] = torch.empty((H, sum(n)), dtype=torch.float32, device="cuda")
            s["dq"], s["dk"], s["dv"] = torch.empty_like(s["q"]), torch.empty_like(s["k"]), torch.empty_like(s["v"])
            s["bws"] = B.workspace_tensor(B.window_attention_backward_workspace_bytes(s["layout"], H, d,
                                                                                      dtype=case["dtype"], **shape))
    return s


# ------------------------------------------------------------------ the pass
def run(s):
    if s["case"]["kind"] == "embed":
        return _embed_own(s) if own else _embed_plain(s)
    return _window_own(s) if own else _window_plain(s)


def _embed_own(s):
    from paper_2609_30379_amd import binding as B
    c = s["case"]
    out = dict(y=B.nt_embedding(s["table"], s["ids"], s["y"], scale=c["scale"]))
    if c["train"]:
        out["dtable"] = B.nt_embedding_backward(s["ids"], s["dy"], s["dtable"], scale=c["scale"], workspace=s["ws"])
    return out


def _window_own(s):
    from paper_2609_30379_amd import binding as B
    c, shape = s["case"], s["shape"]
    if not c["train"]:
        kv_lengths = s["m"] if s["kv_layout"] is not None else None
        return dict(o=B.nt_window_attention(s["layout"], c["heads"], c["d"], s["q"], s["k"], s["v"], s["o"],
                                            kv_lengths=kv_lengths, workspace=s["ws"], **shape))
    B.nt_window_attention(s["layout"], c["heads"], c["d"], s["q"], s["k"], s["v"], s["o"], lse=s["lse"],
                          workspace=s["ws"], **shape)
    B.nt_window_attention_backward(s["layout"], c["heads"], c["d"], s["q"], s["k"], s["v"], s["o"], s["lse"], s["do"],
                                   s["dq"], s["dk"], s["dv"], workspace=s["bws"], **shape)
    return dict(o=s["o"], lse=s["lse"], dq=s["dq"], dk=s["dk"], dv=s["dv"])


def _embed_plain(s):
    c, table, ids = s["case"], s["table"], s["ids"].long()
    inside = ((ids >= 0) & (ids < c["vocab"]))[:, None]
    at = torch.where(inside[:, 0], ids, 0)
    out = dict(y=(torch.where(inside, table[at].float(), 0.0) * c["scale"]).to(table.dtype))
    if c["train"]:
        g = torch.zeros((c["vocab"], c["c"]), dtype=torch.float32, device="cuda")
        out["dtable"] = g.index_add_(0, at, torch.where(inside, s["dy"].float(), 0.0)).mul_(c["scale"])
    return out


def _places(lengths, rows):
    """Sample and position within it of every one of `rows` packed rows."""
    sample = torch.repeat_interleave(torch.arange(lengths.numel(), device="cuda"), lengths.long(), output_size=rows)
    start = torch.cumsum(lengths.long(), 0) - lengths
    return sample, torch.arange(rows, device="cuda") - start[sample]


def _window_plain(s):
    """Every sample padded to the longest, every query against every key."""
    c = s["case"]
    H, K, d, B = c["heads"], c["kv_heads"], c["d"], c["batch"]
    G, n, m = H // K, s["n"].long(), s["m"].long()
    q, k, v = s["q"], s["k"], s["v"]
    N, M = max(_lengths(c)[0]), int(max(_lengths(c)[1]))
    qs, qt = _places(n, q.shape[0])
    ks, kt = _places(s["slots"], k.shape[0])
    used = kt < m[ks]
    ks, kt = ks[used], kt[used]

    def queries(x):                              # packed rows -> [B, K, G * N, d]
        p = torch.zeros((B, N, K, G, d), dtype=torch.float32, device="cuda")
        p[qs, qt] = x.float().view(-1, K, G, d)
        return p.permute(0, 2, 3, 1, 4).reshape(B, K, G * N, d).contiguous()

    def keys(x):                                 # packed rows -> [B, K, M, d]
        p = torch.zeros((B, M, K, d), dtype=torch.float32, device="cuda")
        p[ks, kt] = x[used].float().view(-1, K, d)
        return p.permute(0, 2, 1, 3).contiguous()

    def packed(x):                               # [B, K, G * N, e] -> packed rows
        x = x.view(B, K, G, N, -1).permute(0, 3, 1, 2, 4)[qs, qt]
        return x.reshape(q.shape[0], -1)

    at = (m - n)[:, None, None] + torch.arange(N, device="cuda")[None, :, None]          # position of every query
    j = torch.arange(M, device="cuda")[None, None, :]
    seen = (j < m[:, None, None]) & (torch.arange(N, device="cuda")[None, :, None] < n[:, None, None])
    if c["right"] >= 0:
        seen = seen & (j <= at + c["right"])
    if c["left"] >= 0:
        seen = seen & ((j >= at - c["left"]) | (j < c["sinks"]))
    seen = seen[:, None, None]                   # [B, 1, 1, N, M]
    scale = 1.0 / math.sqrt(d)
    Q, Kp, Vp = queries(q), keys(k), keys(v)
    S = torch.matmul(Q, Kp.transpose(2, 3).contiguous()).mul_(scale).view(B, K, G, N, M)
    S = S.masked_fill_(~seen, -math.inf)
    top = S.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    P = S.sub_(top).exp_()
    total = P.sum(-1, keepdim=True)
    P = P.div_(torch.where(total > 0, total, 1.0)).view(B, K, G * N, M)
    O = torch.matmul(P, Vp)
    o = packed(O).to(q.dtype)
    if not c["train"]:
        return dict(o=o)
    lse = packed((top + torch.log(total)).view(B, K, G * N, 1)).t().contiguous()
    # the backward pass takes the stored (rounded) output, as a training step does
    dO = queries(s["do"])
    delta = (dO * queries(o)).sum(-1, keepdim=True)
    dV = torch.matmul(P.transpose(2, 3).contiguous(), dO)
    dS = torch.matmul(dO, Vp.transpose(2, 3).contiguous()).sub_(delta).mul_(P).mul_(scale)
    dq = packed(torch.matmul(dS, Kp)).to(q.dtype)
    dK = torch.matmul(dS.transpose(2, 3).contiguous(), Q)
    rows = lambda x: x.permute(0, 2, 1, 3)[ks, kt].reshape(-1, K * d).to(k.dtype)   # noqa: E731
    return dict(o=o, lse=lse, dq=dq, dk=rows(dK), dv=rows(dV))


# ------------------------------------------------------------------ what it has to do
def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    if case["kind"] == "embed":
        rows, vocab, c = case["rows"], case["vocab"], case["c"]
        idb = 4 if case["ids"] == "int32" else 8
        b, f = rows * idb + rows * c * e + min(rows, vocab) * c * e, rows * c
        if case["train"]:
            b += rows * c * e + vocab * c * 4
            f += 2 * rows * c
        return {"bytes": b, "flops": f}
    pairs = union = 0
    for n, m in zip(*_lengths(case)):
        p = np.arange(m - n, m)
        hi = np.minimum(m, p + case["right"] + 1) if case["right"] >= 0 else np.full(n, m)
        lo = np.maximum(0, p - case["left"]) if case["left"] >= 0 else np.zeros(n, np.int64)
        sink = np.minimum(np.minimum(lo, hi), case["sinks"])
        pairs += int((hi - lo + sink).sum())
        union += int(hi.max() - lo.min() + sink.max())
    sum_n = sum(_lengths(case)[0])
    H, K, d = case["heads"], case["kv_heads"], case["d"]
    b, f = (2 * sum_n * H + 2 * union * K) * d * e, 4 * d * H * pairs
    if case["train"]:                            # q, k, v, o, do read; dq, dk, dv written; lse written and read
        b += (4 * sum_n * H + 4 * union * K) * d * e + 2 * sum_n * H * 4
        f += 10 * d * H * pairs
    return {"bytes": b, "flops": f}


# ------------------------------------------------------------------ in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "embed":
        table = s["table"].double()
        ids = s["ids"].long()
        ok = torch.nonzero((ids >= 0) & (ids < case["vocab"])).flatten()
        y = torch.zeros((ids.numel(), case["c"]), dtype=torch.float64, device="cuda")
        y[ok] = case["scale"] * torch.index_select(table, 0, ids[ok])
        out = dict(y=y)
        if case["train"]:
            del table
            g = torch.zeros((case["vocab"], case["c"]), dtype=torch.float64, device="cuda")
            g.index_put_((ids[ok],), case["scale"] * s["dy"][ok].double(), accumulate=True)
            out["dtable"] = g
        return out
    H, K, d, train = case["heads"], case["kv_heads"], case["d"], case["train"]
    G = H // K
    n, m = _lengths(case)
    double = lambda x: x.double().requires_grad_(train)   # noqa: E731
    q, k, v = double(s["q"]), double(s["k"]), double(s["v"])
    O = torch.zeros_like(q, requires_grad=False)
    lse = torch.zeros((H, q.shape[0]), dtype=torch.float64, device="cuda")
    grads = [torch.zeros_like(x, requires_grad=False) for x in (q, k, v)]
    a = b = 0
    for N, M, slots in zip(n, m, s["slots"].tolist()):
        far = torch.arange(M - N, M, device="cuda")[:, None] - torch.arange(M, device="cuda")[None, :]
        hidden = torch.zeros((N, M), dtype=torch.bool, device="cuda")
        if case["left"] >= 0:
            hidden |= far > case["left"]
            hidden[:, :case["sinks"]] = False
        if case["right"] >= 0:
            hidden |= far < -case["right"]
        for h in range(H):
            qc, kc = slice(h * d, (h + 1) * d), slice(h // G * d, (h // G + 1) * d)
            x = q[a:a + N, qc].detach().requires_grad_(train)
            y = k[b:b + M, kc].detach().requires_grad_(train)
            z = v[b:b + M, kc].detach().requires_grad_(train)
            score = torch.mm(x, y.t()) / math.sqrt(d)
            score = score.masked_fill(hidden, -math.inf)
            r = torch.mm(torch.softmax(score, 1), z)
            O[a:a + N, qc] = r.detach()
            if train:
                lse[h, a:a + N] = torch.logsumexp(score, 1).detach()
                gx, gy, gz = torch.autograd.grad(r, (x, y, z), s["do"][a:a + N, qc].double())
                grads[0][a:a + N, qc] += gx
                grads[1][b:b + M, kc] += gy
                grads[2][b:b + M, kc] += gz
        a, b = a + N, b + slots
    if not train:
        return dict(o=O)
    return dict(o=O, lse=lse, dq=grads[0], dk=grads[1], dv=grads[2])
