"""Sliding-window attention, forward and backward, against the float64 oracle.

Bars are derived, not chosen.  With u = finfo(type).eps / 2 the relative error of
a rounding: a bf16 call rounds the weights P (and in the backward dS) and the
result, so |o - ref| <= u (A + |o|) with A = sum_j P_j |v_j|, and the gradients
likewise (oracle.tokens.window_attention_backward).  What fp32 arithmetic adds is
covered by fp_rel = 2^-22 (d + 16) (1 + T) + 2^-23 M relative to the same sums: T bounds
|scale| sum_c |q_c k_c|, so a score of d products is off by less than
2^-24 (d + 2) T, a weight by that and a few roundings of the exponential, and a
sum over M keys by 2^-24 M of its terms' sizes."""
import numpy as np
import pytest

from oracle import tokens as T
from paper_2609_30379_amd import synth

from .gpu_util import PARITY_LOG, dev, host

pytestmark = pytest.mark.gpu

U = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


def layout(n):
    from paper_2609_30379_amd import binding as B
    return B.NestedLayout(n, cols=[1] * len(n))


def fp_rel(q, k, d, scale, m):
    t = abs(scale) * d * float(np.abs(q).max(initial=0.0)) * float(np.abs(k).max(initial=0.0)) / 4
    return 2.0 ** -22 * (d + 16) * (1 + t) + 2.0 ** -23 * max(m + [0])


def near(got, ref, bound, what):
    assert got.shape == ref.shape
    assert np.isfinite(got).all(), what
    r = np.abs(got - ref) / np.maximum(bound, 1e-30)
    worst = float(r.max(initial=0.0))
    PARITY_LOG.append((what + " [of the derived bound]", worst, 1.0, float(np.abs(ref).max(initial=0.0))))
    assert worst <= 1.0, f"{what}: {worst:.2f} of the bound at {np.unravel_index(r.argmax(), r.shape)}"


def run(n, m, H, K, d, dtype, left=-1, right=0, sinks=0, scale=None, slots=None, train=True, seed=0, tweak=None):
    """Forward (and backward) of one call against the oracle; returns the device tensors."""
    import torch
    from paper_2609_30379_amd import binding as B
    sq, sk = sum(n), sum(slots or m)
    x = {"q": synth.normal(seed, "w.q", (sq, H * d), 1.0, dtype), "k": synth.normal(seed, "w.k", (sk, K * d), 1.0, dtype),
         "v": synth.normal(seed, "w.v", (sk, K * d), 1.0, dtype), "do": synth.normal(seed, "w.do", (sq, H * d), 1.0, dtype)}
    if tweak:
        tweak(x)
    t = {a: dev(v, dtype) for a, v in x.items()}
    ql = layout(n)
    kl = ql if (slots or m) == n else layout(slots or m)
    kw = dict(kv_layout=kl, kv_heads=K, left=left, right=right, sinks=sinks, scale=scale)
    ok = dict(left=left, right=right, sinks=sinks, scale=scale)
    td = t["q"].dtype
    o = torch.full((sq, H * d), float("nan"), dtype=td, device="cuda")
    lse = torch.full((H, sq), float("nan"), dtype=torch.float32, device="cuda")
    used = torch.tensor(m, dtype=torch.int32, device="cuda") if slots else None
    B.nt_window_attention(ql, H, d, t["q"], t["k"], t["v"], o, lse=lse, kv_lengths=used, **kw)
    ro, rl, A = T.window_attention(x["q"], x["k"], x["v"], n, m, H, K, d, slots=slots, **ok)
    sc = 1 / np.sqrt(d) if scale is None else scale
    fin = {a: np.where(np.isfinite(v), v, 0.0) for a, v in x.items()}
    fp, u = fp_rel(fin["q"], fin["k"], d, sc, m), U[dtype]
    what = f"window {dtype} n={n[:4]} m={m[:4]} H={H}/{K} d={d} [{left},{right}]+{sinks}"
    near(host(o), ro, (u if dtype == "bf16" else 0) * A + u * np.abs(ro) + fp * A, what + " o")
    gl = host(lse)
    assert np.array_equal(np.isneginf(gl), np.isneginf(rl))
    some = np.isfinite(rl)
    near(np.where(some, gl, 0), np.where(some, rl, 0), fp + 2.0 ** -22 * np.abs(np.where(some, rl, 0)), what + " lse")
    if train:
        g = [torch.full_like(t[a], float("nan")) for a in ("q", "k", "v")]
        B.nt_window_attention_backward(ql, H, d, t["q"], t["k"], t["v"], o, lse, t["do"], *g, **kw)
        ref, err = T.window_attention_backward(x["q"], x["k"], x["v"], host(o), host(lse), x["do"], n, m, H, K, d, **ok,
                                               ds_rel=u if dtype == "bf16" else 0.0, p_rel=u if dtype == "bf16" else 0.0,
                                               fp_rel=fp + 2.0 ** -23 * max(n + [0]) * (H // K))
        for name, a, r, e in zip(("dq", "dk", "dv"), g, ref, err):
            near(host(a), r, 1.01 * e + u * np.abs(r), what + " " + name)
        t.update(dq=g[0], dk=g[1], dv=g[2])
    t.update(o=o, lse=lse, ql=ql, kl=kl, kw=kw)
    return t


RAGGED = [0, 1, 5, 33, 64, 0, 130, 31]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [8, 32, 40, 64, 96, 128])
@pytest.mark.parametrize("left,right,sinks", [(-1, 0, 0), (7, 0, 3), (16, 16, 1), (-1, -1, 0)])
def test_head_dims_and_windows(dtype, d, left, right, sinks):
    run(RAGGED, RAGGED, 2, 1, d, dtype, left, right, sinks)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,K", [(1, 1), (3, 3), (6, 2), (5, 1), (16, 2)])
def test_heads(dtype, H, K):
    run([37, 1, 0, 90], [37, 1, 0, 90], H, K, 32, dtype, left=20, sinks=2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,m,left,right,sinks", [
    ([1], [1], -1, 0, 0), ([1], [1], 0, 0, 0),
    ([3, 40], [1, 7], -1, 0, 0),               # more queries than keys: the first see nothing
    ([3, 40], [1, 7], 2, 0, 1),
    ([5, 9], [0, 12], -1, -1, 0),              # no keys at all
    ([0, 4], [70, 4], -1, 0, 0),               # keys without a query: zero gradients
    ([200], [200], 0, 0, 0), ([200], [200], 0, 0, 70),   # only itself; sinks past a tile
    ([200], [200], 3, 0, 199), ([200], [200], 3, 0, 500),
    ([257], [257], 64, 0, 4), ([257], [257], 63, 1, 0),
    ([130], [700], 100, 0, 5), ([130], [700], 600, 0, 65), ([20], [300], 10, 3, 2),
    ([900, 0, 40], [900, 7, 700], 20, 0, 3), ([800], [850], 9, 4, 200),   # sinks seen far past their window
    ([150], [150], -1, 5, 3), ([150], [150], 5, -1, 3),
])
def test_edges(dtype, n, m, left, right, sinks):
    run(n, m, 4, 2, 64 if dtype == "bf16" else 32, dtype, left, right, sinks)


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f32", 64)])
def test_long(dtype, d):
    run([1500, 700], [1500, 700], 2, 1, d, dtype, left=300, sinks=4)
    run([900], [900], 2, 2, d, dtype)


@pytest.mark.parametrize("batch", [1, 63, 64, 200, 5000])
def test_many_samples(batch):
    """Blocks find their sample: in one step of the lanes, in two, with empty samples between."""
    rng = np.random.default_rng(batch)
    n = [int(x) for x in rng.integers(0, 4, batch)]
    n[batch // 2] = 150
    m = [x + int(y) for x, y in zip(n, rng.integers(0, 3, batch))]
    run(n, m, 2, 1, 8, "f32", left=9, sinks=1)


@pytest.mark.parametrize("scale", [0.0, -0.3, 2.0])
def test_scales(scale):
    run([70, 9], [70, 9], 2, 1, 32, "bf16", left=30, sinks=1, scale=scale)
    run([70, 9], [70, 9], 2, 1, 32, "f32", left=30, sinks=1, scale=scale)


def test_large_scores_stay_finite():
    """Scores of thousands: only the running maximum keeps the weights finite."""
    def up(x):
        x["q"] *= 64.0
    run([90], [90], 1, 1, 32, "f32", left=40, tweak=up, train=False)
    run([90], [90], 1, 1, 32, "bf16", left=40, tweak=up, train=False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,K,d", [(4, 4, 64), (8, 1, 128), (12, 3, 32)])
@pytest.mark.parametrize("left,sinks", [(-1, 0), (50, 3)])
def test_single_tokens_over_a_cache(dtype, H, K, d, left, sinks):
    """One query per sample, slots that hold NaN past the keys in use."""
    m, slots = [1, 0, 300, 129, 64, 513], [64, 5, 300, 192, 64, 600]

    def leftovers(x):
        b = 0
        for u, s in zip(m, slots):
            x["k"][b + u:b + s] = np.nan
            x["v"][b + u:b + s] = np.inf
            b += s
    run([1] * 6, m, H, K, d, dtype, left, 0, sinks, slots=slots, train=False, tweak=leftovers)


def test_lengths_on_the_device_are_clamped():
    import torch
    from paper_2609_30379_amd import binding as B
    ql, kl = layout([2, 2, 2]), layout([8, 8, 8])
    q, k, v = (dev(synth.normal(5, a, (r, 32), 1.0, "f32"), "f32") for a, r in (("q", 6), ("k", 24), ("v", 24)))
    out = []
    for used in ([-3, 8, 3], [0, 100, 3]):
        o = torch.empty_like(q)
        B.nt_window_attention(ql, 1, 32, q, k, v, o, kv_layout=kl,
                              kv_lengths=torch.tensor(used, dtype=torch.int32, device="cuda"))
        out.append(host(o))
    assert np.array_equal(out[0], out[1]) and not out[0][:2].any()


def test_strided_operands_and_rows_behind():
    """q, k, v as column slices of one projection; rows past the batch stay as they were."""
    import torch
    from paper_2609_30379_amd import binding as B
    n, H, K, d = [20, 0, 75], 4, 2, 40
    lay = layout(n)
    w = (H + 2 * K) * d + 8
    buf = dev(synth.normal(7, "qkv", (100, w), 1.0, "bf16"), "bf16")
    cut = lambda t: (t[:95, :H * d], t[:95, H * d:(H + K) * d], t[:95, (H + K) * d:(H + 2 * K) * d])   # noqa: E731
    q, k, v = cut(buf)
    o, lse = torch.full((100, H * d + 16), 7.0, dtype=torch.bfloat16, device="cuda"), torch.empty((H, 99), device="cuda")
    do = dev(synth.normal(8, "do", (95, H * d), 1.0, "bf16"), "bf16")
    g = torch.full((100, w), 7.0, dtype=torch.bfloat16, device="cuda")
    kw = dict(kv_heads=K, left=12, sinks=2)
    B.nt_window_attention(lay, H, d, q, k, v, o[:95, :H * d], lse=lse[:, :95], **kw)
    B.nt_window_attention_backward(lay, H, d, q, k, v, o[:95, :H * d], lse[:, :95], do, *cut(g), **kw)
    o2, l2 = torch.empty((95, H * d), dtype=torch.bfloat16, device="cuda"), torch.empty((H, 95), device="cuda")
    g2 = [torch.empty((95, x * d), dtype=torch.bfloat16, device="cuda") for x in (H, K, K)]
    q, k, v = (x.contiguous() for x in (q, k, v))
    B.nt_window_attention(lay, H, d, q, k, v, o2, lse=l2, **kw)
    B.nt_window_attention_backward(lay, H, d, q, k, v, o2, l2, do, *g2, **kw)
    assert torch.equal(o[:95, :H * d], o2) and torch.equal(lse[:, :95], l2)
    assert all(torch.equal(a, b) for a, b in zip(cut(g), g2))
    assert bool((o[95:] == 7).all()) and bool((o[:, H * d:] == 7).all())
    assert bool((g[95:] == 7).all()) and bool((g[:, -8:] == 7).all())


def test_same_bits_every_time_and_on_another_stream():
    import torch
    from paper_2609_30379_amd import binding as B
    t = run([300, 41], [300, 41], 4, 2, 64, "bf16", left=100, sinks=3)
    first = [host(t[a]) for a in ("o", "lse", "dq", "dk", "dv")]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        B.nt_window_attention(t["ql"], 4, 64, t["q"], t["k"], t["v"], t["o"], lse=t["lse"], **t["kw"])
        B.nt_window_attention_backward(t["ql"], 4, 64, t["q"], t["k"], t["v"], t["o"], t["lse"], t["do"], t["dq"],
                                       t["dk"], t["dv"], **t["kw"])
    s.synchronize()
    assert all(np.array_equal(a, host(t[b])) for a, b in zip(first, ("o", "lse", "dq", "dk", "dv")))


def test_captured_graph_follows_the_lengths():
    """A captured single-token call replayed over a growing cache, eager calls in between."""
    import torch
    from paper_2609_30379_amd import binding as B
    H, K, d, cap = 4, 2, 64, 700
    ql, kl = layout([1, 1]), layout([cap, cap])
    q, k, v = (dev(synth.normal(9, a, (r, h * d), 1.0, "bf16"), "bf16") for a, r, h in (("q", 2, H), ("k", 2 * cap, K),
                                                                                   ("v", 2 * cap, K)))
    o, want = torch.empty_like(q), torch.empty_like(q)
    used = torch.tensor([5, 600], dtype=torch.int32, device="cuda")
    kw = dict(kv_layout=kl, kv_heads=K, left=400, sinks=2, kv_lengths=used)
    ws = B.workspace_tensor(B.window_attention_workspace_bytes(ql, H, d, kv_layout=kl, kv_heads=K, left=400, sinks=2))
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        B.nt_window_attention(ql, H, d, q, k, v, o, workspace=ws, **kw)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.nt_window_attention(ql, H, d, q, k, v, o, workspace=ws, **kw)
    for step in range(4):
        used += torch.tensor([37, 11], dtype=torch.int32, device="cuda")
        graph.replay()
        got = host(o)
        B.nt_window_attention(ql, H, d, q, k, v, want, **kw)
        assert np.array_equal(got, host(want)), step


def test_a_row_of_a_long_cache_past_32_bit_offsets():
    """Keys more than 2^32 elements into their buffer."""
    import torch
    from paper_2609_30379_amd import binding as B
    H, d, m = 1, 64, 40
    ld = 1 << 27
    buf = torch.zeros(ld * (m - 1) + 2 * d, dtype=torch.bfloat16, device="cuda")
    kv = buf.as_strided((m, 2 * d), (ld, 1))
    kv.copy_(dev(synth.normal(11, "kv", (m, 2 * d), 1.0, "bf16"), "bf16"))
    q = dev(synth.normal(11, "q", (1, d), 1.0, "bf16"), "bf16")
    o, want = torch.empty_like(q), torch.empty_like(q)
    ql, kl = layout([1]), layout([m])
    B.nt_window_attention(ql, H, d, q, kv[:, :d], kv[:, d:], o, kv_layout=kl)
    B.nt_window_attention(ql, H, d, q, kv[:, :d].contiguous(), kv[:, d:].contiguous(), want, kv_layout=kl)
    assert torch.equal(o, want)


def test_single_tokens_give_a_prompts_rows():
    """A prompt's outputs, token by token over the same cache."""
    import torch
    from paper_2609_30379_amd import binding as B
    N, H, K, d = 70, 4, 2, 32
    q, k, v = (dev(synth.normal(12, a, (N, h * d), 1.0, "f32"), "f32") for a, h in (("q", H), ("k", K), ("v", K)))
    o = torch.empty_like(q)
    kw = dict(kv_heads=K, left=9, sinks=2)
    lay, one = layout([N]), layout([1])
    B.nt_window_attention(lay, H, d, q, k, v, o, **kw)
    for t in range(N):
        r = torch.empty_like(q[:1])
        B.nt_window_attention(one, H, d, q[t:t + 1], k, v, r, kv_layout=lay,
                              kv_lengths=torch.tensor([t + 1], dtype=torch.int32, device="cuda"), **kw)
        # two fp32 orders of the same sums, each within fp_rel of it
        assert float((r - o[t:t + 1]).abs().max()) <= 2 * 2.0 ** -22 * (d + 16) * 8 * float(v.abs().max())


def test_outputs_that_are_operands_are_refused():
    import torch
    from paper_2609_30379_amd import binding as B
    lay = layout([8])
    x = [torch.zeros((8, 32), dtype=torch.bfloat16, device="cuda") for _ in range(8)]
    lse = torch.zeros((1, 8), device="cuda")
    with pytest.raises(B.NtError):
        B.nt_window_attention(lay, 1, 32, x[0], x[1], x[2], x[2])
    for bad in range(3):
        g = [x[5], x[6], x[7]]
        g[bad] = x[bad]
        with pytest.raises(B.NtError):
            B.nt_window_attention_backward(lay, 1, 32, x[0], x[1], x[2], x[3], lse, x[4], *g)
    with pytest.raises(ValueError):
        B.nt_window_attention(lay, 1, 32, x[0].cpu(), x[1], x[2], x[3])
    with pytest.raises(ValueError):
        B.nt_window_attention(lay, 1, 32, x[0], x[1], x[2], x[3][:7])
    with pytest.raises(ValueError):
        B.nt_window_attention(lay, 1, 32, x[0], x[1].float(), x[2], x[3])


def test_keys_without_any_query_get_zero_gradients():
    import torch
    from paper_2609_30379_amd import binding as B
    ql, kl = layout([0, 0]), layout([5, 200])
    q = torch.zeros((0, 64), dtype=torch.bfloat16, device="cuda")
    k = torch.ones((205, 32), dtype=torch.bfloat16, device="cuda")
    v, lse = k.clone(), torch.zeros((2, 0), device="cuda")
    dk, dv = torch.full_like(k, float("nan")), torch.full_like(k, float("nan"))
    B.nt_window_attention(ql, 2, 32, q, k, v, q.clone(), kv_layout=kl, kv_heads=1, lse=lse)
    B.nt_window_attention_backward(ql, 2, 32, q, k, v, q.clone(), lse, q.clone(), q.clone(), dk, dv, kv_layout=kl, kv_heads=1,
                                   left=3, sinks=1)
    assert not bool(dk.any()) and not bool(dv.any())


def test_outputs_that_are_one_another_are_refused():
    import torch
    from paper_2609_30379_amd import binding as B
    lay = B.NestedLayout([3], cols=[1])
    x = [torch.zeros((3, 8), device="cuda") for _ in range(7)]
    q, k, v, o, do, g, h = x
    lse = torch.zeros((1, 3), device="cuda")
    for out in ((g, h, h), (g, g, h), (g, h, g)):
        with pytest.raises(B.NtError, match="one another"):
            B.nt_window_attention_backward(lay, 1, 8, q, k, v, o, lse, do, *out)


def test_many_samples_one_long():
    """More blocks of sinks than are handled apart: the keys' workgroups walk all rows."""
    n = [3] * 1100 + [700]
    run(n, n, 8, 8, 8, "f32", left=5, sinks=3)


@pytest.mark.parametrize("dtype,left,right,sinks", [("bf16", -1, 0, 0), ("f32", 500, 400, 4)])
def test_rows_of_keys_in_parts(dtype, left, right, sinks):
    """320 blocks of keys on 256 places: their rows are cut in two and the sums joined."""
    run([1100, 40], [1100, 40], 64, 32, 72, dtype, left, right, sinks)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_of_few_keys_in_parts(dtype):
    """Blocks of 32 keys that leave places free, groups that end inside a part."""
    run([401, 5], [401, 5], 3, 1, 96, dtype, 110, 110, 4)
    run([300], [350], 5, 1, 24, dtype)


def test_a_token_over_wide_fp32_keys():
    run([1, 2, 1], [733, 300, 0], 8, 1, 128, "f32", left=500, sinks=4, train=False)
