"""Window attention at sizes that reach the kernels of large calls, against float64
with the bars of tests/window_bars.py.

Blocks of 128 rows (keys) are used past 128 blocks of rows (256 of keys) of all
key/value heads, blocks of 32 below.  Each case states which it is for, with a
quarter to spare, and the workspace tells whether keys are cut over workgroups
(partial outputs), rows of keys in parts, and sinks handled apart: all of it is
asserted, so that a moved border cannot drop a kernel from these tests unseen."""
import numpy as np
import pytest

from paper_2609_30379_amd import synth

from . import window_bars as W
from .gpu_util import PARITY_LOG, dev, host

pytestmark = pytest.mark.gpu


def layout(n):
    from paper_2609_30379_amd import binding as B
    return B.NestedLayout(n, cols=[1] * len(n))


def blocks(lengths, mul, heads):
    return sum((x * mul + 127) // 128 for x in lengths) * heads


def near(got, ref, bar, what):
    r = W.worst(got, ref, bar)
    PARITY_LOG.append((what + " [of the derived bar]", r, 1.0, float(np.abs(np.where(np.isfinite(ref), ref, 0)).max(initial=0.0))))
    assert r <= 1.0, f"{what}: {r:.2f} of the bar"


def rows_of(large, n, G, K):
    got = blocks(n, G, K)
    assert got >= 160 if large else got <= 96, got


def forward(n, m, H, K, d, dtype, left=-1, right=0, sinks=0, *, large, cut, slots=None, seed=0, scale=None):
    """One call against float64; `large`: blocks of 128 rows, `cut`: keys over
    several workgroups.  `slots`: room of each sample, of which `m` is in use."""
    import torch
    from paper_2609_30379_amd import binding as B
    rows_of(large, n, H // K, K)
    room = m if slots is None else slots
    x = {"q": synth.normal(seed, "w.q", (sum(n), H * d), 1.0, dtype), "k": synth.normal(seed, "w.k", (sum(room), K * d), 1.0, dtype),
         "v": synth.normal(seed, "w.v", (sum(room), K * d), 1.0, dtype)}
    b = 0
    for i, s in enumerate(room):                           # what is not in use holds anything
        x["k"][b + m[i]:b + s], x["v"][b + m[i]:b + s] = np.nan, np.inf
        b += s
    t = {a: dev(y, dtype) for a, y in x.items()}
    ql = layout(n)
    kl = ql if room == n else layout(room)
    kw = dict(left=left, right=right, sinks=sinks)
    need = B.window_attention_workspace_bytes(ql, H, d, kv_layout=kl, kv_heads=K, dtype=dtype, **kw)
    assert (need > 0) == cut, need
    o = torch.full((sum(n), H * d), float("nan"), dtype=t["q"].dtype, device="cuda")
    lse = torch.full((H, sum(n)), float("nan"), device="cuda")
    ws = B.workspace_tensor(need)
    if ws is not None:
        ws.fill_(0xff)                                     # leftovers of another call: NaN as fp32
    B.nt_window_attention(ql, H, d, t["q"], t["k"], t["v"], o, lse=lse, kv_layout=kl, kv_heads=K, scale=scale, workspace=ws,
                          kv_lengths=None if slots is None else torch.tensor(m, dtype=torch.int32, device="cuda"), **kw)
    f = W.forward({a: np.where(np.isfinite(y), y, 0.0) for a, y in x.items()}, n, m, H, K, d, dtype, slots=room, scale=scale, **kw)
    what = f"window {dtype} n={n[:3]} m={m[:3]} H={H}/{K} d={d} [{left},{right}]+{sinks}"
    near(host(o), *f["o"], what + " o")
    got, (ref, bar) = host(lse), f["lse"]
    assert np.array_equal(np.isneginf(got), np.isneginf(ref))
    some = np.isfinite(ref)
    near(np.where(some, got, 0), np.where(some, ref, 0), bar, what + " lse")
    return dict(x=x, t=t, ql=ql, kl=kl, o=o, lse=lse, kw=kw, what=what)


def training(n, m, H, K, d, dtype, left=-1, right=0, sinks=0, *, large, cut, keys, parts, apart, seed=0):
    """The forward and its gradients; `keys`: blocks of 128 keys, `parts`: into how
    many parts their rows are cut, `apart`: sinks handled apart."""
    import torch
    from paper_2609_30379_amd import binding as B
    r = forward(n, m, H, K, d, dtype, left, right, sinks, large=large, cut=cut, seed=seed)
    got = blocks(m, 1, K)
    assert got >= 288 if keys else got <= 192, got
    x, t, kw = r["x"], r["t"], r["kw"]
    x["do"] = synth.normal(seed, "w.do", (sum(n), H * d), 1.0, dtype)
    do = dev(x["do"], dtype)
    g = [torch.full_like(t[a], float("nan")) for a in ("q", "k", "v")]
    need = B.window_attention_backward_workspace_bytes(r["ql"], H, d, kv_layout=r["kl"], kv_heads=K, dtype=dtype, **kw)
    rest = need - (H * sum(n) * 4 + 15) // 16 * 16 - (parts * 2 * sum(m) * K * d * 4 if parts > 1 else 0)
    assert rest > 0 if apart else rest == 0, (need, rest)
    ws = B.workspace_tensor(need)
    ws.fill_(0xff)
    B.nt_window_attention_backward(r["ql"], H, d, t["q"], t["k"], t["v"], r["o"], r["lse"], do, *g, kv_layout=r["kl"], kv_heads=K,
                                   workspace=ws, **kw)
    ref = W.backward(x, host(r["o"]), host(r["lse"]), n, m, H, K, d, dtype, **kw)
    for a, y in zip(("dq", "dk", "dv"), g):
        near(host(y), *ref[a], r["what"] + " " + a)


WINDOWS = [(-1, 0, 0), (40, 0, 3), (30, 20, 2), (-1, -1, 0)]


@pytest.mark.parametrize("left,right,sinks", WINDOWS)
@pytest.mark.parametrize("d", [32, 56, 64, 128])
def test_blocks_of_128_bf16(d, left, right, sinks):
    n = [300, 0, 140, 1]
    training(n, n, 128, 64, d, "bf16", left, right, sinks, large=True, cut=False, keys=True, parts=1, apart=False)


@pytest.mark.parametrize("left,right,sinks", WINDOWS)
@pytest.mark.parametrize("d", [24, 32, 64, 120])
def test_blocks_of_128_f32(d, left, right, sinks):
    n = [200, 0, 140, 1]
    training(n, n, 128, 64, d, "f32", left, right, sinks, large=True, cut=False, keys=True, parts=1, apart=False)


@pytest.mark.parametrize("dtype,d", [("bf16", 32), ("bf16", 64), ("bf16", 104), ("f32", 32), ("f32", 64)])
def test_blocks_of_128_with_sinks_apart(dtype, d):
    """Few first keys and all the rows past their window, more than 512."""
    training([900, 40], [900, 40], 48, 48, d, dtype, 20, 0, 5, large=True, cut=False, keys=True, parts=1, apart=True)


@pytest.mark.parametrize("dtype,d,parts", [("bf16", 104, 2), ("f32", 40, 2)])
def test_blocks_of_128_in_parts_with_sinks_apart(dtype, d, parts):
    """Rows of a block of keys in parts, and sinks apart: what training on long samples runs."""
    training([1100, 30], [1100, 30], 128, 32, d, dtype, 500, 0, 4, large=True, cut=False, keys=True, parts=parts, apart=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_blocks_of_128_more_keys_than_queries(dtype):
    """Chunks over a cache with their gradients; keys no query sees get zeros."""
    training([150, 3, 90], [700, 260, 91], 64, 32, 64, dtype, 100, 0, 70, large=True, cut=dtype == "f32", keys=True, parts=1, apart=False)


@pytest.mark.parametrize("dtype,d", [("bf16", 32), ("bf16", 64), ("bf16", 128), ("f32", 32), ("f32", 64), ("f32", 128)])
@pytest.mark.parametrize("left,sinks", [(-1, 0), (900, 70)])
def test_chunks_over_a_long_cache(dtype, d, left, sinks):
    """Blocks of 128 rows whose keys are cut over workgroups."""
    forward([200, 0, 130], [2500, 40, 1300], 64, 32, d, dtype, left, 0, sinks, large=True, cut=True)


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 128), ("f32", 64)])
@pytest.mark.parametrize("left,right", [(-1, 0), (-1, -1), (700, 300)])
def test_chunks_over_a_cache_with_room(dtype, d, left, right):
    """Slots for many more keys than are in use: most workgroups of a cut block see
    nothing, and some queries (more of them than keys) see nothing either."""
    forward([200, 130, 60], [230, 100, 0], 64, 32, d, dtype, left, right, 3, large=True, cut=True, slots=[2600, 1300, 1900])


@pytest.mark.parametrize("dtype,d", [("bf16", 8), ("bf16", 32), ("bf16", 64), ("bf16", 128), ("f32", 32), ("f32", 64), ("f32", 128)])
@pytest.mark.parametrize("left,right,sinks", [(-1, 0, 0), (4300, 7, 40)])
def test_tokens_over_a_long_cache(dtype, d, left, right, sinks):
    """Few rows whose keys are cut over workgroups: one token each, and a few with
    a bound on the right that none of them needs."""
    forward([1, 1, 3, 1], [3000, 0, 5200, 2049], 8, 2, d, dtype, left, right, sinks, large=False, cut=True)


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 128), ("f32", 64), ("f32", 128)])
def test_tokens_over_a_cache_with_room(dtype, d):
    """Of 8192 slots a few are in use, none, one, or nearly all; more queries than keys."""
    forward([1, 1, 1, 4, 1], [300, 0, 1, 2, 8000], 16, 4, d, dtype, -1, 0, 0, large=False, cut=True, slots=[8192] * 5)


@pytest.mark.parametrize("left,right,sinks", WINDOWS)
@pytest.mark.parametrize("d", [8, 32, 64, 96, 128])
def test_few_rows_f32_within_fp32_bars(d, left, right, sinks):
    n = [0, 1, 5, 33, 64, 0, 130, 31]
    training(n, n, 4, 2, d, "f32", left, right, sinks, large=False, cut=False, keys=False, parts=1, apart=False)


@pytest.mark.parametrize("scale", [0.0, -0.3, 1.0])
def test_scales_in_blocks_of_128(scale):
    for dtype in ("bf16", "f32"):
        forward([250, 130], [250, 130], 48, 48, 64, dtype, 60, 0, 1, large=True, cut=False, scale=scale)


@pytest.mark.parametrize("dtype,ld", [("bf16", (1 << 22) + 64), ("f32", (1 << 21) + 64)])
@pytest.mark.parametrize("n,H,K", [([260, 0, 30], 128, 64), ([40, 3], 2, 1)])
def test_rows_further_apart_than_32_bit_tiles(dtype, ld, n, H, K):
    """Row strides past 2^23 bytes, forward and backward: the same bits as contiguous operands."""
    import torch
    from paper_2609_30379_amd import binding as B
    T, d = sum(n), 16
    rows_of(H > 2, n, H // K, K)
    lay = layout(n)
    widths = [H * d, K * d, K * d, H * d]
    assert sum(widths) <= ld
    wide = torch.empty((T, ld), dtype=torch.bfloat16 if dtype == "bf16" else torch.float32, device="cuda")
    cols = np.cumsum([0] + widths)
    far = [wide[:, a:a + w] for a, w in zip(cols, widths)]
    for i, (y, w) in enumerate(zip(far, widths)):
        y.copy_(dev(synth.normal(i, "far", (T, w), 1.0, dtype), dtype))
    kw = dict(kv_heads=K, left=50, right=0, sinks=2)
    out = []
    for q, k, v, do in (far, [y.contiguous() for y in far]):
        o, lse = torch.full_like(do, float("nan")), torch.full((H, T), float("nan"), device="cuda")
        B.nt_window_attention(lay, H, d, q, k, v, o, lse=lse, **kw)
        g = [torch.full((T, w), float("nan"), dtype=o.dtype, device="cuda") for w in widths[:3]]
        B.nt_window_attention_backward(lay, H, d, q, k, v, o, lse, do, *g, **kw)
        out.append([o, lse, *g])
    for a, b in zip(*out):
        assert bool(torch.isfinite(a).all()) and torch.equal(a, b)


@pytest.mark.parametrize("n,H,K", [([300, 140], 128, 64), ([300, 41], 4, 2)])
def test_another_stream_writes_every_output(n, H, K):
    """The same bits on another stream, into outputs that were cleared before."""
    import torch
    from paper_2609_30379_amd import binding as B
    T, d = sum(n), 64
    lay = layout(n)
    q, k, v, do = (dev(synth.normal(i, "s", (T, h * d), 1.0, "bf16"), "bf16") for i, h in enumerate((H, K, K, H)))
    o, lse = torch.empty_like(q), torch.empty((H, T), device="cuda")
    g = [torch.empty_like(y) for y in (q, k, v)]
    kw = dict(kv_heads=K, left=100, sinks=3)

    def call():
        for y in (o, lse, *g):
            y.fill_(float("nan"))
        B.nt_window_attention(lay, H, d, q, k, v, o, lse=lse, **kw)
        B.nt_window_attention_backward(lay, H, d, q, k, v, o, lse, do, *g, **kw)

    call()
    first = [host(y) for y in (o, lse, *g)]
    assert all(np.isfinite(y).all() for y in first)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        call()
    s.synchronize()
    assert all(np.array_equal(a, host(b)) for a, b in zip(first, (o, lse, *g)))


def test_missing_or_short_workspaces_are_refused():
    import torch
    from paper_2609_30379_amd import binding as B
    ql, kl = layout([1, 2]), layout([6000, 3000])
    q, o = (torch.zeros((3, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    k, v = (torch.zeros((9000, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    kw = dict(kv_layout=kl, kv_heads=1)
    need = B.window_attention_workspace_bytes(ql, 2, 64, **kw)
    short = torch.zeros(need - 1, dtype=torch.uint8, device="cuda")
    odd = torch.zeros(need + 16, dtype=torch.uint8, device="cuda")[4:]
    for ws, word in ((short, "workspace of"), (odd, "aligned")):
        with pytest.raises(B.NtError, match=word):
            B.nt_window_attention(ql, 2, 64, q, k, v, o, workspace=ws, **kw)
    lse, g = torch.zeros((2, 3), device="cuda"), [torch.zeros_like(y) for y in (q, k, v)]
    need = B.window_attention_backward_workspace_bytes(ql, 2, 64, **kw)
    with pytest.raises(B.NtError, match="workspace of"):
        B.nt_window_attention_backward(ql, 2, 64, q, k, v, o, lse, q, *g, workspace=torch.zeros(need - 1, dtype=torch.uint8, device="cuda"),
                                       **kw)
