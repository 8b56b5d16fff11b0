"""Embedding lookup and its gradient against the float64 oracle.

The lookup is one fp32 product rounded once: off by at most u |y| with u =
finfo(type).eps / 2, plus 2^-24 |y| for the product where it is then rounded to
bf16.  The gradient sums c fp32 terms: off by at most 2^-24 (c + 2) times the sum
of their sizes, plus the rounding of a bf16 table (and of an added start)."""
import numpy as np
import pytest

from oracle import tokens as T
from paper_2609_30379_amd import synth

from .gpu_util import dev, host
from .test_gpu_window import U, near

pytestmark = pytest.mark.gpu


def ids_of(rows, vocab, seed, outside=0.1, hot=0.2):
    r = np.random.default_rng(seed)
    x = r.integers(0, max(vocab, 1), rows)
    x[r.random(rows) < hot] = vocab // 2
    x[r.random(rows) < outside] = -1
    x[r.random(rows) < outside / 2] = vocab
    return x


@pytest.mark.parametrize("tt", ["bf16", "f32"])
@pytest.mark.parametrize("ty", ["bf16", "f32"])
@pytest.mark.parametrize("rows,vocab,c,wide", [(0, 5, 8, 1), (1, 1, 8, 0), (7, 3, 24, 1), (300, 50, 200, 0),
                                               (65, 2000, 768, 1), (33, 9, 2056, 0), (5, 0, 8, 1)])
def test_lookup(tt, ty, rows, vocab, c, wide):
    import torch
    from paper_2609_30379_amd import binding as B
    table, ids = synth.normal(1, "t", (vocab, c), 1.0, tt), ids_of(rows, vocab, 2)
    y = torch.full((rows, c), float("nan"), dtype=dev(np.zeros(1), ty).dtype, device="cuda")
    B.nt_embedding(dev(table, tt), torch.tensor(ids, dtype=torch.int64 if wide else torch.int32, device="cuda"), y, 1.7)
    ref = T.embedding(table, ids, float(np.float32(1.7)))
    near(host(y), ref, (U[ty] + 2.0 ** -24) * np.abs(ref) * 1.001, f"embedding {tt}->{ty} {rows}x{vocab}x{c}")


@pytest.mark.parametrize("td,tg", [("bf16", "f32"), ("f32", "f32"), ("bf16", "bf16"), ("f32", "bf16")])
@pytest.mark.parametrize("rows,vocab,c,wide,acc", [
    (0, 5, 8, 1, 0), (0, 5, 8, 1, 1), (1, 1, 8, 0, 0), (7, 3, 24, 1, 1), (33, 1, 16, 0, 0), (300, 50, 200, 0, 0),
    (300, 50, 200, 1, 1), (65, 3000, 768, 1, 0), (1000, 7, 2056, 0, 1), (5000, 300, 32, 1, 0), (9000, 100000, 8, 0, 1),
    (5, 0, 8, 1, 0),
])
def test_gradient(td, tg, rows, vocab, c, wide, acc):
    import torch
    from paper_2609_30379_amd import binding as B
    ids = ids_of(rows, vocab, 3)
    dy, start = synth.normal(4, "dy", (rows, c), 1.0, td), synth.normal(5, "g", (vocab, c), 1.0, tg)
    g = dev(start, tg)
    i = torch.tensor(ids, dtype=torch.int64 if wide else torch.int32, device="cuda")
    d = dev(dy, td)
    B.nt_embedding_backward(i, d, g, 0.6, accumulate=bool(acc))
    s = float(np.float32(0.6))
    ref, mag, count = T.embedding_backward(ids, dy, vocab, s, start if acc else None)
    mag = mag + (np.abs(start) if acc else 0)
    bound = 1.01 * 2.0 ** -24 * (count[:, None] + 3) * mag + (U["bf16"] * 1.01 * np.abs(ref) if tg == "bf16" else 0)
    near(host(g), ref, bound, f"embedding gradient {td}->{tg} {rows}x{vocab}x{c} acc={acc}")
    if not acc:
        first = host(g)
        g.fill_(float("nan"))
        B.nt_embedding_backward(i, d, g, 0.6)
        assert np.array_equal(first, host(g))


@pytest.mark.parametrize("rows,vocab,what", [(140000, 3, "few"), (16384, 300, "many"), (16385, 70000, "many"), (20000, 5, "few"), (20000, 70000, "many"), (12345, 600000, "one"),
                                             (20000, 9, "none"), (4096, 513, "each")])
def test_gradient_runs(rows, vocab, what):
    """Runs over many chunks, three sort passes, all tokens equal, none inside."""
    import torch
    from paper_2609_30379_amd import binding as B
    r = np.random.default_rng(6)
    ids = {"few": r.integers(0, vocab, rows), "many": r.integers(0, vocab, rows), "one": np.full(rows, vocab - 1),
           "none": np.where(r.random(rows) < 0.5, -7, vocab + 3), "each": np.arange(rows) % vocab}[what]
    c = 8
    dy = synth.normal(7, "dy", (rows, c), 1.0, "f32")
    g = torch.full((vocab, c), float("nan"), device="cuda")
    B.nt_embedding_backward(torch.tensor(ids, device="cuda"), dev(dy, "f32"), g)
    ref, mag, count = np.zeros((vocab, c)), np.zeros((vocab, c)), np.bincount(ids[(ids >= 0) & (ids < vocab)], minlength=vocab)
    ok = (ids >= 0) & (ids < vocab)
    np.add.at(ref, ids[ok], dy[ok].astype(np.float64))
    np.add.at(mag, ids[ok], np.abs(dy[ok].astype(np.float64)))
    near(host(g), ref, 1.01 * 2.0 ** -24 * (count[:, None] + 3) * mag, f"embedding gradient {what}")


def test_strides_and_rows_behind():
    import torch
    from paper_2609_30379_amd import binding as B
    table = dev(synth.normal(8, "t", (40, 96), 1.0, "bf16"), "bf16")
    ids = torch.tensor([3, 39, -1, 3, 0], device="cuda")
    y = torch.full((7, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    B.nt_embedding(table[:, 16:48], ids, y[:5, 8:40])
    assert torch.equal(y[[0, 1, 3, 4], 8:40], table[[3, 39, 3, 0], 16:48]) and not bool(y[2, 8:40].any())
    assert bool((y[5:] == 7).all()) and bool((y[:, :8] == 7).all()) and bool((y[:, 40:] == 7).all())
    g = torch.full((42, 64), 7.0, device="cuda")
    B.nt_embedding_backward(ids, y[:5, 8:40], g[:40, 8:40])
    assert bool((g[40:] == 7).all()) and bool((g[:, :8] == 7).all()) and bool((g[:, 40:] == 7).all())
    assert torch.equal(g[3, 8:40], 2 * table[3, 16:48].float()) and not bool(g[1:3, 8:40].any())


def test_captured_gradient_replays():
    import torch
    from paper_2609_30379_amd import binding as B
    rows, vocab, c = 6000, 700, 64
    ids = torch.randint(-1, vocab, (rows,), device="cuda")
    dy = torch.randn((rows, c), device="cuda")
    g, want = torch.empty((vocab, c), device="cuda"), torch.empty((vocab, c), device="cuda")
    ws = B.workspace_tensor(B.embedding_backward_workspace_bytes(rows, vocab, c))
    B.nt_embedding_backward(ids, dy, g, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.nt_embedding_backward(ids, dy, g, workspace=ws)
    for _ in range(4):
        ids.copy_(torch.randint(-1, vocab, (rows,), device="cuda"))
        g.fill_(3.0)
        graph.replay()
        got = host(g)
        B.nt_embedding_backward(ids, dy, want)
        assert np.array_equal(got, host(want))


@pytest.mark.parametrize("rows,vocab", [(524288, 300), (524289, 70001), (600001, 1), (9000001, 70001), (8500000, 2)])
def test_gradient_of_many_tokens(rows, vocab):
    """Sorts of more than 128 tiles and chunks past 128 rows.  Gradients are small
    whole numbers, so every partial sum is exact and so is the result."""
    import torch
    from paper_2609_30379_amd import binding as B
    r = np.random.default_rng(8)
    ids = r.integers(-1, vocab, rows).astype(np.int32)
    if vocab == 2:
        ids[: rows - 5000] = 1                             # one run over nearly all chunks
    dy = r.integers(-2, 3, (rows, 8)).astype(np.float32)
    g = torch.full((vocab, 8), float("nan"), device="cuda")
    B.nt_embedding_backward(torch.tensor(ids, device="cuda"), torch.tensor(dy, device="cuda"), g)
    ok = ids >= 0
    ref = np.stack([np.bincount(ids[ok], dy[ok, j].astype(np.float64), vocab) for j in range(8)], 1)
    assert np.abs(ref).max() < 2 ** 24
    assert np.array_equal(host(g), ref)


def test_outputs_that_are_operands_are_refused():
    import torch
    from paper_2609_30379_amd import binding as B
    t = torch.zeros((4, 8), device="cuda")
    ids = torch.zeros(4, dtype=torch.int32, device="cuda")
    with pytest.raises(B.NtError):
        B.nt_embedding(t, ids, t)
    with pytest.raises(B.NtError):
        B.nt_embedding_backward(ids, t, t)


@pytest.mark.parametrize("rows", [16384, 16385, 99999, 100000, 131072, 131073, 499999, 500001, 1499999, 1500001])
@pytest.mark.parametrize("vocab", [3, 1000])
def test_gradient_on_both_sides_of_each_plan(rows, vocab):
    """Where chunks, tiles and the way their counts are summed change, and next to a
    power of two.  Whole numbers: every partial sum is exact."""
    import torch
    from paper_2609_30379_amd import binding as B
    r = np.random.default_rng(rows + vocab)
    ids = r.integers(-1, vocab + 1, rows).astype(np.int32)
    dy = r.integers(-2, 3, (rows, 8)).astype(np.float32)
    g = torch.full((vocab, 8), float("nan"), device="cuda")
    B.nt_embedding_backward(torch.tensor(ids, device="cuda"), torch.tensor(dy, device="cuda"), g)
    ok = (ids >= 0) & (ids < vocab)
    ref = np.stack([np.bincount(ids[ok], dy[ok, j].astype(np.float64), vocab) for j in range(8)], 1)
    assert np.abs(ref).max() < 2 ** 24
    assert np.array_equal(host(g), ref)
