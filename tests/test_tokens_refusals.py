"""Argument errors of the token operators, reported on the host before any
device work (CPU: host-only layouts, pointers that are never followed)."""
import ctypes as C

import pytest

from paper_2609_30379_amd import binding as B

P = 4096                                      # an aligned address that no call gets to read
KEEP = []                                     # layouts whose handles the argument structs hold


def host(n):
    return B.NestedLayout(n, cols=[1] * len(n), host_only=True)


def window_args(**kw):
    a = B.WindowArgs()
    lay = host([5, 7])
    KEEP.append(lay)
    a.q_layout = lay.handle
    a.heads, a.kv_heads, a.head_dim, a.left, a.right, a.sinks, a.scale, a.dtype = 4, 2, 32, 3, 0, 1, 0.2, B.NT_BF16
    a.q = a.k = a.v = a.dout = P
    a.o, a.dq, a.dk, a.dv = 2 * P, 3 * P, 4 * P, 5 * P
    a.ld_q = a.ld_o = a.ld_dout = a.ld_dq = 128
    a.ld_k = a.ld_v = a.ld_dk = a.ld_dv = 64
    a.lse, a.ld_lse = P, 12
    a.workspace, a.workspace_bytes = P, 1 << 40
    for k, v in kw.items():
        if isinstance(v, B.NestedLayout):
            KEEP.append(v)
            v = v.handle
        setattr(a, k, v)
    return a


def status(fn, *args):
    return getattr(B.load(), fn)(*args)


def error():
    return B.load().nt_last_error().decode()


WINDOW = [
    (dict(q_layout=None), B.NT_ERR_INVALID_ARG, "q_layout"),
    (dict(dtype=7), B.NT_ERR_INVALID_ARG, "dtype"),
    (dict(heads=0), B.NT_ERR_INVALID_ARG, "heads"),
    (dict(heads=3), B.NT_ERR_INVALID_ARG, "heads"),
    (dict(kv_heads=0), B.NT_ERR_INVALID_ARG, "heads"),
    (dict(heads=1 << 17), B.NT_ERR_UNSUPPORTED, "heads"),
    (dict(head_dim=0), B.NT_ERR_INVALID_ARG, "head_dim"),
    (dict(head_dim=36), B.NT_ERR_UNSUPPORTED, "head_dim"),
    (dict(head_dim=136), B.NT_ERR_UNSUPPORTED, "head_dim"),
    (dict(left=-2), B.NT_ERR_INVALID_ARG, "left"),
    (dict(right=-2), B.NT_ERR_INVALID_ARG, "right"),
    (dict(sinks=-1), B.NT_ERR_INVALID_ARG, "sinks"),
    (dict(scale=float("nan")), B.NT_ERR_INVALID_ARG, "scale"),
    (dict(scale=float("inf")), B.NT_ERR_INVALID_ARG, "scale"),
    (dict(q=None), B.NT_ERR_INVALID_ARG, "q is NULL"),
    (dict(k=P + 8), B.NT_ERR_INVALID_ARG, "k must be 16-byte"),
    (dict(ld_v=60), B.NT_ERR_INVALID_ARG, "v's row stride"),
    (dict(ld_v=68), B.NT_ERR_INVALID_ARG, "v's row stride"),
    (dict(ld_o=120), B.NT_ERR_INVALID_ARG, "o's row stride"),
    (dict(scale=2e38), B.NT_ERR_INVALID_ARG, "scale"),
    (dict(o=P), B.NT_ERR_INVALID_ARG, "alias"),
    (dict(ld_lse=11), B.NT_ERR_INVALID_ARG, "lse"),
    (dict(lse=P + 2), B.NT_ERR_INVALID_ARG, "lse"),
]


@pytest.mark.parametrize("fn", ["nt_window_attention", "nt_window_attention_backward"])
@pytest.mark.parametrize("kw,code,word", WINDOW)
def test_window_refusals(fn, kw, code, word):
    assert status(fn, C.byref(window_args(**kw)), None) == code
    assert word in error()


def test_window_layout_refusals():
    assert status("nt_window_attention", C.byref(window_args(kv_layout=host([5]))), None) == B.NT_ERR_LAYOUT_MISMATCH
    assert status("nt_window_attention", C.byref(window_args()), None) == B.NT_ERR_INVALID_ARG
    assert "host-only" in error()
    assert status("nt_window_attention", None, None) == B.NT_ERR_INVALID_ARG


@pytest.mark.parametrize("kw,word", [(dict(kv_lengths=P), "kv_lengths"), (dict(lse=None), "lse"), (dict(dout=None), "dout"),
                                     (dict(ld_dq=127), "dq"), (dict(dk=P + 4), "dk"), (dict(dv=None), "dv")])
def test_window_backward_refusals(kw, word):
    a = window_args(**kw)
    got = status("nt_window_attention_backward", C.byref(a), None)
    assert got == B.NT_ERR_INVALID_ARG and (word in error() or "host-only" in error())


def test_window_workspace_queries_read_no_pointers():
    a = window_args(q=None, k=None, v=None, o=None, lse=None, scale=float("nan"))
    n = C.c_uint64(77)
    assert status("nt_window_attention_workspace", C.byref(a), C.byref(n)) == B.NT_OK
    assert status("nt_window_attention_backward_workspace", C.byref(a), C.byref(n)) == B.NT_OK and n.value >= 4 * 12 * 4
    assert status("nt_window_attention_workspace", C.byref(a), None) == B.NT_ERR_INVALID_ARG
    assert status("nt_window_attention_backward_workspace", C.byref(window_args(heads=3)), C.byref(n)) == B.NT_ERR_INVALID_ARG


def embed(**kw):
    a = dict(table=P, vocab=10, ld_table=64, table_dtype=B.NT_BF16, ids=P, wide=1, rows=5, c=64, scale=1.0, y=P, ld_y=64,
             y_dtype=B.NT_BF16)
    a.update(kw)
    return status("nt_embedding", *a.values(), None)


def embed_backward(**kw):
    a = dict(ids=P, wide=1, rows=5, vocab=10, c=64, dy=P, ld_dy=64, dtype=B.NT_BF16, scale=1.0, dtable=P, ld=64,
             table_dtype=B.NT_F32, acc=0, ws=P, ws_bytes=1 << 40)
    a.update(kw)
    return status("nt_embedding_backward", *a.values(), None)


@pytest.mark.parametrize("kw,code", [
    (dict(rows=-1), B.NT_ERR_INVALID_ARG), (dict(vocab=-1), B.NT_ERR_INVALID_ARG), (dict(c=0), B.NT_ERR_INVALID_ARG),
    (dict(c=12), B.NT_ERR_INVALID_ARG), (dict(rows=1 << 31), B.NT_ERR_OVERFLOW), (dict(vocab=1 << 31), B.NT_ERR_OVERFLOW),
    (dict(ids=None), B.NT_ERR_INVALID_ARG), (dict(ids=P + 4), B.NT_ERR_INVALID_ARG), (dict(wide=2), B.NT_ERR_INVALID_ARG),
])
def test_embedding_refusals(kw, code):
    assert embed(**kw) == code and error()
    assert embed_backward(**kw) == code and error()


@pytest.mark.parametrize("kw", [dict(table=None), dict(y=None), dict(table=P + 8), dict(ld_table=60), dict(ld_y=68),
                                dict(y_dtype=5), dict(table_dtype=-1)])
def test_lookup_refusals(kw):
    assert embed(**kw) == B.NT_ERR_INVALID_ARG and error()


@pytest.mark.parametrize("kw", [dict(dy=None), dict(dtable=None), dict(dy=P + 8), dict(ld=62), dict(ld_dy=56), dict(acc=2),
                                dict(dtype=9), dict(table_dtype=9), dict(ws=None), dict(ws_bytes=8), dict(ws=P + 8)])
def test_embedding_gradient_refusals(kw):
    assert embed_backward(**kw) == B.NT_ERR_INVALID_ARG and error()


def test_embedding_outputs_that_are_operands():
    assert embed() == B.NT_ERR_INVALID_ARG and "alias" in error()
    assert embed_backward() == B.NT_ERR_INVALID_ARG and "alias" in error()
    assert embed(c=1 << 25, ld_table=1 << 25, ld_y=1 << 25) == B.NT_ERR_OVERFLOW
    assert embed_backward(c=1 << 25, ld=1 << 25, ld_dy=1 << 25) == B.NT_ERR_OVERFLOW


def test_workspaces_stay_bounded():
    """Many blocks of sinks, of which one long sample uses a few; tokens by the ten million."""
    lengths = [40] * 499 + [20000]
    a = window_args(q_layout=host(lengths), kv_layout=host(lengths), heads=8, kv_heads=8, head_dim=128, left=64, sinks=20000,
                    ld_q=1024, ld_k=1024, ld_v=1024, ld_o=1024)
    n = C.c_uint64()
    assert status("nt_window_attention_backward_workspace", C.byref(a), C.byref(n)) == B.NT_OK
    assert n.value < 1 << 30
    assert status("nt_embedding_backward_workspace", 1 << 30, 1000, 512, C.byref(n)) == B.NT_OK
    assert n.value < 18 << 30                              # 16 bytes a token, 65536 chunks of two partial rows


def test_nothing_to_do_is_ok():
    assert embed(rows=0, ids=None, y=None) == B.NT_OK
    assert embed_backward(vocab=0, dtable=None) == B.NT_OK
    assert embed_backward(rows=0, acc=1, ids=None, dy=None, ws=None, ws_bytes=0) == B.NT_OK
    a = window_args(q_layout=host([0, 0]), kv_layout=host([0, 0]))
    assert status("nt_window_attention", C.byref(a), None) == B.NT_ERR_INVALID_ARG      # host-only layout, checked first


BACKWARD = [
    (dict(kv_lengths=P), "takes no kv_lengths"), (dict(lse=None), "needs the forward's lse"),
    (dict(dout=None), "dout is NULL"), (dict(dout=P + 8), "dout must be 16-byte"), (dict(ld_dout=120), "dout's row stride"),
    (dict(dq=None), "dq is NULL"), (dict(dq=P + 8), "dq must be 16-byte"), (dict(ld_dq=127), "dq's row stride"),
    (dict(dk=None), "dk is NULL"), (dict(dk=4 * P + 4), "dk must be 16-byte"), (dict(ld_dk=60), "dk's row stride"),
    (dict(dv=None), "dv is NULL"), (dict(dv=5 * P + 2), "dv must be 16-byte"), (dict(ld_dv=68), "dv's row stride"),
    (dict(dq=P), "must not alias the operands"), (dict(dk=2 * P), "must not alias the operands"),
    (dict(dv=P), "must not alias the operands"), (dict(dk=3 * P), "must not alias one another"),
    (dict(dv=3 * P), "must not alias one another"), (dict(dv=4 * P), "must not alias one another"),
]


@pytest.mark.parametrize("kw,words", BACKWARD)
def test_window_backward_names_the_operand(kw, words):
    """Every operand of the backward is looked at before the layouts' device."""
    assert status("nt_window_attention_backward", C.byref(window_args(**kw)), None) == B.NT_ERR_INVALID_ARG
    assert words in error()


def test_window_forward_names_the_lengths():
    assert status("nt_window_attention", C.byref(window_args(kv_lengths=P + 2)), None) == B.NT_ERR_INVALID_ARG
    assert "kv_lengths" in error()


@pytest.mark.parametrize("n,m,left,right,sinks", [(1, 32000, 1023, 0, 0), (1, 32000, 1023, 1, 0), (1, 32000, 1023, 1, 4),
                                                  (3, 32000, 500, 40, 2), (5, 30000, 900, 5, 0)])
def test_a_window_past_the_last_query_keeps_the_plan_small(n, m, left, right, sinks):
    """A bound `right` that no query needs (right >= N) leaves the window of `left`
    keys: a few queries over a long cache are not cut, and need no partial sums."""
    a = window_args(q_layout=host([n]), kv_layout=host([m]), heads=12, kv_heads=12, head_dim=64, left=left, right=right,
                    sinks=sinks)
    bytes_ = C.c_uint64(77)
    assert status("nt_window_attention_workspace", C.byref(a), C.byref(bytes_)) == B.NT_OK
    assert bytes_.value == 0


def test_all_keys_of_a_long_cache_are_cut():
    """The same without a window on the left: 500 tiles for one block of rows."""
    bytes_ = C.c_uint64()
    for left in (-1, 32000):
        a = window_args(q_layout=host([1]), kv_layout=host([32000]), heads=12, kv_heads=12, head_dim=64, left=left, right=1,
                        sinks=0)
        assert status("nt_window_attention_workspace", C.byref(a), C.byref(bytes_)) == B.NT_OK
        assert bytes_.value >= 2 * 12 * (64 + 2) * 4


@pytest.mark.parametrize("head_dim", [0, -8])
def test_the_default_scale_leaves_a_bad_head_dim_to_the_library(head_dim):
    lay = host([5])
    a = B._window_args(lay, 4, head_dim, None, 2, -1, 0, 0, None, B.NT_BF16)
    assert status("nt_window_attention", C.byref(a), None) == B.NT_ERR_INVALID_ARG and "head_dim" in error()
    assert B._window_args(lay, 4, 64, None, 2, -1, 0, 0, None, B.NT_BF16).scale == 0.125


def test_embedding_gradient_has_no_border_at_powers_of_two():
    """Chunks and tiles change where both sides were measured, not next to a round
    number of tokens: one token more never changes the workspace by a hundredth."""
    def need(rows):
        n = C.c_uint64()
        assert status("nt_embedding_backward_workspace", rows, 30000, 64, C.byref(n)) == B.NT_OK
        return n.value
    for p in range(15, 24):
        a, b, c = (need((1 << p) + x) for x in (-1, 0, 1))
        assert abs(b - a) < 0.01 * a and abs(c - b) < 0.01 * b, p
