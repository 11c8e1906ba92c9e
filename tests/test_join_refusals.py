"""The C entry points of the join refuse bad arguments before anything is queued (no GPU needed: the addresses are never
followed)."""
import ctypes as C

import pytest

from paper_2605_04711_b200 import binding as B

P = 1 << 20                       # a 256-byte aligned address that nothing reads


def _e(**kw):
    d = {n: 0 for n, _ in B.JoinForm._fields_} | dict(dim=16, kind=1, stream_dtype=1, branch_dtype=0, grad_dtype=0, eps=1e-6, scale=1.0) | kw
    return B.JoinForm(*[d[n] for n, _ in B.JoinForm._fields_])


def _join(e, **kw):
    a = dict(x=P, f=P << 1, post_w=P << 2, post_b=P << 3, gate=P << 4, pre_w=P << 5, pre_b=P << 6, rows=4, y=P << 7, h=P << 8) | kw
    return B._lib.baoc_join(e, *a.values(), None)


def _grad(e, **kw):
    a = dict(y=P, f=P << 1, dy=P << 2, dh=P << 3, post_w=P << 4, post_b=P << 5, gate=P << 6, pre_w=P << 7, rows=4, dx=P << 8, df=P << 9, dpost_w=P << 10,
             dpost_b=P << 11, dgate=P << 12, dpre_w=P << 13, dpre_b=P << 14, ws=P << 15, ws_bytes=1 << 20) | kw
    return B._lib.baoc_join_grad(e, *a.values(), None)


@pytest.mark.parametrize("kw", [dict(dim=0), dict(dim=8193), dict(kind=2), dict(stream_dtype=2), dict(branch_dtype=-1), dict(grad_dtype=3), dict(eps=0.0),
                                dict(eps=float("inf")), dict(scale=float("nan")), dict(rows_per_gate=-1), dict(x_stride=15), dict(h_stride=(1 << 28) + 1),
                                dict(stream_dtype=0, branch_dtype=1)])
def test_descriptors(kw):
    e, n = C.byref(_e(**kw)), C.c_size_t()
    assert _join(e) == B.E_INVALID and _grad(e) == B.E_INVALID
    assert B._lib.baoc_join_grad_workspace_bytes(e, 4, C.byref(n)) == B.E_INVALID
    assert b"baoc_join_grad_workspace_bytes" in B._lib.baoc_join_last_error()


def test_join_arguments():
    e = C.byref(_e())
    assert _join(None) == B.E_INVALID and _join(e, rows=-1) == B.E_INVALID and _join(e, rows=(1 << 31) + 1) == B.E_INVALID
    for k in ("f", "pre_w", "y", "h", "post_w"):                        # (the last: a bias without its weight)
        assert _join(e, **{k: None}) == B.E_INVALID
    assert _join(C.byref(_e(kind=0))) == B.E_INVALID                    # biases of RMS norms
    for k in ("x", "f", "post_w", "post_b", "gate", "pre_w", "pre_b", "y", "h"):
        assert _join(e, **{k: (P << 10) + 1}) == B.E_ALIGN
    for kw in (dict(y=P + 64), dict(y=(P << 1) + 32), dict(h=(P << 1) + 32), dict(h=P), dict(h=(P << 7) + 16)):
        assert _join(e, **kw) == B.E_INVALID
    assert _join(C.byref(_e(x_stride=32)), y=P) == B.E_INVALID          # the same array at another stride
    assert _join(e, x=None, f=None, pre_w=None, y=None, h=None, rows=0) == B.OK


def test_grad_arguments():
    e, n = C.byref(_e()), C.c_size_t()
    assert _grad(None) == B.E_INVALID and _grad(e, rows=-1) == B.E_INVALID
    for k in ("y", "f", "dh", "pre_w", "df", "ws", "post_w", "gate"):
        assert _grad(e, **{k: None}) == B.E_INVALID
    for k in ("y", "f", "dy", "dh", "post_w", "post_b", "gate", "pre_w", "dx", "df"):
        assert _grad(e, **{k: (P << 20) + 1}) == B.E_ALIGN
    for k in ("dpost_w", "dpost_b", "dgate", "dpre_w", "dpre_b"):
        assert _grad(e, **{k: (P << 20) + 1}) == B.E_ALIGN
    assert _grad(e, ws=(P << 15) + 128) == B.E_ALIGN
    for kw in (dict(dx=P), dict(dx=(P << 2) + 64), dict(df=(P << 3) + 32), dict(df=P << 1), dict(dx=P << 3), dict(df=(P << 8) + 64)):
        assert _grad(e, **kw) == B.E_INVALID
    assert B._lib.baoc_join_grad_workspace_bytes(e, 4, None) == B.E_INVALID
    assert B._lib.baoc_join_grad_workspace_bytes(e, 4, C.byref(n)) == B.OK
    assert _grad(e, ws_bytes=n.value - 1) == B.E_WORKSPACE
    assert b"workspace too small" in B._lib.baoc_join_last_error()
    for kw in (dict(dy_stride=15), dict(df_stride=(1 << 28) + 1)):
        assert _grad(C.byref(_e(**kw))) == B.E_INVALID


def test_plans():
    for kw in (dict(dim=0), dict(dim=8193), dict(dim=8, kind="batch"), dict(dim=8, eps=0.0), dict(dim=8, scale=float("inf"))):
        with pytest.raises(B.BaocError):
            B.Join(**kw)


def test_groups_longer_than_the_rows():
    """A gate for more rows than there are, however many, is one gate: the descriptor is taken."""
    n = C.c_size_t()
    for rows_per_gate in (4, 5, 1 << 31, 1 << 32, (1 << 63) - 1):
        assert B._lib.baoc_join_grad_workspace_bytes(C.byref(_e(rows_per_gate=rows_per_gate)), 4, C.byref(n)) == B.OK


@pytest.mark.parametrize("dim", [1, 200, 256, 257, 512, 513, 768, 769, 2048, 8192])
def test_a_workspace_serves_fewer_rows(dim):
    """The size never falls as rows rise (rows around every change of how they are spread)."""
    n, last = C.c_size_t(), 0
    for rows in [0, 1, 2, 3, 4, 5, 147, 148, 149, 295, 296, 297, 443, 444, 445, 591, 592, 593, 596, 597, 740, 888, 1184, 1185, 1776, 2368, 2369, 5000, 1 << 20, 1 << 31]:
        assert B._lib.baoc_join_grad_workspace_bytes(C.byref(_e(dim=dim)), rows, C.byref(n)) == B.OK
        assert n.value >= last
        last = n.value


VECTORS = ("post_w", "post_b", "gate", "pre_w", "pre_b")


@pytest.mark.parametrize("v", VECTORS)
def test_outputs_that_lie_on_a_vector(v):
    """A row of another CTA would be normed by what one has written: 4 rows of 16 columns, 256 bytes of y and 128 of h."""
    e = C.byref(_e())
    for out, size in (("y", 256), ("h", 128)):
        for off in (0, 60, size - 4, -60):
            assert _join(e, **{v: P << 9, out: (P << 9) - off // 4 * 4}) == B.E_INVALID
    assert b"overlap" in B._lib.baoc_join_last_error()


def test_gates_that_an_output_lies_on():
    """Every group's gate counts: 2 rows a gate are 2 gates of 64 bytes, one a gate are 4."""
    for per, gates in ((2, 2), (1, 4), (3, 2)):
        e = C.byref(_e(rows_per_gate=per))
        assert _join(e, y=(P << 4) + 64 * gates - 64) == B.E_INVALID and _grad(e, dx=(P << 6) + 64 * gates - 64) == B.E_INVALID
        assert _grad(e, dpre_w=(P << 12) + 32 * gates - 32) == B.E_INVALID


SUMS = ("dpost_w", "dpost_b", "dgate", "dpre_w", "dpre_b")


@pytest.mark.parametrize("out", SUMS)
def test_column_sums_that_lie_on_another_array(out):
    e = C.byref(_e())
    for at in (P, (P << 1) + 96, (P << 2) + 224, P << 3, P << 4, P << 5, (P << 6) + 32, P << 7, P << 8, (P << 9) + 96, (P << 15) + 256):
        assert _grad(e, **{out: at}) == B.E_INVALID
        assert b"overlap" in B._lib.baoc_join_last_error()
    for other in SUMS:
        if other != out:
            assert _grad(e, **{out: P << 20, other: (P << 20) + 16}) == B.E_INVALID


def test_a_workspace_that_lies_on_another_array():
    e = C.byref(_e())
    for at in (P, P << 1, P << 2, P << 3, P << 4, P << 5, P << 6, P << 7, P << 8, P << 9):
        assert _grad(e, ws=at) == B.E_INVALID
    for at in (P, P << 2):
        assert _grad(e, ws=at - 256) == B.E_INVALID


def test_a_gate_for_its_own_gradient():
    e = C.byref(_e(grad_dtype=1, rows_per_gate=2))
    assert _grad(e, dgate=P << 6) == B.E_INVALID and b"overlap" in B._lib.baoc_join_last_error()
