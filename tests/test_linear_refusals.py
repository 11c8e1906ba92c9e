"""The C entry points of the matrix product refuse bad arguments before anything is queued (no GPU needed: the addresses are
never followed)."""
import ctypes as C

import pytest

from paper_2605_04711_b200 import binding as B

P = 1 << 20                       # a 256-byte aligned address that nothing reads


def _e(**kw):
    d = {n: 0 for n, _ in B.LinearForm._fields_} | dict(n_in=16, n_out=24, act=1) | kw
    return B.LinearForm(*[d[n] for n, _ in B.LinearForm._fields_])


def _product(e, **kw):
    a = dict(x=P, w=P << 1, bias=P << 2, residual=P << 3, tokens=4, out=P << 4, pre=P << 5, ws=None, ws_bytes=0) | kw
    return B._lib.baoc_linear(e, *a.values(), None)


def _grad(e, **kw):
    a = dict(x=P, w=P << 1, dout=P << 2, pre=P << 3, tokens=4, dx=P << 4, dw=P << 5, db=P << 6, ws=P << 7, ws_bytes=1 << 16) | kw
    return B._lib.baoc_linear_grad(e, *a.values(), None)


@pytest.mark.parametrize("kw", [dict(n_in=0), dict(n_out=(1 << 24) + 1), dict(act=5), dict(act=-1), dict(layout=2), dict(out_dtype=2), dict(grad_dtype=-1),
                                dict(x_stride=15), dict(w_stride=15), dict(layout=1, w_stride=20), dict(out_stride=23), dict(residual_stride=(1 << 28) + 1),
                                dict(dw_stride=-16), dict(dx_stride=15), dict(pre_stride=23), dict(dout_stride=23)])
def test_descriptors(kw):
    e, n = C.byref(_e(**kw)), C.c_size_t()
    assert _product(e) == B.E_INVALID and _grad(e) == B.E_INVALID
    assert B._lib.baoc_linear_workspace_bytes(e, 4, 0, C.byref(n)) == B.E_INVALID
    assert B._lib.baoc_linear_grad_workspace_bytes(e, 4, 0, C.byref(n)) == B.E_INVALID
    assert b"baoc_linear_grad_workspace_bytes" in B._lib.baoc_linear_last_error()


def test_product_arguments():
    e = C.byref(_e())
    assert _product(None) == B.E_INVALID and _product(e, tokens=-1) == B.E_INVALID and _product(e, tokens=(1 << 30) + 1) == B.E_INVALID
    for k in ("x", "w", "out"):
        assert _product(e, **{k: None}) == B.E_INVALID
    for k in ("x", "w", "bias", "residual", "out", "pre"):
        assert _product(e, **{k: (P << 12) + 1}) == B.E_ALIGN
    for kw in (dict(out=P), dict(out=(P << 1) + 16), dict(out=(P << 3) + 16), dict(pre=P), dict(pre=P << 4), dict(pre=P << 3), dict(ws=None, ws_bytes=64),
               dict(ws=P, ws_bytes=256)):
        assert _product(e, **kw) == B.E_INVALID
    assert _product(C.byref(_e(out_stride=32)), out=P << 3) == B.E_INVALID       # the residual at another stride
    assert _product(e, ws=(P << 8) + 16, ws_bytes=256) == B.E_ALIGN
    assert _product(e, x=P + 2) == B.E_WORKSPACE                                 # has to be laid out first
    assert _product(C.byref(_e(n_in=17)), ws=P << 8, ws_bytes=1000) == B.E_WORKSPACE
    assert b"workspace too small" in B._lib.baoc_linear_last_error()
    assert _product(e, x=None, w=None, out=None, tokens=0) == B.OK


def test_grad_arguments():
    e, n = C.byref(_e()), C.c_size_t()
    assert _grad(None) == B.E_INVALID and _grad(e, tokens=-1) == B.E_INVALID and _grad(e, tokens=(1 << 30) + 1) == B.E_INVALID
    for k in ("x", "w", "dout", "pre", "ws"):
        assert _grad(e, **{k: None}) == B.E_INVALID
    for k in ("x", "w", "dout", "pre", "dx", "dw", "db"):
        assert _grad(e, **{k: (P << 12) + 1}) == B.E_ALIGN
    assert _grad(e, ws=(P << 7) + 64) == B.E_ALIGN
    for kw in (dict(dx=P), dict(dx=P << 5), dict(dw=P << 1), dict(db=(P << 5) + 8), dict(dw=P << 7), dict(db=P << 2), dict(ws=P << 3)):
        assert _grad(e, **kw) == B.E_INVALID
    size = B._lib.baoc_linear_grad_workspace_bytes
    assert size(e, 4, 0, None) == B.E_INVALID and B._lib.baoc_linear_workspace_bytes(e, 4, 0, None) == B.E_INVALID
    for kw in (dict(), dict(grad_dtype=1), dict(n_in=17), dict(n_out=25), dict(act=0)):
        d = C.byref(_e(**kw))
        assert size(d, 4, 0, C.byref(n)) == B.OK and n.value > 0
        assert _grad(d, ws_bytes=n.value - 1) == B.E_WORKSPACE
        small = n.value
        assert size(d, 4, 1, C.byref(n)) == B.OK and n.value >= small


def test_plans():
    for kw in (dict(n_in=0, n_out=4), dict(n_in=4, n_out=1 << 25), dict(n_in=4, n_out=4, act="tanh"), dict(n_in=4, n_out=4, layout="nk")):
        with pytest.raises(B.BaocError):
            B.Linear(**kw)
    assert B.Linear(64, 128).workspace_bytes(1000) == 0 and B.Linear(65, 128).workspace_bytes(1000) > 0


def test_outputs_that_lie_on_the_bias():
    """4 rows of 24 columns, 192 bytes of out and pre; 96 bytes of bias."""
    e = C.byref(_e())
    for out in ("out", "pre"):
        for off in (0, 92, -188):
            assert _product(e, **{out: (P << 2) + off}) == B.E_INVALID and b"overlap" in B._lib.baoc_linear_last_error()
    assert _product(e, bias=(P << 8) + 4096, ws=P << 8, ws_bytes=8192) == B.E_INVALID
