"""The C entry points of the token table and of the clip refuse bad arguments before anything is queued (no GPU needed: the
addresses are never followed)."""
import ctypes as C

import pytest

from paper_2605_04711_b200 import binding as B

P = 1 << 20                       # a 256-byte aligned address that nothing reads


def _e(**kw):
    d = dict(vocab=100, dim=16, table_dtype=1, act_dtype=0, grad_dtype=0, id_bits=64, scale=1.0, pad_id=-1, table_stride=0,
             act_stride=0, grad_stride=0) | kw
    return B.Embed(*[d[n] for n, _ in B.Embed._fields_])


BAD = [dict(vocab=0), dict(vocab=1 << 31), dict(dim=0), dict(dim=(1 << 24) + 1), dict(table_dtype=2), dict(act_dtype=-1),
       dict(grad_dtype=7), dict(id_bits=16), dict(scale=float("inf")), dict(scale=float("nan")), dict(pad_id=-2), dict(pad_id=100),
       dict(table_stride=15), dict(act_stride=-16), dict(grad_stride=(1 << 28) + 1)]


@pytest.mark.parametrize("kw", BAD)
def test_descriptors(kw):
    e, n = _e(**kw), C.c_size_t()
    assert B._lib.baoc_embed(C.byref(e), P, P << 1, 4, P << 2, None) == B.E_INVALID
    assert B._lib.baoc_embed_grad(C.byref(e), P, P << 1, 4, P << 2, 0, P << 3, 1 << 20, None) == B.E_INVALID
    assert B._lib.baoc_embed_grad_workspace_bytes(C.byref(e), 4, C.byref(n)) == B.E_INVALID
    assert b"baoc_embed_grad_workspace_bytes" in B._lib.baoc_embed_last_error()


def test_embed_arguments():
    e = C.byref(_e())
    f = B._lib.baoc_embed
    assert f(None, P, P << 1, 4, P << 2, None) == B.E_INVALID
    for args in ((None, P, 4, P), (P, None, 4, P), (P, P, 4, None), (P, P << 1, -1, P << 2), (P, P << 1, 1 << 41, P << 2),
                 (P, P << 1, 4, P + 64)):                               # the last: out inside the table
        assert f(e, *args, None) == B.E_INVALID
    for args in ((P + 2, P, 4, P << 2), (P, P + 4, 4, P << 2), (P, P << 1, 4, (P << 2) + 1)):
        assert f(e, *args, None) == B.E_ALIGN
    assert f(e, None, None, 0, None, None) == B.OK                      # no tokens: nothing to do


def test_grad_arguments():
    d, n = _e(), C.c_size_t()
    e = C.byref(d)
    size = B._lib.baoc_embed_grad_workspace_bytes
    assert size(e, 1000, None) == B.E_INVALID and size(e, -1, C.byref(n)) == B.E_INVALID
    assert size(e, (1 << 30) + 1, C.byref(n)) == B.E_INVALID and size(e, 1000, C.byref(n)) == B.OK
    need, f = n.value, B._lib.baoc_embed_grad
    assert 0 < need < 1 << 22
    W = P << 6
    for args in ((None, P, 1000, P << 2, 0, W, need), (P, None, 1000, P << 2, 0, W, need), (P, P << 1, 1000, None, 0, W, need),
                 (P, P << 1, 1000, P << 2, 0, None, need), (P, P << 1, -1, P << 2, 0, W, need), (P, P << 1, (1 << 30) + 1, P << 2, 0, W, need),
                 (P, P << 1, 1000, (P << 1) + 32, 0, W, need), (P, P << 1, 1000, W + 32, 0, W, need)):
        assert f(e, *args, None) == B.E_INVALID
    for args in ((P + 4, P << 1, 1000, P << 2, 0, W, need), (P, (P << 1) + 1, 1000, P << 2, 0, W, need),
                 (P, P << 1, 1000, (P << 2) + 1, 0, W, need), (P, P << 1, 1000, P << 2, 0, W + 128, need)):
        assert f(e, *args, None) == B.E_ALIGN
    assert f(e, P, P << 1, 1000, P << 2, 0, W, need - 1, None) == B.E_WORKSPACE
    assert b"workspace too small" in B._lib.baoc_embed_last_error()


def test_clip_arguments():
    h = B.Baoc([(64, 8, 8), (5, 5, 1)], B.default_configs())
    L = B._lib
    assert L.baoc_clip_workspace_bytes(None, C.byref(C.c_size_t())) == B.E_INVALID and L.baoc_clip_workspace_bytes(h._h, None) == B.E_INVALID
    need = h.clip_workspace_bytes()
    assert L.baoc_bind_clip_workspace(None, P, need, None) == B.E_INVALID and L.baoc_bind_clip_workspace(h._h, None, need, None) == B.E_INVALID
    assert L.baoc_bind_clip_workspace(h._h, P + 16, need, None) == B.E_ALIGN
    assert L.baoc_bind_clip_workspace(h._h, P, need - 1, None) == B.E_WORKSPACE
    tab = (C.c_void_p * 2)(P, P + 1024)
    assert L.baoc_grad_norm(None, tab, 0, P, None) == B.E_INVALID and L.baoc_grad_norm(h._h, None, 0, P, None) == B.E_INVALID
    assert L.baoc_grad_norm(h._h, tab, 0, None, None) == B.E_INVALID and L.baoc_grad_norm(h._h, tab, 2, P, None) == B.E_INVALID
    assert L.baoc_grad_norm(h._h, tab, 0, P + 2, None) == B.E_ALIGN
    assert L.baoc_grad_norm(h._h, tab, 0, P, None) == B.E_STATE
    assert "no clip workspace" in h.last_error()
    assert L.baoc_clip_grads(None, tab, 0, tab, 0, 1.0, P, None) == B.E_INVALID
    assert L.baoc_clip_grads(h._h, tab, 0, tab, 0, 1.0, P, None) == B.E_STATE


def test_workspace_covers_every_vocabulary():
    """The grouping's tables: at least one start per row of the table and one more, and a place per token."""
    n = C.c_size_t()
    for vocab in (1, 2, 127, 128, 129, 50257, 131072, 131073, 10 ** 6, (1 << 31) - 1):
        for tokens in (0, 1, 1000):
            assert B._lib.baoc_embed_grad_workspace_bytes(C.byref(_e(vocab=vocab)), tokens, C.byref(n)) == B.OK
            assert n.value >= 4 * (vocab + 1) + 4 * tokens
