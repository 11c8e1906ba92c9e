"""The C entry points of the log probabilities refuse bad arguments before anything is queued (no GPU needed: the addresses
are never followed)."""
import ctypes as C

import pytest

from paper_2605_04711_b200 import binding as B

P = 1 << 20                       # a 256-byte aligned address that nothing reads


def _e(**kw):
    d = dict(vocab=100, dtype=0, id_bits=64, scale=1.0, top=2, stride=0, grad_stride=0) | kw
    return B.Logp(*[d[n] for n, _ in B.Logp._fields_])


@pytest.mark.parametrize("kw", [dict(vocab=0), dict(vocab=1 << 31), dict(dtype=2), dict(id_bits=16), dict(scale=0.0), dict(scale=-1.0),
                                dict(scale=float("inf")), dict(scale=float("nan")), dict(top=-1), dict(top=33), dict(vocab=3, top=4),
                                dict(stride=99), dict(grad_stride=-100), dict(stride=(1 << 32) + 1)])
def test_descriptors(kw):
    e = C.byref(_e(**kw))
    assert B._lib.baoc_logp(e, P, P, 4, P, P, P, P, P, None) == B.E_INVALID
    assert B._lib.baoc_logp_grad(e, P, P, P, P, None, 4, P << 4, None) == B.E_INVALID
    assert b"baoc_logp_grad" in B._lib.baoc_logp_last_error()


def test_arguments():
    e, f, g = C.byref(_e()), B._lib.baoc_logp, B._lib.baoc_logp_grad
    good = [P, P << 1, 4, P << 2, P << 3, P << 4, P << 5, P << 6]
    assert f(None, *good, None) == B.E_INVALID
    for i in (0, 1, 3, 4, 5, 6, 7):
        assert f(e, *(None if j == i else a for j, a in enumerate(good)), None) == B.E_INVALID
        assert f(e, *(a + 1 if j == i else a for j, a in enumerate(good)), None) == B.E_ALIGN
    for n in (-1, 1 << 31):
        assert f(e, *good[:2], n, *good[3:], None) == B.E_INVALID
    assert f(e, None, None, 0, *([None] * 5), None) == B.OK
    good = [P, P << 1, P << 2, P << 3, P << 4, 4, P << 5]
    assert g(None, *good, None) == B.E_INVALID
    for i in (0, 1, 2, 3, 6):
        assert g(e, *(None if j == i else a for j, a in enumerate(good)), None) == B.E_INVALID
    for i in (0, 1, 2, 3, 4, 6):
        assert g(e, *(a + 1 if j == i else a for j, a in enumerate(good)), None) == B.E_ALIGN
    for d in (P + 2, P + 200, P - 2):                                   # inside the logits, but not the logits
        assert g(e, *good[:6], d, None) == B.E_INVALID
    assert g(C.byref(_e(stride=128)), *good[:6], P, None) == B.E_INVALID    # the same array at another stride
    assert g(e, *good[:5], 1 << 31, P << 5, None) == B.E_INVALID
    assert g(e, None, None, None, None, None, 0, None, None) == B.OK


def test_plans():
    for kw in (dict(vocab=0), dict(vocab=10, top=11), dict(vocab=10, scale=0.0), dict(vocab=1 << 31), dict(vocab=10, top=-1)):
        with pytest.raises(B.BaocError):
            B.LogProbs(**kw)


def test_outputs_that_lie_on_another_array():
    """4 rows of 100 bf16 logits (800 bytes), 32 bytes of ids, 16 of logp and entropy, 48 of stats, 32 of each of the alternatives."""
    e, f = C.byref(_e()), B._lib.baoc_logp
    good = [P, P << 1, 4, P << 2, P << 3, P << 4, P << 5, P << 6]
    for i in (3, 4, 5, 6, 7):
        for at in [P, P + 796, P << 1, (P << 1) + 28] + [a for j, a in enumerate(good) if j > 2 and j != i]:
            assert f(e, *(at if j == i else a for j, a in enumerate(good)), None) == B.E_INVALID
            assert b"overlaps" in B._lib.baoc_logp_last_error()


def test_gradients_that_lie_on_another_array():
    e, g = C.byref(_e()), B._lib.baoc_logp_grad
    good = [P, P << 1, P << 2, P << 3, P << 4, 4, P << 5]
    for i, size in ((1, 32), (2, 48), (3, 16), (4, 16)):
        for at in (good[i], good[i] + size - 4, good[i] - 796):
            assert g(e, *good[:6], at, None) == B.E_INVALID and b"overlaps" in B._lib.baoc_logp_last_error()
    wide = C.byref(_e(stride=128, grad_stride=128))                     # 256 bytes from row to row, 200 of them logits
    for at in (P + 192, P + 216, P - 4):                                # (48 bytes of stats: from 200 to 208 on they would lie in a gap)
        assert g(wide, P, P << 1, at, P << 3, P << 4, 4, P, None) == B.E_INVALID


@pytest.mark.parametrize("name", ["logits", "dlogp", "dentropy", "dlogits"])
def test_gradients_that_autograd_would_lose(name):
    """Like the other plans: what requires a gradient is refused while gradients are on (before the devices are looked at)."""
    import torch
    t = dict(logits=torch.zeros(4, 10), ids=torch.zeros(4, dtype=torch.int64), stats=torch.zeros(4, 3), dlogp=torch.zeros(4), dentropy=torch.zeros(4), dlogits=torch.zeros(4, 10))
    t[name].requires_grad_(True)
    with pytest.raises(B.BaocError, match="autograd does not see.*detach " + name):
        B.LogProbs(10).grad(**t)
    for call in (dict(t), t | {name: t[name].detach()}):
        with torch.no_grad(), pytest.raises(B.BaocError, match="CUDA device"):
            B.LogProbs(10).grad(**call)


def test_scales_that_leave_the_numbers():
    """Above 2^127 the scale in base 2 is infinite, and every row was NaN."""
    for scale in (2.4e38, 3.4e38):
        e = C.byref(_e(scale=scale))
        assert B._lib.baoc_logp(e, None, None, 0, None, None, None, None, None, None) == B.E_INVALID
        assert B._lib.baoc_logp_grad(e, None, None, None, None, None, 0, None, None) == B.E_INVALID
        with pytest.raises(B.BaocError, match="2\\^127"):
            B.LogProbs(10, scale=scale)
    for scale in (2.0 ** 127, 1e-45):
        B.LogProbs(10, scale=scale)
