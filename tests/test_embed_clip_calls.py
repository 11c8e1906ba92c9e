"""What a program may count on from the token table's and the clip's calls, without a GPU."""
import ctypes as C

import pytest
import torch

from paper_2605_04711_b200 import binding as B


def _workspace(vocab, dim, tokens):
    e, n = B.Embed(vocab, dim, 1, 0, 0, 64, 1.0, -1, 0, 0, 0), C.c_size_t()
    assert B._lib.baoc_embed_grad_workspace_bytes(C.byref(e), tokens, C.byref(n)) == B.OK
    return n.value


@pytest.mark.parametrize("vocab,dim", [(1, 8), (300, 256), (4096, 2048), (32000, 128), (32000, 2048), (50257, 64), (50257, 512), (50257, 768),
                                       (98304, 256), (98305, 256), (128256, 64), (131072, 4096), (600000, 1), (600000, 16384)])
def test_a_workspace_serves_every_smaller_batch(vocab, dim):
    """The size never falls as the number of tokens grows: every count up to 3000, then steps that are odd and below the
    distance at which the tables' sizes move by their alignment."""
    last = 0
    for n in list(range(3000)) + list(range(3001, 300000, 37)) + [1 << 20, (1 << 20) + 1, 1 << 27, 1 << 30]:
        size = _workspace(vocab, dim, n)
        assert size >= last, n
        last = size


# ---- devices: tensors of several GPUs stood in for by what the calls look at --------------------------------------------
class _OnDevice:
    """A contiguous array of some GPU as the binding sees one."""

    def __init__(self, device, numel, dtype, address=1 << 20):
        self.device_index, self.n, self.dtype, self.address = device, numel, dtype, address
        self.is_cuda = True

    def get_device(self):
        return self.device_index

    def numel(self):
        return self.n

    def element_size(self):
        return {torch.uint8: 1, torch.bfloat16: 2, torch.float32: 4}[self.dtype]

    def data_ptr(self):
        return self.address

    def is_contiguous(self):
        return True


@pytest.fixture
def queued(monkeypatch):
    """Calls that would be queued, as (device, entry point)."""
    log = []

    def queue(device, call, *args):
        log.append((device, call))
        return B.OK
    monkeypatch.setattr(B, "_queue", queue)
    monkeypatch.setattr(B, "_stream", lambda: pytest.fail("queued on whatever device is current"))
    return log


def test_a_clip_workspace_is_bound_on_its_own_device(queued):
    h = B.Baoc([(64, 8, 8), (5, 5, 1)], B.default_configs())
    h.bind_clip_workspace(_OnDevice(1, h.clip_workspace_bytes(), torch.uint8))
    assert queued == [(1, B._lib.baoc_bind_clip_workspace)]


def test_a_clip_workspace_is_contiguous_device_memory(queued):
    h = B.Baoc([(64, 8, 8), (5, 5, 1)], B.default_configs())
    with pytest.raises(B.BaocError) as err:
        h.bind_clip_workspace(torch.empty(h.clip_workspace_bytes(), dtype=torch.uint8))
    assert err.value.code == B.E_INVALID and queued == []


def test_clip_arrays_are_on_the_workspaces_device(queued):
    h = B.Baoc([(64, 8, 8), (5, 5, 1)], B.default_configs())
    h.bind_clip_workspace(_OnDevice(1, h.clip_workspace_bytes(), torch.uint8))
    del queued[:]
    arrays = lambda *devices: [_OnDevice(d, n, torch.bfloat16) for d, n in zip(devices, (64, 5))]
    here, there = _OnDevice(1, 3, torch.float32), _OnDevice(0, 3, torch.float32)
    for call in (lambda: h.grad_norm(arrays(1, 1), there), lambda: h.grad_norm(arrays(1, 0), here), lambda: h.grad_norm(arrays(0, 0), here),
                 lambda: h.grad_norm(arrays(0, 0), there), lambda: h.clip_grads(arrays(1, 1), arrays(0, 1), 1.0, here),
                 lambda: h.clip_grads(arrays(1, 1), None, 1.0, there)):
        with pytest.raises(B.BaocError) as err:
            call()
        assert err.value.code == B.E_INVALID and queued == []
    h.grad_norm(arrays(1, 1), here)
    h.clip_grads(arrays(1, 1), arrays(1, 1), 1.0, here)
    assert queued == [(1, B._lib.baoc_grad_norm), (1, B._lib.baoc_clip_grads)]


def test_binding_the_same_workspace_again_keeps_one_reference(queued):
    h = B.Baoc([(64, 8, 8), (5, 5, 1)], B.default_configs())
    ws = _OnDevice(0, h.clip_workspace_bytes(), torch.uint8)
    for _ in range(3):
        h.bind_clip_workspace(ws)
    assert sum(k is ws for k in h._keep) == 1


# ---- shapes -------------------------------------------------------------------------------------------------------------
def test_ids_and_rows_that_do_not_belong_together_are_refused():
    """As many rows as ids are not enough: [30, 3] ids and rows [3, 30] pair up wrongly."""
    e = B.Embedding(10, 8)
    table = torch.zeros(10, 8)
    for ids_shape, lead in (((30, 3), (3, 30)), ((2, 3, 5), (2, 5, 3)), ((6, 1), (2, 3))):
        ids, rows = torch.zeros(ids_shape, dtype=torch.int64), torch.zeros(*lead, 8)
        for call in (lambda: e.lookup(table, ids, out=rows), lambda: e.grad(ids, rows, table)):
            with pytest.raises(B.BaocError, match="shape") as err:
                call()
            assert err.value.code == B.E_INVALID


@pytest.mark.parametrize("ids_shape,lead", [((6,), (6,)), ((2, 3), (2, 3)), ((2, 3), (6,)), ((6,), (2, 3)), ((), ()), ((), (1,)), ((1, 6), (6,)),
                                            ((0, 3), (0, 3))])
def test_ids_and_rows_that_belong_together_are_queued(queued, monkeypatch, ids_shape, lead):
    """Equal leading shapes, or one of the two in a row."""
    e = B.Embedding(10, 8)
    monkeypatch.setattr(torch.Tensor, "get_device", lambda t: 0)
    ids, rows, table = torch.zeros(ids_shape, dtype=torch.int64), torch.zeros(*lead, 8), torch.zeros(10, 8)
    assert e.lookup(table, ids, out=rows) is rows
    assert e.grad(ids, rows, table, ws=torch.zeros(e.grad_workspace_bytes(6), dtype=torch.uint8)) is table
    assert queued == [(0, B._lib.baoc_embed), (0, B._lib.baoc_embed_grad)]


def test_a_refused_call_leaves_the_plan_as_it_was(monkeypatch):
    """A row stride above 2^28 is refused by the library; what comes after the refusal is not refused for it."""
    e, other = B.Embedding(2, 8), B.Embedding(2, 8)
    monkeypatch.setattr(torch.Tensor, "get_device", lambda t: 0)
    monkeypatch.setattr(B, "_queue", lambda device, call, *args: call(*args, None))
    stride = (1 << 28) + 1
    wide = torch.empty(stride + 8, device="meta").as_strided((2, 8), (stride, 1))
    ids, rows, ws = torch.zeros(2, dtype=torch.int64), torch.zeros(2, 8), torch.zeros(1 << 20, dtype=torch.uint8)
    for call in (lambda: e.lookup(wide, ids, out=rows), lambda: e.lookup(torch.zeros(2, 8), ids, out=wide), lambda: e.grad(ids, wide, rows, ws=ws),
                 lambda: e.grad(ids, rows, wide, ws=ws)):
        for _ in range(2):
            with pytest.raises(B.BaocError, match="row stride") as err:
                call()
            assert err.value.code == B.E_INVALID
        assert e.grad_workspace_bytes(1000) == other.grad_workspace_bytes(1000)


def test_a_lookup_that_autograd_would_lose_is_refused(queued, monkeypatch):
    """The output carries no history: a table that requires a gradient would silently get none."""
    monkeypatch.setattr(torch.Tensor, "get_device", lambda t: 0)
    e, ids, rows = B.Embedding(10, 8), torch.zeros(4, dtype=torch.int64), torch.zeros(4, 8)
    table = torch.zeros(10, 8, requires_grad=True)
    with pytest.raises(B.BaocError, match="detach") as err:
        e.lookup(table, ids, out=rows)
    assert err.value.code == B.E_INVALID and queued == []
    e.lookup(table.detach(), ids, out=rows)
    with torch.no_grad():
        e.lookup(table, ids, out=rows)
    assert len(queued) == 2
