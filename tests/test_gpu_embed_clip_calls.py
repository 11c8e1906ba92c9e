"""The token table's and the clip's calls as a program makes them one after another: workspaces that are kept, plans that
have refused a call, captures, devices."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2605_04711_b200 import binding
    return binding


@pytest.fixture(scope="module")
def G():
    from paper_2605_04711_b200 import harness
    return harness


def _integers(shape, seed, most=3):
    """Small whole numbers: their sums are exact in fp32 in every order."""
    g = torch.Generator().manual_seed(seed)
    return torch.randint(-most, most + 1, shape, generator=g).float()


@pytest.mark.parametrize("vocab,dim,largest,batches", [(32000, 128, 81700, (81000, 40000, 300)), (50257, 64, 63500, (63000, 257)),
                                                       (50257, 512, 6530, (6400, 6529, 1))])
def test_one_workspace_for_the_largest_batch(B, G, vocab, dim, largest, batches):
    e = B.Embedding(vocab, dim)
    guard, ws = G.guarded_alloc(e.grad_workspace_bytes(largest), "cuda:0")
    for n in (largest, *batches):
        ids = torch.randint(0, vocab, (n,), generator=torch.Generator().manual_seed(n))
        dout = _integers((n, dim), n)
        d = torch.full((vocab, dim), float("nan"), device="cuda:0")
        e.grad(ids.to("cuda:0"), dout.to("cuda:0"), d, ws=ws)
        assert torch.equal(d.cpu(), torch.zeros(vocab, dim).index_add_(0, ids, dout))
    assert G.guards_intact(guard)


def test_a_clip_workspace_is_not_bound_in_a_capture(B):
    """Refused before anything is queued; the capture goes on and the handle works afterwards."""
    h = B.Baoc([(64, 8, 8), (5, 5, 1)], B.default_configs())
    ws = torch.empty(h.clip_workspace_bytes(), dtype=torch.uint8, device="cuda:0")
    gs, norms = [torch.full((64,), 2.0, device="cuda:0"), torch.ones(5, device="cuda:0")], torch.zeros(3, device="cuda:0")
    x, graph = torch.zeros(4, device="cuda:0"), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        x.add_(1)
        with pytest.raises(B.BaocError) as err:
            h.bind_clip_workspace(ws)
    assert err.value.code == B.E_STATE
    graph.replay()
    assert bool((x == 1).all())
    with pytest.raises(B.BaocError) as err:
        h.grad_norm(gs, norms)
    assert err.value.code == B.E_STATE
    h.bind_clip_workspace(ws)
    with torch.cuda.graph(graph := torch.cuda.CUDAGraph()):
        h.grad_norm(gs, norms)
    graph.replay()
    assert norms[1] == 16.0 and abs(float(norms[2]) - 5.0 ** 0.5) < 1e-6


def test_a_sessions_first_clip_is_not_captured(B, G):
    from paper_2605_04711_b200 import workloads as W
    sess = G.Session(W.Workload("clip_capture", [W.Block("w", 16, 8), W.Block("b", 5, 1)], window=2, mem_budget_frac=1.0, time_budget=2.0, seed=0))
    sess.grads[0].fill_(1.0)
    graph = torch.cuda.CUDAGraph()
    x = torch.zeros(4, device="cuda:0")
    with torch.cuda.graph(graph):
        x.add_(1)
        with pytest.raises(B.BaocError) as err:
            sess.clip_grads(0, 1.0)
    assert err.value.code == B.E_STATE
    norm = sess.clip_grads(0, 100.0)[0]
    assert abs(float(norm) - 133.0 ** 0.5) < 1e-5
    with torch.cuda.graph(graph := torch.cuda.CUDAGraph()):
        sess.clip_grads(0, 100.0)
    sess.grads[0].fill_(2.0)
    graph.replay()
    assert abs(float(sess.clip_norms[0]) - 2 * 133.0 ** 0.5) < 1e-5
