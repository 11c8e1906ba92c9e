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
