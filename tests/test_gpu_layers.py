"""The operators between the token table and the loss as a model runs them together: the residual model of the examples, forwards
and backwards, eagerly and as a captured graph."""
import importlib.util
import math
import os
import subprocess
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
DEV = "cuda:0"


@pytest.fixture(scope="module")
def lm():
    spec = importlib.util.spec_from_file_location("residual_lm", os.path.join(ROOT, "examples", "residual_lm.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def _setup(lm, seed=3):
    gen = torch.Generator().manual_seed(seed)
    p = {name: torch.empty(s, device=DEV) for name, s in lm.blocks()}
    lm.initialise(p, gen)
    for name, v in p.items():
        if v.dim() == 1:
            v.add_(0.2 * torch.randn(v.shape, generator=gen).to(DEV))
    ids = lm.sequences(gen)
    inputs, targets = ids[:, :-1].reshape(-1), ids[:, 1:].reshape(-1)
    return p, inputs, torch.where((inputs != lm.PAD) & (targets != lm.PAD), targets, -1)


def _reference(lm, p, ids, follow):
    """The same model in 64 bits with automatic differentiation, from the bf16 matrices."""
    q = {k: (v.to(torch.bfloat16).double() if v.dim() == 2 else v.double()).requires_grad_(True) for k, v in p.items()}
    rms = lambda v, w: v * torch.rsqrt(v.square().mean(1, keepdim=True) + 1e-6) * w
    table = q["table"]
    y = torch.where((ids != lm.PAD)[:, None], table[ids], table[ids].detach()) * lm.DIM ** 0.5       # the pad row takes no gradient here
    h = rms(y, q["pre.0"])
    for i in range(lm.LAYERS):
        f = torch.nn.functional.gelu(h @ q[f"w1.{i}"].t() + q[f"b1.{i}"]) @ q[f"w2.{i}"].t()
        y = y + q[f"gate.{i}"] * rms(f, q[f"post.{i}"])
        h = rms(y, q[f"pre.{i + 1}"])
    logp = torch.log_softmax(h @ table.t(), 1)
    kept = follow >= 0
    loss = -(logp.gather(1, follow.clamp(min=0)[:, None])[:, 0] * kept).sum() / kept.sum()
    loss.backward()
    return float(loss), {k: v.grad for k, v in q.items()}


def test_gradients_of_the_whole_model(lm):
    """Every rounding of an activation or of its gradient to bf16 adds at most 2^-8 of it; along the longest way, the embedding's,
    there are 4 roundings per block and 3 more forwards and as many backwards, 22 for two blocks.  Their effects on a whole
    gradient add up like independent ones or better (root of 22) but may be magnified by the blocks: a factor of 4 for that."""
    p, ids, follow = _setup(lm)
    g = {k: torch.full(v.shape, float("nan"), dtype=torch.bfloat16, device=DEV) for k, v in p.items()}
    loss = float(lm.Model().loss_and_gradients(p, g, ids, follow))
    want, grads = _reference(lm, p, ids, follow)
    assert abs(loss - want) <= 4 * math.sqrt(22) * 2 ** -8 * want
    for k, w in grads.items():
        err = float((g[k].double() - w).norm() / w.norm())
        assert err <= 4 * math.sqrt(22) * 2 ** -8, (k, err)


def test_captured_model(lm):
    """The whole model, forwards and backwards, in a graph, replayed on other inputs: the bits of the eager calls."""
    p, ids, follow = _setup(lm)
    model = lm.Model()
    new = lambda: {k: torch.zeros(v.shape, dtype=torch.bfloat16, device=DEV) for k, v in p.items()}
    g, at_ids, at_follow = new(), ids.clone(), follow.clone()
    model.loss_and_gradients(p, g, at_ids, at_follow)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph := torch.cuda.CUDAGraph()):
        loss = model.loss_and_gradients(p, g, at_ids, at_follow)
    for seed in (3, 4):
        _, ids, follow = _setup(lm, seed)
        want = new()
        eager = lm.Model().loss_and_gradients(p, want, ids, follow)
        at_ids.copy_(ids)
        at_follow.copy_(follow)
        for v in g.values():
            v.fill_(7)
        graph.replay()
        assert torch.equal(loss, eager) and all(torch.equal(g[k], want[k]) for k in want)


def test_two_models_on_two_streams(lm):
    """Two plans' calls that overlap on the GPU leave the bits of calls one after another."""
    sets = [_setup(lm, seed) for seed in (5, 6)]
    new = lambda p: {k: torch.zeros(v.shape, dtype=torch.bfloat16, device=DEV) for k, v in p.items()}
    want = [new(s[0]) for s in sets]
    for s, g in zip(sets, want):
        lm.Model().loss_and_gradients(s[0], g, *s[1:])
    torch.cuda.synchronize()
    got, streams, models = [new(s[0]) for s in sets], [torch.cuda.Stream() for _ in sets], [lm.Model() for _ in sets]
    torch.cuda.synchronize()
    for _ in range(5):
        for s, g, stream, m in zip(sets, got, streams, models):
            with torch.cuda.stream(stream):
                m.loss_and_gradients(s[0], g, *s[1:])
    torch.cuda.synchronize()
    assert all(torch.equal(a[k], b[k]) for a, b in zip(got, want) for k in a)


def test_example_runs(lm):
    losses, norms = lm.train(steps=4, window=3)
    assert len(losses) == 4 and all(math.isfinite(x) and x > 0 for x in losses + norms)


def test_gradients_run_clean_under_the_checked_build():
    """The join's cases on the library whose kernels validate their workspace ranges first."""
    from paper_2605_04711_b200 import build
    if os.environ.get("BAOC_CHECKED") == "1":
        return                                                          # this is the child
    build.build(checked=True)
    r = subprocess.run([sys.executable, "-m", "pytest", "tests/test_gpu_join.py", "-m", "gpu", "-x", "-q"], cwd=ROOT, env=dict(os.environ, BAOC_CHECKED="1"),
                       capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr[-2000:]
    assert " passed" in r.stdout and "failed" not in r.stdout
