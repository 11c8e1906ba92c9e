"""Norm, clip and table gradient at the sizes where large models run them: shares of many rounds, the clip's long tiles, more
segments than the joint finish stages, warps with more tokens than a list entry can address.

Whole numbers first: their squares and sums are exact in fp32 and in double, so every norm is the correctly rounded root of
an integer and every gradient an integer.  An element that is left out or counted twice shows whatever its place.

Real numbers, with u = 2^-24.  A thread sums the squares of four 16-byte words in four fp32 sums: chains of 8 (bf16) or 4
(fp32) multiply-adds, then two additions, all of non-negative terms, so a round is off by at most (8 + 2) u; doubles from
there on.  The root halves that: 5 u before the norm's one rounding to fp32.  The clip factor adds its own rounding, 6 u, and
the product is rounded once to the output type (bf16: once to fp32 first).  Rounding is monotone, so an output has to lie
between the rounded ends of the interval that the errors before it allow; 0.1 u covers the second-order terms, the doubles
and the factor's 1e-6."""
import os
import subprocess
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
NORM, CLIP = 5.1 * U, 6.1 * U
BF, F = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def B():
    from paper_2605_04711_b200 import binding
    return binding


@pytest.fixture(scope="module")
def G():
    from paper_2605_04711_b200 import harness
    return harness


def _gen(seed):
    return torch.Generator(device="cuda:0").manual_seed(seed)


def _handle(B, sizes):
    h = B.Baoc([(n, n, 1) for n in sizes], B.default_configs())
    h.bind_clip_workspace(torch.empty(h.clip_workspace_bytes(), dtype=torch.uint8, device="cuda:0"))
    return h


def _views(flat, sizes, step=8):
    """The blocks in one array, each starting at a multiple of 16 bytes."""
    out, at = [], 0
    for n in sizes:
        out.append(flat[at:at + n])
        at += (n + step - 1) // step * step
    return out


def _length(sizes, step=8):
    return sum((n + step - 1) // step * step for n in sizes)


def _whole(sizes, dtype, seed):
    flat = torch.randint(0, 4, (_length(sizes),), generator=_gen(seed), device="cuda:0").to(dtype)
    return _views(flat, sizes)


def _normal(sizes, dtype, seed):
    """Blocks of different scales."""
    flat = torch.empty(_length(sizes), device="cuda:0").normal_(0.0, 1.0, generator=_gen(seed))
    views = _views(flat, sizes)
    for i, v in enumerate(views):
        v *= 10.0 ** (i % 4 - 2)
    return _views(flat.to(dtype), sizes)


def _sum_squares(gs):
    return torch.stack([g.double().square().sum() for g in gs])


def _want(gs):
    sq = _sum_squares(gs)
    return torch.cat([sq.sum()[None], sq]).sqrt()


def _within(got, want, rel):
    lo, hi = ((want + sign * rel * want.abs()).float().to(got.dtype).double() for sign in (-1.0, 1.0))
    low, high = torch.minimum(lo, hi), torch.maximum(lo, hi)
    bad = ~((got.double() >= low) & (got.double() <= high))
    assert not bool(bad.any()), (int(bad.sum()), float(((got.double() - want).abs() / want.abs().clamp(min=1e-300)).max()) / U)


MANY = [1 + (7 * i) % 50 for i in range(5000)]
SIZES = {"one": [20_000_003], "mixed": [8193, 12_000_005, 1, 16384, 9_000_000, 77], "many": MANY, "many_and_large": MANY[:2500] + [20_000_001] + MANY[2500:]}


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("sizes", SIZES.values(), ids=SIZES)
def test_norm_of_whole_numbers(B, sizes, dtype):
    h, gs = _handle(B, sizes), _whole(sizes, dtype, 1)
    norms = torch.full((1 + len(sizes),), -1.0, device="cuda:0")
    h.grad_norm(gs, norms)
    assert torch.equal(norms, _want(gs).float())


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("sizes", SIZES.values(), ids=SIZES)
def test_norm(B, sizes, dtype):
    h, gs = _handle(B, sizes), _normal(sizes, dtype, 2)
    norms = torch.full((1 + len(sizes),), -1.0, device="cuda:0")
    h.grad_norm(gs, norms)
    _within(norms, _want(gs), NORM)


@pytest.mark.parametrize("sizes", [[1], [7, 8, 9], [255, 4096, 16385, 100003], [300] * 700, [3_000_000]])
@pytest.mark.parametrize("dtype", [BF, F])
def test_norm_of_smaller_blocks(B, sizes, dtype):
    h, gs = _handle(B, sizes), _normal(sizes, dtype, 3)
    norms = torch.empty(1 + len(sizes), device="cuda:0")
    h.grad_norm(gs, norms)
    _within(norms, _want(gs), NORM)


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("spike", [1e25, 3e36, 1e-12])
def test_norm_with_a_value_outside_the_fp32_squares_in_any_round(B, dtype, spike):
    """The value stands in the first, a middle and a last round of shares, and in the tail; what surrounds it is 20 orders
    of magnitude smaller, so nothing but the value's own square makes the norm."""
    n = 20_000_003
    h, g, norms = _handle(B, [n]), torch.full((n,), spike * 1e-20, device="cuda:0").to(dtype), torch.empty(2, device="cuda:0")
    rest = g[0].clone()
    for at in (0, 8191, 8192, 3 * 8192 + 17, 4 * 8192 - 1, 4 * 8192, 9_999_999, 12_345_678, n - 8193, n - 20, n - 4, n - 1):
        g[at] = spike
        h.grad_norm([g], norms)
        want = (g[at].double().square() + (n - 1) * rest.double().square()).sqrt()
        _within(norms, want.expand(2), NORM)
        g[at] = rest


# 2^25 elements and more: the clip's long tiles
LONG = [(1 << 25) + 5, 3 * 16384 + 1, 7, 100_003]


@pytest.mark.parametrize("src,dst", [(BF, BF), (F, F), (F, BF)])
@pytest.mark.parametrize("max_norm", [0.5, 1e9])
def test_clip(B, G, src, dst, max_norm):
    h, gs = _handle(B, LONG), _normal(LONG, src, 4)
    nb = 2 if dst == BF else 4
    guard, flat = G.guarded_alloc(_length(LONG) * nb, "cuda:0")
    flat.fill_(0xFF)
    outs = _views(flat.view(dst), LONG)
    norms = torch.empty(1 + len(LONG), device="cuda:0")
    before = [g.clone() for g in gs]
    h.clip_grads(gs, outs, max_norm, norms)
    want = _want(gs)
    _within(norms, want, NORM)
    factor = (max_norm / (want[0] + 1e-6)).clamp(max=1.0)
    for g, b, o in zip(gs, before, outs):
        assert torch.equal(g, b)
        if factor == 1.0:
            assert torch.equal(o, g.to(dst))
        else:
            _within(o, g.double() * factor, CLIP)
    if src == dst:
        h.clip_grads(gs, None, max_norm, norms)
        assert all(torch.equal(g, o) for g, o in zip(gs, outs))
    assert G.guards_intact(guard)


def test_clip_of_smaller_blocks(B):
    sizes = [255, 8, 16385, 1, 100_003]
    for src, dst in ((BF, BF), (F, F), (F, BF)):
        h, gs = _handle(B, sizes), _normal(sizes, src, 5)
        outs = [torch.empty(n, dtype=dst, device="cuda:0") for n in sizes]
        norms = torch.empty(1 + len(sizes), device="cuda:0")
        h.clip_grads(gs, outs, 0.25, norms)
        factor = 0.25 / (_want(gs)[0] + 1e-6)
        for g, o in zip(gs, outs):
            _within(o, g.double() * factor, CLIP)


@pytest.mark.parametrize("kind", ["uniform", "half_alike"])
def test_gradient_of_more_tokens_than_a_list_entry_addresses(B, kind):
    """70 M tokens: a warp's stretch of the grouping is longer than 2^19, so its lists hold no offsets and every id is read
    again."""
    n, vocab, dim = 70_000_003, 1000, 2
    gen = _gen(6)
    ids = torch.randint(-1, vocab, (n,), generator=gen, device="cuda:0", dtype=torch.int32)
    if kind == "half_alike":
        ids[torch.rand(n, generator=gen, device="cuda:0") < 0.5] = 389
    dout = torch.randint(-1, 2, (n, dim), generator=gen, device="cuda:0").to(BF)
    d = torch.full((vocab, dim), float("nan"), device="cuda:0")
    B.Embedding(vocab, dim, pad_id=7).grad(ids, dout, d)
    kept = (ids >= 0) & (ids != 7)
    want = torch.zeros((vocab, dim), dtype=torch.float64, device="cuda:0").index_add_(0, ids[kept].long(), dout[kept].double())
    assert torch.equal(d.double(), want)


def test_these_cases_run_clean_under_the_checked_build():
    """The same cases, and those of the calls one after another, on the library whose kernels validate their tables first."""
    from paper_2605_04711_b200 import build
    if os.environ.get("BAOC_CHECKED") == "1":
        return                                                          # this is the child
    build.build(checked=True)
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-m", "pytest", "tests/test_gpu_embed_clip_sizes.py", "tests/test_gpu_embed_clip_calls.py", "-m", "gpu", "-x", "-q"],
                       cwd=root, env=dict(os.environ, BAOC_CHECKED="1"), capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr[-2000:]
    assert " passed" in r.stdout and "failed" not in r.stdout
