"""Log probabilities of given tokens, entropy, most probable tokens and the logits' gradient, against plain 64-bit forms.

With u = 2^-24, t the scaled distance of a logit to the row's largest and n the longest chain of additions of one thread:
  * e^t: the distance, its scaling and the scale in base 2 are rounded (3 u |t|), the exponential is off by at most 4 u;
  * S: n additions, a rescaling by such an exponential per 32 of them at most, 16 joins of two sums: (1.3 n + 100) u, and
    what the terms are off by, 3 u times the mean of |t|, which is below log S + H;
  * log S is off by S's relative error and 2 u |log S|; logp by that, 3 u |t| and a rounding; H by log S's error and twice S's
    relative error of the second sum, which is at most H;
  * p of the gradient: 4 u (|t| + log S + 2) relative; a gradient by that of its terms, and four roundings.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U, SUB = 2.0 ** -24, 2.0 ** -126
BF, F = torch.bfloat16, torch.float32
INF = float("inf")


@pytest.fixture(scope="module")
def B():
    from paper_2605_04711_b200 import binding
    return binding


def _within(got, want, tol):
    lo, hi = ((want + sign * (tol + SUB)).float().to(got.dtype).double() for sign in (-1.0, 1.0))
    g = got.double().cpu()
    same = (g == want) | (torch.isnan(g) & torch.isnan(want))
    bad = ~(((g >= lo) & (g <= hi)) | same)
    assert not bool(bad.any()), (int(bad.sum()), g[bad][:4], want[bad][:4])


def _logits(n, v, dtype, seed, spread=3.0):
    g = torch.Generator().manual_seed(seed)
    return (spread * torch.randn((n, v), generator=g)).to(dtype)


def _want(x, ids, scale, top):
    """(logp, entropy, log S, largest, top ids, top logp, log q) in 64 bits of rows of finite logits or -inf, ids inside."""
    z = x.double() * float(torch.tensor(scale, dtype=F))
    m = z.max(1, keepdim=True)[0]
    logq = torch.log_softmax(z, 1)
    q = logq.exp()
    h = -torch.where(q > 0, q * logq, 0.0).sum(1)
    ti = torch.sort(x.float(), dim=1, descending=True, stable=True)[1][:, :top]
    return logq.gather(1, ids[:, None].long())[:, 0], h, torch.logsumexp(z, 1) - m[:, 0], ti, logq.gather(1, ti), logq


def _tolerance(v, logs, h, t):
    chain = 1.3 * (math.ceil(v / 256) + 16) + 100
    s = U * (chain + 3 * (logs + h))
    return s + U * (2 * logs.abs() + 4 * t.abs()), 3 * s + U * (4 * logs.abs() + 4 * h)


def _check(B, x, ids, scale, top, view=None):
    plan = B.LogProbs(x.shape[1], scale=scale, top=top)
    out = plan.logprobs(x.to("cuda:0") if view is None else view, ids.to("cuda:0"))
    logp, h, logs, ti, tl, _ = _want(x, ids, scale, top)
    tol, tol_h = _tolerance(x.shape[1], logs, h, torch.where(torch.isinf(logp), 0.0, logp))
    _within(out.logp, logp, tol)
    _within(out.entropy, h, tol_h)
    _within(out.stats[:, 1], logs, tol)
    assert torch.equal(out.stats[:, 0].cpu(), x.float().max(1)[0]) and torch.equal(out.stats[:, 2], out.entropy)
    if top:
        assert torch.equal(out.top_ids.cpu().long(), ti)
        _within(out.top_logp, tl, tol[:, None] + U * 4 * torch.where(torch.isinf(tl), 0.0, tl.abs()))
    return out


@pytest.mark.parametrize("n,v", [(1, 1), (1, 2), (3, 3), (5, 7), (2, 40), (3, 255), (1, 4099), (300, 257), (1, 50257), (2, 32000), (20, 32771),
                                 (40, 16384), (100, 9001), (150, 8192), (300, 50257), (1, 131072), (4, 262144)])
@pytest.mark.parametrize("dtype,idt,scale,top", [(BF, torch.int64, 1.0, 5), (BF, torch.int32, 1.25, 32), (F, torch.int64, 0.7, 0), (F, torch.int32, 1.0, 20)])
def test_forward(B, n, v, dtype, idt, scale, top):
    x = _logits(n, v, dtype, n * 7 + v)
    ids = torch.randint(0, v, (n,), generator=torch.Generator().manual_seed(v)).to(idt)
    x[torch.arange(n), ids.long()] += torch.linspace(0, 12, n).to(dtype)          # some rows are sure of their token
    _check(B, x, ids, scale, min(top, v))


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("n,v", [(6, 5003), (200, 5003), (6, 50000)])
def test_shapes_of_rows(B, dtype, n, v):
    """Rows that are constant, rise, fall, are mostly masked, repeat few values, lie far from zero."""
    x = _logits(n, v, dtype, 3)
    x[0] = 1.5
    x[1] = torch.arange(v).float().div(v).to(dtype)
    x[2] = -torch.arange(v).float().div(v).to(dtype)
    x[3, torch.arange(v) % 997 != 5] = -INF
    x[4] = (torch.arange(v) % 3).to(dtype)
    x[5] = x[5] + 3.0e4
    x[5, 17] = torch.finfo(dtype).min                                              # a mask of the type's lowest value
    ids = torch.randint(0, v, (n,), generator=torch.Generator().manual_seed(4))
    for top in (1, 7, 32):
        _check(B, x, ids, 1.0, top)


def test_few_threads_hold_the_largest(B):
    """Thousands of logits above the 32nd of the threads' largest: the threads' elements are counted instead of listed."""
    n, v = 150, 131072
    x = torch.full((n, v), -5.0, dtype=BF)
    vec = torch.arange(v) // 8 % 256
    g = torch.Generator().manual_seed(8)
    x[:, vec < 31] = (10 + 6 * torch.rand((n, int((vec < 31).sum())), generator=g)).to(BF)
    x[:, vec == 31] = 9.0
    x[1, vec < 31] = 12.0
    _check(B, x, torch.randint(0, v, (n,), generator=g), 1.0, 32)


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("v", [9, 300, 40000])
def test_rows_without_a_value(B, dtype, v):
    """Nothing but -inf; the type's lowest value throughout; infinities; NaN; ignored ids."""
    lowest = torch.finfo(dtype).min
    x = _logits(8, v, dtype, 5)
    x[0] = -INF
    x[1] = lowest
    x[2, v // 2] = INF
    x[3, v // 3] = float("nan")
    x[4], x[5] = float("nan"), float("nan")                                        # not read: the ids are outside
    ids = torch.tensor([1, 2, 3, 4, -1, v, 0, 5], dtype=torch.int64)
    x[6, 0] = -INF                                                                 # the given token cannot follow
    plan = B.LogProbs(v, top=3)
    d = x.to("cuda:0")
    out = plan.logprobs(d, ids.to("cuda:0"))
    logp, h, ti, tl = out.logp.cpu(), out.entropy.cpu(), out.top_ids.cpu(), out.top_logp.cpu()
    assert logp[0] == -INF and h[0] == 0 and ti[0].tolist() == [0, 1, 2] and bool((tl[0] == -INF).all())
    assert abs(float(logp[1]) + math.log(v)) <= 1e-5 and abs(float(h[1]) - math.log(v)) <= 1e-5 and ti[1].tolist() == [0, 1, 2]
    assert math.isnan(logp[2]) and math.isnan(h[2]) and ti[2, 0] == v // 2
    assert math.isnan(logp[3]) and math.isnan(h[3]) and ti[3, 0] == v // 3
    assert bool((logp[4:6] == 0).all()) and bool((h[4:6] == 0).all()) and bool((ti[4:6] == -1).all()) and bool((tl[4:6] == 0).all())
    assert logp[6] == -INF and float(h[6]) > 0
    one = torch.ones(8, device="cuda:0")
    g = plan.grad(d, ids.to("cuda:0"), out.stats, one, 0.5 * one).cpu().float()
    assert bool((g[0] == 0).all()) and bool((g[4:6] == 0).all())
    assert bool(torch.isnan(g[2]).any()) and bool(torch.isnan(g[3]).all())
    assert bool(torch.isfinite(g[[1, 6, 7]]).all())


def _want_grad(x, ids, scale, g, h, stats):
    s = float(torch.tensor(scale, dtype=F))
    x64, ok = x.double(), (ids >= 0) & (ids < x.shape[1])
    st = stats.double()
    logq = (x64 - st[:, :1]) * s - st[:, 1:2]
    q = logq.exp()
    ent = torch.where(q > 0, q * (logq + st[:, 2:]), 0.0)
    d = -g.double()[:, None] * q - h.double()[:, None] * ent
    mag = g.double().abs()[:, None] * q + h.double().abs()[:, None] * torch.where(q > 0, q * (logq.abs() + st[:, 2:]), 0.0)
    eps = U * 4 * (torch.where(q > 0, (x64 - st[:, :1]).abs() * s, 0.0) + st[:, 1:2].abs() + 4)
    tol = mag * (eps + 4 * U) + (h.double().abs()[:, None] * q) * U * 4 * (torch.where(q > 0, logq.abs(), 0.0) + st[:, 2:])
    rows = torch.nonzero(ok).flatten()
    d[rows, ids[rows].long()] += g.double()[rows]
    tol = tol + U * (d.abs() + mag) * 3
    return torch.where(ok[:, None], d * s, 0.0), torch.where(ok[:, None], tol * s, 0.0)


@pytest.mark.parametrize("n,v", [(1, 1), (3, 2), (5, 7), (1, 4099), (300, 257), (33, 32000), (7, 50257), (2, 131072)])
@pytest.mark.parametrize("dtype,scale,entropy", [(BF, 1.0, True), (BF, 1.25, False), (F, 0.5, True), (F, 1.0, False)])
def test_grad(B, n, v, dtype, scale, entropy):
    x = _logits(n, v, dtype, n + v)
    gen = torch.Generator().manual_seed(v)
    ids = torch.randint(0, v, (n,), generator=gen)
    if n > 2:
        ids[1] = -1
    if v > 100:
        x[0, ::3] = -INF
        x[0, ids[0]] = 2.0
    g, h = torch.randn(n, generator=gen), 0.3 * torch.randn(n, generator=gen) if entropy else torch.zeros(n)
    z = x.double() * float(torch.tensor(scale, dtype=F))
    q = torch.softmax(z, 1)
    stats = torch.stack([x.float().max(1)[0].double(), torch.logsumexp(z, 1) - z.max(1)[0], torch.special.entr(q).sum(1)], 1).float()
    want, tol = _want_grad(x, ids, scale, g, h, stats)
    plan, d, dev = B.LogProbs(v, scale=scale), x.to("cuda:0"), "cuda:0"
    args = (ids.to(dev), stats.to(dev), g.to(dev), h.to(dev) if entropy else None)
    got = plan.grad(d, *args)
    assert got.dtype == dtype
    _within(got, want, tol)
    again = d.clone()
    plan.grad(again, *args, dlogits=again)                                         # in place: the same bits
    assert torch.equal(again, got)
    for left, width in ((1, v + 3), (8, v + 16)):                                  # rows in a wider buffer, in and out unlike
        wide = torch.full((n, width), 7.0, dtype=dtype, device=dev)
        plan.grad(d, *args, dlogits=wide[:, left:left + v])
        assert torch.equal(wide[:, left:left + v], got) and bool((wide[:, :left] == 7).all()) and bool((wide[:, left + v:] == 7).all())


def test_grad_against_differences(B):
    """The gradient of sum(g logp + h H), by differences of the 64-bit form."""
    n, v, scale = 3, 50, 1.3
    x = _logits(n, v, F, 1, 1.5)
    ids = torch.tensor([4, 49, 0])
    g, h = torch.tensor([0.7, -1.2, 0.3]), torch.tensor([0.4, 0.1, -0.8])
    s = float(torch.tensor(scale, dtype=F))

    def value(z):
        q = torch.log_softmax(z * s, 1)
        return float((g.double() * q.gather(1, ids[:, None])[:, 0] - h.double() * (q.exp() * q).sum(1)).sum())

    plan, dev = B.LogProbs(v, scale=scale), "cuda:0"
    out = plan.logprobs(x.to(dev), ids.to(dev))
    got = plan.grad(x.to(dev), ids.to(dev), out.stats, g.to(dev), h.to(dev)).cpu().double()
    step = 1e-5                        # third derivatives of order 1: the difference is off by about 1e-10 / 6
    for i in range(n):
        for j in range(0, v, 7):
            e = torch.zeros_like(x, dtype=torch.float64)
            e[i, j] = step
            assert abs((value(x.double() + e) - value(x.double() - e)) / (2 * step) - float(got[i, j])) <= 2e-6


def test_strides_shapes_and_offsets(B):
    x, dev = _logits(24, 301, BF, 9), "cuda:0"
    ids = torch.randint(0, 301, (4, 6), generator=torch.Generator().manual_seed(1))
    plain = _check(B, x, ids.reshape(-1), 1.0, 4)
    out = B.LogProbs(301, top=4).logprobs(x.to(dev).view(4, 6, 301), ids.to(dev))
    assert tuple(out.top_ids.shape) == (4, 6, 4) and tuple(out.stats.shape) == (4, 6, 3)
    assert torch.equal(out.logp.view(-1), plain.logp) and torch.equal(out.top_ids.view(-1, 4), plain.top_ids)
    for left, width in ((0, 304), (1, 333), (3, 308), (8, 320)):
        wide = torch.full((24, width), float("nan"), dtype=BF, device=dev)
        wide[:, left:left + 301] = x.to(dev)
        _check(B, x, ids.reshape(-1), 1.0, 4, view=wide[:, left:left + 301])


def test_long_offsets(B):
    """Rows whose bytes start beyond 32 bits."""
    n, v, dev = 90000, 32000, "cuda:0"
    x = torch.zeros((n, v), dtype=BF, device=dev)                                   # 5.8 GB
    last = _logits(2, v, BF, 2)
    x[n - 2:] = last.to(dev)
    ids = torch.arange(n, device=dev) % v
    plan = B.LogProbs(v, top=2)
    out = plan.logprobs(x, ids)
    logp, h, logs, ti, _, _ = _want(last, ids[n - 2:].cpu(), 1.0, 2)
    tol, _ = _tolerance(v, logs, h, logp)
    _within(out.logp[n - 2:], logp, tol)
    assert torch.equal(out.top_ids[n - 2:].cpu().long(), ti) and abs(float(out.logp[7]) + math.log(v)) < 1e-5
    plan.grad(x, ids, out.stats, torch.ones(n, device=dev), dlogits=x)
    p = torch.softmax(last.double(), 1)
    p[torch.arange(2), ids[n - 2:].cpu()] -= 1
    _within(x[n - 2:], -p, (p.abs() + 1e-3) * U * 200)


def test_same_bits_in_a_graph_and_on_another_stream(B):
    x, dev = _logits(5, 50257, BF, 3).to("cuda:0"), "cuda:0"
    ids = torch.arange(5, device=dev)
    plan = B.LogProbs(50257, top=20)
    want = plan.logprobs(x, ids)
    one = torch.ones(5, device=dev)
    wg = plan.grad(x, ids, want.stats, one, one)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = plan.logprobs(x, ids)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    buf, grad = plan.buffers(5, dev), torch.empty_like(x)
    with torch.cuda.graph(graph := torch.cuda.CUDAGraph()):
        plan.logprobs(x, ids, out=buf)
        plan.grad(x, ids, buf.stats, one, one, dlogits=grad)
    graph.replay()
    assert all(torch.equal(a, b) for a, b in zip(buf, want)) and torch.equal(grad, wg)


def test_refusals(B):
    dev = "cuda:0"
    x, ids = torch.zeros((4, 10), device=dev), torch.zeros(4, dtype=torch.int64, device=dev)
    plan = B.LogProbs(10, top=2)
    for bad in (lambda: plan.logprobs(x[:, :9], ids), lambda: plan.logprobs(x, ids[:3]), lambda: plan.logprobs(x.half(), ids),
                lambda: plan.logprobs(x, ids.float()), lambda: plan.logprobs(x.cpu(), ids), lambda: plan.logprobs(x, ids.cpu()),
                lambda: plan.logprobs(x, ids, out=plan.buffers(3, dev)), lambda: plan.logprobs(x, ids, out=B.LogProbs(10).buffers(4, dev)),
                lambda: plan.logprobs(x.t().contiguous().t(), ids), lambda: plan.logprobs(x.clone().requires_grad_(True), ids),
                lambda: plan.grad(x, ids, torch.zeros(4, 2, device=dev), torch.zeros(4, device=dev)),
                lambda: plan.grad(x, ids, torch.zeros(4, 3, device=dev), torch.zeros(4, device=dev, dtype=torch.float64)),
                lambda: plan.grad(x, ids, torch.zeros(4, 3, device=dev), torch.zeros(4, device=dev), dlogits=x.bfloat16())):
        with pytest.raises(B.BaocError):
            bad()
    out = plan.logprobs(x, ids)                                                     # the plan works on
    assert out.top_ids.tolist() == [[0, 1]] * 4
    wide = torch.zeros(100, device=dev)
    with pytest.raises(B.BaocError, match="overlaps"):
        plan.grad(wide[:40].view(4, 10), ids, out.stats, torch.zeros(4, device=dev), dlogits=wide[10:50].view(4, 10))
    both = torch.zeros((4, 20), device=dev)                                         # side by side in one buffer is no overlap
    plan.grad(both[:, :10], ids, out.stats, torch.ones(4, device=dev), dlogits=both[:, 10:])
    empty = plan.logprobs(x[:0], ids[:0])
    assert empty.logp.numel() == 0 and plan.grad(x[:0], ids[:0], empty.stats, empty.logp).numel() == 0


def test_outputs_that_are_not_there(B):
    dev = "cuda:0"
    x, ids, plan = torch.zeros((4, 10), device=dev), torch.zeros(4, dtype=torch.int64, device=dev), B.LogProbs(10)
    for name in ("logp", "entropy", "stats"):
        with pytest.raises(B.BaocError):
            plan.logprobs(x, ids, out=plan.buffers(4, dev)._replace(**{name: None}))


@pytest.mark.parametrize("dtype", [BF, F])
def test_scales_at_their_ends(B, dtype):
    """All of the probability with the largest logits, or the same for every token."""
    dev = "cuda:0"
    x = torch.tensor([[0.0, 1.0, 1.0, -INF, 0.99]], device=dev).to(dtype)
    ids = torch.tensor([1], device=dev)
    cold, hot = B.LogProbs(5, scale=2.0 ** 127, top=3), B.LogProbs(5, scale=2.0 ** -149, top=3)
    for plan, kept in ((cold, 2), (hot, 4)):
        out = plan.logprobs(x, ids)
        assert abs(float(out.logp) + math.log(kept)) <= 1e-6 and abs(float(out.entropy) - math.log(kept)) <= 1e-6 and out.top_ids.tolist() == [[1, 2, 4]]
        one = torch.ones(1, device=dev)
        assert bool(torch.isfinite(plan.grad(x, ids, out.stats, one)).all())
