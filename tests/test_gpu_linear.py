"""The matrix product with bias, activation and residual, and its gradient, against plain 64-bit forms.

Most operands are small whole numbers or dyadic fractions: every product and every sum of them is exact in fp32 in any order, so
that outputs have to be equal to the last bit (a bf16 output: to the rounded value).  Elsewhere, with u = 2^-24:
  * a sum of k products: 2 (k + 4) u of the sum of their sizes (additions in any order, truncated ones among them);
  * relu is exact; of z = -90 .. 90: silu (12 + 4 |z|) u relative, gelu (16 + 4 z^2) u (the argument of erfc is rounded twice and
    its relative slope is up to 2 z^2 there), gelu_tanh (16 + 10 |v|) u with v its exponent; derivatives the same of their terms'
    sizes.  The fast division returns 0 for divisors above 2^126: 2^-118 absolute (|z| e^-87).
  * dz is rounded to bf16: numbers in [1, 2) are 2^-7 apart, so a rounding is off by 2^-8 of the value; where what is left is
    rounded to bf16 twice more, by 2^-8 of at most 2^-16 of the value, 2^-24.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U, TINY = 2.0 ** -24, 2.0 ** -118
BF, F = torch.bfloat16, torch.float32
DEV = "cuda:0"
ACTS = ["none", "relu", "gelu", "gelu_tanh", "silu"]


@pytest.fixture(scope="module")
def B():
    from paper_2605_04711_b200 import binding
    return binding


@pytest.fixture(scope="module")
def G():
    from paper_2605_04711_b200 import harness
    return harness


@pytest.fixture(autouse=True)
def _no_wait_ran_out(B):
    yield
    assert B.linear_status() == 0


def _ints(shape, seed, most=3, dtype=BF):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return torch.randint(-most, most + 1, shape, generator=g, device=DEV).to(dtype)


def _rand(shape, seed, scale=1.0, dtype=BF):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return (scale * torch.randn(shape, generator=g, device=DEV)).to(dtype)


def _within(got, want, tol):
    lo, hi = ((want + s * tol).float().to(got.dtype).double() for s in (-1.0, 1.0))
    g = got.double()
    bad = ~((g >= lo) & (g <= hi))
    assert not bool(bad.any()), (int(bad.sum()), g[bad][:4], want[bad][:4], float(((g - want).abs() / (tol + 1e-300)).max()))


def _act(z, act):
    if act == "relu":
        return z.clamp(min=0.0)
    if act == "gelu":
        return 0.5 * z * torch.special.erfc(-z * math.sqrt(0.5))
    if act == "gelu_tanh":
        return z * torch.sigmoid(math.sqrt(8.0 / math.pi) * (z + 0.044715 * z ** 3))
    return z * torch.sigmoid(z) if act == "silu" else z


def _rel(z, act):
    if act == "silu":
        return (12 + 4 * z.abs()) * U
    if act == "gelu":
        return (16 + 4 * z * z) * U
    if act == "gelu_tanh":
        return (16 + 10 * 1.6 * (z + 0.044715 * z ** 3).abs()) * U
    return U * torch.ones_like(z)


def _slope(z, act):
    z = z.clone().requires_grad_(True)
    with torch.enable_grad():
        if act == "relu":
            return (z.detach() > 0).double()
        return torch.autograd.grad(_act(z, act).sum(), z)[0] if act != "none" else torch.ones_like(z)


def _slope_tol(z, act):
    if act in ("none", "relu"):
        return torch.zeros_like(z)
    phi = torch.exp(-0.5 * z * z)
    if act == "gelu":
        return (torch.special.erfc(-z * math.sqrt(0.5)) + z.abs() * phi) * (20 + 4 * z * z) * U
    v = math.sqrt(8.0 / math.pi) * (z + 0.044715 * z ** 3) if act == "gelu_tanh" else z
    s = torch.sigmoid(v)
    steep = v.abs() * 3 + z.abs()
    return (s + s * (1 - s) * steep) * (24 + 10 * v.abs()) * U + s * steep * 4 * U * (v > 0)


def _w(w, layout):
    return w if layout == "out_in" else w.t().contiguous()


SHAPES = [(1, 1, 1), (1, 64, 64), (1, 2048, 512), (3, 8, 5), (2, 65, 63), (7, 513, 1001), (128, 64, 256), (129, 128, 257), (100, 200, 300), (300, 1000, 96),
          (513, 96, 4099), (1000, 72, 136), (4, 8192, 2048), (1, 2048, 8192), (2048, 256, 4096), (4000, 520, 1000), (16384, 64, 768), (33, 4096, 33)]


@pytest.mark.parametrize("m,k,n", SHAPES)
@pytest.mark.parametrize("layout", ["out_in", "in_out"])
@pytest.mark.parametrize("dtype,bias,residual,pre,act", [(F, False, False, False, "none"), (BF, True, True, True, "relu"), (F, True, True, True, "relu")])
def test_exact_sums(B, m, k, n, layout, dtype, bias, residual, pre, act):
    x, w = _ints((m, k), 1), _ints((n, k), 2)
    b, r = (_ints((n,), 3, 9, F) if bias else None), (_ints((m, n), 4, 9, dtype) if residual else None)
    kept = torch.full((m, n), float("nan"), dtype=BF, device=DEV) if pre else None
    out = torch.full((m, n), float("nan"), dtype=dtype, device=DEV)
    B.Linear(k, n, act, layout).product(x, _w(w, layout), bias=b, residual=r, out=out, pre=kept)
    z = x.double() @ w.double().t() + (0 if b is None else b.double())
    want = _act(z, act) + (0 if r is None else r.double())
    assert torch.equal(out, want.to(dtype))
    if pre:
        assert torch.equal(kept, z.to(BF))


@pytest.mark.parametrize("m,k,n", SHAPES)
@pytest.mark.parametrize("layout", ["out_in", "in_out"])
@pytest.mark.parametrize("dtype,act", [(F, "none"), (BF, "relu"), (F, "relu")])
def test_exact_gradients(B, m, k, n, layout, dtype, act):
    x, w, dout = _ints((m, k), 1), _ints((n, k), 2), _ints((m, n), 5)
    pre = _ints((m, n), 6) if act != "none" else None
    dx = torch.full((m, k), float("nan"), dtype=BF, device=DEV)
    dw = torch.full_like(_w(w, layout), float("nan"), dtype=dtype)
    db = torch.full((n,), float("nan"), dtype=dtype, device=DEV)
    B.Linear(k, n, act, layout).grad(x, _w(w, layout), dout, pre=pre, dx=dx, dw=dw, db=db)
    dz = dout.double() * (1 if pre is None else (pre > 0).double())
    assert torch.equal(dx, (dz @ w.double()).to(BF))
    want = dz.t() @ x.double()
    assert torch.equal(dw, (want if layout == "out_in" else want.t()).to(dtype))
    assert torch.equal(db, dz.sum(0).to(dtype))


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("dtype", [F, BF])
def test_activations(B, act, dtype):
    """z runs over -90 .. 90 in fine steps: x holds it in three bf16 pieces."""
    m, n = 300, 257
    z = torch.cat([torch.linspace(-90, 90, 200 * n, dtype=torch.float64), torch.linspace(-6, 6, 100 * n, dtype=torch.float64)]).float().view(m, n).to(DEV)
    pieces, rest = [], z.clone()
    for _ in range(3):
        pieces.append(rest.to(BF))
        rest = rest - pieces[-1].float()
    assert float(rest.abs().max()) == 0.0
    # x = one-hot rows would need k = n; instead one output column at a time is a row of the batch
    x = torch.stack(pieces, -1).reshape(m * n, 3)
    w = torch.ones((1, 3), dtype=BF, device=DEV)
    out = B.Linear(3, 1, act).product(x, w, out_dtype=dtype)
    zd = z.double().reshape(-1, 1)
    want = _act(zd, act)
    sums = 2 * (3 + 4) * U * zd.abs() * _slope(zd, act).abs() * 1.01          # the sum of the pieces
    _within(out, want, want.abs() * _rel(zd, act) + sums + TINY)
    r = _ints((m * n, 1), 3, 5, dtype)
    _within(B.Linear(3, 1, act).product(x, w, residual=r, out_dtype=dtype), want + r.double(), want.abs() * _rel(zd, act) + sums + (want + r.double()).abs() * U + TINY)


@pytest.mark.parametrize("act", ACTS)
def test_activation_slopes(B, act):
    """One row: its column sums in fp32 are dz itself, before any rounding."""
    z = torch.linspace(-100, 100, 4001, dtype=torch.float64).to(BF).to(DEV).view(1, -1)
    z[0, :1000] = torch.linspace(-5, 5, 1000).to(BF)
    n = z.shape[1]
    dout = _rand((1, n), 1)
    db = torch.empty(n, device=DEV)
    B.Linear(8, n, act).grad(None, None, dout, pre=z if act != "none" else None, db=db)
    zd, d = z.double()[0], dout.double()[0]
    want = d * _slope(zd, act)
    _within(db, want, d.abs() * (_slope_tol(zd, act) + TINY) + want.abs() * U * 2)


def test_odd_activations(B):
    """Infinities and NaN before the activation; huge finite values."""
    z = torch.tensor([float("inf"), float("-inf"), float("nan"), 3e38, -3e38, 0.0, -0.0], device=DEV)
    x = torch.ones((1, 1), dtype=BF, device=DEV)
    w = z.to(BF).view(-1, 1)
    for act in ACTS:
        got = B.Linear(1, 7, act).product(x, w, out_dtype=F)[0]
        assert got[0] == float("inf") and math.isnan(got[2]) and float(got[3]) > 2.9e38
        assert bool((got[5:] == 0).all())
        if act == "none":
            assert float(got[4]) < -2.9e38
        else:
            assert float(got[4].abs()) <= 1e-30
        db = torch.empty(7, device=DEV)
        B.Linear(1, 7, act).grad(None, None, torch.ones((1, 7), dtype=BF, device=DEV), pre=w.view(1, -1) if act != "none" else None, db=db)
        assert float(db[0]) == 1.0 and float(db[3]) == 1.0
        if act != "none":
            assert float(db[1]) == 0.0 and float(db[4]) == 0.0 and math.isnan(db[2])


@pytest.mark.parametrize("m,k,n", [(1, 2048, 1000), (200, 1000, 777), (1500, 768, 2304), (5, 100, 9)])
@pytest.mark.parametrize("act,layout,dtype", [("gelu", "out_in", BF), ("silu", "in_out", F), ("gelu_tanh", "out_in", F), ("none", "in_out", BF)])
def test_random_values(B, m, k, n, act, layout, dtype):
    x, w, b = _rand((m, k), 1), _rand((n, k), 2, k ** -0.5), _rand((n,), 3, 0.1, F)
    r, pre = _rand((m, n), 4, 1.0, dtype), torch.empty((m, n), dtype=BF, device=DEV)
    p = B.Linear(k, n, act, layout)
    out = p.product(x, _w(w, layout), bias=b, residual=r, pre=pre)
    z = x.double() @ w.double().t() + b.double()
    dz_err = 2 * (k + 4) * U * (x.double().abs() @ w.double().abs().t() + b.double().abs())
    a = _act(z, act)
    _within(pre, z, dz_err)
    _within(out, a + r.double(), 1.13 * dz_err + a.abs() * _rel(z, act) + (a + r.double()).abs() * U + TINY)
    dout = _rand((m, n), 5)
    dx, dw, db = torch.empty((m, k), dtype=BF, device=DEV), torch.empty_like(_w(w, layout), dtype=dtype), torch.empty(n, dtype=dtype, device=DEV)
    p.grad(x, _w(w, layout), dout, pre=pre if act != "none" else None, dx=dx, dw=dw, db=db)
    slope = _slope(pre.double(), act)
    dz, tol = dout.double() * slope, dout.double().abs() * (_slope_tol(pre.double(), act) + TINY) + (dout.double() * slope).abs() * U
    _within(db, dz.sum(0), tol.sum(0) + m * U * dz.abs().sum(0))
    rounded = tol + (dz.abs() * 2 ** -8 * 1.01 if act != "none" else 0)
    _within(dx, dz @ w.double(), rounded @ w.double().abs() + 2 * (n + 4) * U * (dz.abs() @ w.double().abs()))
    split = tol + (dz.abs() * (2 ** -24 if dtype == F else 2 ** -8) * 1.01 if act != "none" else 0)
    want, err = dz.t() @ x.double(), split.t() @ x.double().abs() + 2 * (3 * m + 4) * U * (dz.abs().t() @ x.double().abs())
    _within(dw, want if layout == "out_in" else want.t(), err if layout == "out_in" else err.t())


def test_gradient_against_differences(B):
    """<dout, act(x w^T + b)> by differences of the 64-bit form."""
    m, k, n = 3, 8, 6
    x, w, b = (_ints((m, k), 1).double() / 4).to(BF), (_ints((n, k), 2).double() / 4).to(BF), _ints((n,), 3, 3, F) / 8
    dout = _ints((m, n), 4)
    for act in ACTS:
        p = B.Linear(k, n, act)
        pre = torch.empty((m, n), dtype=BF, device=DEV)
        p.product(x, w, bias=b, pre=pre)
        z0 = x.double() @ w.double().t() + b.double()
        assert torch.equal(pre.double(), z0) or act == "none" or float((pre.double() - z0).abs().max()) <= 2 ** -7
        dw, db = torch.empty((n, k), device=DEV), torch.empty(n, device=DEV)
        p.grad(x, w, dout, pre=pre if act != "none" else None, dw=dw, db=db)
        if not torch.equal(pre.double(), z0) or act == "relu":           # (relu has no derivative at 0, where some z lie)
            continue
        value = lambda q, c: float((dout.double() * _act(x.double() @ q.t() + c, act)).sum())
        step = 1e-4                          # third derivatives below 2 k 27 / 64 |dout|: off by less than 1e-7
        for i in range(n):
            e = torch.zeros(n, dtype=torch.float64, device=DEV)
            e[i] = step
            assert abs((value(w.double(), b.double() + e) - value(w.double(), b.double() - e)) / (2 * step) - float(db[i])) <= 1e-5
            f = torch.zeros((n, k), dtype=torch.float64, device=DEV)
            f[i, i % k] = step
            assert abs((value(w.double() + f, b.double()) - value(w.double() - f, b.double())) / (2 * step) - float(dw[i, i % k])) <= 1e-4


@pytest.mark.parametrize("m,k,n", [(50, 96, 200), (50, 96, 257), (300, 65, 130)])
@pytest.mark.parametrize("layout", ["out_in", "in_out"])
def test_strides_and_offsets(B, m, k, n, layout):
    x, w, dout, pre, r = _ints((m, k), 1), _ints((n, k), 2), _ints((m, n), 3), _ints((m, n), 4), _ints((m, n), 5)
    wl = _w(w, layout)
    z = x.double() @ w.double().t()
    dz = dout.double() * (pre > 0)
    for left, extra in ((8, 16), (1, 3), (4, 8), (0, 1)):
        cut = lambda t: (wide := torch.full((t.shape[0], t.shape[1] + extra), 7.0, dtype=t.dtype, device=DEV), wide[:, left:left + t.shape[1]])
        held, views = [], []
        for t in (x, wl, dout, pre, r):
            a, v = cut(t)
            v.copy_(t)
            held.append(a)
            views.append(v)
        if left + n > n + extra or left + k > k + extra:
            continue
        vx, vw, vd, vp, vr = views
        (ho, out), (hp, kept) = cut(r), cut(r)
        p = B.Linear(k, n, "relu", layout)
        p.product(vx, vw, residual=vr, out=out, pre=kept)
        assert torch.equal(out, (z.clamp(min=0) + r.double()).to(BF)) and torch.equal(kept, z.to(BF))
        (hx, dx), (hw, dw) = cut(x), cut(wl)
        p.grad(vx, vw, vd, pre=vp, dx=dx, dw=dw)
        want = dz.t() @ x.double()
        assert torch.equal(dx, (dz @ w.double()).to(BF)) and torch.equal(dw, (want if layout == "out_in" else want.t()).to(BF))
        for a in (ho, hp, hx, hw):
            assert bool((a[:, :left] == 7).all()) and bool((a[:, a.shape[1] - extra + left:] == 7).all())
        vr2 = vr.clone()
        p.product(vx, vw, residual=vr2, out=vr2)                                   # in place of the residual
        assert torch.equal(vr2, out)


def test_leading_dimensions_and_empty_batches(B):
    x, w = _ints((4, 6, 40), 1), _ints((24, 40), 2)
    p = B.Linear(40, 24)
    out = p.product(x, w)
    assert tuple(out.shape) == (4, 6, 24) and torch.equal(out.view(-1, 24), p.product(x.view(-1, 40), w))
    none = x[:0].reshape(0, 40)
    assert p.product(none, w).numel() == 0
    dx, dw, db = torch.empty((0, 40), dtype=BF, device=DEV), torch.full((24, 40), 3.0, device=DEV), torch.full((24,), 3.0, device=DEV)
    p.grad(none, w, torch.empty((0, 24), dtype=BF, device=DEV), dx=dx, dw=dw, db=db)
    assert bool((dw == 0).all()) and bool((db == 0).all())


def test_workspaces(B, G):
    """One workspace serves every smaller batch; nothing is written outside it."""
    for k, n in ((64, 64), (513, 1001), (64, 1001), (513, 64)):
        for act in ("none", "silu"):
            p, last = B.Linear(k, n, act), (0, 0)
            for m in (0, 1, 7, 8, 9, 100, 1183 * 8, 1184 * 8, 1185 * 8, 10 ** 5, 1 << 30):
                now = (p.workspace_bytes(m), p.grad_workspace_bytes(m))
                assert now[0] >= last[0] and now[1] >= last[1]
                last = now
    m, k, n = 321, 513, 1001
    p = B.Linear(k, n, "silu")
    x, w, dout, pre = _rand((m, k), 1), _rand((n, k), 2, 0.05), _rand((m, n), 3), _rand((m, n), 4)
    guard, ws = G.guarded_alloc(p.workspace_bytes(m), DEV)
    want = p.product(x, w)
    assert torch.equal(p.product(x, w, ws=ws), want) and G.guards_intact(guard)
    guard, ws = G.guarded_alloc(p.grad_workspace_bytes(m), DEV)
    outs = []
    for space in (None, ws, ws):
        dx, dw, db = torch.empty_like(x), torch.empty((n, k), device=DEV), torch.empty(n, device=DEV)
        p.grad(x, w, dout, pre=pre, dx=dx, dw=dw, db=db, ws=space)
        outs.append((dx, dw, db))
    assert all(torch.equal(a, b) for o in outs[1:] for a, b in zip(o, outs[0])) and G.guards_intact(guard)
    for some in (dict(dx=torch.empty_like(x)), dict(dw=torch.empty((n, k), device=DEV)), dict(db=torch.empty(n, device=DEV))):
        p.grad(x if "dw" in some else None, w if "dx" in some else None, dout, pre=pre, ws=ws, **some)
        (key, got), = some.items()
        assert torch.equal(got, outs[0][{"dx": 0, "dw": 1, "db": 2}[key]])


def test_long_offsets(B):
    """Rows whose bytes start beyond 32 bits."""
    m, k, n = 700000, 64, 2048
    x = torch.zeros((m, k), dtype=BF, device=DEV)
    last = _ints((5, k), 1)
    x[m - 5:] = last
    w = _ints((n, k), 2)
    out = B.Linear(k, n).product(x, w, out_dtype=F)                                # 5.7 GB
    assert torch.equal(out[m - 5:], (last.double() @ w.double().t()).float()) and bool((out[:1000] == 0).all())
    del out
    dout = torch.zeros((m, n), dtype=BF, device=DEV)
    d = _ints((5, n), 3)
    dout[m - 5:] = d
    dx, dw, db = torch.empty_like(x), torch.empty((n, k), device=DEV), torch.empty(n, device=DEV)
    B.Linear(k, n).grad(x, w, dout, dx=dx, dw=dw, db=db)
    assert torch.equal(dx[m - 5:], (d.double() @ w.double()).to(BF)) and torch.equal(dw, (d.double().t() @ last.double()).float()) and torch.equal(db, d.float().sum(0))


def test_same_bits_in_a_graph_and_on_another_stream(B):
    m, k, n = 700, 513, 1000
    p = B.Linear(k, n, "gelu")
    x, w, dout = _rand((m, k), 1), _rand((n, k), 2, 0.05), _rand((m, n), 3)
    pre = torch.empty((m, n), dtype=BF, device=DEV)
    ws, gws = (torch.empty(b, dtype=torch.uint8, device=DEV) for b in (p.workspace_bytes(m), p.grad_workspace_bytes(m)))

    def both():
        out = p.product(x, w, pre=pre, ws=ws)
        dx, dw, db = torch.empty_like(x), torch.empty((n, k), device=DEV), torch.empty(n, device=DEV)
        p.grad(x, w, dout, pre=pre, dx=dx, dw=dw, db=db, ws=gws)
        return out, dx, dw, db

    want = both()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = both()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    with torch.cuda.graph(graph := torch.cuda.CUDAGraph()):
        got = both()
    for _ in range(2):
        for g in got:
            g.fill_(7)
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_refusals(B):
    p = B.Linear(16, 24, "relu")
    x, w = _ints((5, 16), 1), _ints((24, 16), 2)
    for kw in (dict(x=x[:, :15]), dict(x=x.float()), dict(w=w.t().contiguous()), dict(w=w.float()), dict(x=x.cpu()), dict(bias=torch.zeros(24, dtype=BF, device=DEV)),
               dict(bias=torch.zeros(23, device=DEV)), dict(residual=torch.zeros((5, 24), device=DEV), out=torch.zeros((5, 24), dtype=BF, device=DEV)),
               dict(out=torch.zeros((4, 24), dtype=BF, device=DEV)), dict(out=torch.zeros((5, 24), dtype=torch.float16, device=DEV)),
               dict(pre=torch.zeros((5, 24), device=DEV)), dict(x=x.clone().requires_grad_(True)), dict(w=w.clone().requires_grad_(True)), dict(x=x.t().contiguous().t())):
        with pytest.raises(B.BaocError):
            p.product(**(dict(x=x, w=w) | kw))
    both = torch.zeros(5 * 24 + 8, dtype=BF, device=DEV)
    with pytest.raises(B.BaocError, match="overlap"):
        p.product(x, w, residual=both[:120].view(5, 24), out=both[8:].view(5, 24))
    dout, pre = _ints((5, 24), 3), _ints((5, 24), 4)
    dw = torch.zeros((24, 16), device=DEV)
    for kw in (dict(pre=None, dw=dw), dict(dw=dw, x=None), dict(dx=torch.zeros((5, 16), dtype=BF, device=DEV), w=None), dict(dw=dw.t().contiguous()),
               dict(dw=dw, db=torch.zeros(24, dtype=BF, device=DEV)), dict(dx=torch.zeros((5, 16), device=DEV)), dict(dout=dout.float(), dw=dw),
               dict(dw=dw, ws=torch.empty(16, dtype=torch.uint8, device=DEV)), dict(dx=x, dw=dw)):
        with pytest.raises(B.BaocError):
            p.grad(**(dict(x=x, w=w, dout=dout, pre=pre) | kw))
    assert torch.equal(p.product(x, w), (x.double() @ w.double().t()).clamp(min=0).to(BF))


@pytest.mark.parametrize("m,k,n", [(9, 16, 8), (130, 40, 24), (257, 8, 40), (40, 264, 8)])
def test_narrow_outputs_on_the_grid(B, m, k, n):
    """Fewer columns than an output copy's box, on the 16-byte grid, between guards."""
    x, w = _ints((m, k), 1), _ints((n, k), 2)
    want = x.double() @ w.double().t()
    for dtype in (BF, F):
        wide = torch.full((m + 2, n + 16), 7.0, dtype=dtype, device=DEV)
        B.Linear(k, n).product(x, w, out=wide[1:m + 1, :n])
        assert torch.equal(wide[1:m + 1, :n], want.to(dtype)) and bool((wide[:, n:] == 7).all()) and bool((wide[0] == 7).all()) and bool((wide[m + 1] == 7).all())


@pytest.mark.parametrize("dtype", [F, BF])
def test_long_sums_keep_their_low_bits(B, dtype):
    """131072 positive products: within a chunk of 512, 32 additions of 16 products cut at most 2^-23 each (2^-18 of the sum); 256
    chunks are added up to nearest, 2^-24 each (2^-16): below 2^-15 in all.  (Additions cut throughout would lose 2^-12.)"""
    m, k, n = 131072, 128, 192
    x, d = _rand((m, k), 1).abs() + 0.5, _rand((m, n), 2).abs() + 0.5
    dw = torch.empty((n, k), dtype=dtype, device=DEV)
    B.Linear(k, n).grad(x, None, d, dw=dw)
    want = d.double().t() @ x.double()
    _within(dw, want, want * 2.0 ** -15)


@pytest.mark.parametrize("m,k,n", [(8192, 768, 768), (16384, 776, 520), (9001, 600, 1000), (16384, 2304, 768), (4096, 1024, 1030), (12288, 256, 250), (130, 8192, 2048), (300, 8000, 1025)])
@pytest.mark.parametrize("layout", ["out_in", "in_out"])
@pytest.mark.parametrize("dtype", [F, BF])
def test_long_sums_of_few_tiles(B, m, k, n, layout, dtype):
    """Sums over many steps of outputs with few tiles, which several CTAs share: dw of narrow layers, products of few rows."""
    x, w, dout = _ints((m, k), 1), _ints((n, k), 2), _ints((m, n), 5)
    p, r = B.Linear(k, n, "none", layout), _ints((m, n), 4, 9, dtype)
    out = p.product(x, _w(w, layout), residual=r)
    assert torch.equal(out, (x.double() @ w.double().t() + r.double()).to(dtype))
    dx, dw, db = torch.empty((m, k), dtype=BF, device=DEV), torch.empty_like(_w(w, layout), dtype=dtype), torch.empty(n, dtype=dtype, device=DEV)
    p.grad(x, _w(w, layout), dout, dx=dx, dw=dw, db=db)
    want = dout.double().t() @ x.double()
    assert torch.equal(dx, (dout.double() @ w.double()).to(BF)) and torch.equal(db, dout.double().sum(0).to(dtype))
    assert torch.equal(dw, (want if layout == "out_in" else want.t()).to(dtype))
    again = torch.empty_like(dw)
    p.grad(x, _w(w, layout), dout, dw=again)
    assert torch.equal(dw, again)


def test_these_cases_run_clean_under_the_checked_build():
    """Shapes whose operands go through the workspace, on the library whose kernels validate what they touch of it first."""
    import os
    import subprocess
    import sys
    from paper_2605_04711_b200 import build
    if os.environ.get("BAOC_CHECKED") == "1":
        return                                                          # this is the child
    build.build(checked=True)
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-m", "pytest", "tests/test_gpu_linear.py", "-m", "gpu", "-x", "-q", "-k", "exact or random or strides or workspaces or few_tiles"],
                       cwd=root, env=dict(os.environ, BAOC_CHECKED="1"), capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr[-2000:]
    assert " passed" in r.stdout and "failed" not in r.stdout


@pytest.mark.parametrize("m,k,n,stride", [(391, 11, 7, 8), (80, 6, 7, 8), (1, 64, 5, 8), (3, 2048, 513, 520), (300, 64, 257, 264), (1000, 72, 1001, 1008), (4000, 200, 1005, 1024), (4096, 2048, 770, 784)])
@pytest.mark.parametrize("act", ["none", "relu"])
def test_what_lies_behind_a_rows_end_stays(B, m, k, n, stride, act):
    """Rows on the 16-byte grid that end off it, in buffers of wider rows: the columns behind them and the row behind the last stay."""
    x, w, dout = _ints((m, k), 1), _ints((n, k), 2), _ints((m, n), 3)
    z = x.double() @ w.double().t()
    for dtype in (BF, F):
        r = _ints((m, n), 4, 9, dtype)
        out, res, pre = (torch.full((m + 1, stride), 7.0, dtype=t, device=DEV) for t in (dtype, dtype, BF))
        res[:m, :n] = r
        p = B.Linear(k, n, act)
        p.product(x, w, residual=res[:m, :n], out=out[:m, :n], pre=pre[:m, :n])
        assert torch.equal(out[:m, :n], (_act(z, act) + r.double()).to(dtype)) and torch.equal(pre[:m, :n], z.to(BF))
        p.product(x, w, residual=res[:m, :n], out=res[:m, :n])
        assert torch.equal(res[:m, :n], out[:m, :n])
        for a in (out, res, pre):
            assert bool((a[:, n:] == 7).all()) and bool((a[m] == 7).all())
        # dx is [m, n] of a layer from n to k columns, dw [n, k] or [k, n]
        dz = dout.double().t() @ x.double()
        dw, dx = torch.full((k + 1, stride), 7.0, dtype=dtype, device=DEV), torch.full((m + 1, stride), 7.0, dtype=BF, device=DEV)
        B.Linear(k, n, layout="in_out").grad(x, None, dout, dw=dw[:k, :n])
        B.Linear(n, k).grad(None, w.t().contiguous(), x, dx=dx[:m, :n])
        assert torch.equal(dw[:k, :n], dz.t().to(dtype)) and torch.equal(dx[:m, :n], z.to(BF))
        for a, rows in ((dw, k), (dx, m)):
            assert bool((a[:, n:] == 7).all()) and bool((a[rows] == 7).all())


@pytest.mark.parametrize("m,k,n,stride", [(40, 7, 16, 8), (391, 13, 64, 16), (5, 513, 512, 520), (300, 1001, 256, 1008), (1000, 70, 520, 80), (2000, 515, 1024, 1024)])
def test_what_lies_behind_a_rows_end_is_not_read(B, m, k, n, stride):
    """The same of operands: NaN behind their rows reaches no sum, whichever of their dimensions is summed over."""
    def cut(t):
        wide = torch.full((t.shape[0] + 1, stride), float("nan"), dtype=BF, device=DEV)
        wide[:t.shape[0], :t.shape[1]] = t
        return wide[:t.shape[0], :t.shape[1]]

    x, w, d = _ints((m, k), 1), _ints((n, k), 2), _ints((m, n), 3)
    p, dw, dx = B.Linear(k, n), torch.empty((n, k), device=DEV), torch.empty((m, n), dtype=BF, device=DEV)
    assert torch.equal(p.product(cut(x), cut(w), out_dtype=F), (x.double() @ w.double().t()).float())
    p.grad(cut(x), None, d, dw=dw)                                                 # dw = d^T x
    assert torch.equal(dw, (d.double().t() @ x.double()).float())
    back = B.Linear(n, k, layout="in_out")                                         # w [n, k]: dx = dz w^T, summed over k
    back.grad(None, cut(w), cut(x), dx=dx)
    assert torch.equal(dx, (x.double() @ w.double().t()).to(BF))
    assert torch.equal(B.Linear(n, k, layout="in_out").product(d, cut(w), out_dtype=F), (d.double() @ w.double()).float())
