"""The norms around a block's join and their gradient, against plain 64-bit forms.

The bounds are running ones: ``E`` carries a 64-bit value and how far an fp32 evaluation of it may be off.  With u = 2^-24 every
operation adds u times its result's size; a mean over a row adds 20 u times the mean size (8 additions of a thread, at most 10
levels of sums between threads, a product); a reciprocal root adds 4 u of itself; a sum over n rows in any order adds n u times
the sum of sizes.  Outputs have to lie between the rounded ends of the interval that this gives.
"""
import pytest
import torch

pytestmark = pytest.mark.gpu

U, SUB = 2.0 ** -24, 2.0 ** -126
BF, F = torch.bfloat16, torch.float32
DEV = "cuda:0"


@pytest.fixture(scope="module")
def B():
    from paper_2605_04711_b200 import binding
    return binding


@pytest.fixture(scope="module")
def G():
    from paper_2605_04711_b200 import harness
    return harness


class E:
    def __init__(self, v, e=None):
        self.v = v.double()
        self.e = torch.zeros_like(self.v) if e is None else e

    def __add__(self, o):
        v = self.v + o.v
        return E(v, self.e + o.e + U * v.abs())

    def __sub__(self, o):
        return self + E(-o.v, o.e)

    def __mul__(self, o):
        v = self.v * o.v
        return E(v, self.v.abs() * o.e + o.v.abs() * self.e + self.e * o.e + U * v.abs())

    def mean(self):
        return E(self.v.mean(1, keepdim=True), self.e.mean(1, keepdim=True) + 20 * U * self.v.abs().mean(1, keepdim=True))

    def rsqrt(self):
        v = self.v.rsqrt()
        return E(v, 0.5 * v.pow(3) * self.e + 4 * U * v)

    def rows(self, groups=1):
        n, d = self.v.shape
        s = lambda t: t.view(groups, -1, d).sum(1)
        return E(s(self.v), s(self.e) + (n / groups) * U * s(self.v.abs()))


def _one(x):
    return E(torch.tensor(float(torch.tensor(x, dtype=F)), dtype=torch.float64))


def _hat(v, layer, eps):
    c = v - v.mean() if layer else v
    r = ((c * c).mean() + _one(eps)).rsqrt()
    return c * r, r


def _norm_grad(dn, n, r, layer):
    inner = dn - n * (dn * n).mean()
    return r * (inner - dn.mean() if layer else inner)


def _within(got, want):
    lo, hi = ((want.v + s * (want.e + SUB)).float().to(got.dtype).double() for s in (-1.0, 1.0))
    g = got.double().cpu()
    bad = ~((g >= lo) & (g <= hi))
    assert not bool(bad.any()), (int(bad.sum()), g[bad][:4], want.v.expand_as(g)[bad][:4], want.e.expand_as(g)[bad][:4])


def _data(n, dim, layer, post, gates, stream, branch, seed=0, offset=0.0):
    g = torch.Generator().manual_seed(seed + n * 131 + dim)
    r = lambda *s: torch.randn(s, generator=g)
    d = {"x": (2 * r(n, dim) + offset).to(stream), "f": (0.5 * r(n, dim) + 0.2).to(branch), "pre_w": 1 + 0.1 * r(dim), "pre_b": 0.1 * r(dim) if layer else None,
         "post_w": 0.5 + 0.1 * r(dim) if post else None, "post_b": 0.1 * r(dim) if post and layer else None, "gate": 0.5 + 0.3 * r(gates, dim) if gates else None}
    d["dy"], d["dh"] = (0.01 * r(n, dim)).to(stream), (0.01 * r(n, dim)).to(branch)
    return d


def _spread(gate, n):
    return E(gate.repeat_interleave(n // gate.shape[0], 0))


def _want_branch(d, layer, eps):
    u, nf, rf = E(d["f"]), None, None
    if d["post_w"] is not None:
        nf, rf = _hat(u, layer, eps)
        u = nf * E(d["post_w"])
        if layer and d["post_b"] is not None:
            u = u + E(d["post_b"])
    return u, nf, rf


def _want(d, layer, scale, eps):
    n = d["f"].shape[0]
    u, _, _ = _want_branch(d, layer, eps)
    if d["gate"] is not None:
        u = u * _spread(d["gate"], n)
    y = u if d["x"] is None else _one(scale) * E(d["x"]) + u
    h = _hat(y, layer, eps)[0] * E(d["pre_w"])
    return y, (h + E(d["pre_b"]) if d["pre_b"] is not None else h)


def _want_grad(d, y, layer, scale, eps):
    n = d["f"].shape[0]
    u, nf, rf = _want_branch(d, layer, eps)
    dh = E(d["dh"])
    ny, ry = _hat(E(y), layer, eps)
    dn = _norm_grad(dh * E(d["pre_w"]), ny, ry, layer)
    t = dn if d["dy"] is None else E(d["dy"]) + dn
    got = {"dpre_w": (dh * ny).rows(), "dx": _one(scale) * t}
    if layer:
        got["dpre_b"] = dh.rows()
    du = t
    if d["gate"] is not None:
        got["dgate"] = (t * u).rows(d["gate"].shape[0])
        du = t * _spread(d["gate"], n)
    got["df"] = du
    if nf is not None:
        got["dpost_w"] = (du * nf).rows()
        if d["post_b"] is not None:
            got["dpost_b"] = du.rows()
        got["df"] = _norm_grad(du * E(d["post_w"]), nf, rf, layer)
    return got


def _dev(d):
    return {k: None if v is None else v.to(DEV) for k, v in d.items()}


def _vectors(c):
    return dict(pre_b=c["pre_b"], post_w=c["post_w"], post_b=c["post_b"], gate=c["gate"])


def _run_grad(p, c, y, grad=F, **more):
    names = {"dpre_w": "pre_w", "dpre_b": "pre_b", "dpost_w": "post_w", "dpost_b": "post_b", "dgate": "gate"}
    out = {k: torch.full_like(c[of], float("nan"), dtype=grad) for k, of in names.items() if c[of] is not None}
    dx, df = p.grad(y, c["f"], c["dh"], c["pre_w"], dy=c["dy"], post_w=c["post_w"], post_b=c["post_b"], gate=c["gate"], **out, **more)
    return out | {"dx": dx, "df": df}


def _check(B, d, layer, scale=1.0, eps=1e-6, grad=F):
    p, c = B.Join(d["f"].shape[1], "layer" if layer else "rms", eps=eps, scale=scale), _dev(d)
    y, h = p.join(c["x"], c["f"], c["pre_w"], **_vectors(c), y=None if c["x"] is not None else torch.empty_like(c["dy"]))
    for got, want in zip((y, h), _want(d, layer, scale, eps)):
        _within(got, want)
    got = _run_grad(p, c, y, grad)
    for k, want in _want_grad(d, y.cpu(), layer, scale, eps).items():
        _within(got[k], want)
    return y, h, got


SHAPES = [(1, 1), (3, 2), (1, 8), (2, 2048), (1, 8192), (5, 7), (33, 64), (70, 256), (9, 257), (300, 513), (64, 520), (40, 768), (20, 1000), (1000, 96),
          (3000, 128), (700, 1024), (6, 2049), (12, 4096), (6, 4104), (7, 5000), (700, 8192), (5, 8191)]


@pytest.mark.parametrize("n,dim", SHAPES)
@pytest.mark.parametrize("stream,branch,layer,post,gates,grad", [(F, BF, False, True, 1, BF), (BF, BF, True, True, 1, F), (F, F, True, False, 0, F),
                                                                (F, BF, False, False, 1, F), (BF, BF, False, True, 0, BF)])
def test_join_and_gradient(B, n, dim, stream, branch, layer, post, gates, grad):
    _check(B, _data(n, dim, layer, post, gates, stream, branch), layer, scale=0.7 if layer else 1.0, grad=grad)


@pytest.mark.parametrize("n,gates", [(12, 12), (12, 3), (600, 5), (4000, 2), (4000, 1000), (6000, 7), (5929, 77)])
@pytest.mark.parametrize("dim", [64, 100, 520, 2048])
def test_gate_per_group(B, n, gates, dim):
    n = n // gates * gates
    _check(B, _data(n, dim, True, True, gates, F, BF), True)


@pytest.mark.parametrize("layer", [False, True])
@pytest.mark.parametrize("dim", [40, 513, 4096])
def test_special_rows(B, layer, dim):
    """Rows of zeros, of one value, far from zero, nearly constant: eps and the mean's removal carry them."""
    d = _data(8, dim, layer, True, 1, F, F)
    d["x"][0], d["f"][0] = 0, 0
    d["f"][1] = 3.0
    d["x"][2] += 1000.0
    d["f"][3] += 100.0
    d["f"][4], d["x"][4] = 0, 1e-6
    _check(B, d, layer, eps=1e-5)


def test_without_a_stream(B):
    d = _data(50, 300, False, False, 0, F, BF)
    d["x"] = None
    y, h, _ = _check(B, d, False)
    assert torch.equal(y.cpu(), d["f"].float())
    c = _dev(d)
    dx, df = B.Join(300).grad(y, None, c["dh"], c["pre_w"], want_dx=False)       # nothing but the norm
    assert dx is None
    _within(df, _want_grad(d | {"dy": None}, y.cpu(), False, 1.0, 1e-6)["df"])


@pytest.mark.parametrize("dim", [64, 2048, 100])
def test_in_place_strides_and_guards(B, G, dim):
    n = 37
    d = _data(n, dim, True, True, 1, F, BF)
    p, c = B.Join(dim, "layer"), _dev(d)
    y, h = p.join(c["x"], c["f"], c["pre_w"], **_vectors(c))
    x2, f2 = c["x"].clone(), c["f"].clone()
    p.join(x2, f2, c["pre_w"], **_vectors(c), y=x2, h=f2)
    assert torch.equal(x2, y) and torch.equal(f2, h)
    want = _run_grad(p, c, y)
    dy2, dh2 = c["dy"].clone(), c["dh"].clone()
    got = _run_grad(p, c | {"dy": dy2, "dh": dh2}, y, dx=dy2, df=dh2)
    assert all(torch.equal(got[k], want[k]) for k in want) and torch.equal(dy2, want["dx"])
    for left, width in ((8, dim + 16), (1, dim + 3), (4, dim + 9)):
        wide = {k: torch.full((n, width), 9.0, dtype=c[k].dtype, device=DEV) for k in ("x", "f", "dy", "dh")}
        for k in wide:
            wide[k][:, left:left + dim] = c[k]
        cut = {k: v[:, left:left + dim] for k, v in wide.items()}
        oy, oh = torch.full((n, width), 9.0, device=DEV), torch.full((n, width), 9.0, dtype=BF, device=DEV)
        p.join(cut["x"], cut["f"], c["pre_w"], **_vectors(c), y=oy[:, left:left + dim], h=oh[:, left:left + dim])
        for o, w in zip((oy, oh), _want(d, True, 1.0, 1e-6)):
            _within(o[:, left:left + dim], w)
            assert bool((o[:, :left] == 9).all()) and bool((o[:, left + dim:] == 9).all())
        got = _run_grad(p, c | cut, y, dx=cut["dy"], df=cut["dh"])
        for k, w in _want_grad(d, y.cpu(), True, 1.0, 1e-6).items():
            _within(got[k], w)
        assert bool((wide["dy"][:, :left] == 9).all()) and bool((wide["dh"][:, left + dim:] == 9).all())
    guard, ws = G.guarded_alloc(p.grad_workspace_bytes(n), DEV)
    again = _run_grad(p, c, y, ws=ws)
    assert all(torch.equal(again[k], want[k]) for k in want) and G.guards_intact(guard)


def test_one_workspace_serves_fewer_rows(B):
    for dim in (64, 100, 1000, 2048, 4096, 8192, 8191):
        p, last = B.Join(dim), 0
        for n in (0, 1, 2, 147, 148, 149, 591, 592, 593, 1000, 4735, 4736, 4737, 10 ** 5, 10 ** 6, 1 << 31):
            assert p.grad_workspace_bytes(n) >= last
            last = p.grad_workspace_bytes(n)


def test_no_rows(B):
    p, w = B.Join(16), torch.ones(16, device=DEV)
    e = torch.empty((0, 16), device=DEV)
    y, h = p.join(e, e, w)
    dw = torch.full((16,), float("nan"), device=DEV)
    p.grad(y, e, h, w, dpre_w=dw)
    assert y.numel() == 0 and bool((dw == 0).all())


def test_nothing_wanted_but_the_branch(B):
    d = _data(20, 200, True, True, 1, F, BF)
    p, c = B.Join(200, "layer"), _dev(d)
    y, _ = p.join(c["x"], c["f"], c["pre_w"], **_vectors(c))
    all_ = _run_grad(p, c, y)
    dx, df = p.grad(y, c["f"], c["dh"], c["pre_w"], dy=c["dy"], post_w=c["post_w"], post_b=c["post_b"], gate=c["gate"])
    assert torch.equal(dx, all_["dx"]) and torch.equal(df, all_["df"])


def test_gradient_against_differences(B):
    """<dy, y> + <dh, h> by differences of the 64-bit form, at some of every input's elements."""
    n, dim, layer, scale, eps = 4, 12, True, 0.8, 1e-5
    d = _data(n, dim, layer, True, 2, F, F, offset=0.5)
    p, c = B.Join(dim, "layer", eps=eps, scale=scale), _dev(d)
    y, _ = p.join(c["x"], c["f"], c["pre_w"], **_vectors(c))
    got = _run_grad(p, c, y)

    def value(q):
        v, w = _want(q, layer, scale, eps)
        return float((v.v * d["dy"].double()).sum() + (w.v * d["dh"].double()).sum())

    step = 1e-4                              # third derivatives of order 0.01 at most: off by 1e-10
    for of, k in (("x", "dx"), ("f", "df"), ("pre_w", "dpre_w"), ("pre_b", "dpre_b"), ("post_w", "dpost_w"), ("post_b", "dpost_b"), ("gate", "dgate")):
        base = {a: None if b is None else b.double() for a, b in d.items()}
        flat = got[k].reshape(-1).cpu().double()
        for i in range(0, flat.numel(), 5):
            at = [base | {of: base[of].clone()} for _ in range(2)]
            for q, s in zip(at, (step, -step)):
                q[of].view(-1)[i] += s
            # fp32 terms below 0.1 each, a few roundings; y itself was rounded once
            assert abs((value(at[0]) - value(at[1])) / (2 * step) - float(flat[i])) <= 2e-6, (k, i)


def test_long_offsets(B):
    """Rows whose bytes start beyond 32 bits."""
    n, dim = 600000, 2048
    x = torch.zeros((n, dim), device=DEV)                                          # 4.9 GB
    f = torch.zeros((n, dim), dtype=BF, device=DEV)
    d = _data(3, dim, False, True, 1, F, BF)
    x[n - 3:], f[n - 3:] = d["x"].to(DEV), d["f"].to(DEV)
    c = _dev(d)
    p = B.Join(dim)
    y, h = p.join(x, f, c["pre_w"], post_w=c["post_w"], gate=c["gate"], y=x)
    for got, want in zip((y, h), _want(d, False, 1.0, 1e-6)):
        _within(got[n - 3:], want)
    dh = torch.zeros((n, dim), dtype=BF, device=DEV)
    dh[n - 3:] = c["dh"]
    dw = torch.empty(dim, device=DEV)
    _, df = p.grad(y, f, dh, c["pre_w"], post_w=c["post_w"], gate=c["gate"], df=dh, dpre_w=dw, want_dx=False)
    want = _want_grad(d | {"dy": None}, y[n - 3:].cpu(), False, 1.0, 1e-6)
    _within(df[n - 3:], want["df"])
    _within(dw, want["dpre_w"])


def test_same_bits_in_a_graph_and_on_another_stream(B):
    d = _data(500, 768, True, True, 5, BF, BF)
    p, c = B.Join(768, "layer"), _dev(d)
    y, h = p.join(c["x"], c["f"], c["pre_w"], **_vectors(c))
    want = _run_grad(p, c, y)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        y2, h2 = p.join(c["x"], c["f"], c["pre_w"], **_vectors(c))
        got = _run_grad(p, c, y2)
    side.synchronize()
    assert torch.equal(y, y2) and torch.equal(h, h2) and all(torch.equal(got[k], want[k]) for k in want)
    y3, h3 = torch.empty_like(y), torch.empty_like(h)
    out = {k: torch.empty_like(v) for k, v in want.items()}
    ws = torch.empty(p.grad_workspace_bytes(500), dtype=torch.uint8, device=DEV)
    with torch.cuda.graph(graph := torch.cuda.CUDAGraph()):
        p.join(c["x"], c["f"], c["pre_w"], **_vectors(c), y=y3, h=h3)
        p.grad(y3, c["f"], c["dh"], c["pre_w"], dy=c["dy"], post_w=c["post_w"], post_b=c["post_b"], gate=c["gate"], ws=ws, **out)
    for _ in range(2):
        graph.replay()
        assert torch.equal(y, y3) and torch.equal(h, h3) and all(torch.equal(out[k], want[k]) for k in want)


def test_refusals(B):
    d = _data(6, 32, True, True, 3, F, BF)
    p, c = B.Join(32, "layer"), _dev(d)
    v = _vectors(c)
    join = lambda **kw: p.join(*[(c | kw)[k] for k in ("x", "f", "pre_w")], **(v | {k: a for k, a in kw.items() if k not in ("x", "f", "pre_w")}))
    for kw in (dict(x=c["x"][:5]), dict(x=c["x"][:, :31]), dict(f=c["f"].half()), dict(x=c["x"].cpu()), dict(pre_w=c["pre_w"][:31]), dict(pre_w=c["pre_w"].bfloat16()),
               dict(gate=c["gate"][:2].repeat(2, 1)), dict(gate=c["gate"].t()), dict(y=c["x"].bfloat16()), dict(h=c["x"]), dict(x=c["x"].bfloat16(), f=c["f"].float()),
               dict(post_w=None), dict(y=c["f"].float()[:, ::2]), dict(x=c["x"].clone().requires_grad_(True)), dict(pre_w=c["pre_w"].clone().requires_grad_(True))):
        with pytest.raises(B.BaocError):
            join(**kw)
    both = torch.zeros(7 * 32, device=DEV)
    with pytest.raises(B.BaocError, match="overlap"):
        join(x=both[:192].view(6, 32), y=both[16:208].view(6, 32))
    with pytest.raises(B.BaocError):
        B.Join(32, "rms").join(c["x"], c["f"], c["pre_w"], pre_b=c["pre_b"])       # a bias of an RMS norm
    y, h = join()
    for kw in (dict(dgate=torch.empty(2, 32, device=DEV)), dict(dpre_w=torch.empty(31, device=DEV)), dict(dpre_w=torch.empty(32, device=DEV), dpre_b=torch.empty(32, dtype=BF, device=DEV)),
               dict(ws=torch.empty(16, dtype=torch.uint8, device=DEV)), dict(df=c["f"], post_w=c["post_w"]), dict(dpost_w=torch.empty(32, device=DEV))):
        with pytest.raises(B.BaocError):
            p.grad(y, c["f"], c["dh"], c["pre_w"], **kw)
    _check(B, d, True)                                                              # the plan's module works on


def test_one_gate_for_more_rows_than_there_are(B):
    """rows_per_gate at and beyond the number of rows, beyond 32 bits too, through the C entries."""
    import ctypes as C
    d = _data(6, 64, False, True, 1, F, BF)
    p, c = B.Join(64), _dev(d)
    y, h = p.join(c["x"], c["f"], c["pre_w"], **_vectors(c))
    want = _run_grad(p, c, y)
    for rpg in (6, 7, 1 << 31, 1 << 32, (1 << 63) - 1):
        p._e.rows_per_gate = p._g.rows_per_gate = rpg
        y2, h2, dx, df, dg = torch.empty_like(y), torch.empty_like(h), torch.empty_like(y), torch.empty_like(h), torch.empty(64, device=DEV)
        ws = torch.empty(p.grad_workspace_bytes(6), dtype=torch.uint8, device=DEV)
        q = lambda t: t.data_ptr()
        p._g.grad_dtype = 1
        assert B._lib.baoc_join(p._ref, q(c["x"]), q(c["f"]), q(c["post_w"]), None, q(c["gate"]), q(c["pre_w"]), None, 6, q(y2), q(h2), B._stream()) == 0
        assert B._lib.baoc_join_grad(p._gref, q(y), q(c["f"]), q(c["dy"]), q(c["dh"]), q(c["post_w"]), None, q(c["gate"]), q(c["pre_w"]), 6, q(dx), q(df), None, None,
                                     q(dg), None, None, q(ws), ws.numel(), B._stream()) == 0
        assert torch.equal(y2, y) and torch.equal(h2, h) and torch.equal(dx, want["dx"]) and torch.equal(df, want["df"]) and torch.equal(dg, want["dgate"][0])


@pytest.mark.parametrize("gates", [0, 3])
def test_gates_without_rows(B, gates):
    """An empty batch (no sequences, or sequences of no tokens): nothing to join, and every gate's gradient is zero."""
    p, x, f, w = B.Join(40), torch.empty(0, 40, device=DEV), torch.empty(0, 40, dtype=BF, device=DEV), torch.ones(40, device=DEV)
    gate, dgate, dw = torch.ones(gates, 40, device=DEV), torch.full((gates, 40), 7.0, dtype=BF, device=DEV), torch.full((40,), 7.0, dtype=BF, device=DEV)
    y, h = p.join(x, f, w, gate=gate)
    dx, df = p.grad(y, f, h, w, gate=gate, dgate=dgate, dpre_w=dw)
    assert y.shape == h.shape == dx.shape == df.shape == (0, 40) and not dgate.any() and not dw.any()
    with pytest.raises(B.BaocError):
        p.join(torch.zeros(2, 40, device=DEV), torch.zeros(2, 40, dtype=BF, device=DEV), w, gate=torch.ones(0, 40, device=DEV))
    with pytest.raises(B.BaocError):
        p.join(x, f, w, gate=torch.ones((), device=DEV))


def test_a_refused_join_leaves_the_gradient_alone(B):
    """A form of the join that is refused (an fp32 branch on a bf16 stream) says nothing of the gradient's form."""
    p, w = B.Join(32), torch.ones(32, device=DEV)
    x, f = torch.ones(4, 32, dtype=BF, device=DEV), torch.ones(4, 32, dtype=BF, device=DEV)
    with pytest.raises(B.BaocError, match="fp32 stream"):
        p.join(x, f.float(), w)
    dx, df = p.grad(x, None, f, w)
    assert torch.isfinite(dx).all() and torch.equal(dx, df)


@pytest.mark.parametrize("n,dim", [(592, 768), (593, 768), (594, 513), (1500, 300), (1201, 512), (700, 765), (2000, 600)])
@pytest.mark.parametrize("stream,branch,layer,gates", [(F, BF, False, 1), (BF, BF, True, 1), (F, F, True, 1), (BF, BF, False, 0), (BF, BF, True, 2)])
def test_more_than_a_few_rows(B, n, dim, stream, branch, layer, gates):
    """Rows of 257 to 768 columns: from some number of them on, a warp takes one alone."""
    _check(B, _data(n // max(gates, 1) * max(gates, 1), dim, layer, True, gates, stream, branch), layer, grad=F)


@pytest.mark.parametrize("n,dim", [(9000, 256), (7000, 512), (5000, 768), (1500, 5000), (1500, 8192)])
@pytest.mark.parametrize("layer,gates", [(False, 0), (True, 5)])
@pytest.mark.parametrize("want_dx", [True, False])
def test_rows_requested_ahead(B, n, dim, layer, gates, want_dx):
    """Many bf16 rows per CTA, each requested while the one before is worked on, dy's place behind the store that holds it: dy itself
    in place of dx, dx apart, and no dx."""
    d = _data(n, dim, layer, True, gates, BF, BF)
    d["dy"] *= 100
    p, c = B.Join(dim, "layer" if layer else "rms"), _dev(d)
    y, _ = p.join(c["x"], c["f"], c["pre_w"], **_vectors(c))
    want, first = _want_grad(d, y.cpu(), layer, 1.0, 1e-6), None
    for dx in (None, "dy", None) if want_dx else (None, None):
        call = c | {"dy": c["dy"].clone()}
        got = _run_grad(p, call, y, **({"dx": call["dy"]} if dx else {}), want_dx=want_dx)
        for k, w in want.items() if first is None else ():
            if k != "dx" or want_dx:
                _within(got[k], w)
        first = first or got
        assert all(torch.equal(got[k], first[k]) for k in first if first[k] is not None)


@pytest.mark.parametrize("n,dim", [(1, 1), (3, 2), (5, 7), (33, 64), (9, 257), (300, 513), (40, 768), (594, 513), (700, 765), (2000, 600), (3000, 128), (700, 1024), (6, 2049), (12, 4096),
                                   (6, 4104), (300, 8192), (5, 8191)])
@pytest.mark.parametrize("stream,branch,layer,groups", [(F, BF, True, 1), (F, F, True, 1), (F, BF, True, 3), (F, F, False, 2), (BF, BF, True, 1), (BF, BF, True, 4), (BF, BF, False, 3)])
def test_gates_of_a_branch_without_a_norm(B, n, dim, stream, branch, layer, groups):
    """post(f) is f itself, whatever its mean: the gate's gradient sums Dy f, not Dy (f - mean(f))."""
    groups = min(groups, n)
    d = _data(n // groups * groups, dim, layer, False, groups, stream, branch)
    d["f"] += 1
    _check(B, d, layer, scale=0.7, grad=F)


def test_gate_gradient_of_a_branch_without_a_norm_against_differences(B):
    """<dy, y> + <dh, h> by differences of the 64-bit form along every gate."""
    n, dim, scale, eps = 4, 12, 0.8, 1e-5
    d = _data(n, dim, True, False, 2, F, F, offset=0.5)
    p, c = B.Join(dim, "layer", eps=eps, scale=scale), _dev(d)
    y, _ = p.join(c["x"], c["f"], c["pre_w"], **_vectors(c))
    got = _run_grad(p, c, y)

    def value(q):
        v, w = _want(q, True, scale, eps)
        return float((v.v * d["dy"].double()).sum() + (w.v * d["dh"].double()).sum())

    step = 1e-4                              # third derivatives of order 0.01 at most: off by 1e-10
    for of, k in (("gate", "dgate"), ("f", "df"), ("x", "dx")):
        base = {a: None if b is None else b.double() for a, b in d.items()}
        flat = got[k].reshape(-1).cpu().double()
        for i in range(flat.numel()):
            at = [base | {of: base[of].clone()} for _ in range(2)]
            for q, s in zip(at, (step, -step)):
                q[of].view(-1)[i] += s
            # fp32 terms below 0.1 each, a few roundings; y itself was rounded once
            assert abs((value(at[0]) - value(at[1])) / (2 * step) - float(flat[i])) <= 2e-6, (k, i)


@pytest.mark.parametrize("n,dim,stream,branch", [(6, 40, F, BF), (21, 513, F, F), (702, 768, BF, BF), (6, 8192, BF, BF)])
@pytest.mark.parametrize("layer,post,gates", [(a, b, c) for a in (False, True) for b in (False, True) for c in (0, 1, 3)])
def test_every_form(B, n, dim, stream, branch, layer, post, gates):
    """Each of what may be left out, left out: the stream, dy, the biases; each column sum wanted alone or not at all."""
    n -= n % 3
    full = _data(n, dim, layer, post, gates, stream, branch)
    for without in ((), ("dy",), ("x",), ("x", "dy"), ("pre_b",), ("post_b",), ("pre_b", "post_b", "dy")):
        d = full | {k: None for k in without}
        p, c = B.Join(dim, "layer" if layer else "rms", scale=0.7), _dev(d)
        y, h = p.join(c["x"], c["f"], c["pre_w"], **_vectors(c), y=torch.empty((n, dim), dtype=stream, device=DEV))
        for got, want in zip((y, h), _want(d, layer, 0.7, 1e-6)):
            _within(got, want)
        want, all_ = _want_grad(d, y.cpu(), layer, 0.7, 1e-6), _run_grad(p, c, y)
        for k, w in want.items():
            if k in all_:                            # (a bias that was left out has no gradient's place in it)
                _within(all_[k], w)
        for k in all_:
            if k not in ("dx", "df"):
                one = torch.full_like(all_[k], float("nan"))
                _, df = p.grad(y, c["f"], c["dh"], c["pre_w"], dy=c["dy"], post_w=c["post_w"], post_b=c["post_b"], gate=c["gate"], want_dx=False, **{k: one})
                assert torch.equal(one, all_[k]) and torch.equal(df, all_["df"])
