"""The token table's lookup and gradient and the gradient norm and clip, against plain 64-bit forms.

Every kernel computes in fp32 (or wider) and rounds to its output type at the end.  With u = 2^-24, the rounding of one
fp32 operation relative to its result, and 2^-149 where that result is subnormal, the fp32 value lies in want +- tol:
  * lookup: one product, u |want|;
  * gradient of a row named c times: c additions in any order and one product, (c + 2) u of scale * sum |dout|;
    accumulated, one addition more, of |old| too;
  * norm: chains of at most 64 squares and three additions of non-negative terms in fp32 (68 u of the squares at most, half
    of it for the root), doubles from there on, one rounding to fp32: 36 u relative;
  * clip: the norm's 34 u before its output rounding, one rounding of the factor, one product: 37 u.
Rounding is monotone, so the output has to lie between the rounded ends of that interval: for a bf16 output those are
neighbours at most, and mostly one value.
"""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

U, SUB = 2.0 ** -24, 2.0 ** -149
BF, F = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def B():
    from paper_2605_04711_b200 import binding
    return binding


@pytest.fixture(scope="module")
def G():
    from paper_2605_04711_b200 import harness
    return harness


def _dev(t):
    return t.to("cuda:0")


def _rand(shape, dtype, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (scale * torch.randn(shape, generator=g, dtype=torch.float32)).to(dtype)


def _ids(n, vocab, seed, kind="uniform", dtype=torch.int64):
    g = torch.Generator().manual_seed(seed)
    if kind == "same":
        return torch.full((n,), vocab // 2, dtype=dtype)
    if kind == "skewed":
        u = torch.rand(n, generator=g, dtype=torch.float64)
        return (torch.exp(u * math.log(vocab + 1.0)) - 1.0).long().clamp_(0, vocab - 1).to(dtype)
    return torch.randint(0, vocab, (n,), generator=g).to(dtype)


def _want_lookup(table, ids, scale):
    out = torch.zeros((ids.numel(), table.shape[1]), dtype=torch.float64)
    ok = (ids >= 0) & (ids < table.shape[0])
    out[ok] = table.double()[ids[ok].long()] * float(np.float32(scale))
    return out


def _want_grad(dout, ids, vocab, scale, pad):
    """(sum, sum of magnitudes, count) per row in 64 bits."""
    ok = (ids >= 0) & (ids < vocab) & (ids != (-1 if pad is None else pad))
    k, x = ids[ok].long(), dout.double()[ok]
    total = torch.zeros((vocab, dout.shape[1]), dtype=torch.float64)
    mag, count = torch.zeros_like(total), torch.zeros(vocab, dtype=torch.float64)
    total.index_add_(0, k, x)
    mag.index_add_(0, k, x.abs())
    count.index_add_(0, k, torch.ones(k.numel(), dtype=torch.float64))
    s = float(np.float32(scale))
    return total * s, mag * abs(s), count


def _within(got, want, tol):
    lo, hi = ((want + sign * (tol + SUB)).float().to(got.dtype).double() for sign in (-1.0, 1.0))
    g = got.double().cpu()
    bad = ~((g >= lo) & (g <= hi))
    assert not bool(bad.any()), (int(bad.sum()), float(((g - want).abs() / (tol + SUB)).max()))


# ---- lookup -------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("n,vocab,dim", [(1, 1, 1), (1, 300, 2048), (2, 7, 3), (5, 100, 8), (33, 1000, 257), (64, 130, 64), (257, 4099, 513),
                                         (1000, 129, 136), (7, 3, 4100), (4096, 512, 100), (50, 60, 66), (50, 60, 362), (50, 60, 2)])
@pytest.mark.parametrize("tdt,odt,idt,scale", [(F, BF, torch.int64, 45.25), (F, F, torch.int32, 1.0), (BF, BF, torch.int32, -0.3),
                                               (BF, F, torch.int64, 1.0)])
def test_lookup(B, n, vocab, dim, tdt, odt, idt, scale):
    table, ids = _rand((vocab, dim), tdt, 1), _ids(n, vocab, 2, dtype=idt)
    ids[n // 2] = -1 if n > 1 else ids[0]
    if n > 4:
        ids[3] = vocab
        ids[4] = torch.iinfo(idt).min
    out = B.Embedding(vocab, dim, scale=scale).lookup(_dev(table), _dev(ids), out_dtype=odt)
    assert out.dtype == odt and tuple(out.shape) == (n, dim)
    want = _want_lookup(table, ids, scale)
    _within(out, want, U * want.abs())


def test_lookup_shapes_strides_and_offsets(B):
    table = _rand((50, 40), F, 3)
    ids = _ids(24, 50, 4).view(4, 6)
    e = B.Embedding(50, 40)
    dt = _dev(table)
    out = e.lookup(dt, _dev(ids))
    assert tuple(out.shape) == (4, 6, 40)
    want = _want_lookup(table, ids.reshape(-1), 1.0)
    assert torch.equal(out.cpu().view(-1, 40), want.to(BF))
    # a slice of the ids that is not contiguous
    out = e.lookup(dt, _dev(ids)[:, :-1])
    assert torch.equal(out.cpu().view(-1, 40), _want_lookup(table, ids[:, :-1].reshape(-1), 1.0).to(BF))
    # rows inside wider buffers: the wide path with strides, and odd offsets that only elements are aligned to
    for left, width in ((8, 64), (1, 47), (3, 48), (2, 46), (4, 47)):
        wt = torch.zeros((50, width))
        wt[:, left:left + 40] = table
        wo = torch.full((24, width), 7.0, dtype=BF, device="cuda:0")
        e.lookup(_dev(wt)[:, left:left + 40], _dev(ids).view(-1), out=wo[:, left:left + 40])
        assert torch.equal(wo[:, left:left + 40].cpu(), want.to(BF))
        assert bool((wo[:, :left] == 7).all()) and bool((wo[:, left + 40:] == 7).all())
    # no tokens
    assert e.lookup(dt, torch.empty(0, dtype=torch.int64, device="cuda:0")).shape == (0, 40)


def test_lookup_keeps_infinities_and_nan_in_their_rows(B):
    table = _rand((9, 24), F, 5)
    table[2, 3], table[2, 4], table[5, 0] = float("inf"), float("-inf"), float("nan")
    ids = torch.tensor([0, 2, -1, 5, 9, 1], dtype=torch.int32)
    out = B.Embedding(9, 24, scale=2.0).lookup(_dev(table), _dev(ids), out_dtype=F).cpu()
    want = torch.zeros(6, 24)
    for t, v in enumerate(ids.tolist()):
        if 0 <= v < 9:
            want[t] = 2.0 * table[v]
    assert torch.equal(torch.nan_to_num(out, nan=123.0), torch.nan_to_num(want, nan=123.0))


def test_lookup_offsets_beyond_32_bits(B):
    """A bf16 table of 4.4 G elements: rows whose element offsets pass 2^31 and 2^32."""
    vocab, dim = 537000, 8192
    table = torch.zeros((vocab, dim), dtype=BF, device="cuda:0")
    ids = torch.tensor([0, 262143, 262144, 524288, vocab - 1], device="cuda:0")
    rows = _rand((5, dim), BF, 6)
    table[ids] = _dev(rows)
    out = B.Embedding(vocab, dim).lookup(table, ids)
    assert torch.equal(out.cpu(), rows)


# ---- gradient -----------------------------------------------------------------------------------------------------
GRAD_SHAPES = [(1, 1, 1, "uniform"), (1, 300, 2048, "uniform"), (3, 5, 2, "uniform"), (64, 130, 64, "skewed"), (200, 7, 257, "uniform"),
               (333, 1000, 100, "skewed"), (1000, 129, 136, "same"), (31, 128, 8, "same"), (32, 127, 16, "same"), (33, 50, 24, "same"),
               (2049, 300, 40, "skewed"), (5000, 3, 33, "uniform"), (4099, 513, 520, "skewed"), (70000, 40, 16, "skewed"),
               (40000, 17, 300, "same"), (256, 50, 40, "same"), (257, 50, 40, "same"), (200, 30, 1500, "skewed"), (256, 5, 511, "uniform"),
               (300, 90, 362, "skewed"), (5000, 100, 98, "skewed"), (900, 33, 50, "skewed"), (900, 33, 130, "skewed"), (60, 30000, 600, "skewed")]


@pytest.mark.parametrize("n,vocab,dim,kind", GRAD_SHAPES)
@pytest.mark.parametrize("adt,gdt,idt,scale", [(BF, BF, torch.int64, 45.25), (F, F, torch.int32, 1.0), (BF, F, torch.int32, -0.3),
                                               (F, BF, torch.int64, 1.0)])
def test_grad(B, G, n, vocab, dim, kind, adt, gdt, idt, scale):
    dout, ids = _rand((n, dim), adt, 7), _ids(n, vocab, 8, kind, idt)
    pad = vocab // 3 if n > 40 else None
    if n > 4:
        ids[0], ids[n // 2] = -1, vocab
    e = B.Embedding(vocab, dim, scale=scale, pad_id=pad)
    nb = 2 if gdt == BF else 4
    guard_t, flat = G.guarded_alloc(vocab * dim * nb, "cuda:0")
    guard_w, ws = G.guarded_alloc(e.grad_workspace_bytes(n), "cuda:0")
    flat.fill_(0xFF)                                                    # NaN in both types: every row has to be written
    ws.fill_(0xA5)
    dtable = flat.view(gdt).view(vocab, dim)
    e.grad(_dev(ids), _dev(dout), dtable, ws=ws)
    want, mag, count = _want_grad(dout, ids, vocab, scale, pad)
    _within(dtable, want, (count[:, None] + 2) * U * mag)
    first = dtable.clone()
    # accumulated on top of what is there: rows that no token named keep their bits
    base = _rand((vocab, dim), gdt, 9)
    dtable.copy_(base)
    e.grad(_dev(ids), _dev(dout), dtable, accumulate=True, ws=ws)
    _within(dtable, want + base.double(), (count[:, None] + 3) * U * (mag + base.double().abs()))
    untouched = count == 0
    assert torch.equal(dtable.cpu()[untouched], base[untouched])
    # equal inputs, equal bits (other contents of the workspace, another stream)
    ws.fill_(0x3C)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        e.grad(_dev(ids), _dev(dout), dtable, ws=ws)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(dtable, first)
    assert G.guards_intact(guard_t) and G.guards_intact(guard_w)


@pytest.mark.parametrize("n", [3000, 32767, 32768, 70003])
@pytest.mark.parametrize("vocab", [1, 127, 128, 129, 98304, 98305, 131071, 262145, 600000])
def test_grad_vocabularies(B, vocab, n):
    """Vocabularies and token counts around the sizes where the grouping changes its geometry."""
    dim = 4
    ids = _ids(n, vocab, 10, "uniform")
    ids[:50] = vocab - 1
    dout = _rand((n, dim), F, 11)
    dtable = torch.full((vocab, dim), float("nan"), device="cuda:0")
    B.Embedding(vocab, dim).grad(_dev(ids), _dev(dout), dtable)
    want, mag, count = _want_grad(dout, ids, vocab, 1.0, None)
    _within(dtable, want, (count[:, None] + 2) * U * mag)


def test_grad_masked_positions_are_not_read(B):
    """NaN and infinities at padded and ignored positions reach no row; at a named position they reach that row alone."""
    n, vocab, dim = 300, 20, 40
    ids = _ids(n, vocab, 12)
    ids[::7], ids[1::7] = 4, -100
    dout = _rand((n, dim), F, 13)
    clean = dout.clone()
    dout[::7], dout[1::7] = float("nan"), float("inf")
    for name, x in (("clean", clean), ("dirty", dout)):
        d = torch.empty((vocab, dim), device="cuda:0")
        B.Embedding(vocab, dim, pad_id=4).grad(_dev(ids), _dev(x), d)
        want, mag, count = _want_grad(clean, ids, vocab, 1.0, 4)
        _within(d, want, (count[:, None] + 2) * U * mag)
        assert bool((d[4] == 0).all())
    at = int((ids == 9).nonzero()[0])
    clean[at, 5] = float("inf")
    B.Embedding(vocab, dim, pad_id=4).grad(_dev(ids), _dev(clean), d)
    d = d.cpu()
    assert d[9, 5] == float("inf") and int((~torch.isfinite(d)).sum()) == 1


def test_grad_of_no_tokens_and_of_masked_tokens_only(B):
    for n, ids in ((0, torch.empty(0, dtype=torch.int64)), (70, torch.full((70,), 3)), (70, torch.full((70,), -1))):
        d = torch.full((10, 24), 5.0, dtype=BF, device="cuda:0")
        e = B.Embedding(10, 24, pad_id=3)
        e.grad(_dev(ids), _dev(_rand((n, 24), BF, 14)), d, accumulate=True)
        assert bool((d == 5).all())
        e.grad(_dev(ids), _dev(_rand((n, 24), BF, 14)), d)
        assert bool((d == 0).all())


def test_grad_strides_and_offsets(B):
    n, vocab, dim = 90, 30, 40
    ids, dout = _ids(n, vocab, 15, "skewed"), _rand((n, dim), BF, 16)
    want, mag, count = _want_grad(dout, ids, vocab, 1.0, None)
    tol = (count[:, None] + 2) * U * mag
    for left, width in ((8, 64), (1, 47), (3, 48), (2, 46), (4, 47)):
        wd = torch.full((n, width), float("nan"), dtype=BF)
        wd[:, left:left + dim] = dout
        wt = torch.full((vocab, width), 7.0, dtype=BF, device="cuda:0")
        B.Embedding(vocab, dim).grad(_dev(ids), _dev(wd)[:, left:left + dim], wt[:, left:left + dim])
        _within(wt[:, left:left + dim], want, tol)
        assert bool((wt[:, :left] == 7).all()) and bool((wt[:, left + dim:] == 7).all())
    # a batch of sequences: ids [3, 30], dout [3, 30, dim]
    d = torch.empty((vocab, dim), dtype=BF, device="cuda:0")
    B.Embedding(vocab, dim).grad(_dev(ids).view(3, 30), _dev(dout).view(3, 30, dim), d)
    _within(d, want, tol)


def test_grad_offsets_beyond_32_bits(B):
    """dout of 2.2 G bf16 elements with two long and some short rows, whose last tokens lie past 2^31 elements."""
    n, vocab, dim = 270000, 1000, 8192
    dout = torch.zeros((n, dim), dtype=BF, device="cuda:0")
    ids = torch.full((n,), -1)
    pos = torch.cat([torch.arange(0, 100), torch.arange(n - 100, n)])
    ids[pos] = _ids(200, 5, 17) * 199
    rows = _rand((200, dim), BF, 18)
    dout[_dev(pos)] = _dev(rows)
    d = torch.empty((vocab, dim), device="cuda:0")
    B.Embedding(vocab, dim).grad(_dev(ids), dout, d)
    want, mag, count = _want_grad(rows, ids[pos], vocab, 1.0, None)
    _within(d, want, (count[:, None] + 2) * U * mag)


def test_grad_is_the_lookups_derivative(B):
    """Differences of L(table) = sum(w * lookup(table)) in each of some entries: L is linear, so a central difference in
    fp32 with step 1/2 is exact up to its roundings."""
    n, vocab, dim, scale = 60, 11, 16, 1.5
    table, ids, w = _rand((vocab, dim), F, 19), _ids(n, vocab, 20, "skewed"), _rand((n, dim), F, 21)
    ids[5] = -1
    e = B.Embedding(vocab, dim, scale=scale)
    d = torch.empty((vocab, dim), device="cuda:0")
    e.grad(_dev(ids), _dev(w), d)
    for v, c in ((0, 0), (1, 7), (5, 15), (10, 3)):
        val = []
        for step in (0.5, -0.5):
            t2 = table.clone()
            t2[v, c] += step
            out = e.lookup(_dev(t2), _dev(ids), out_dtype=F).cpu().double()
            val.append(float((out * w.double()).sum()))
        count = int((ids == v).sum())
        # each of the count outputs is off by two roundings (t2 and the product) of about |table| * scale <= 8
        tol = 2 * count * 2 * U * 8 * float(w.abs().max()) + (count + 2) * U * scale * float(w[ids == v].abs().sum())
        assert abs((val[0] - val[1]) - float(d[v, c])) <= tol


# ---- norm and clip --------------------------------------------------------------------------------------------------
BLOCKS = [1, 2, 7, 8, 9, 255, 4096, 16383, 16384, 16385, 32769, 100003, 3, 131072]


def _handle(B, sizes):
    h = B.Baoc([(n, n, 1) for n in sizes], B.default_configs())
    h.bind_clip_workspace(torch.empty(h.clip_workspace_bytes(), dtype=torch.uint8, device="cuda:0"))
    return h


def _grads(sizes, dtype, seed, scale=1.0):
    return [_rand((n,), dtype, seed + i, scale * 10.0 ** (i % 5 - 2)) for i, n in enumerate(sizes)]


def _want_norms(gs):
    sq = [float((g.double() ** 2).sum()) for g in gs]
    return torch.tensor([math.sqrt(sum(sq))] + [math.sqrt(x) for x in sq], dtype=torch.float64)


@pytest.mark.parametrize("sizes", [[1], [5], BLOCKS, [300] * 700, [3000000]])
@pytest.mark.parametrize("dtype", [BF, F])
def test_grad_norm(B, sizes, dtype):
    h, gs = _handle(B, sizes), _grads(sizes, dtype, 30)
    norms = torch.full((1 + len(sizes),), -1.0, device="cuda:0")
    dg = [_dev(g) for g in gs]
    want = _want_norms(gs)
    h.grad_norm(dg, norms)
    _within(norms, want, 36 * U * want)
    first = norms.clone()
    for _ in range(3):                                                  # the workspace is ready for the next call; equal bits
        h.grad_norm(dg, norms)
        assert torch.equal(norms, first)
    assert h.query().kernel_launches >= 4


@pytest.mark.parametrize("src,dst", [(BF, BF), (F, F), (F, BF)])
@pytest.mark.parametrize("sizes", [[1], BLOCKS, [130] * 700])
@pytest.mark.parametrize("max_norm", [0.0, 0.5, 1e9])
def test_clip(B, G, src, dst, sizes, max_norm):
    h, gs = _handle(B, sizes), _grads(sizes, src, 40)
    norms = torch.empty(1 + len(sizes), device="cuda:0")
    want_n = _want_norms(gs)
    factor = min(1.0, max_norm / (float(want_n[0]) + 1e-6))
    dg, outs, guards = [_dev(g) for g in gs], [], []
    for g in gs:
        whole, view = G.guarded_alloc(g.numel() * (2 if dst == BF else 4), "cuda:0")
        view.fill_(0xFF)
        guards.append(whole)
        outs.append(view.view(dst))
    h.clip_grads(dg, outs, max_norm, norms)
    _within(norms, want_n, 36 * U * want_n)
    for g, d, o in zip(gs, dg, outs):
        want = g.double() * factor
        _within(o, want, 37 * U * (factor < 1.0) * want.abs())
        assert torch.equal(d.cpu(), g)                                  # the source is left alone
    if src == dst:                                                      # in place: the same bits
        h.clip_grads(dg, None, max_norm, norms)
        for d, o in zip(dg, outs):
            assert torch.equal(d, o)
    assert all(G.guards_intact(w) for w in guards)


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("scale", [1e-30, 1e-22, 1e-18, 1e18, 1e25, 3e36])
def test_norm_of_values_whose_squares_leave_fp32(B, dtype, scale):
    sizes = [20000, 33, 1]
    gs = [_rand((n,), dtype, 50 + i, scale) for i, n in enumerate(sizes)]
    h = _handle(B, sizes)
    norms = torch.empty(4, device="cuda:0")
    out = [torch.empty(n, device="cuda:0", dtype=dtype) for n in sizes]
    h.clip_grads([_dev(g) for g in gs], out, 1.0, norms)
    want = _want_norms(gs)
    f = min(1.0, 1.0 / (float(want[0]) + 1e-6))
    ok = want < 3.4e38
    _within(norms.cpu()[ok], want[ok], 36 * U * want[ok])
    assert bool(torch.isinf(norms.cpu()[~ok]).all())
    # (a factor below the smallest normal fp32 number is rounded to a multiple of 2^-149)
    for g, o in zip(gs, out):
        w = g.double() * f
        _within(o, w, 37 * U * w.abs() + g.double().abs() * 2.0 ** -150)


def test_mixed_magnitudes_in_one_thread(B):
    """One block holds zeros, values whose squares vanish in fp32 and values whose squares overflow it."""
    g = torch.zeros(16384 * 3)
    g[5::64], g[6::64], g[40000:] = 1e-25, 1e-30, 1e-24
    for big in (None, 2e25):
        if big:
            g[777] = big
        h = _handle(B, [g.numel()])
        norms = torch.empty(2, device="cuda:0")
        h.grad_norm([_dev(g)], norms)
        want = _want_norms([g])
        _within(norms, want, 36 * U * want)


def test_zero_infinite_and_nan_gradients(B):
    sizes = [100, 20000, 3]
    h = _handle(B, sizes)
    norms = torch.empty(4, device="cuda:0")
    for dtype in (BF, F):
        gs = [torch.zeros(n, dtype=dtype, device="cuda:0") for n in sizes]
        out = [torch.full_like(g, 3.0) for g in gs]
        h.clip_grads(gs, out, 1.0, norms)
        assert bool((norms == 0).all()) and all(bool((o == 0).all()) for o in out)
        gs[1][7777], gs[0][3] = float("inf"), 2.0
        h.clip_grads(gs, out, 1.0, norms)
        assert norms[0] == float("inf") and norms[2] == float("inf") and norms[1] == 2.0 and norms[3] == 0
        assert bool((out[0] == 0).all()) and int(torch.isnan(out[1]).sum()) == 1 and bool(torch.isnan(out[1][7777]))
        gs[2][0] = float("nan")
        h.clip_grads(gs, out, 1.0, norms)
        assert bool(torch.isnan(norms[0])) and bool(torch.isnan(norms[3])) and all(bool(torch.isnan(o).all()) for o in out)


def test_other_arrays_streams_and_a_captured_graph(B):
    sizes = BLOCKS
    h = _handle(B, sizes)
    a, b = ([_dev(g) for g in _grads(sizes, BF, s)] for s in (60, 80))
    want = [_want_norms([g.cpu() for g in x]) for x in (a, b)]
    norms = torch.empty(1 + len(sizes), device="cuda:0")
    s = torch.cuda.Stream()
    for k in range(4):                                                  # alternating arrays and streams, ordered by the caller
        st = s if k & 1 else torch.cuda.current_stream()
        st.wait_stream(torch.cuda.current_stream() if k & 1 else s)
        with torch.cuda.stream(st):
            h.grad_norm((a, b)[k // 2], norms)
        torch.cuda.synchronize()
        _within(norms, want[k // 2], 36 * U * want[k // 2])
    out = [torch.empty_like(g) for g in a]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        h.clip_grads(a, out, 0.25, norms)
    h.grad_norm(b, norms)                                               # the tables hold other pointers now
    torch.cuda.synchronize()
    graph.replay()
    torch.cuda.synchronize()
    _within(norms, want[0], 36 * U * want[0])
    for g, o in zip(a, out):
        w = g.cpu().double() * (0.25 / (float(want[0][0]) + 1e-6))
        _within(o, w, 37 * U * w.abs())
    h.grad_norm(b, norms)
    _within(norms, want[1], 36 * U * want[1])


def test_captured_embedding(B):
    n, vocab, dim = 500, 100, 64
    e = B.Embedding(vocab, dim)
    table, ids = _dev(_rand((vocab, dim), F, 90)), _dev(_ids(n, vocab, 91, "skewed"))
    out = torch.empty((n, dim), dtype=BF, device="cuda:0")
    d = torch.empty((vocab, dim), dtype=BF, device="cuda:0")
    ws = torch.empty(e.grad_workspace_bytes(n), dtype=torch.uint8, device="cuda:0")

    def call():
        e.lookup(table, ids, out=out)
        e.grad(ids, out, d, ws=ws)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    ids.copy_(_dev(_ids(n, vocab, 92, "same")))
    graph.replay()
    got = out.clone(), d.clone()
    call()
    assert torch.equal(got[0], out) and torch.equal(got[1], d)


def test_binding_refuses_what_it_can_see(B):
    e = B.Embedding(10, 16)
    t, ids, d = torch.zeros(10, 16, device="cuda:0"), torch.zeros(4, dtype=torch.int64, device="cuda:0"), torch.zeros(4, 16, device="cuda:0")
    bad = [lambda: e.lookup(t[:9], ids), lambda: e.lookup(t, ids.float()), lambda: e.lookup(t.cpu(), ids), lambda: e.lookup(t.half(), ids),
           lambda: e.lookup(t, ids, out=torch.zeros(5, 16, device="cuda:0")), lambda: e.lookup(t, ids, out=t[:4]),
           lambda: e.lookup(t.t().contiguous().t(), ids), lambda: e.lookup(t, ids.cpu()),
           lambda: e.grad(ids, d[:3], t), lambda: e.grad(ids, d, t[:, :8]), lambda: e.grad(ids, d.double(), t),
           lambda: e.grad(ids, d[:1].expand(4, 16), t), lambda: e.grad(ids, t[:4], t),
           lambda: e.grad(ids, d, t, ws=torch.empty(16, dtype=torch.uint8, device="cuda:0"))]
    for k, f in enumerate(bad):
        with pytest.raises(B.BaocError):
            f()
            raise AssertionError(k)
    h = B.Baoc([(64, 8, 8), (5, 5, 1)], B.default_configs())
    norms = torch.zeros(3, device="cuda:0")
    gs = [torch.zeros(64, dtype=BF, device="cuda:0"), torch.zeros(5, dtype=BF, device="cuda:0")]
    with pytest.raises(B.BaocError) as x:
        h.grad_norm(gs, norms)
    assert x.value.code == B.E_STATE
    with pytest.raises(B.BaocError) as x:
        h.bind_clip_workspace(torch.empty(16, dtype=torch.uint8, device="cuda:0"))
    assert x.value.code == B.E_WORKSPACE
    h.bind_clip_workspace(torch.empty(h.clip_workspace_bytes(), dtype=torch.uint8, device="cuda:0"))
    f32 = [g.float() for g in gs]
    bad = [(lambda: h.grad_norm(gs[:1], norms), B.E_INVALID), (lambda: h.grad_norm([gs[0], gs[0]], norms), B.E_INVALID),
           (lambda: h.grad_norm([gs[0], f32[1]], norms), B.E_INVALID), (lambda: h.grad_norm([g.half() for g in gs], norms), B.E_INVALID),
           (lambda: h.grad_norm(gs, norms[:2]), B.E_INVALID), (lambda: h.grad_norm(gs, norms.double()), B.E_INVALID),
           (lambda: h.clip_grads(gs, f32, 1.0, norms), B.E_INVALID), (lambda: h.clip_grads(gs, None, -1.0, norms), B.E_INVALID),
           (lambda: h.clip_grads(gs, None, float("nan"), norms), B.E_INVALID), (lambda: h.clip_grads(gs, None, float("inf"), norms), B.E_INVALID),
           (lambda: h.grad_norm([torch.zeros(72, dtype=BF, device="cuda:0")[1:65], gs[1]], norms), B.E_ALIGN)]
    for f, code in bad:
        with pytest.raises(B.BaocError) as x:
            f()
        assert x.value.code == code
    buf = torch.zeros(200, dtype=BF, device="cuda:0")
    with pytest.raises(B.BaocError):
        h.clip_grads([buf[:64], gs[1]], [buf[8:72], torch.zeros_like(gs[1])], 1.0, norms)
    h.clip_grads(gs, None, 1.0, norms)                                  # and the handle still works
    assert float(norms[0]) == 0.0


def test_example_trains():
    """The bigram model's operators together: its loss falls below half of a uniform guess's, and the clip acts."""
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "bigram_lm.py")
    spec = importlib.util.spec_from_file_location("bigram_lm", path)
    lm = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(lm)
    losses, norms = lm.train(steps=150)
    assert losses[0] > 0.8 * math.log(lm.VOCAB)
    assert np.mean(losses[-10:]) < 0.5 * math.log(lm.VOCAB)
    assert all(math.isfinite(x) and x > 0 for x in norms) and max(norms) > 0.25


def test_these_cases_run_clean_under_the_checked_build():
    """The same cases on the library whose kernels validate their tables and workspace ranges first."""
    import os
    import subprocess
    import sys
    from paper_2605_04711_b200 import build
    if os.environ.get("BAOC_CHECKED") == "1":
        return                                                          # this is the child
    build.build(checked=True)
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-m", "pytest", "tests/test_gpu_embed_clip.py", "-m", "gpu", "-x", "-q"], cwd=root,
                       env=dict(os.environ, BAOC_CHECKED="1"), capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr[-2000:]
    assert " passed" in r.stdout and "failed" not in r.stdout
