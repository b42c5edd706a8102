"""nm_layer_norm and nm_layer_norm_grad against binary64 on the CPU: rows of one element to 32768, odd widths, means far from zero, strides, types, none and many rows."""
import pytest
import torch

from gpu_util import DEV

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
E32 = 2.0 ** -24
EPS = 1e-5


def _inputs(R, C, xt, wt, seed=0, offset=0.3):
    gen = torch.Generator().manual_seed(seed + 7 * R + C)
    new = lambda *s: torch.randn(*s, generator=gen)                          # noqa: E731
    return ((new(R, C) + offset * new(R, 1) * 3).to(xt), (1 + 0.3 * new(C)).to(wt), new(C).to(wt), new(R, C).to(xt))


def _half(t):
    return torch.finfo(t).eps / 2


def _want(x, w, b, g, eps=EPS):
    """{name: (value, bound)}.  n: a sum's terms; errors at their largest, added up.  mean: n half steps of the mean magnitude.  A deviation d: the mean's error and one
    rounding.  Variance: n half steps, and 2 |d| times d's error in the mean; rstd: half the variance's relative error, and 4 steps of root and quotient."""
    R, C = x.shape
    X, W, B, G = x.double(), w.double(), b.double(), g.double()
    n = C + 16
    mean = X.mean(1, keepdim=True)
    emean = n * E32 * X.abs().mean(1, keepdim=True)
    d = X - mean
    ed = emean + E32 * d.abs()
    var = (d * d).mean(1, keepdim=True)
    # (the deviations' sum of products with their error: the mean's own error enters squared, since they add up to zero, but is taken in full)
    evar = n * E32 * var + 2 * (d.abs() * ed).mean(1, keepdim=True) + (ed * ed).mean(1, keepdim=True)
    r = 1 / (var + eps).sqrt()
    rr = 0.5 * evar / (var + eps) * (1 + 2 * evar / (var + eps)) + 6 * E32   # relative
    h = d * r
    eh = ed * r + h.abs() * (rr + 2 * E32)
    ux = _half(x.dtype)
    y = h * W + B
    ey = eh * W.abs() + 3 * E32 * ((h * W).abs() + B.abs())
    u = G * W
    eu = E32 * u.abs()
    mu, muh = u.mean(1, keepdim=True), (u * h).mean(1, keepdim=True)
    emu = n * E32 * u.abs().mean(1, keepdim=True) + eu.mean(1, keepdim=True)
    emuh = n * E32 * (u * h).abs().mean(1, keepdim=True) + (u.abs() * eh + eu * h.abs()).mean(1, keepdim=True) * 2
    t = u - mu - h * muh
    et = eu + emu + eh * muh.abs() + h.abs() * emuh + eh * emuh + 4 * E32 * (u.abs() + mu.abs() + (h * muh).abs())
    dx = t * r
    edx = et * r * (1 + rr) + dx.abs() * (rr + E32)
    uw = _half(w.dtype)
    dw, db = (G * h).sum(0), G.sum(0)
    edw = (G.abs() * eh).sum(0) + (R + 4) * E32 * (G * h).abs().sum(0)
    edb = (R + 4) * E32 * G.abs().sum(0)
    out = lambda v, e, half: (v, e + half * (v.abs() + e) + 1e-37)           # noqa: E731
    return {"y": out(y, ey, ux), "mean": (mean[:, 0], emean[:, 0] + 1e-37), "rstd": (r[:, 0], (r * rr)[:, 0]), "dx": out(dx, edx, ux), "dw": out(dw, edw, uw), "db": out(db, edb, uw)}


def _check(name, got, want):
    off = (got.cpu().double() - want[0]).abs()
    assert got.shape == want[0].shape and bool((off <= want[1]).all()), f"{name}: {(off / want[1]).max().item():.3g} of the bound"


def _compare(x, w, b, g, view=lambda t: t):
    import paper_2203_10991_amd as nm
    want = _want(x, w, b, g)
    xd, gd = view(x.to(DEV)), view(g.to(DEV))
    y, mean, rstd = nm.nm_layer_norm(xd, w.to(DEV), b.to(DEV), EPS, want_stats=True)
    dx, dw, db = nm.nm_layer_norm_grad(gd, xd, w.to(DEV), mean, rstd)
    assert y.dtype == dx.dtype == x.dtype and dw.dtype == db.dtype == w.dtype
    for name, got in (("y", y), ("mean", mean), ("rstd", rstd), ("dx", dx), ("dw", dw), ("db", db)):
        _check(name, got, want[name])
    return y, dx, dw, db


@pytest.mark.parametrize("xt,wt", [(BF16, F32), (BF16, BF16), (F32, F32), (F32, BF16)])
@pytest.mark.parametrize("R,C", [(1, 1), (3, 2), (5, 7), (2, 8), (9, 9), (4, 33), (70, 64), (13, 511), (6, 512), (5, 513), (300, 1001), (1, 1024), (7, 1025), (33, 2047), (3, 2048), (5, 4097),
                                 (2, 8191), (3, 8192), (2, 8193), (3, 16384), (2, 16391), (2, 32768), (2500, 40), (1700, 264)])
def test_against_binary64(R, C, xt, wt):
    _compare(*_inputs(R, C, xt, wt))


@pytest.mark.parametrize("xt", [BF16, F32])
def test_means_far_from_zero(xt):
    """a mean of hundreds of deviations: sums of squares would cancel"""
    for C in (100, 3000):
        _compare(*_inputs(6, C, xt, F32, offset=100.0))


@pytest.mark.parametrize("xt", [BF16, F32])
@pytest.mark.parametrize("C", [5, 100, 1024, 2500])
def test_views(xt, C):
    """rows apart, starting on any element, columns apart, a shared row, more dimensions"""
    import paper_2203_10991_amd as nm
    x, w, b, g = _inputs(12, C, xt, F32)

    def shifted(t):
        wide = torch.full((t.shape[0], C + 11), float("nan"), dtype=t.dtype, device=DEV)
        wide[:, 3:3 + C] = t
        return wide[:, 3:3 + C]
    got, plain = _compare(x, w, b, g, shifted), _compare(x, w, b, g)
    assert all(torch.equal(a, c) for a, c in zip(got, plain))
    got = _compare(x, w, b, g, lambda t: torch.stack((t, t), -1)[..., 0])
    assert all(torch.equal(a, c) for a, c in zip(got, plain))
    xd, wd, bd = x.to(DEV), w.to(DEV), b.to(DEV)
    assert torch.equal(nm.nm_layer_norm(xd.view(3, 4, C), wd, bd).view(12, C), plain[0])
    assert torch.equal(nm.nm_layer_norm(xd[:1].expand(5, C), wd, bd), plain[0][:1].expand(5, C))


def test_without_weights():
    import paper_2203_10991_amd as nm
    x, w, b, g = _inputs(40, 300, F32, F32)
    one, nil = torch.ones(300), torch.zeros(300)
    xd, gd = x.to(DEV), g.to(DEV)
    y, mean, rstd = nm.nm_layer_norm(xd, want_stats=True)
    _check("y", y, _want(x, one, nil, g)["y"])
    dx, dw, db = nm.nm_layer_norm_grad(gd, xd, None, mean, rstd, want_weight=False, want_bias=False)
    _check("dx", dx, _want(x, one, nil, g)["dx"])
    assert dw is None and db is None
    _check("y", nm.nm_layer_norm(xd, w.to(DEV)), _want(x, w, nil, g)["y"])
    _check("y", nm.nm_layer_norm(xd, None, b.to(DEV)), _want(x, one, b, g)["y"])
    dx, dw, db = nm.nm_layer_norm_grad(gd, xd, w.to(DEV), mean, rstd, want_weight=False)
    assert dw is None
    _check("db", db, _want(x, w, nil, g)["db"])
    dx, dw, db = nm.nm_layer_norm_grad(gd, xd, w.to(DEV), mean, rstd, want_bias=False)
    assert db is None
    _check("dw", dw, _want(x, w, nil, g)["dw"])


def test_no_rows_equal_rows_and_what_is_not_finite():
    import paper_2203_10991_amd as nm
    x = torch.empty(0, 70, device=DEV)
    y, mean, rstd = nm.nm_layer_norm(x, torch.ones(70, device=DEV), want_stats=True)
    dx, dw, db = nm.nm_layer_norm_grad(x, x, torch.ones(70, device=DEV), mean, rstd)
    assert y.shape == dx.shape == (0, 70) and not bool(dw.any()) and not bool(db.any())
    same = torch.full((5, 1000), 3.0, device=DEV)                            # variance zero
    y, mean, rstd = nm.nm_layer_norm(same, want_stats=True)
    assert not bool(y.any()) and bool(((rstd - EPS ** -0.5).abs() <= EPS ** -0.5 * 8 * E32).all())
    same[1, 700], same[3, 2] = float("nan"), float("inf")                    # ... stays in its row
    y = nm.nm_layer_norm(same)
    assert bool(torch.isnan(y[[1, 3]]).all()) and not bool(y[[0, 2, 4]].any())


def test_same_bits_streams_and_a_graph():
    import paper_2203_10991_amd as nm
    x, w, b, g = (t.to(DEV) for t in _inputs(3000, 700, BF16, F32))

    def both():
        y, mean, rstd = nm.nm_layer_norm(x, w, b, want_stats=True)
        return y, mean, rstd, *nm.nm_layer_norm_grad(g, x, w, mean, rstd)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        apart = both()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = both()
    for turn in range(4):
        want = both()
        if turn == 0:
            assert all(torch.equal(a, c) for a, c in zip(want, apart))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(want, held))
        x.copy_(torch.randn(x.shape, device=DEV))


def test_offsets_past_32_bits():
    """rows 2^31 elements apart, and 5 x 10^9 bytes of rows"""
    import paper_2203_10991_amd as nm
    x, w, b, g = _inputs(3, 300, BF16, F32)
    store = torch.empty((2 << 31) + 1000, dtype=BF16, device=DEV)
    far = store.as_strided((3, 300), (1 << 31, 1))
    far.copy_(x)
    assert torch.equal(nm.nm_layer_norm(far, w.to(DEV), b.to(DEV)), nm.nm_layer_norm(x.to(DEV), w.to(DEV), b.to(DEV)))
    rows = store[:(1 << 32) // 1024 * 1000].view(-1, 1000)
    rows.normal_()
    y = nm.nm_layer_norm(rows)
    assert torch.equal(y[-5:], nm.nm_layer_norm(rows[-5:].clone())) and torch.equal(y[:5], nm.nm_layer_norm(rows[:5].clone()))


def test_gradients_against_differences():
    import paper_2203_10991_amd as nm
    x, w, b, g = _inputs(5, 37, F32, F32)
    y, mean, rstd = nm.nm_layer_norm(x.to(DEV), w.to(DEV), b.to(DEV), EPS, want_stats=True)
    got = nm.nm_layer_norm_grad(g.to(DEV), x.to(DEV), w.to(DEV), mean, rstd)
    bounds = _want(x, w, b, g)
    at = [t.double() for t in (x, w, b)]
    gen = torch.Generator().manual_seed(1)
    for i, name in enumerate(("dx", "dw", "db")):
        d = torch.randn(at[i].shape, generator=gen, dtype=torch.float64)
        f = []
        for step in (1e-5, -1e-5):
            X, W, B = (t + step * d if k == i else t for k, t in enumerate(at))
            f.append((g.double() * torch.nn.functional.layer_norm(X, (37,), W, B, EPS)).sum())
        assert abs((f[0] - f[1]) / 2e-5 - (got[i].cpu().double() * d).sum()) <= (bounds[name][1] * d.abs()).sum() + 1e-7 * d.abs().sum()


def test_refusals():
    import paper_2203_10991_amd as nm
    x, w = torch.zeros(4, 10, device=DEV), torch.ones(10, device=DEV)
    y, mean, rstd = nm.nm_layer_norm(x, w, want_stats=True)
    for call in (lambda: nm.nm_layer_norm(x.cpu()), lambda: nm.nm_layer_norm(x, w[:5]), lambda: nm.nm_layer_norm(x, w.cpu()), lambda: nm.nm_layer_norm_grad(x[:2], x, w, mean, rstd),
                 lambda: nm.nm_layer_norm_grad(x, x, w, mean[:2], rstd), lambda: nm.nm_layer_norm_grad(x.to(BF16), x, w, mean, rstd), lambda: nm.nm_layer_norm_grad(x, x, w, mean, rstd.double())):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: nm.nm_layer_norm(x.half()), lambda: nm.nm_layer_norm(x, w, w.to(BF16))):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: nm.nm_layer_norm(x, eps=-1.0), lambda: nm.nm_layer_norm(x, eps=float("nan")), lambda: nm.nm_layer_norm(torch.zeros(1, 32769, device=DEV)),
                 lambda: nm.nm_layer_norm(torch.zeros(1, 0, device=DEV))):
        with pytest.raises(nm.NmError):
            call()


@pytest.mark.parametrize("xt", [BF16, F32])
@pytest.mark.parametrize("R,C", [(2700, 1030), (1400, 2500), (1300, 5000), (1283, 9000), (530, 16384), (1290, 16391), (260, 32768)])
def test_workgroups_with_several_rows(R, C, xt):
    """rows of several waves, more of them than the forward pass (1280) and the gradients (256 or 512) have workgroups: statistics exchanged row after row, the next row on its way, sums over rows"""
    import paper_2203_10991_amd as nm
    x, w, b, g = _inputs(R, C, xt, F32)
    got = _compare(x, w, b, g)
    # every row's result is what the row alone gives
    xd = x.to(DEV)
    for at in (0, R // 2, R - 1):
        assert torch.equal(got[0][at:at + 1], nm.nm_layer_norm(xd[at:at + 1], w.to(DEV), b.to(DEV), EPS))


@pytest.mark.parametrize("C", [1500, 4000, 9000, 20000])
def test_rows_of_several_waves_again_and_again(C):
    """the same bits from every call, for rows that differ by far from one to the next"""
    import paper_2203_10991_amd as nm
    gen = torch.Generator(device=DEV).manual_seed(C)
    x = torch.randn(3000, C, generator=gen, device=DEV) * torch.exp2(torch.randint(-20, 20, (3000, 1), generator=gen, device=DEV).float()) + torch.randn(3000, 1, generator=gen, device=DEV) * 1000
    w, g = torch.rand(C, generator=gen, device=DEV) + 0.5, torch.randn(3000, C, generator=gen, device=DEV)

    def both():
        y, mean, rstd = nm.nm_layer_norm(x, w, want_stats=True)
        return y, mean, rstd, *nm.nm_layer_norm_grad(g, x, w, mean, rstd)
    first = both()
    for _ in range(5):
        assert all(torch.equal(a, b) for a, b in zip(first, both()))
    # (rows in another order: results move with them)
    order = torch.randperm(3000, generator=gen, device=DEV)
    y, mean, rstd = nm.nm_layer_norm(x[order], w, want_stats=True)
    assert torch.equal(y, first[0][order]) and torch.equal(mean, first[1][order]) and torch.equal(rstd, first[2][order])
