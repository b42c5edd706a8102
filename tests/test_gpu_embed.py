"""nm_embed, nm_embed_grad and NMEmbedding against binary64 on the CPU: tokens from none to tens of thousands, one token everywhere, every kind of order;
odd widths, strides, bases; both sorts on either side of their border."""
import pytest
import torch

from gpu_util import DEV, kernels_of

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def _ids(kind, N, V, gen):
    if kind == "uniform":
        return torch.randint(0, V, (N,), generator=gen)
    if kind == "frequent":
        return (torch.rand(N, generator=gen, dtype=torch.float64) * torch.log(torch.tensor(V + 1.0, dtype=torch.float64))).exp().sub(1).long().clamp(0, V - 1)
    if kind == "one":
        return torch.full((N,), V // 2)
    if kind == "falling":
        return torch.arange(N).flip(0) % V
    if kind == "two":                                                    # runs that end on, before and behind the borders of a chunk
        return (torch.arange(N) // 31) % min(V, 2)
    if kind == "runs":                                                   # rows of 1 to 70 tokens in turn: either side of what one workgroup sums
        length = torch.arange(N) % 70 + 1
        return torch.repeat_interleave(torch.arange(N), length)[:N].remainder(V)[torch.randperm(N, generator=gen)]
    raise ValueError(kind)


def _want(g, ids, V, scale, padding=-1):
    """(sums, sums of magnitudes) in binary64"""
    out, size = torch.zeros(V, g.shape[1], dtype=torch.float64), torch.zeros(V, g.shape[1], dtype=torch.float64)
    ok = (ids >= 0) & (ids < V) & (ids != padding)
    out.index_add_(0, ids[ok], g[ok].double())
    size.index_add_(0, ids[ok], g[ok].double().abs())
    return out * scale, size * abs(scale)


def _check(got, want, size, n_most):
    """n additions in binary32, in any order: at most n 2^-24 of the sum of magnitudes, and two roundings more; bf16 adds half a unit in the last place"""
    eps = 2.0 ** -8 * want.abs() if got.dtype == BF16 else 0
    assert bool(((got.cpu().double() - want).abs() <= (n_most + 3) * 2.0 ** -24 * size + eps + 1e-38).all())


@pytest.mark.parametrize("table,out", [(F32, F32), (F32, BF16), (BF16, BF16), (BF16, F32)])
@pytest.mark.parametrize("N,V,D,bits", [(0, 5, 8, 64), (1, 1, 1, 32), (7, 100, 33, 64), (8, 1000, 1024, 32), (513, 300, 64, 64), (100, 50, 2049, 32), (3, 9, 8200, 64)])
def test_lookup(table, out, N, V, D, bits):
    import paper_2203_10991_amd as nm
    gen = torch.Generator().manual_seed(N + V)
    t = torch.randn(V, D, generator=gen).to(table).to(DEV)
    ids = _ids("uniform", N, V, gen).to(torch.int64 if bits == 64 else torch.int32).to(DEV)
    got = nm.nm_embed(t, ids, 1.7, out)
    assert got.shape == (N, D) and torch.equal(got, (t[ids.long()].float() * torch.tensor(1.7, device=DEV)).to(out))
    # a view whose rows start anywhere, tokens in two dimensions
    wide = torch.randn(V, D + 13, generator=gen).to(table).to(DEV)
    got = nm.nm_embed(wide[:, 3:3 + D], ids.reshape(1, N, 1))
    assert got.shape == (1, N, 1, D) and torch.equal(got.reshape(N, D), wide[:, 3:3 + D][ids.long()])


def test_lookup_of_tokens_outside_and_other_layouts():
    import paper_2203_10991_amd as nm
    t = torch.randn(10, 40, device=DEV)
    ids = torch.tensor([[0, -1, 9], [10, 1 << 40, 3]], device=DEV)
    got = nm.nm_embed(t, ids.t())                                         # (not contiguous)
    bad = (ids.t() < 0) | (ids.t() > 9)
    assert bool(torch.isnan(got[bad]).all()) and torch.equal(got[~bad], t[ids.t()[~bad]])
    assert torch.equal(nm.nm_embed(t.t(), torch.tensor([5], device=DEV))[0], t[:, 5])
    assert nm.nm_embed(t[:, :0], ids).shape == (2, 3, 0)
    assert bool(torch.isnan(nm.nm_embed(t[:0], ids)).all())


GRADS = [(1, 1, 1), (2, 7, 5), (15, 3, 8), (16, 40, 33), (17, 1000, 64), (64, 2, 1024), (65, 300, 100), (200, 1, 64), (255, 300, 8), (256, 40, 600), (256, 9000, 1030), (257, 40, 600), (512, 300, 100), (300, 30000, 600), (513, 40, 64), (1000, 50, 520), (4095, 30011, 72), (4096, 77, 40), (4097, 30011, 72), (8192, 500, 136)]
LARGE = [(8193, 500, 72), (8200, 3, 64), (16384, 40000, 40), (16385, 200, 24), (20000, 70000, 40), (32768, 511, 16), (32769, 511, 16), (33000, 511, 24), (33000, 512, 33), (65536, 300000, 16), (65537, 513, 8), (70001, 300000, 16)]


@pytest.mark.parametrize("kind", ["uniform", "frequent", "one", "falling", "two", "runs"])
@pytest.mark.parametrize("N,V,D", GRADS + LARGE)
def test_gradient(kind, N, V, D):
    import paper_2203_10991_amd as nm
    gen = torch.Generator().manual_seed(N + V + D)
    ids = _ids(kind, N, V, gen)
    g = torch.randn(N, D, generator=gen)
    gd, idd = g.to(DEV), ids.to(torch.int32).to(DEV)
    want, size = _want(g, ids, V, 0.5)
    most = int(torch.bincount(ids).max())
    got = nm.nm_embed_grad(gd, idd, V, 0.5)
    assert got.shape == (V, D) and got.dtype == F32
    _check(got, want, size, most)
    assert torch.equal(got, nm.nm_embed_grad(gd, idd.long(), V, 0.5))
    names = kernels_of(lambda: nm.nm_embed_grad(gd, idd, V, 0.5))
    assert any(("embed_few_kernel" if D >= 8 and (N <= 256 or N <= 512 and V * D < 500000) else "embed_rank_kernel" if N <= 4096 else "embed_merge_kernel" if N <= 32768 else "embed_move_kernel") in k for k in names), names


@pytest.mark.parametrize("gt", [F32, BF16])
@pytest.mark.parametrize("out", [F32, BF16])
@pytest.mark.parametrize("N,V,D", [(300, 40, 64), (300, 40, 37), (9000, 100, 264), (40, 7, 4100)])
def test_gradient_types_views_and_accumulation(gt, out, N, V, D):
    import paper_2203_10991_amd as nm
    gen = torch.Generator().manual_seed(D)
    ids = _ids("frequent", N, V, gen)
    ids[::7], ids[1::50], ids[2::50] = 5, -3, V + 2                         # padding tokens, tokens outside
    wide = torch.full((N, D + 11), float("nan"))
    wide[:, 2:2 + D] = torch.randn(N, D, generator=gen)
    wide = wide.to(gt).to(DEV)
    g, idd = wide[:, 2:2 + D], ids.to(DEV)
    want, size = _want(g.cpu(), ids, V, -3.0, padding=5)
    most = int(torch.bincount(ids[(ids >= 0) & (ids < V)]).max())
    got = nm.nm_embed_grad(g, idd, V, -3.0, padding_idx=5, out_dtype=out)
    assert got.dtype == out
    _check(got, want, size, most)
    assert bool((got[5] == 0).all())
    # into a view: with what was there, or in its place; nothing beside it
    hold = torch.full((V, D + 9), 7.0, dtype=out, device=DEV)
    into = hold[:, 4:4 + D]
    assert nm.nm_embed_grad(g, idd, V, -3.0, padding_idx=5, out=into) is into
    assert torch.equal(into, got)
    nm.nm_embed_grad(g, idd, V, -3.0, padding_idx=5, out=into, accumulate=True)
    before = got.cpu().double()
    eps = 2.0 ** -8 if out == BF16 else 2.0 ** -23
    assert bool(((into.cpu().double() - before - want).abs() <= eps * (before + want).abs() + (most + 4) * 2.0 ** -24 * size + 1e-38).all())
    absent = torch.ones(V, dtype=torch.bool)
    absent[ids[(ids >= 0) & (ids < V) & (ids != 5)]] = False
    assert bool((into[absent.to(DEV)] == 0).all())
    assert bool((hold[:, :4] == 7).all()) and bool((hold[:, 4 + D:] == 7).all())


def test_gradient_without_tokens_and_with_nan():
    import paper_2203_10991_amd as nm
    g = torch.zeros(0, 24, device=DEV)
    assert bool((nm.nm_embed_grad(g, torch.zeros(0, dtype=torch.int64, device=DEV), 33) == 0).all())
    out = torch.ones(33, 24, device=DEV)
    nm.nm_embed_grad(g, torch.zeros(0, dtype=torch.int64, device=DEV), 33, out=out, accumulate=True)
    assert bool((out == 1).all())
    assert nm.nm_embed_grad(torch.zeros(4, 0, device=DEV), torch.zeros(4, dtype=torch.int64, device=DEV), 33).shape == (33, 0)
    g = torch.ones(50, 24, device=DEV)
    g[3], g[4, 0] = float("nan"), float("inf")                              # of a padding token, and of one that counts
    ids = torch.arange(50, device=DEV) % 10
    ids[3] = 9
    got = nm.nm_embed_grad(g, ids, 10, padding_idx=9)
    assert bool(torch.isfinite(got[[0, 1, 2, 3, 5, 6, 7, 8, 9]]).all()) and torch.isinf(got[4, 0]) and bool(torch.isfinite(got[4, 1:]).all())


def test_gradient_on_another_stream_and_from_a_graph():
    import paper_2203_10991_amd as nm
    gen = torch.Generator().manual_seed(2)
    ids, g = _ids("frequent", 9000, 2000, gen).to(DEV), torch.randn(9000, 64, generator=gen).to(DEV)
    want = nm.nm_embed_grad(g, ids, 2000)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = nm.nm_embed_grad(g, ids, 2000)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = nm.nm_embed_grad(g, ids, 2000)
    for k in range(4):
        g.mul_(2)
        ids.add_(1).remainder_(2000)
        graph.replay()
        assert torch.equal(got, nm.nm_embed_grad(g, ids, 2000))
        torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_layer(dtype):
    from paper_2203_10991_amd.autograd import NMEmbedding
    torch.manual_seed(1)
    layer = NMEmbedding(50, 48, padding_idx=3, scale=48 ** 0.5, device=DEV, dtype=dtype)
    ids = torch.randint(0, 50, (4, 30), device=DEV)
    out = layer(ids)
    gy = torch.randn(4, 30, 48, device=DEV).to(dtype)
    out.backward(gy)
    ref = layer.weight.detach().double().cpu().requires_grad_()
    want = torch.nn.functional.embedding(ids.cpu(), ref, padding_idx=3) * 48 ** 0.5
    want.backward(gy.cpu().double())
    eps = 2.0 ** -8 if dtype == BF16 else 2.0 ** -20
    assert bool(((out.detach().cpu().double() - want.detach()).abs() <= eps * want.detach().abs()).all())
    assert layer.weight.grad.dtype == dtype
    assert bool(((layer.weight.grad.cpu().double() - ref.grad).abs() <= eps * ref.grad.abs() + 1e-4).all())
    # the gradient of the function, against differences: it is linear in the table
    if dtype == F32:
        d = torch.randn_like(layer.weight)
        d[3] = 0
        with torch.no_grad():
            a = (layer(ids).double() * gy).sum()
            layer.weight.add_(d)
            b = (layer(ids).double() * gy).sum()
            got = (layer.weight.grad.double() * d).sum()
            size = (layer(ids).detach().double() * gy).abs().sum()
        assert abs(float(b - a - got.detach())) <= 1e-4 * float(size)
    with pytest.raises(ValueError):
        NMEmbedding(5, 4, max_norm=1.0)


def test_refusals():
    import paper_2203_10991_amd as nm
    t, ids = torch.zeros(5, 8, device=DEV), torch.zeros(4, dtype=torch.int64, device=DEV)
    for bad in (lambda: nm.nm_embed(t.cpu(), ids), lambda: nm.nm_embed(t, ids.cpu()), lambda: nm.nm_embed(t[0], ids), lambda: nm.nm_embed_grad(t, ids, 5),
                lambda: nm.nm_embed_grad(t[:4], ids, 5, out=torch.zeros(6, 8, device=DEV)), lambda: nm.nm_embed_grad(t[:4], ids, 5, accumulate=True)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: nm.nm_embed(t.half(), ids), lambda: nm.nm_embed(t, ids.short()), lambda: nm.nm_embed(t, ids, out_dtype=torch.float16),
                lambda: nm.nm_embed_grad(t[:4].half(), ids, 5)):
        with pytest.raises(TypeError):
            bad()
    with pytest.raises(nm.NmError) as e:
        nm.nm_embed_grad(t[:4], ids, 5, out=t)
    assert e.value.status == 5
