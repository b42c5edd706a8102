"""nm_rotary and rotary_freqs against binary64 on the CPU: both layouts, parts of a head, positions from negative to past 2^31, strides, in place."""
import math

import pytest
import torch

from gpu_util import DEV

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def _want(x, freqs, positions, interleaved, scale=1.0, inverse=False):
    """(value, bound): the pairs as complex numbers times a unit one.  Bound: the angle's turn is rounded once (2^-25 of half a turn: 2 pi 2^-26 of an angle; in binary64
    before), cosine and sine are off by 2 steps of one (2^-23), as products and sum are by 3 roundings of theirs, and the result by its own."""
    r, X = 2 * freqs.numel(), x.double()
    z = torch.polar(torch.ones((), dtype=torch.float64), positions.double().unsqueeze(-1) * freqs.cpu() * (-1 if inverse else 1)).unsqueeze(2) * scale
    pairs = X[..., :r].unflatten(-1, (r // 2, 2)) if interleaved else X[..., :r].unflatten(-1, (2, r // 2)).transpose(-1, -2)
    turned = torch.view_as_real(torch.complex(pairs[..., 0].contiguous(), pairs[..., 1].contiguous()) * z)
    size = pairs.abs().sum(-1, keepdim=True).expand_as(pairs) * abs(scale)
    back = (lambda t: t.flatten(-2)) if interleaved else (lambda t: t.transpose(-1, -2).flatten(-2))
    value, bound = X.clone(), torch.zeros_like(X)
    value[..., :r] = back(turned)
    # a position times a frequency has 53 bits too: 2^-52 of the angle, here as there
    angle = (positions.double().abs().max() if positions.numel() else 0) * freqs.abs().max().item() * 2.0 ** -50
    bound[..., :r] = back(size) * (2 * math.pi * 2.0 ** -26 + 2.0 ** -22 + 4 * 2.0 ** -24 + angle)
    half = torch.finfo(x.dtype).eps / 2
    bound[..., :r] += half * (value[..., :r].abs() + bound[..., :r])
    return value, bound


def _check(got, want):
    off = (got.cpu().double() - want[0]).abs()
    assert got.shape == want[0].shape and bool((off <= want[1] + 1e-37).all()), f"{(off / (want[1] + 1e-37)).max().item():.3g} of the bound"


CASES = [(1, 1, 1, 2, 2), (2, 3, 1, 8, 4), (1, 70, 3, 64, 64), (2, 33, 5, 80, 32), (3, 7, 2, 40, 22), (1, 9, 4, 128, 96), (2, 5, 72, 128, 128), (1, 4, 2, 30, 10), (1, 3, 2, 7, 6), (2, 300, 1, 16, 16),
         (1, 2, 3, 1024, 1024), (1, 2, 300, 24, 24), (1, 2, 2, 1023, 1022), (5, 1, 20, 64, 64)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("B,T,H,D,part", CASES)
def test_against_binary64(B, T, H, D, part, interleaved, dtype):
    import paper_2203_10991_amd as nm
    gen = torch.Generator().manual_seed(D + part)
    x = torch.randn(B, T, H, D, generator=gen).to(dtype)
    freqs = nm.rotary_freqs(part, device=DEV)
    xd = x.to(DEV)
    _check(nm.nm_rotary(xd, freqs, interleaved=interleaved), _want(x, freqs, torch.arange(T).expand(B, T), interleaved))
    far = torch.randint(-(1 << 20), 1 << 20, (B, T), generator=gen)
    got = nm.nm_rotary(xd, freqs, far.to(DEV), interleaved=interleaved, scale=1.3)
    _check(got, _want(x, freqs, far, interleaved, 1.3))
    assert torch.equal(got, nm.nm_rotary(xd, freqs, far.int().to(DEV), interleaved=interleaved, scale=1.3))
    shared = far[0]
    _check(nm.nm_rotary(xd, freqs, shared.to(DEV), interleaved=interleaved, inverse=True), _want(x, freqs, shared.expand(B, T), interleaved, inverse=True))
    place = xd.clone()
    assert nm.nm_rotary(place, freqs, far.to(DEV), interleaved=interleaved, scale=1.3, out=place) is place and torch.equal(place, got)


def test_positions_past_31_bits():
    import paper_2203_10991_amd as nm
    x, freqs = torch.randn(1, 3, 2, 16), nm.rotary_freqs(16, device=DEV)
    pos = torch.tensor([1 << 31, (1 << 33) + 5, -(1 << 32)])
    _check(nm.nm_rotary(x.to(DEV), freqs, pos.to(DEV)), _want(x, freqs, pos[None], False))


@pytest.mark.parametrize("interleaved", [False, True])
def test_inverse_is_the_gradient(interleaved):
    """<g, turned x> = <turned back g, x>, up to the roundings of both"""
    import paper_2203_10991_amd as nm
    gen = torch.Generator().manual_seed(3)
    x, g = (torch.randn(2, 9, 3, 24, generator=gen) for _ in range(2))
    freqs = nm.rotary_freqs(16, device=DEV)
    pos = torch.arange(9).expand(2, 9) * 1000
    fwd, back = nm.nm_rotary(x.to(DEV), freqs, pos.to(DEV), interleaved, 0.7), nm.nm_rotary(g.to(DEV), freqs, pos.to(DEV), interleaved, 0.7, inverse=True)
    bound = (_want(x, freqs, pos, interleaved, 0.7)[1] * g.abs()).sum() + (_want(g, freqs, pos, interleaved, 0.7, True)[1] * x.abs()).sum()
    # the elements behind the part pass unscaled on both sides
    assert abs((fwd.cpu().double() * g.double()).sum() - (back.cpu().double() * x.double()).sum()) <= bound


def test_views():
    """parts of a wider tensor, heads before tokens, elements apart, rows that start anywhere; what lies outside stays as it was"""
    import paper_2203_10991_amd as nm
    x = torch.randn(2, 11, 6, 33, device=DEV).to(BF16)
    freqs = nm.rotary_freqs(8, device=DEV)
    part = x[:, :, 1:4, 1:17]
    want = nm.nm_rotary(part.contiguous(), freqs)
    assert torch.equal(nm.nm_rotary(part, freqs), want)
    assert torch.equal(nm.nm_rotary(part.transpose(1, 2).contiguous().transpose(1, 2), freqs), want)
    assert torch.equal(nm.nm_rotary(torch.stack((part, part), -1)[..., 0], freqs), want)
    assert torch.equal(nm.nm_rotary(part[:1].expand(2, -1, -1, -1), freqs), want[:1].expand(2, -1, -1, -1))
    kept = x.clone()
    nm.nm_rotary(part, freqs, out=part)
    assert torch.equal(part, want)
    kept[:, :, 1:4, 1:17] = want
    assert torch.equal(x, kept)


def test_nothing_to_do_streams_and_a_graph():
    import paper_2203_10991_amd as nm
    freqs = nm.rotary_freqs(8, device=DEV)
    for shape in ((0, 3, 2, 8), (2, 0, 2, 8), (2, 3, 0, 8)):
        assert nm.nm_rotary(torch.zeros(shape, device=DEV), freqs).shape == shape
    x = torch.randn(4, 50, 3, 8, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        apart = nm.nm_rotary(x, freqs)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(apart, nm.nm_rotary(x, freqs))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = nm.nm_rotary(x, freqs)
    for _ in range(3):
        x.normal_()
        graph.replay()
        assert torch.equal(held, nm.nm_rotary(x, freqs))


def test_frequencies():
    import paper_2203_10991_amd as nm
    f = nm.rotary_freqs(64, 500.0)
    assert f.dtype == torch.float64 and torch.equal(f, torch.tensor([500.0 ** -(2 * j / 64) for j in range(32)], dtype=torch.float64).to(f)) or bool(((f - torch.tensor(
        [500.0 ** -(2 * j / 64) for j in range(32)], dtype=torch.float64)).abs() <= 1e-14).all())
    assert bool(((nm.rotary_freqs(64, scaling="linear", factor=4.0) * 4 - nm.rotary_freqs(64)).abs() <= 1e-15).all())
    b = nm.rotary_freqs(64, scaling="base", factor=4.0) / nm.rotary_freqs(64)
    assert abs(b[0] - 1) < 1e-14 and abs(b[-1] - 0.25) < 1e-14 and bool((b[1:] < b[:-1]).all())
    p = nm.rotary_freqs(64, scaling="parts", factor=4.0, original_length=2048) / nm.rotary_freqs(64)
    turns = nm.rotary_freqs(64) * 2048 / (2 * math.pi)
    assert bool(((p[turns >= 32] - 1).abs() < 1e-14).all()) and bool(((p[turns <= 1] - 0.25).abs() < 1e-14).all()) and bool((p[1:] <= p[:-1] + 1e-14).all())
    assert nm.rotary_freqs(2, scaling="base", factor=4.0).tolist() == [1.0]
    for bad in (lambda: nm.rotary_freqs(3), lambda: nm.rotary_freqs(0), lambda: nm.rotary_freqs(8, scaling="other"), lambda: nm.rotary_freqs(8, scaling="parts"), lambda: nm.rotary_freqs(8, -1.0)):
        with pytest.raises(ValueError):
            bad()


def test_refusals():
    import paper_2203_10991_amd as nm
    x, freqs = torch.zeros(2, 5, 3, 16, device=DEV), nm.rotary_freqs(16, device=DEV)
    for call in (lambda: nm.nm_rotary(x.cpu(), freqs), lambda: nm.nm_rotary(x[0], freqs), lambda: nm.nm_rotary(x, freqs, torch.zeros(4, dtype=torch.int64, device=DEV)),
                 lambda: nm.nm_rotary(x, freqs, torch.zeros(5, dtype=torch.int64)), lambda: nm.nm_rotary(x, freqs, out=x[:1]),
                 lambda: nm.nm_rotary(x.transpose(2, 3), freqs[:1], out=x)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: nm.nm_rotary(x.half(), freqs), lambda: nm.nm_rotary(x, freqs.float()), lambda: nm.nm_rotary(x, freqs.cpu()), lambda: nm.nm_rotary(x, freqs, torch.zeros(5, device=DEV))):
        with pytest.raises(TypeError):
            call()
    wide = torch.zeros(2, 5, 4, 16, device=DEV)
    for call in (lambda: nm.nm_rotary(x, nm.rotary_freqs(18, device=DEV)), lambda: nm.nm_rotary(wide[:, :, :3], freqs, out=wide[:, :, 1:]), lambda: nm.nm_rotary(x, freqs, scale=float("nan")),
                 lambda: nm.nm_rotary(torch.zeros(1, 1, 1, 1026, device=DEV), freqs), lambda: nm.nm_rotary(x, freqs, out=wide[:, :, :1].expand(2, 5, 3, 16))):
        with pytest.raises(nm.NmError):
            call()


@pytest.mark.parametrize("interleaved", [False, True])
def test_cosines_and_sines_of_unrounded_angles(interleaved):
    """Pairs (1, 0), which become the cosine and the sine themselves.  The 2-norm of their errors stays below that of exact functions of a fraction of a turn rounded to binary32, rounded once:
    whatever rounds the fraction has that error, and its functions' own beside it"""
    import paper_2203_10991_amd as nm
    T, part = 4000, 64
    freqs = nm.rotary_freqs(part, 300.0)
    pos = torch.arange(T) * 261 + 7
    x = torch.zeros(1, T, 1, part)
    x[..., 0::2 if interleaved else 1][..., :part // 2] = 1.0
    y = nm.nm_rotary(x.to(DEV), freqs.to(DEV), pos.to(DEV), interleaved).cpu().double()[0, :, 0]
    got = torch.stack((y[:, 0::2], y[:, 1::2]) if interleaved else (y[:, :part // 2], y[:, part // 2:]))
    angle = pos.double()[:, None] * freqs
    want = torch.stack((angle.cos(), angle.sin()))
    turn = angle / (2 * math.pi)
    rounded = (turn - turn.round()).float().double() * 2 * math.pi
    limit = (torch.stack((rounded.cos(), rounded.sin())).float().double() - want).norm()
    assert float((got - want).norm()) < float(limit), float((got - want).norm() / limit)
