"""nm_adamw and NMAdamW against the step in binary64 on the CPU: every combination of types, sizes around a block of 256 and a vector of four,
arrays that start anywhere, more tensors than a launch holds, gradients that are not finite, layouts; 8-bit states against their definition."""
import math

import numpy as np
import pytest
import torch

from gpu_util import DEV

pytestmark = pytest.mark.gpu

B1, B2, EPS, LR, WD = 0.9, 0.999, 1e-8, 1e-2, 0.1
SIZES = [1, 3, 4, 255, 256, 257, 1000, 4096, 4097, 16384 + 5]


def _philox(counter, key):
    """Philox4x32-10 of counters [n, 4] (uint64 arrays of 32-bit words)"""
    c, k, m32 = [counter[:, i].copy() for i in range(4)], list(key), np.uint64(0xffffffff)
    for _ in range(10):
        p0, p1 = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(p1 >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), p1 & m32, (p0 >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), p0 & m32]
        k = [(k[0] + 0x9E3779B9) & 0xffffffff, (k[1] + 0xBB67AE85) & 0xffffffff]
    return np.stack(c, 1)


def _halves(n, number, step, seed):
    quads = -(-n // 4)
    c = np.zeros((quads, 4), dtype=np.uint64)
    c[:, 0], c[:, 2], c[:, 3] = np.arange(quads), number, (1 << 31) + step
    w = _philox(c, (seed & 0xffffffff, seed >> 32)).reshape(-1)[:n]
    return (w & np.uint64(0xffff)).astype(np.float64) / 65536, (w >> np.uint64(16)).astype(np.float64) / 65536


def _values(state):
    codes, scale = state
    return codes.detach().cpu().float().double().reshape(-1) * scale.detach().cpu().double().repeat_interleave(256)[:codes.numel()]


def _step64(p, g, m, v, step):
    m = B1 * m + (1 - B1) * g
    v = B2 * v + (1 - B2) * g * g
    up = LR / (1 - B1 ** step) * m / ((v / (1 - B2 ** step)).sqrt() + EPS)
    return p * (1 - LR * WD) - up, m, v, up


def _near(got, want, size, eps):
    assert bool(((got.detach().cpu().double().reshape(-1) - want).abs() <= eps * size + 1e-37).all())


def _made(n, offset, dtype, gen, scale=1.0, positive=False):
    """n values in the middle of a larger array, `offset` elements behind a 16-byte boundary"""
    x = torch.randn(n + 64, generator=gen) * scale
    return (x.abs() if positive else x).to(dtype).to(DEV)[offset:offset + n]


@pytest.mark.parametrize("param,grad,master", [("float32", "float32", False), ("float32", "bfloat16", False), ("bfloat16", "float32", False),
                                               ("bfloat16", "bfloat16", False), ("bfloat16", "float32", True), ("bfloat16", "bfloat16", True)])
@pytest.mark.parametrize("offset", [0, 1])
def test_binary32_states(param, grad, master, offset):
    import paper_2203_10991_amd as nm
    gen = torch.Generator().manual_seed(3)
    pt, gt = getattr(torch, param), getattr(torch, grad)
    p, g = [_made(n, offset, pt, gen) for n in SIZES], [_made(n, offset, gt, gen, 0.1) for n in SIZES]
    m, v = [_made(n, offset, torch.float32, gen, 0.03) for n in SIZES], [_made(n, offset, torch.float32, gen, 1e-2, True) for n in SIZES]
    w = [x.float() + 1e-3 for x in p] if master else None
    want = [_step64((w[k] if master else p[k]).cpu().double(), g[k].cpu().double(), m[k].cpu().double(), v[k].cpu().double(), 7) for k in range(len(p))]
    around = [x._base.clone() if x._base is not None else None for x in p]
    versions = [x._version for x in p]
    nm.nm_adamw(p, g, m, v, 7, lr=LR, betas=(B1, B2), eps=EPS, weight_decay=WD, masters=w)
    torch.cuda.synchronize()
    for k, (wp, wm, wv, up) in enumerate(want):
        # a few binary32 roundings of each term; bf16: half a unit in the last place
        size = wp.abs() + up.abs()
        _near(m[k], wm, wm.abs() + (1 - B1) * g[k].cpu().double().abs() + (B1 * wm).abs(), 2.0 ** -21)
        _near(v[k], wv, wv, 2.0 ** -21)
        if master:
            _near(w[k], wp, size, 2.0 ** -21)
            assert torch.equal(p[k], w[k].to(torch.bfloat16))
        else:
            _near(p[k], wp, size, 2.0 ** -21 if pt == torch.float32 else 2.0 ** -8 + 2.0 ** -21)
        assert p[k]._version > versions[k]
        if around[k] is not None:                                            # nothing beside the tensor
            b, n = p[k]._base, SIZES[k]
            assert torch.equal(b[:offset], around[k][:offset]) and torch.equal(b[offset + n:], around[k][offset + n:])


@pytest.mark.parametrize("param,grad,master", [("float32", "float32", False), ("float32", "bfloat16", False), ("bfloat16", "float32", False),
                                               ("bfloat16", "bfloat16", False), ("bfloat16", "float32", True), ("bfloat16", "bfloat16", True)])
@pytest.mark.parametrize("offset", [0, 1])
def test_8_bit_states(param, grad, master, offset):
    """Codes are the neighbour that the random word picks, but where the fraction comes within 1e-4 of it; scales are the power of two of the block."""
    import paper_2203_10991_amd as nm
    gen = torch.Generator().manual_seed(4)
    pt, gt, seed, step = getattr(torch, param), getattr(torch, grad), 0x123456789ab, 3
    p, g, m, v = [], [], [], []
    for n in SIZES:
        p.append(_made(n, offset, pt, gen))
        size = torch.randn(n, generator=gen).mul_(3).exp_()                  # magnitudes over many octaves: codes below the smallest normal one
        buf = torch.zeros(n + 64, dtype=gt, device=DEV)
        buf[offset:offset + n] = (torch.randn(n, generator=gen) * size).to(gt)
        if n > 600:
            buf[offset + 256:offset + 512] = 0                               # a block of zeros
        g.append(buf[offset:offset + n])
        pair = []
        for top in (0x100, 0x80):
            codes = torch.randint(0, 0x7f, (n + 64,), generator=gen, dtype=torch.uint8)
            if top == 0x100:
                codes |= (torch.randint(0, 2, (n + 64,), generator=gen, dtype=torch.uint8) << 7)
            if n > 600:
                codes[offset + 256:offset + 512] = 0
            scale = torch.exp2(torch.randint(-12, -6, (-(-n // 256),), generator=gen).float())
            pair.append((codes.to(DEV)[offset:offset + n].view(torch.float8_e4m3fn), scale.to(DEV)))
        m.append(pair[0])
        v.append(pair[1])
    w = [x.float() + 1e-3 for x in p] if master else None
    before = [(_values(m[k]), _values(v[k])) for k in range(len(p))]
    start = [(w[k] if master else p[k]).cpu().double() for k in range(len(p))]
    nm.nm_adamw(p, g, m, v, step, lr=LR, betas=(B1, B2), eps=EPS, weight_decay=WD, masters=w, seed=seed)
    torch.cuda.synchronize()
    for k, n in enumerate(SIZES):
        g64 = g[k].cpu().double()
        wp, wm, wv, up = _step64(start[k], g64, before[k][0], before[k][1] ** 2, step)
        _near(w[k] if master else p[k], wp, wp.abs() + up.abs() * 4, 2.0 ** -21 if master or pt == torch.float32 else 2.0 ** -8 + 2.0 ** -20)
        if master:
            assert torch.equal(p[k], w[k].to(torch.bfloat16))
        for (codes, scale), want, chance in ((m[k], wm, _halves(n, k, step, seed)[0]), (v[k], wv.sqrt(), _halves(n, k, step, seed)[1])):
            want, scale = want.numpy(), scale.cpu().double().numpy()
            code = codes.view(torch.uint8).cpu().numpy().astype(np.int64)
            for b, at in enumerate(range(0, n, 256)):
                block, got = want[at:at + 256], code[at:at + 256]
                top = np.abs(block).max()
                exponent = math.ceil(math.log2(top / 448)) if top > 0 else 0
                assert scale[b] == 2.0 ** exponent or abs(top / 448 / 2.0 ** round(math.log2(top / 448)) - 1) < 1e-6
                y = np.abs(block) / scale[b]
                grid = 2.0 ** (np.maximum(np.floor(np.log2(np.maximum(y, 1e-300))), -6) - 3)
                at_grid = y / grid + chance[at:at + 256]
                low = np.floor(at_grid) * grid
                sure = np.abs(at_grid - np.round(at_grid)) > 1e-4
                value = np.where((got & 0x7f) < 8, (got & 7) * 2.0 ** -9, 2.0 ** ((got >> 3 & 15) - 7.0) * (1 + (got & 7) / 8))
                if codes is v[k][0]:
                    low = np.where((y > 0) & (low == 0), 2.0 ** -9, low)
                assert np.array_equal(value[sure], low[sure]) and np.abs(value - low).max() <= grid.max() * 1.001
                assert bool((np.abs(value - low) <= 1.001 * np.maximum(grid, 2.0 ** -9)).all())
                signs = block < 0
                assert np.array_equal((got >> 7 & 1)[value > 0], signs[value > 0].astype(np.int64))


def test_rounding_of_8_bit_states_has_no_bias():
    """v moves by a hundredth of a step of its codes each time: under gradients of one size it comes to their square.  Rounded to nearest it would not move
    at all.  200 steps at beta2 = 0.99 from sqrt(v) = 1 to a gradient of 0.5: sqrt(v) = 0.574 in exact arithmetic, and the mean over 65536
    elements holds to 2 % (each element's own error, at most a step of 12.5 % a time, averages out; what stays is that of the square of a noisy value)."""
    import paper_2203_10991_amd as nm
    n = 65536
    p, g = torch.zeros(n, device=DEV), torch.full((n,), 0.5, device=DEV)
    m, v = nm.alloc_adamw_state(p, q8=True), nm.alloc_adamw_state(p, q8=True)
    v[0].view(torch.uint8).fill_(0x38)                                        # 1.0
    for step in range(1, 201):
        nm.nm_adamw([p], [g], [m], [v], step, lr=0.0, betas=(0.9, 0.99), seed=11)
    want = math.sqrt(0.25 + 0.75 * 0.99 ** 200)
    assert abs(float(_values(v).mean()) / want - 1) < 0.02
    assert abs(float(_values(m).mean()) / 0.5 - 1) < 0.02
    # the same steps give the same bits, another seed others
    runs = []
    for seed in (5, 5, 6):
        m, v = nm.alloc_adamw_state(p, q8=True), nm.alloc_adamw_state(p, q8=True)
        noise = torch.randn(n, generator=torch.Generator().manual_seed(1)).to(DEV)
        nm.nm_adamw([p], [noise], [m], [v], 1, lr=0.0, seed=seed)
        runs.append(m[0].view(torch.uint8).clone())
    assert torch.equal(runs[0], runs[1]) and not torch.equal(runs[0], runs[2])


@pytest.mark.parametrize("q8", [False, True])
def test_many_tensors_and_a_scale_on_the_device(q8):
    """More tensors than a launch holds, empty ones among them; the gradients' factor from device memory or as a number gives the same bits."""
    import paper_2203_10991_amd as nm
    gen = torch.Generator().manual_seed(5)
    sizes = [(0,), (7,), (300, 5), ()] * 30
    p0 = [torch.randn(s, generator=gen).to(DEV) for s in sizes]
    g = [torch.randn(s, generator=gen).to(DEV) for s in sizes]
    out = []
    for scale in (0.25, torch.tensor([0.25], device=DEV), None):
        p = [x.clone() for x in p0]
        m, v = ([nm.alloc_adamw_state(x, q8) for x in p] for _ in range(2))
        if scale is None:
            for k in range(len(p)):                                          # one by one
                nm.nm_adamw([p[k]], [g[k]], [m[k]], [v[k]], 1, grad_scale=0.25, seed=9, numbers=[k])
        else:
            nm.nm_adamw(p, g, m, v, 1, grad_scale=scale, seed=9)
        out.append([x.clone() for x in p] + [x.view(torch.uint8).clone() if q8 else x for s in m + v for x in (s if q8 else [s])])
    for other in out[1:]:
        assert all(torch.equal(a, b) for a, b in zip(out[0], other))
    assert all(bool((a != b).all()) for a, b in zip(out[0], p0) if a.numel())


@pytest.mark.parametrize("q8", [False, True])
def test_what_is_not_finite_stays_where_it_is(q8):
    import paper_2203_10991_amd as nm
    p = torch.ones(1024, device=DEV)
    g = torch.full((1024,), 0.5, device=DEV)
    g[5], g[300], g[301] = float("nan"), float("inf"), -float("inf")
    m, v = nm.alloc_adamw_state(p, q8), nm.alloc_adamw_state(p, q8)
    nm.nm_adamw([p], [g], [m], [v], 1, seed=1)
    torch.cuda.synchronize()
    bad = torch.zeros(1024, dtype=torch.bool)
    bad[[5, 300, 301]] = True
    values = [_values(s) if q8 else s.cpu() for s in (m, v)]
    assert bool(torch.isnan(p.cpu())[bad].all()) and bool(torch.isfinite(p.cpu())[~bad].all())
    for x in values:
        assert not bool(torch.isfinite(x)[bad].any()) and bool(torch.isfinite(x)[~bad].all()) and bool((x[~bad] > 0).all())


def test_layouts_and_mixed_lists():
    """Parameters in any dense layout; a gradient in another one; tensors of several types in one list."""
    import paper_2203_10991_amd as nm
    gen = torch.Generator().manual_seed(6)
    conv = torch.randn(8, 16, 3, 3, generator=gen).to(DEV).to(memory_format=torch.channels_last)
    turned = torch.randn(40, 24, generator=gen).to(DEV).t()
    low = torch.randn(33, generator=gen).to(torch.bfloat16).to(DEV)
    p = [conv, turned, low]
    g = [torch.randn(8, 16, 3, 3, generator=gen).to(DEV), torch.randn(24, 40, generator=gen).to(torch.bfloat16).to(DEV), torch.randn(33, generator=gen).to(DEV)]
    m, v = [nm.alloc_adamw_state(x) for x in p], [nm.alloc_adamw_state(x) for x in p]
    assert m[0].stride() == conv.stride() and m[1].stride() == turned.stride()
    want = [_step64(x.cpu().double(), y.cpu().double(), torch.zeros_like(x.cpu()).double(), torch.zeros_like(x.cpu()).double(), 1) for x, y in zip(p, g)]
    nm.nm_adamw(p, g, m, v, 1, lr=LR, betas=(B1, B2), eps=EPS, weight_decay=WD, masters=[None, None, low.float()])
    torch.cuda.synchronize()
    for x, (wp, wm, _, up), y in zip(p, want, m):
        eps = 2.0 ** -8 + 2.0 ** -20 if x.dtype == torch.bfloat16 else 2.0 ** -20
        assert bool(((x.cpu().double() - wp).abs() <= eps * (wp.abs() + up.abs())).all())
        assert bool(((y.cpu().double() - wm).abs() <= 2.0 ** -20 * wm.abs()).all())


def test_refusals():
    import paper_2203_10991_amd as nm
    p = torch.zeros(8, 8, device=DEV)
    s = lambda: nm.alloc_adamw_state(p)                                         # noqa: E731
    with pytest.raises(ValueError):
        nm.nm_adamw([p], [p, p], [s()], [s()], 1)
    with pytest.raises(ValueError):
        nm.nm_adamw([p], [torch.zeros(8, device=DEV)], [s()], [s()], 1)
    with pytest.raises(ValueError):
        nm.nm_adamw([p.cpu()], [p.cpu()], [s().cpu()], [s().cpu()], 1)
    with pytest.raises(TypeError):
        nm.nm_adamw([p.half()], [p.clone()], [s()], [s()], 1)
    with pytest.raises(TypeError):
        nm.nm_adamw([p], [p.clone()], [s().double()], [s()], 1)
    with pytest.raises(ValueError):
        nm.nm_adamw([p[:, :4]], [p[:, :4].clone()], [s()[:, :4]], [s()[:, :4]], 1)         # gaps
    with pytest.raises(ValueError):
        nm.nm_adamw([p], [p.clone()], [s().t()], [s()], 1)
    with pytest.raises(ValueError):
        codes, scale = nm.alloc_adamw_state(p, q8=True)
        nm.nm_adamw([p], [p.clone()], [(codes, scale[:0])], [(codes, scale)], 1)
    for bad in (dict(step=0), dict(step=1, betas=(1.0, 0.9)), dict(step=1, eps=-1.0), dict(step=1, lr=float("nan")), dict(step=1, masters=[p.clone()])):
        with pytest.raises(nm.NmError):
            nm.nm_adamw([p], [p.clone()], [s()], [s()], **bad)
    with pytest.raises(nm.NmError) as e:
        one = s()
        nm.nm_adamw([p], [p.clone()], [one], [one], 1)
    assert e.value.status == 5
    assert bool((p == 0).all())


@pytest.mark.parametrize("states,master", [("f32", False), ("f32", True), ("q8", True)])
def test_optimizer_trains_and_comes_back_from_its_state(states, master):
    """A least-squares problem: the optimizer brings the loss down as torch's does, and one made from its state_dict goes on bit for bit."""
    from paper_2203_10991_amd.optim import NMAdamW
    gen = torch.Generator().manual_seed(8)
    x, y = torch.randn(256, 64, generator=gen).to(DEV), torch.randn(256, 32, generator=gen).to(DEV)
    w0 = torch.randn(32, 64, generator=gen).mul_(0.1).to(DEV)

    def run(opt, w, steps):
        for _ in range(steps):
            opt.zero_grad()
            loss = (x @ w.float().t() - y).square().mean()
            loss.backward()
            opt.step()
        return float(loss.detach())
    dtype = torch.bfloat16 if master else torch.float32
    w = torch.nn.Parameter(w0.to(dtype, copy=True))
    idle = torch.nn.Parameter(torch.ones(3, device=DEV))                       # without a gradient
    opt = NMAdamW([{"params": [idle]}, {"params": [w], "weight_decay": 0.0}], lr=1e-2, states=states, master=master, seed=4)
    run(opt, w, 60)
    other = torch.nn.Parameter(w.detach().clone())
    idle2 = torch.nn.Parameter(torch.ones(3, device=DEV))
    opt2 = NMAdamW([{"params": [idle2]}, {"params": [other], "weight_decay": 0.0}], lr=1e-2, states=states, master=master, seed=4)
    opt2.load_state_dict(opt.state_dict())
    for k, t in opt.state[w].items():
        u = opt2.state[other][k]
        assert (t.dtype == u.dtype and t.data_ptr() != u.data_ptr()) if isinstance(t, torch.Tensor) else t == u
    a, b = run(opt, w, 60), run(opt2, other, 60)
    assert a == b and torch.equal(w, other)
    ref = torch.nn.Parameter(w0.clone())
    want = run(torch.optim.AdamW([ref], lr=1e-2, weight_decay=0.0), ref, 120)
    first = float((x @ w0.t() - y).square().mean())
    assert abs(a - want) < 0.05 * (first - want)
    assert bool((idle == 1).all()) and not opt.state[idle]
