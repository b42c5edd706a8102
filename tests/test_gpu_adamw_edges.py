"""NMAdamW and nm_adamw at their edges: captured graphs, steps that fail, second moments below binary32's normal numbers."""
import pytest
import torch

from gpu_util import DEV

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("states", ["f32", "q8"])
def test_a_step_is_not_captured(states):
    from paper_2203_10991_amd.optim import NMAdamW
    w = torch.nn.Parameter(torch.ones(300, device=DEV))
    opt = NMAdamW([w], lr=0.1, states=states)
    w.grad = torch.ones(300, device=DEV)
    opt.step()
    torch.cuda.synchronize()
    before, x = w.detach().clone(), torch.zeros(4, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        x.add_(1)
        with pytest.raises(RuntimeError, match="captured"):
            opt.step()
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert bool((x == 3).all()) and torch.equal(w, before) and opt.state[w]["step"] == 1
    opt.step()
    assert opt.state[w]["step"] == 2 and bool((w < before).all())


def test_a_tensor_of_more_workgroups_than_a_grid_has():
    """2^34 elements and more are 2^32 threads"""
    import paper_2203_10991_amd as nm
    n = (1 << 34) + 1111
    p, g = torch.zeros(n, dtype=torch.bfloat16, device=DEV), torch.zeros(n, dtype=torch.bfloat16, device=DEV)
    m, v = (nm.alloc_adamw_state(p, q8=True) for _ in range(2))
    tail = 3000
    parts = [slice(0, tail), slice((1 << 33) - 1024, (1 << 33) - 1024 + tail), slice(n - tail, n)]
    small = torch.randn(tail, device=DEV).to(torch.bfloat16), torch.randn(tail, device=DEV).to(torch.bfloat16)
    for at in parts:
        p[at], g[at] = small
    nm.nm_adamw([p], [g], [m], [v], 1, lr=0.1, seed=3)
    ps, gs = small[0].clone(), small[1]
    ms, vs = (nm.alloc_adamw_state(ps) for _ in range(2))
    nm.nm_adamw([ps], [gs], [ms], [vs], 1, lr=0.1)
    for at in parts:
        assert torch.equal(p[at], ps)
        assert bool((m[0][at].view(torch.uint8) != 0).any())
    assert bool((p[tail:1 << 20] == 0).all()) and bool((p[n - (1 << 20):n - tail] == 0).all())
    del p, g, m, v
    torch.cuda.empty_cache()


@pytest.mark.parametrize("n", [4096, 4099])
@pytest.mark.parametrize("param", [torch.float32, torch.bfloat16])
def test_second_moments_below_the_normal_numbers(n, param):
    """v from 2^-148 to 2^-90, halved exactly by beta2 = 0.5 with a gradient of zero, m near its root, eps = 0: the step is lr m' / (sqrt(v') sqrt(2)) twice over, to a few
    roundings of binary32 (and half a unit of a bf16 parameter)."""
    import paper_2203_10991_amd as nm
    gen = torch.Generator().manual_seed(n)
    v = torch.exp2(torch.randint(-148, -90, (n,), generator=gen).double()) * (1 + torch.randint(0, 2, (n,), generator=gen))
    m = (v.sqrt() * torch.randn(n, generator=gen).double()).float()
    v = v.float()
    assert bool((v > 0).all()) and int((v < 2.0 ** -126).sum()) > n // 4
    p0 = torch.randn(n, generator=gen).to(param)
    p, md, vd = p0.to(DEV), m.to(DEV), v.to(DEV)
    nm.nm_adamw([p], [torch.zeros(n, device=DEV)], [md], [vd], 1, lr=0.5, betas=(0.5, 0.5), eps=0.0, weight_decay=0.0)
    assert torch.equal(vd.cpu(), v / 2) and torch.equal(md.cpu(), m / 2)
    up = 0.5 / 0.5 * (m.double() / 2) / ((v.double() / 2).sqrt() * 2.0 ** 0.5)
    want = p0.double() - up
    eps = 2.0 ** -21 + (2.0 ** -8 if param == torch.bfloat16 else 0)
    assert bool(((p.cpu().double() - want).abs() <= eps * (p0.double().abs() + up.abs())).all())
