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
