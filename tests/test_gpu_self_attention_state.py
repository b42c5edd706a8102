"""What NMSelfAttention keeps between calls: its frequencies, whichever call comes first."""
import copy

import pytest
import torch

from gpu_util import DEV

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


def _layer(**kw):
    from paper_2203_10991_amd.autograd import NMConfig, NMSelfAttention
    torch.manual_seed(5)
    return NMSelfAttention(64, 4, 2, cfg=NMConfig(seed=1), **{**dict(device=DEV, dtype=BF16), **kw})


def _train(layer, x):
    x = x.detach().clone().requires_grad_()
    y = layer(x)
    dx, db = torch.autograd.grad(y, (x, layer.proj.bias), torch.ones_like(y))
    return y.detach(), dx, db


def test_an_evaluation_in_front_of_training():
    """under inference_mode and no_grad, as built and after a move from the host"""
    x = torch.randn(2, 20, 64, device=DEV).to(BF16)
    want = _train(_layer(), x)
    for first in (torch.inference_mode, torch.no_grad):
        for layer in (_layer(), _layer(device="cpu").to(DEV), copy.deepcopy(_layer())):
            layer.load_state_dict(_layer().state_dict())
            with first():
                y = layer(x)
            assert torch.equal(y, want[0])
            assert all(torch.equal(a, b) for a, b in zip(_train(layer, x), want))


def test_built_on_the_meta_device():
    x = torch.randn(1, 9, 64, device=DEV).to(BF16)
    with torch.device("meta"):
        layer = _layer(device=None)
    layer = layer.to_empty(device=DEV)
    layer.load_state_dict(_layer().state_dict())
    assert all(torch.equal(a, b) for a, b in zip(_train(layer, x), _train(_layer(), x)))


def test_the_first_call_captured():
    """a layer of its own for the graph; libraries and streams are warm from another one"""
    x = torch.randn(2, 20, 64, device=DEV).to(BF16)
    other, layer = _layer(), _layer()
    with torch.no_grad():
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            other(x)
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            held = layer(x)
        for _ in range(3):
            want = other(x)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(held, want)
            x.copy_(torch.randn(x.shape, device=DEV))


def test_saved_and_loaded_onto_the_host():
    """(a file of this test's own) ... and moved back"""
    import io
    x = torch.randn(1, 9, 64, device=DEV).to(BF16)
    layer = _layer()
    want = _train(layer, x)
    file = io.BytesIO()
    torch.save(layer, file)
    file.seek(0)
    again = torch.load(file, map_location="cpu", weights_only=False)
    assert again.qkv.weight.device.type == "cpu"
    # (the configuration's state travels with the module; its seed's step is the same)
    assert all(torch.equal(a, b) for a, b in zip(_train(again.to(DEV), x), want))
