"""The operators together: layers with 8-bit integer dense products, and the example's training steps."""
import importlib.util
import os

import pytest
import torch

from gpu_util import DEV, kernels_of

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("relu", [False, True])
def test_layers_with_8_bit_dense_products(dtype, relu):
    """Forward and input gradient are nm_linear_i8's bit for bit and near the dense ones; the weight and bias gradients are those of the layer without."""
    import paper_2203_10991_amd as nm
    from paper_2203_10991_amd.autograd import NMConfig, NMLinear, NMLinearReLU
    torch.manual_seed(3)
    cls = NMLinearReLU if relu else NMLinear
    layer = cls(72, 104, cfg=NMConfig(seed=5, dense="i8"), device=DEV, dtype=dtype)
    plain = cls(72, 104, cfg=NMConfig(seed=5), device=DEV, dtype=dtype)
    plain.load_state_dict(layer.state_dict())
    x = torch.randn(2, 40, 72, device=DEV).to(dtype).requires_grad_()
    gy = torch.randn(2, 40, 104, device=DEV).to(dtype)
    y = layer(x)
    assert torch.equal(y, nm.nm_linear_i8(x.detach(), *nm.nm_quant_i8(layer.weight.detach()), layer.bias.detach(), relu=relu))
    dx, dw, db = torch.autograd.grad(y, (x, layer.weight, layer.bias), gy)
    g = gy * (y > 0).to(dtype) if relu else gy
    assert torch.equal(dx, nm.nm_linear_i8(g.reshape(-1, 104), *nm.nm_quant_i8_t(layer.weight.detach())).reshape(x.shape))
    yp = plain(x)
    dxp, dwp, dbp = torch.autograd.grad(yp, (x, plain.weight, plain.bias), gy)
    # 127 steps of each row's and channel's largest value, rounded to nearest on both sides: about 1 % of the products' 2-norm
    for a, b in ((y, yp), (dx, dxp)):
        assert float((a.detach().double() - b.detach().double()).norm() / b.detach().double().norm()) < (0.1 if relu else 0.03)
    if not relu:
        assert torch.equal(dw, dwp) and torch.equal(db, dbp)
    names = kernels_of(lambda: layer(x.detach()))
    assert any("gemm_i8" in k for k in names)
    with pytest.raises(ValueError):
        cls(72, 104, cfg=NMConfig(dense="i4"), device=DEV, dtype=dtype)(x)


def test_second_derivatives_take_the_dense_way():
    from paper_2203_10991_amd.autograd import NMConfig, NMLinear
    layer = NMLinear(16, 24, cfg=NMConfig(dense="i8"), device=DEV)
    x, gy = torch.randn(32, 16, device=DEV, requires_grad=True), torch.randn(32, 24, device=DEV, requires_grad=True)
    dx, = torch.autograd.grad(layer(x), x, gy, create_graph=True)
    second, = torch.autograd.grad(dx.sum(), gy)
    assert torch.allclose(second, layer.weight.detach().sum(1).expand(32, 24), atol=1e-5)


def test_the_example_learns():
    spec = importlib.util.spec_from_file_location("lm_step", os.path.join(ROOT, "examples", "lm_step.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    first = mod.train(60)
    assert first[0] > 5.0 and first[-1] < 0.6 * first[0]
    plain = mod.train(60, dense="native", states="f32")
    assert abs(first[-1] - plain[-1]) < 0.25 * plain[0]
