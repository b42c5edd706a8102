"""Matrices whose rows share memory -- expanded along their rows, as autograd makes the gradient of a sum over tokens, or overlapping -- give what their copies give, through
the C++ binding and without it."""
import pytest
import torch

from gpu_util import DEV

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(params=["binding", "ctypes"])
def way(request, monkeypatch):
    from paper_2203_10991_amd import api
    api.load()
    if request.param == "ctypes":
        monkeypatch.setattr(api, "_native", api._NoNative)


def _shared(T, C, dtype):
    """(T x C) matrices without rows of their own"""
    row = torch.randn(C + T, device=DEV).to(dtype)
    return [row[:C].expand(T, C), row[:1].expand(T, C), row.as_strided((T, C), (1, 1)), torch.randn(T, 1, device=DEV).to(dtype).expand(T, C)]


def _same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b)) if isinstance(a, tuple) else torch.equal(a, b)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T,C", [(2, 1), (3, 40), (70, 200), (600, 33)])
def test_functions(way, T, C, dtype):
    import paper_2203_10991_amd as nm
    wq, ws = nm.nm_quant_i8(torch.randn(24, C, device=DEV))
    ids = torch.randint(0, 9, (T,), device=DEV)
    for x in _shared(T, C, dtype):
        for f in (nm.nm_quant_i8, nm.nm_quant_i8_t, lambda t: nm.nm_linear_i8(t, wq, ws), lambda t: nm.nm_embed_grad(t, ids, 9), lambda t: nm.nm_embed(t, ids.clamp(max=T - 1)),
                  lambda t: nm.nm_linear_i8(t.reshape(1, T, C), wq, ws), lambda t: nm.nm_embed_grad(t.reshape(1, T, C), ids.reshape(1, T), 9)):
            assert _same(f(x), f(x.contiguous()))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_embedding_in_front_of_a_sum(way, dtype):
    from paper_2203_10991_amd.autograd import NMEmbedding
    layer = NMEmbedding(50, 48, padding_idx=3, device=DEV, dtype=dtype)
    for shape, dims in (((30,), (0,)), ((1, 30), (1,)), ((4, 30), (0, 1)), ((4, 30), (0, 1, 2))):
        ids = torch.randint(0, 50, shape, device=DEV)
        layer.weight.grad = None
        gy = torch.randint(-3, 4, (48,), device=DEV).to(dtype)
        pooled = layer(ids).sum(dims)
        pooled.backward(gy.expand_as(pooled) if pooled.dim() else gy[0])
        count = torch.bincount(ids.flatten(), minlength=50).double()
        count[3] = 0
        want = count[:, None] * (gy if pooled.dim() else gy[:1]).double()
        assert torch.equal(layer.weight.grad.double(), want.expand(50, 48))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("relu", [False, True])
def test_layers_on_expanded_rows(way, dtype, relu):
    """A class token's rows in, a sum over tokens behind: output and gradients are those of the same values with rows of their own."""
    from paper_2203_10991_amd.autograd import NMConfig, NMLinear, NMLinearReLU
    torch.manual_seed(2)
    layer = (NMLinearReLU if relu else NMLinear)(72, 104, cfg=NMConfig(seed=5, dense="i8"), device=DEV, dtype=dtype)
    cls = torch.randn(1, 1, 72, device=DEV).to(dtype)
    gy = torch.randn(104, device=DEV).to(dtype)
    out = []
    for own in (False, True):
        x = (cls.expand(48, 1, 72).contiguous() if own else cls.expand(48, 1, 72)).detach().requires_grad_()
        y = layer(x)
        grad = gy.expand(y.shape)
        out.append((y, *torch.autograd.grad(y, (x, layer.weight, layer.bias), grad.contiguous() if own else grad)))
    assert all(torch.equal(a, b) for a, b in zip(out[0][:3], out[1][:3]))
    # (the bias gradient: the framework's or the library's sum of 48 rows, in an order that goes by the layout: 48 2^-24 of the magnitudes each, rounded once)
    a, b = out[0][3].double(), out[1][3].double()
    assert bool(((a - b).abs() <= 2 * 48 * 2.0 ** -24 * 48 * gy.double().abs() + (2.0 ** -7 * b.abs() if dtype == BF16 else 0)).all())
    x = torch.randn(40, 72, device=DEV).to(dtype).requires_grad_()
    layer(x).sum(0).backward(gy)
    assert x.grad.shape == x.shape and bool(torch.isfinite(x.grad).all())
