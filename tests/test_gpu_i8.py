"""nm_quant_i8, nm_quant_i8_t, nm_gemm_i8 and nm_linear_i8 against binary64: codes and scales exactly, products against exact integer sums, at the edges of
tiles, stages of 128 bytes, chunks of 16 and groups of eight features; odd sizes and strides, what stands behind the rows, rows that are zero or not finite."""
import numpy as np
import pytest
import torch

from gpu_util import DEV, kernels_of

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def _codes(x):
    """the definition, in binary32 on the CPU"""
    x = x.detach().cpu().float().numpy()
    top = np.abs(x).max(1, keepdims=True) if x.shape[1] else np.zeros((x.shape[0], 1), np.float32)
    q, s = np.zeros(x.shape, np.int8), np.zeros(x.shape[0], np.float32)
    for r in range(x.shape[0]):
        a = top[r, 0]
        if not np.isfinite(a):
            s[r] = np.nan
        elif a >= 2.0 ** -110:
            q[r], s[r] = np.rint(x[r] * (np.float32(127) * (np.float32(1) / a))).astype(np.int8), a / np.float32(127)
    return torch.from_numpy(q), torch.from_numpy(s)


def _view(t, left, right, fill):
    """t inside a wider tensor, `fill` around it"""
    wide = torch.full((t.shape[0] + 2, left + t.shape[1] + right), fill, dtype=t.dtype, device=DEV)
    wide[1:-1, left:left + t.shape[1]] = t.to(DEV)
    return wide[1:-1, left:left + t.shape[1]]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("R,C", [(1, 1), (3, 7), (5, 8), (70, 33), (4, 512), (9, 513), (300, 1000), (2, 1025), (7, 4096), (3, 4104), (2, 8193), (5, 20001), (200, 2112), (130, 4160), (257, 2080)])
def test_codes(dtype, R, C):
    import paper_2203_10991_amd as nm
    gen = torch.Generator().manual_seed(R + C)
    x = (torch.randn(R, C, generator=gen) * torch.randn(R, 1, generator=gen).mul_(3).exp_()).to(dtype)
    x[R // 2, :C // 2] = 0
    for t in (x.to(DEV), _view(x, 8, 24, float("nan")), _view(x, 3, 2, float("nan"))):
        q, s = nm.nm_quant_i8(t)
        want, ws = _codes(x)
        assert torch.equal(q.cpu(), want) and torch.equal(s.cpu(), ws)
        assert q.stride(0) % 128 == 0 or R == 1
        assert bool((q._base[:, C:] == 0).all()) if q._base is not None else q.shape[1] % 128 == 0
        q, s = nm.nm_quant_i8_t(t)
        want, ws = _codes(x.t())
        assert torch.equal(q.cpu(), want) and torch.equal(s.cpu(), ws)
        assert bool((q._base[:, R:] == 0).all()) if q._base is not None else q.shape[1] % 128 == 0


def test_codes_of_rows_without_a_scale():
    import paper_2203_10991_amd as nm
    x = torch.randn(9, 40)
    x[1], x[2, 3], x[3, 0], x[4] = 0, float("nan"), float("inf"), 1e-38
    x[5] *= 1e30
    x[6] *= 1e-30
    x[7] = -0.0
    for f, t in ((nm.nm_quant_i8, x), (nm.nm_quant_i8_t, x.t().contiguous())):
        q, s = f(t.to(DEV))
        want, ws = _codes(x)
        assert torch.equal(q.cpu(), want) and torch.equal(torch.nan_to_num(s.cpu(), nan=7.0), torch.nan_to_num(ws, nan=7.0))
    y = nm.nm_linear_i8(x.to(DEV), *nm.nm_quant_i8(torch.randn(24, 40, device=DEV)), torch.ones(24, device=DEV), relu=True)
    bad = torch.zeros(9, dtype=torch.bool)
    bad[[2, 3]] = True
    assert bool(torch.isnan(y.cpu()[bad]).all()) and bool(torch.isfinite(y.cpu()[~bad]).all()) and bool((y.cpu()[[1, 4, 7]] == 1).all())
    assert nm.nm_quant_i8(torch.zeros(0, 5, device=DEV))[0].shape == (0, 5) and bool((nm.nm_quant_i8(torch.zeros(5, 0, device=DEV))[1] == 0).all())
    assert bool((nm.nm_quant_i8_t(torch.zeros(0, 5, device=DEV))[1] == 0).all()) and nm.nm_quant_i8_t(torch.zeros(5, 0, device=DEV))[0].shape == (0, 5)


def _random_codes(R, C, gen, layout):
    """codes over the whole range, in the layout of nm_quant_i8 or in rows of 16-byte multiples with 99s behind them"""
    q = torch.randint(-127, 128, (R, C), generator=gen, dtype=torch.int8)
    ld = -(-C // 128) * 128 if layout == "padded" else -(-C // 16) * 16 + 16
    wide = torch.full((R, ld), 0 if layout == "padded" else 99, dtype=torch.int8, device=DEV)
    wide[:, :C] = q.to(DEV)
    return q, wide[:, :C]


def _check(y, q, xs, w, ws, bias, relu):
    """Integer sums are exact in binary64.  Conversion, two products and a sum in binary32, half a unit in the last place of the result."""
    product = (q.double() @ w.double().t()) * (xs.double()[:, None] * ws.double())
    want = product + (0 if bias is None else bias.cpu().double())
    size = product.abs() + (0 if bias is None else bias.cpu().double().abs())
    if relu:
        want = want.clamp_min(0)
    eps = 2.0 ** -8 * want.abs() if y.dtype == BF16 else 0
    assert y.shape == want.shape
    assert bool(((y.cpu().double() - want).abs() <= 2.0 ** -21 * size + eps).all())


SIZES = [(1, 1, 1), (1, 4096, 1024), (2, 33, 16), (16, 40, 127), (17, 8, 128), (31, 129, 129), (33, 1000, 250), (64, 64, 384), (65, 72, 4096), (100, 1333, 1001),
         (197, 264, 256), (300, 135, 2050), (1, 300, 8192), (7, 5000, 515), (32, 70, 3000), (32, 16, 20000), (33, 70, 3000), (5, 1, 40), (512, 512, 640)]
# each tile, for bf16 and binary32 results: one of them to a workgroup and several, ragged on every side
TILES = [(1010, 956, 510, BF16, "2, 2, 1, 1, 4"), (2471, 1608, 118, BF16, "2, 2, 1, 1, 4"), (437, 838, 68, F32, "2, 2, 1, 1, 4"), (40, 36000, 300, F32, "2, 2, 1, 1, 4"), (914, 1381, 503, BF16, "2, 2, 2, 1, 3"), (13379, 1184, 189, BF16, "2, 2, 2, 1, 3"),
         (914, 1381, 503, F32, "2, 2, 2, 1, 3"), (12187, 337, 1947, F32, "2, 2, 2, 1, 3"), (12187, 337, 1947, BF16, "2, 2, 2, 2, 2"), (10270, 2192, 1508, BF16, "2, 2, 2, 2, 2"),
         (6303, 935, 2390, F32, "2, 2, 2, 2, 2"), (10270, 2189, 1508, F32, "2, 2, 2, 2, 2"), (7484, 482, 2938, BF16, "2, 4, 2, 1, 4"), (7484, 482, 2938, F32, "2, 4, 2, 1, 4"),
         (6343, 2547, 128, F32, "2, 4, 2, 1, 4"), (6343, 2547, 127, BF16, "2, 4, 4, 2, 2"), (9727, 3107, 1251, BF16, "2, 4, 4, 2, 2"), (12052, 1187, 2622, F32, "2, 4, 4, 2, 2")]
# few tokens, or few features: blocks of 16 or 32 tokens and of 16 or 32 features
FEW = [(1, 4096, 1024, "1, 2, false"), (16, 70, 3000, "1, 1, false"), (9, 9000, 500, "1, 2, false"), (17, 70, 3000, "1, 1, false"), (32, 9001, 1300, "2, 2, false"),
       (600, 200, 2001, "1, 2, false"), (1000, 200, 2001, "1, 2, false"), (700, 90, 77, "1, 2, false"), (64, 4096, 1023, "1, 2, false"), (2771, 65, 77, "1, 2, false"),
       (2231, 113, 61, "1, 2, false"), (500, 1000, 4001, "2, 2, false"), (130, 300, 9000, "1, 1, false")]


@pytest.mark.parametrize("layout", ["padded", "loose"])
@pytest.mark.parametrize("out", [F32, BF16])
@pytest.mark.parametrize("T,O,I", SIZES)
def test_product(T, O, I, out, layout):
    import paper_2203_10991_amd as nm
    gen = torch.Generator().manual_seed(T + O + I)
    q, xq = _random_codes(T, I, gen, layout)
    w, wq = _random_codes(O, I, gen, layout)
    xs, ws = torch.rand(T, generator=gen) + 0.1, torch.rand(O, generator=gen) + 0.1
    for bias, relu in ((None, False), (torch.randn(O, generator=gen) * 1e3, True), ((torch.randn(O, generator=gen) * 1e3).to(BF16), False)):
        b = None if bias is None else bias.to(DEV)
        y = nm.nm_gemm_i8(xq, xs.to(DEV), wq, ws.to(DEV), b, relu=relu, out_dtype=out)
        assert y.dtype == out
        _check(y, q, xs, w, ws, bias, relu)


def _route(T, O, I, out):
    import paper_2203_10991_amd as nm
    gen = torch.Generator().manual_seed(T)
    q, xq = _random_codes(T, I, gen, "loose")
    w, wq = _random_codes(O, I, gen, "loose")
    xs, ws, bias = torch.rand(T, generator=gen) + 0.1, torch.rand(O, generator=gen) + 0.1, torch.randn(O, generator=gen) * 1e3
    args = (xq, xs.to(DEV), wq, ws.to(DEV), bias.to(DEV))
    _check(nm.nm_gemm_i8(*args, out_dtype=out), q, xs, w, ws, bias, False)
    return kernels_of(lambda: nm.nm_gemm_i8(*args, out_dtype=out))


@pytest.mark.parametrize("T,O,I,out,kernel", TILES)
def test_every_tile(T, O, I, out, kernel):
    names = _route(T, O, I, out)
    assert any(f"gemm_i8_kernel<{kernel}, " in k for k in names), names


@pytest.mark.parametrize("T,O,I,kernel", FEW)
def test_few_tokens_or_features(T, O, I, kernel):
    names = _route(T, O, I, BF16)
    assert any(f"gemm_i8_few_kernel<{kernel}>" in k for k in names), names


@pytest.mark.parametrize("T,I,fused", [(1, 1024, True), (4, 4000, True), (4, 4100, False), (1, 16000, True), (1, 17000, False), (5, 64, False)])
def test_tokens_rounded_inside_the_product(T, I, fused):
    import paper_2203_10991_amd as nm
    wq, ws = nm.nm_quant_i8(torch.randn(100, I, device=DEV))
    x = torch.randn(T, I, device=DEV)
    names = kernels_of(lambda: nm.nm_linear_i8(x, wq, ws))
    assert any("quant_rows_kernel" in k for k in names) != fused and any("gemm_i8_few_kernel<1, " in k and ", true>" in k for k in names) == fused, names


def test_sums_that_fill_32_bits():
    import paper_2203_10991_amd as nm
    for I in (131072, 131071):
        for a, b in ((127, 127), (-127, 127)):
            xq, wq = torch.full((3, I + 128 - I % 128 if I % 128 else I), a, dtype=torch.int8, device=DEV)[:, :I], torch.full((5, 131072), b, dtype=torch.int8, device=DEV)[:, :I]
            y = nm.nm_gemm_i8(xq, torch.ones(3, device=DEV), wq, torch.ones(5, device=DEV), out_dtype=F32)
            assert bool((y == float(np.float32(a * b * I))).all())
    with pytest.raises(nm.NmError):
        xq = torch.zeros(3, 131073, dtype=torch.int8, device=DEV)
        nm.nm_gemm_i8(xq, torch.ones(3, device=DEV), xq, torch.ones(3, device=DEV))


@pytest.mark.parametrize("dtype,out", [(F32, F32), (BF16, BF16), (BF16, F32), (F32, BF16)])
@pytest.mark.parametrize("T,O,I", [(1, 1, 1), (1, 4096, 1024), (4, 100, 77), (16, 1000, 2048), (33, 65, 130), (1, 70, 16000), (1, 70, 17000), (4, 33, 4031), (4, 33, 4097), (3, 1000, 15), (2, 17, 64), (197, 264, 1001), (1576, 1333, 1001), (40, 24, 9000)])
def test_layer(dtype, out, T, O, I):
    """nm_linear_i8 is the rounding of x and the product, bit for bit; x a view with NaN around it, in three dimensions"""
    import paper_2203_10991_amd as nm
    gen = torch.Generator().manual_seed(T + I)
    x = torch.randn(T, I, generator=gen).to(dtype)
    wq, ws = nm.nm_quant_i8(torch.randn(O, I, generator=gen).to(DEV))
    bias = torch.randn(O, generator=gen).to(dtype).to(DEV)
    q, xs = nm.nm_quant_i8(x.to(DEV))
    want = nm.nm_gemm_i8(q, xs, wq, ws, bias, relu=True, out_dtype=out)
    _check(want, q.cpu(), xs.cpu(), wq.cpu(), ws.cpu(), bias, True)
    for t in (x.to(DEV), _view(x, 5, 6, float("nan")), _view(x, 8, 16, float("nan"))):
        assert torch.equal(nm.nm_linear_i8(t, wq, ws, bias, relu=True, out_dtype=out), want)
    assert torch.equal(nm.nm_linear_i8(x.to(DEV).reshape(T, 1, I), wq, ws, bias, relu=True, out_dtype=out), want.reshape(T, 1, O))
    if T == 1:
        assert torch.equal(nm.nm_linear_i8(x.to(DEV)[0], wq, ws, bias, relu=True, out_dtype=out), want[0])
    # codes whose rows start anywhere
    loose = wq.clone(memory_format=torch.contiguous_format)
    assert torch.equal(nm.nm_linear_i8(x.to(DEV), loose, ws, bias, relu=True, out_dtype=out), want)


def test_layer_on_another_stream_from_a_graph_and_without_tokens():
    import paper_2203_10991_amd as nm
    gen = torch.Generator().manual_seed(1)
    wq, ws = nm.nm_quant_i8(torch.randn(300, 200, generator=gen).to(DEV))
    x = torch.randn(70, 200, generator=gen).to(DEV)
    want = nm.nm_linear_i8(x, wq, ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = nm.nm_linear_i8(x, wq, ws)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = nm.nm_linear_i8(x, wq, ws)
    for _ in range(4):
        x.mul_(1.5)
        graph.replay()
        assert torch.equal(got, nm.nm_linear_i8(x, wq, ws))
        torch.cuda.synchronize()
    assert nm.nm_linear_i8(x[:0], wq, ws).shape == (0, 300) and nm.nm_linear_i8(x, wq[:0], ws[:0]).shape == (70, 0)


def test_refusals():
    import paper_2203_10991_amd as nm
    x = torch.zeros(4, 32, device=DEV)
    wq, ws = nm.nm_quant_i8(torch.zeros(8, 32, device=DEV))
    for bad in (lambda: nm.nm_quant_i8(x.cpu()), lambda: nm.nm_quant_i8(x[0]), lambda: nm.nm_linear_i8(x.cpu(), wq, ws), lambda: nm.nm_linear_i8(x[:, :31], wq, ws),
                lambda: nm.nm_linear_i8(x, wq, ws[:7]), lambda: nm.nm_linear_i8(x, wq, ws, torch.zeros(7, device=DEV)), lambda: nm.nm_linear_i8(x[:, :0], wq[:, :0], ws),
                lambda: nm.nm_linear_i8(x, wq.cpu(), ws)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: nm.nm_quant_i8(x.half()), lambda: nm.nm_linear_i8(x.half(), wq, ws), lambda: nm.nm_linear_i8(x, wq.to(torch.uint8), ws),
                lambda: nm.nm_linear_i8(x, wq, ws.double()), lambda: nm.nm_linear_i8(x, wq, ws, out_dtype=torch.float16)):
        with pytest.raises(TypeError):
            bad()
