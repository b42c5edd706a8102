"""Layer norm, rotary positions and attention together, as a transformer block uses them: modules with their gradients, the example, a captured step, one token after another."""
import importlib.util
import os

import pytest
import torch
import torch.nn.functional as F

from gpu_util import DEV, kernels_of

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
F32, BF16, F64 = torch.float32, torch.bfloat16, torch.float64


def _example():
    spec = importlib.util.spec_from_file_location("lm_block", os.path.join(ROOT, "examples", "lm_block.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def _plain_attention(x, w, b, heads, kv_heads, freqs, causal, lens):
    """self-attention up to the projection behind it, in x's type on the CPU"""
    B, T, width = x.shape
    D = width // heads
    qkv = F.linear(x, w, b).view(B, T, heads + 2 * kv_heads, D)
    q, k, v = qkv[:, :, :heads], qkv[:, :, heads:heads + kv_heads], qkv[:, :, heads + kv_heads:]
    if freqs is not None:
        r = 2 * len(freqs)
        angle = (torch.arange(T, dtype=F64)[:, None] * freqs)[None, :, None]
        c, s = angle.cos().to(x.dtype), angle.sin().to(x.dtype)
        turn = lambda t: torch.cat((t[..., :r // 2] * c - t[..., r // 2:r] * s, t[..., :r // 2] * s + t[..., r // 2:r] * c, t[..., r:]), -1)    # noqa: E731
        q, k = turn(q), turn(k)
    k, v = (t.repeat_interleave(heads // kv_heads, 2) for t in (k, v))
    scores = torch.einsum("bihd,bjhd->bhij", q, k) * D ** -0.5
    i, j = torch.arange(T)[:, None], torch.arange(T)[None]
    see = (j < lens[:, None, None, None]) & (i < lens[:, None, None, None])
    if causal:
        see = see & (j <= i)
    p = torch.nan_to_num(torch.softmax(scores.masked_fill(~see, -float("inf")), -1))
    return torch.einsum("bhij,bjhd->bihd", p, v).reshape(B, T, width)


@pytest.mark.parametrize("heads,kv_heads,width,turned,causal", [(4, 4, 64, None, True), (6, 2, 240, 16, False), (8, 1, 128, 0, True)])
def test_self_attention_and_its_gradients(heads, kv_heads, width, turned, causal):
    """the module in binary32 against binary64: outputs, the input's gradient (dense products) and the biases'.  A sum of n products in binary32 is off by up to n 2^-24 of the sum of
    magnitudes; ten sums of at most 400 terms follow one another, magnitudes add up to at most about ten times a result's 2-norm: 10 x 400 x 10 x 2^-24 = 2.4e-3"""
    from paper_2203_10991_amd.autograd import NMConfig, NMSelfAttention
    torch.manual_seed(1)
    layer = NMSelfAttention(width, heads, kv_heads, causal, rotary=turned, cfg=NMConfig(seed=1), device=DEV)
    B, T = 3, 48
    lens = torch.tensor([48, 17, 1], dtype=torch.int32)
    x = torch.randn(B, T, width, device=DEV, requires_grad=True)
    g = torch.randn(B, T, width, device=DEV)
    y = layer(x, lens=lens.to(DEV))
    dx, dqkv, dproj = torch.autograd.grad(y, (x, layer.qkv.bias, layer.proj.bias), g)
    plain = [t.detach().cpu().double().requires_grad_() for t in (x, layer.qkv.weight, layer.qkv.bias, layer.proj.weight, layer.proj.bias)]
    freqs = None if turned == 0 else layer._freqs
    want = F.linear(_plain_attention(*plain[:3], heads, kv_heads, freqs, causal, lens), *plain[3:])
    wdx, wdqkv, wdproj = torch.autograd.grad(want, (plain[0], plain[2], plain[4]), g.cpu().double())
    for name, a, b in (("y", y, want), ("dx", dx, wdx), ("dqkv", dqkv, wdqkv), ("dproj", dproj, wdproj)):
        off = float((a.detach().cpu().double() - b.detach()).norm() / b.detach().norm())
        assert off < 2.4e-3, (name, off)
    names = kernels_of(lambda: layer(x.detach(), lens=lens.to(DEV)))
    assert any("attention_kernel" in k for k in names) and (turned == 0) != any("rotary_kernel" in k for k in names)


def test_functions_with_gradients():
    """attention and rotary as functions: what the calls behind them give, also for gradients that autograd expands"""
    import paper_2203_10991_amd as nm
    from paper_2203_10991_amd.autograd import attention, rotary
    q, k, v = (torch.randn(2, 30, h, 32, device=DEV, requires_grad=True) for h in (4, 2, 2))
    freqs, pos = nm.rotary_freqs(16, device=DEV), torch.arange(30, device=DEV) * 7
    y = rotary(q, freqs, pos, True, 1.5)
    assert torch.equal(y, nm.nm_rotary(q.detach(), freqs, pos, True, 1.5))
    dq, = torch.autograd.grad(y.sum(), q)                                     # (a gradient with strides of zero)
    assert torch.equal(dq, nm.nm_rotary(torch.ones_like(q.detach()), freqs, pos, True, 1.5, inverse=True))
    lens = torch.tensor([30, 11], dtype=torch.int32, device=DEV)
    o = attention(q, k, v, True, 0.3, lens, lens)
    plain = [t.detach() for t in (q, k, v)]
    want, lse = nm.nm_attention(*plain, True, 0.3, lens, lens, want_lse=True)
    assert torch.equal(o, want)
    for a, b in zip(torch.autograd.grad(o.sum(), (q, k, v)), nm.nm_attention_grad(torch.ones_like(want), *plain, want, lse, True, 0.3, lens, lens)):
        assert torch.equal(a, b)
    with pytest.raises(RuntimeError):                                         # no second derivatives
        d, = torch.autograd.grad(attention(q, k, v).sum(), q, create_graph=True)
        d.sum().backward()


@pytest.mark.parametrize("affine,bias", [(True, True), (True, False), (False, False)])
def test_layer_norm_module(affine, bias):
    import paper_2203_10991_amd as nm
    from paper_2203_10991_amd.autograd import NMLayerNorm
    layer = NMLayerNorm(100, elementwise_affine=affine, bias=bias, device=DEV)
    x = torch.randn(4, 7, 100, device=DEV, requires_grad=True)
    y = layer(x)
    w, b = (None if p is None else p.detach() for p in (layer.weight, layer.bias))
    want, mean, rstd = nm.nm_layer_norm(x.detach(), w, b, layer.eps, want_stats=True)
    assert torch.equal(y, want)
    params = [p for p in (layer.weight, layer.bias) if p is not None]
    got = torch.autograd.grad(y.sum(), [x, *params])
    dx, dw, db = nm.nm_layer_norm_grad(torch.ones_like(want), x.detach(), w, mean, rstd)
    assert torch.equal(got[0], dx) and all(torch.equal(a, c) for a, c in zip(got[1:], (dw, db)))
    assert layer.state_dict().keys() == torch.nn.LayerNorm(100, elementwise_affine=affine, bias=bias).state_dict().keys()
    with pytest.raises(ValueError):
        NMLayerNorm((3, 4))
    with pytest.raises(ValueError):
        layer(x[..., :50])


def test_the_example_runs():
    mod = _example()
    losses = mod.train(3, layers=1, batch=8)
    assert len(losses) == 3 and all(0 < x < 20 for x in losses)


def test_the_examples_gradients():
    """the whole model in binary32: gradients of the embedding and the norms, which the dense products alone decide, against binary64.  Tolerance as above, through two
    blocks of six sums each and back: 24 x 260 x 10 x 2^-24 = 3.7e-3"""
    mod = _example()
    from paper_2203_10991_amd.autograd import NMConfig
    torch.manual_seed(2)
    model = mod.Model(40, 64, 2, 4, 2, NMConfig(seed=1), device=DEV, dtype=F32)
    ids, target = torch.randint(40, (3, 24), device=DEV), torch.randint(40, (3, 24), device=DEV)
    lens = torch.tensor([24, 9, 1], dtype=torch.int32, device=DEV)
    loss = mod.loss_of(model, ids, target, lens)
    loss.backward()
    p = {k: v.detach().cpu().double().requires_grad_() for k, v in model.named_parameters()}
    x = F.embedding(ids.cpu(), p["embed.weight"]) * 8
    for n in range(2):
        at = f"blocks.{n}."
        h = F.layer_norm(x, (64,), p[at + "norm1.weight"], p[at + "norm1.bias"])
        h = _plain_attention(h, p[at + "attn.qkv.weight"], p[at + "attn.qkv.bias"], 4, 2, model.blocks[n].attn._freqs, True, lens.cpu())
        x = x + F.linear(h, p[at + "attn.proj.weight"], p[at + "attn.proj.bias"])
        h = F.layer_norm(x, (64,), p[at + "norm2.weight"], p[at + "norm2.bias"])
        x = x + F.linear(F.linear(h, p[at + "up.weight"], p[at + "up.bias"]).relu(), p[at + "down.weight"], p[at + "down.bias"])
    logits = F.linear(F.layer_norm(x, (64,), p["norm.weight"], p["norm.bias"]), p["head.weight"], p["head.bias"])
    there = torch.arange(24) < lens.cpu()[:, None]
    want = F.cross_entropy(logits.flatten(0, 1), torch.where(there, target.cpu(), -100).flatten(), ignore_index=-100)
    assert abs(float(loss) - float(want)) < 1e-4 * float(want)
    want.backward()
    checked = 0
    for k, v in model.named_parameters():
        if "norm" in k or "embed" in k or k.endswith("bias"):
            off = float((v.grad.cpu().double() - p[k].grad).norm() / p[k].grad.norm().clamp(min=1e-12))
            # (the keys' biases have a gradient of zero: every score of a row moves alike.  Together with the others they are held to the same bound)
            assert off < 3.7e-3, (k, off)
            checked += 1
    assert checked == 1 + 2 * 2 * 2 + 2 + 2 * 4 + 1


def test_a_block_captured_in_a_graph():
    """forward and backward of a block, captured once and replayed on new data between eager calls"""
    from paper_2203_10991_amd.autograd import NMConfig
    mod = _example()
    torch.manual_seed(3)
    block = mod.Block(64, 4, 2, NMConfig(seed=1), device=DEV, dtype=BF16)
    x, g = torch.randn(2, 32, 64, device=DEV).to(BF16).requires_grad_(), torch.randn(2, 32, 64, device=DEV).to(BF16)
    params = [block.norm1.weight, block.norm1.bias, block.norm2.weight, block.attn.qkv.bias]

    def step():
        y = block(x)
        return (y.detach(), *torch.autograd.grad(y, [x, *params], g))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(2):
            step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for _ in range(4):
        want = step()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, want))
        with torch.no_grad():
            x.copy_(torch.randn(x.shape, device=DEV))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_tokens_one_after_another(dtype):
    """a prompt at once, and its last tokens one at a time over a cache: the same attention up to the roundings of both.  bf16: probabilities and results rounded on both
    sides, 4 x 2^-8 of values that sum to at most the largest |v|; binary32: 2 x (40 + 64 + 8) 2^-24 x 8 of it (scores' errors at 8 units)"""
    import paper_2203_10991_amd as nm
    B, T, H, K, D = 2, 40, 4, 2, 32
    q, k, v = (torch.randn(B, T, h, D, device=DEV).to(dtype) for h in (H, K, K))
    freqs = nm.rotary_freqs(D, device=DEV)
    whole = nm.nm_attention(nm.nm_rotary(q, freqs), nm.nm_rotary(k, freqs), v, causal=True)
    caches = [torch.full((B, 64, K, D), float("nan"), device=DEV, dtype=dtype) for _ in range(2)]
    bound = float(v.float().abs().max()) * (4 * 2.0 ** -8 if dtype == BF16 else 2 * 112 * 8 * 2.0 ** -24)
    for t in range(T):
        at = torch.full((B, 1), t, device=DEV)
        caches[0][:, t:t + 1] = nm.nm_rotary(k[:, t:t + 1], freqs, at)
        caches[1][:, t:t + 1] = v[:, t:t + 1]
        lens = torch.full((B,), t + 1, dtype=torch.int32, device=DEV)
        o = nm.nm_attention(nm.nm_rotary(q[:, t:t + 1], freqs, at), *caches, causal=True, k_lens=lens)
        assert float((o[:, 0].float() - whole[:, t].float()).abs().max()) <= bound


def test_modules_refuse():
    from paper_2203_10991_amd.autograd import NMSelfAttention
    for bad in (dict(width=100, heads=3), dict(width=64, heads=4, kv_heads=3), dict(width=60, heads=5), dict(width=512, heads=2), dict(width=64, heads=4, rotary=7), dict(width=64, heads=4, rotary=18)):
        with pytest.raises(ValueError):
            NMSelfAttention(**bad, device=DEV)
