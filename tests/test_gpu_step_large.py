"""Offsets past 32 bits in the operators around the update phase: tables, gradients, weights, tokens, outputs and parameters of more than 2^31 elements or 2^32 bytes,
checked at their far ends against the same call on what lies there."""
import pytest
import torch

from gpu_util import DEV

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


def test_embedding_of_a_large_table():
    import paper_2203_10991_amd as nm
    V, D = 1_100_000, 2056                                                # 2.26e9 elements
    table = torch.zeros(V, D, dtype=BF16, device=DEV)
    ids = torch.tensor([0, 1, V - 1, V - 2, 1_050_000, V - 1, 5], device=DEV)
    table[ids] = torch.randn(len(ids), D, device=DEV).to(BF16)
    out = nm.nm_embed(table, ids, 2.0)
    assert torch.equal(out, (table[ids].float() * 2).to(BF16))
    del table
    g = torch.randn(len(ids), D, device=DEV).to(BF16)
    grad = nm.nm_embed_grad(g, ids, V, out_dtype=torch.float32)
    small = torch.zeros(V - 1_049_999, D, device=DEV)
    far = ids >= 1_050_000
    small.index_add_(0, ids[far] - 1_049_999, g[far].float())
    assert torch.equal(grad[1_049_999:], small)
    assert torch.equal(grad[0], g[0].float()) and torch.equal(grad[5], g[6].float())
    assert bool((grad[6:1_049_999] == 0).all())


def test_gradient_of_many_tokens():
    """More than 2^31 elements of incoming gradient"""
    import paper_2203_10991_amd as nm
    N, D, V = 540_000, 4096, 70_001
    g = torch.ones(N, D, dtype=BF16, device=DEV)
    g[N - 3:] = 2
    ids = torch.arange(N, device=DEV) % V
    ids[N - 3:] = V - 1
    got = nm.nm_embed_grad(g, ids, V, out_dtype=torch.float32)
    want = torch.bincount(ids[:N - 3], minlength=V).float()
    want[V - 1] += 6
    assert torch.equal(got, want[:, None].expand(V, D))


def test_products_with_large_operands():
    import paper_2203_10991_amd as nm
    gen = torch.Generator(device=DEV).manual_seed(1)

    def codes(R, C):
        return torch.randint(-127, 128, (R, C), generator=gen, device=DEV, dtype=torch.int8), torch.rand(R, generator=gen, device=DEV) + 0.1
    # weights of 2.3e9 bytes, few tokens and many
    wq, ws = codes(140_008, 16384)
    for T in (3, 130):
        xq, xs = codes(T, 16384)
        y = nm.nm_gemm_i8(xq, xs, wq, ws)
        assert torch.equal(y[:, -520:], nm.nm_gemm_i8(xq, xs, wq[-520:], ws[-520:])) and torch.equal(y[:, :64], nm.nm_gemm_i8(xq, xs, wq[:64], ws[:64]))
    del wq
    # tokens of 2.3e9 bytes, and 4.6e9 bytes of results
    x = torch.randn(70_001, 32768, generator=gen, device=DEV, dtype=BF16)
    wq, ws = codes(72, 32768)
    y = nm.nm_linear_i8(x, wq, ws)
    assert torch.equal(y[-300:], nm.nm_linear_i8(x[-300:], wq, ws))
    del x
    xq, xs = codes(70_001, 64)
    wq, ws = codes(32775, 64)
    y = nm.nm_gemm_i8(xq, xs, wq, ws)
    assert torch.equal(y[-300:], nm.nm_gemm_i8(xq[-300:], xs[-300:], wq, ws))
    y = nm.nm_gemm_i8(xq, xs, wq, ws, out_dtype=torch.float32)
    assert torch.equal(y[-300:], nm.nm_gemm_i8(xq[-300:], xs[-300:], wq, ws, out_dtype=torch.float32))


def test_adamw_on_more_than_32_bits_of_elements():
    import paper_2203_10991_amd as nm
    n = (1 << 32) + 777
    p, g = torch.zeros(n, dtype=BF16, device=DEV), torch.zeros(n, dtype=BF16, device=DEV)
    m, v = (nm.alloc_adamw_state(p, q8=True) for _ in range(2))
    tail = 3000
    p[-tail:], g[-tail:] = torch.randn(tail, device=DEV).to(BF16), torch.randn(tail, device=DEV).to(BF16)
    p[:tail], g[:tail] = p[-tail:], g[-tail:]
    ps, gs = p[-tail:].clone(), g[-tail:].clone()
    ms, vs = (nm.alloc_adamw_state(ps) for _ in range(2))
    nm.nm_adamw([p], [g], [m], [v], 1, lr=0.1, seed=3)
    nm.nm_adamw([ps], [gs], [ms], [vs], 1, lr=0.1)
    assert torch.equal(p[-tail:], ps) and torch.equal(p[:tail], ps)
    assert bool((p[tail:1 << 20] == 0).all()) and bool((p[-(1 << 20):-tail] == 0).all())
    for codes, scale, want in ((*m, ms), (*v, vs.sqrt())):
        got = codes[-tail:].float() * scale.repeat_interleave(256)[-(tail + 256 * len(scale) - n):][:tail]
        # (the last block is short: its scales end with 256 for it)
        assert bool(((got - want).abs() <= 0.13 * want.abs() + scale[-20:].max() * 2.0 ** -9).all())
        # another word for the same value a whole 2^32 elements further on
    assert not torch.equal(m[0][:tail].view(torch.uint8), m[0][-tail:].view(torch.uint8))
