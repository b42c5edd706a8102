"""nm_attention and nm_attention_grad against binary64 on the CPU: one query to hundreds, shared heads, lengths that leave sequences or queries without a key, NaN in
what does not count, strides, splits, streams, graphs, offsets past 32 bits."""
import pytest
import torch

from attention_reference import check, inputs, reference
from gpu_util import DEV, kernels_of

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def _all(q, k, v, g, causal, scale, ql=None, kl=None):
    import paper_2203_10991_amd as nm
    dev = [t.to(DEV) for t in (q, k, v, g)]
    lens = [None if t is None else torch.tensor(t, dtype=torch.int32, device=DEV) for t in (ql, kl)]
    mask = dict(causal=causal, scale=scale, q_lens=lens[0], k_lens=lens[1])
    o, lse = nm.nm_attention(*dev[:3], want_lse=True, **mask)
    dq, dk, dv = nm.nm_attention_grad(dev[3], *dev[:3], o, lse, **mask)
    return dict(o=o, lse=lse[0], dq=dq, dk=dk, dv=dv)


def _compare(q, k, v, g, causal, scale, ql=None, kl=None):
    got, want = _all(q, k, v, g, causal, scale, ql, kl), reference(q, k, v, g, causal, scale, ql, kl)
    for name in got:
        check(name, got[name], want[name])
    return got


SIZES = [(1, 1, 1, 1, 1, 8), (1, 1, 40, 2, 1, 32), (2, 2, 1, 2, 2, 16), (1, 31, 33, 1, 1, 64), (2, 32, 32, 2, 1, 40), (1, 33, 65, 3, 1, 128), (2, 64, 64, 4, 2, 64), (1, 100, 127, 7, 1, 80),
         (1, 129, 128, 2, 2, 96), (1, 128, 257, 1, 1, 104), (3, 200, 200, 2, 2, 24), (1, 300, 300, 4, 4, 120), (1, 5, 700, 8, 2, 128), (1, 260, 70, 2, 1, 48)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("B,Tq,Tk,H,K,D", SIZES)
def test_against_binary64(B, Tq, Tk, H, K, D, causal, dtype):
    _compare(*inputs(B, Tq, Tk, H, K, D, dtype), causal, D ** -0.5)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("B,Tq,Tk,H,K,D,ql,kl", [(3, 150, 600, 2, 1, 24, [150, 33, 0], [600, 31, 555]), (2, 129, 513, 2, 2, 64, [129, 128], [513, 480]), (2, 520, 520, 2, 1, 48, [520, 400], [520, 33]),
                                                 (2, 140, 530, 3, 1, 80, [140, 1], [530, 1]), (1, 200, 1100, 2, 2, 128, [200], [1030]), (2, 100, 100, 2, 2, 64, [100, 97], [96, 65])])
def test_few_workgroups(B, Tq, Tk, H, K, D, ql, kl, causal, dtype):
    """two waves to a block of rows: halves of a tile that hold no key, or none that a row sees"""
    _compare(*inputs(B, Tq, Tk, H, K, D, dtype, seed=13), causal, D ** -0.5, ql, kl)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("Tq,Tk,ql,kl", [(70, 70, [70, 1, 0, 33, 69, 32], [70, 1, 0, 33, 69, 32]), (40, 90, [40, 40, 3, 0, 40, 7], [90, 20, 0, 64, 1, 65]),
                                         (1, 130, [1, 1, 1, 0, 1, 1], [130, 0, 1, 64, 129, 33])])
def test_lengths_and_what_lies_behind(Tq, Tk, ql, kl, causal, dtype):
    """tokens behind a sequence hold NaN and infinities; results there are zeros"""
    B, H, K, D = 6, 4, 2, 72
    q, k, v, g = inputs(B, Tq, Tk, H, K, D, dtype, seed=1)
    for b in range(B):
        q[b, ql[b]:], g[b, ql[b]:] = float("nan"), float("inf")
        k[b, kl[b]:], v[b, kl[b]:] = float("inf"), float("nan")
        dead = max(0, ql[b] - kl[b]) if causal else (ql[b] if kl[b] == 0 else 0)
        g[b, :dead] = float("nan")                                           # queries that see nothing
    got = _compare(q, k, v, g, causal, 0.3, ql, kl)
    for b in range(B):
        for name, n in (("o", ql[b]), ("dq", ql[b]), ("dk", kl[b]), ("dv", kl[b])):
            assert not bool(got[name][b, n:].any()) and not bool(torch.isnan(got[name][b]).any()), (name, b)
        assert bool((got["lse"][b, :, ql[b]:] == -float("inf")).all())


def test_lengths_beyond_the_tensors():
    """... count as the tensors' own, and 64-bit lengths as 32-bit ones"""
    import paper_2203_10991_amd as nm
    q, k, v, _ = (t.to(DEV) for t in inputs(3, 20, 50, 2, 2, 64, BF16))
    lens = torch.tensor([1 << 40, 51, -5], device=DEV)
    got = nm.nm_attention(q, k, v, k_lens=lens)
    assert torch.equal(got[:2], nm.nm_attention(q, k, v)[:2]) and not bool(got[2].any())


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_scores_far_apart(dtype):
    """scores of hundreds: maxima that move many times, probabilities of zero and one; rising and falling along the keys"""
    for order in (1, -1):
        q, k, v, g = inputs(1, 50, 300, 2, 1, 64, dtype, seed=3, spread=4.0)
        k = (k.float() * torch.linspace(0.1, 3, 300)[::1][torch.arange(300) if order > 0 else torch.arange(299, -1, -1)].view(1, -1, 1, 1)).to(dtype)
        _compare(q, k, v, g, False, 1.0)
        _compare(q, k, v, g, True, 1.0)


@pytest.mark.parametrize("T,K,D,spread", [(900, 2, 32, 5.0), (300, 2, 128, 4.0)])
def test_rows_that_look_at_few_keys(T, K, D, spread):
    """bf16: 2-norms of dq's and dk's errors.  The result's rounding is 0.166 % (half a step, 2^-9 to 2^-8 of a value, over sqrt(3), over a binade); what rounding P for o adds, and dS where P
    is small, is allowed as much again, sqrt(2) times that; dS rounded everywhere would be as much a third time"""
    q, k, v, g = inputs(2, T, T, 4, K, D, BF16, seed=15, spread=spread)
    got, want = _all(q, k, v, g, True, D ** -0.5), reference(q, k, v, g, True, D ** -0.5)
    for name in ("dq", "dk"):
        w = want[name][0]
        assert float((got[name].double().cpu() - w).norm() / w.norm()) < 0.0024, name


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_gradients_against_differences(dtype):
    """the sum of g o along a direction, by central differences in binary64 around the rounded inputs"""
    q, k, v, g = inputs(1, 9, 13, 4, 2, 16, dtype, seed=4)
    got = _all(q, k, v, g, True, 0.25)
    gen = torch.Generator().manual_seed(5)
    for name, t in (("dq", q), ("dk", k), ("dv", v)):
        d = torch.randn(t.shape, generator=gen, dtype=torch.float64)
        at = {"q": q.double(), "k": k.double(), "v": v.double()}
        value = []
        for h in (1e-4, -1e-4):
            moved = dict(at)
            moved[name[1]] = at[name[1]] + h * d
            o = torch.zeros(1, 9, 4, 16, dtype=torch.float64)
            for head in range(4):
                s = (moved["q"][0, :, head] @ moved["k"][0, :, head // 2].t() * 0.25).masked_fill(~(torch.arange(13)[None] <= torch.arange(9)[:, None] + 4), -float("inf"))
                o[0, :, head] = torch.softmax(s, 1) @ moved["v"][0, :, head // 2]
            value.append((g.double() * o).sum())
        slope = (value[0] - value[1]) / 2e-4
        bound = (reference(q, k, v, g, True, 0.25)[name][1] * d.abs()).sum() + 1e-6 * d.abs().sum()       # differences: h^2 times third derivatives of a few units
        assert abs((got[name].cpu().double() * d).sum() - slope) <= bound


def test_queries_that_look_at_few_keys():
    """scores of a deviation of ten: dP and delta nearly cancel.  With what rounding took from o the errors' 2-norm stays near that of rounding dS and the result (two roundings of
    at most 2^-8, 0.58 of that in the mean: 0.32 %); without it they are at least half as large again"""
    import paper_2203_10991_amd as nm
    q, k, v, g = inputs(1, 256, 256, 4, 4, 64, BF16, seed=14, spread=10.0)
    want = reference(q, k, v, g, True, 0.125)
    dev = [t.to(DEV) for t in (q, k, v, g)]
    o, lse = nm.nm_attention(*dev[:3], causal=True, scale=0.125, want_lse=True)
    assert lse.shape == (33, 1, 4, 256)
    error = []
    for stats in (lse, lse[:1]):
        got = nm.nm_attention_grad(dev[3], *dev[:3], o, stats, causal=True, scale=0.125)
        error.append([float((a.cpu().double() - want[name][0]).norm() / want[name][0].norm()) for name, a in zip(("dq", "dk"), got)])
        for name, a in zip(("dq", "dk", "dv"), got):
            check(name, a, want[name])
    assert max(error[0]) < 0.0032 and all(b > 1.5 * a for a, b in zip(*error)), error
    plain = nm.nm_attention(*dev[:3], causal=True, scale=0.125)
    assert torch.equal(plain, o)


def test_views():
    """parts of one tensor, heads before tokens, an expanded batch, elements apart, rows off a 16-byte boundary"""
    import paper_2203_10991_amd as nm
    B, T, H, K, D = 2, 45, 4, 2, 32
    qkv = torch.randn(B, T, H + 2 * K, D, device=DEV).to(BF16)
    q, k, v = qkv[:, :, :H], qkv[:, :, H:H + K], qkv[:, :, H + K:]
    plain = [t.contiguous() for t in (q, k, v)]
    g = torch.randn(B, T, H, D, device=DEV).to(BF16)
    o, lse = nm.nm_attention(*plain, causal=True, want_lse=True)
    want = nm.nm_attention_grad(g, *plain, o, lse, causal=True)
    assert torch.equal(o, nm.nm_attention(q, k, v, causal=True))
    dqkv = torch.full_like(qkv, float("nan"))
    parts = dqkv[:, :, :H], dqkv[:, :, H:H + K], dqkv[:, :, H + K:]
    nm.nm_attention_grad(g, q, k, v, o, lse, causal=True, out=parts)
    assert torch.equal(dqkv, torch.cat(want, 2))
    by_head = [t.transpose(1, 2).contiguous().transpose(1, 2) for t in plain]
    assert torch.equal(o, nm.nm_attention(*by_head, causal=True))
    assert all(torch.equal(a, b) for a, b in zip(want, nm.nm_attention_grad(g.transpose(1, 2).contiguous().transpose(1, 2), *by_head, o, lse, causal=True)))
    apart = [torch.stack((t, t), -1)[..., 0] for t in plain]
    assert torch.equal(o, nm.nm_attention(*apart, causal=True))
    off = [torch.cat((t[..., :1], t), -1)[..., 1:] for t in plain]
    assert torch.equal(o, nm.nm_attention(*off, causal=True))
    one = [t[:1].expand(3, -1, -1, -1) for t in plain]
    assert torch.equal(nm.nm_attention(*one, causal=True), nm.nm_attention(*(t.contiguous() for t in one), causal=True))
    wide_k = plain[1][:, :, :1].expand(-1, -1, 2, -1)                        # heads that are one
    assert torch.equal(nm.nm_attention(plain[0], wide_k, plain[2]), nm.nm_attention(plain[0], wide_k.contiguous(), plain[2]))


def test_nothing_to_do():
    import paper_2203_10991_amd as nm
    for B, Tq, Tk in ((0, 4, 4), (2, 0, 4), (2, 4, 0)):
        q, k, v, g = (t.to(DEV) for t in inputs(B, Tq, Tk, 4, 2, 32, BF16))
        o, lse = nm.nm_attention(q, k, v, want_lse=True)
        assert o.shape == q.shape and not bool(o.any()) and bool((lse[0] == -float("inf")).all())
        for d, t in zip(nm.nm_attention_grad(g, q, k, v, o, lse), (q, k, v)):
            assert d.shape == t.shape and not bool(d.any())


def test_same_bits_and_routes():
    """keys split among workgroups where rows are few, rows where keys are few; the same call gives the same bits"""
    import paper_2203_10991_amd as nm
    q, k, v, _ = (t.to(DEV) for t in inputs(2, 1, 3000, 8, 2, 64, BF16, seed=6))
    assert any("join" in n for n in kernels_of(lambda: nm.nm_attention(q, k, v))) and nm.load().nm_attention_workspace(2, 1, 3000, 8, 2, 64, 1) > 0
    assert torch.equal(nm.nm_attention(q, k, v), nm.nm_attention(q, k, v))
    q, k, v, g = (t.to(DEV) for t in inputs(1, 900, 100, 8, 1, 64, BF16, seed=7))
    o, lse = nm.nm_attention(q, k, v, want_lse=True)
    assert any("sum" in n for n in kernels_of(lambda: nm.nm_attention_grad(g, q, k, v, o, lse)))
    first = nm.nm_attention_grad(g, q, k, v, o, lse)
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(first, nm.nm_attention_grad(g, q, k, v, o, lse)))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("B,Tq,Tk,H,K,D,kl", [(2, 1, 3000, 8, 2, 64, [3000, 1777]), (1, 3, 2049, 4, 1, 128, None), (2, 1, 5000, 2, 2, 80, [5000, 0])])
def test_few_queries_over_many_keys(B, Tq, Tk, H, K, D, kl, dtype):
    for causal in (False, True):
        _compare(*inputs(B, Tq, Tk, H, K, D, dtype, seed=8), causal, D ** -0.5, None, kl)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_many_rows_over_few_keys(dtype):
    for causal in (False, True):
        _compare(*inputs(1, 700, 100, 4, 1, 64, dtype, seed=9), causal, 0.125)


@pytest.mark.parametrize("B,Tq,Tk,H,K,D,kl", [(32, 40, 2048, 2, 1, 128, None), (32, 33, 2050, 1, 1, 96, "ragged"), (16, 9, 4100, 2, 1, 72, "ragged")])
def test_many_keys_of_many_heads(B, Tq, Tk, H, K, D, kl):
    """eight waves to a tile of rows: from 2048 keys on, where there are workgroups for every CU"""
    import paper_2203_10991_amd as nm
    lens = None if kl is None else [Tk - 97 * b for b in range(B)]
    ins = inputs(B, Tq, Tk, H, K, D, BF16, seed=12)
    for causal in (False, True):
        _compare(*ins, causal, D ** -0.5, None, lens)
    q, k, v, g = (t.to(DEV) for t in ins)
    o, lse = nm.nm_attention(q, k, v, want_lse=True)
    assert any("attention_dkdv_kernel<1, %d, 32, 8," % (-(-D // 32)) in n for n in kernels_of(lambda: nm.nm_attention_grad(g, q, k, v, o, lse)))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("B,T,H,K,D", [(20, 130, 16, 16, 32), (9, 300, 16, 16, 64), (3, 600, 30, 15, 40)])
def test_many_workgroups(B, T, H, K, D, dtype):
    """more than the 256 that are dealt to the XCDs at a time, and what is left behind the last 256; lengths from all to none"""
    lens = [T - (T * b) // max(1, B - 1) for b in range(B)]
    _compare(*inputs(B, T, T, H, K, D, dtype, seed=13), True, D ** -0.5, lens, lens)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("B,T,H,K,D", [(3, 300, 48, 6, 16), (4, 1100, 15, 15, 72), (3, 130, 576, 9, 8)])
def test_tiles_of_many_heads_together(B, T, H, K, D, dtype):
    """all heads' tiles in one list, of rows and of keys, and eight heads' at a time with three heads left over"""
    lens = [T - (T * b) // (2 * B) for b in range(B)]
    _compare(*inputs(B, T, T, H, K, D, dtype, seed=14), True, D ** -0.5, lens, lens)


def test_another_stream_and_two_graphs():
    """two captured calls with workspaces of their own, replayed in turn with eager calls between"""
    import paper_2203_10991_amd as nm
    sets = [[t.to(DEV) for t in inputs(2, n, m, 8, 2, 64, BF16, seed=n)] for n, m in ((1, 2500), (200, 200))]

    def both(q, k, v, g):
        o, lse = nm.nm_attention(q, k, v, causal=True, want_lse=True)
        return [o, lse, *nm.nm_attention_grad(g, q, k, v, o, lse, causal=True)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        apart = [both(*s) for s in sets]
    torch.cuda.current_stream().wait_stream(side)
    graphs = []
    for s in sets:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = both(*s)
        graphs.append((graph, out))
    gen = torch.Generator(device=DEV).manual_seed(1)
    for turn in range(4):
        want = [both(*s) for s in sets]
        if turn == 0:
            assert all(torch.equal(a, b) for x, y in zip(want, apart) for a, b in zip(x, y))
        for graph, _ in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for (_, out), w in zip(graphs, want):
            assert all(torch.equal(a, b) for a, b in zip(out, w))
        for s in sets:
            for t in s:
                t.copy_(torch.randn(t.shape, generator=gen, device=DEV))


def test_offsets_past_32_bits():
    """keys 2^24 elements apart (10 GB of cache), sequences 2^31 apart"""
    import paper_2203_10991_amd as nm
    q, k, v, g = (t.to(DEV) for t in inputs(2, 40, 300, 2, 1, 32, BF16, seed=11))
    cache = torch.empty(300 << 24, dtype=BF16, device=DEV)
    far = [cache.as_strided((1, 300, 1, 32), (0, 1 << 24, 32, 1), at) for at in (0, 32)]
    for f, t in zip(far, (k, v)):
        f.copy_(t[:1])
    o, lse = nm.nm_attention(q[:1], *far, want_lse=True)
    near = nm.nm_attention(q[:1], k[:1], v[:1], want_lse=True)
    assert torch.equal(o, near[0])
    out = torch.empty_like(q[:1]), cache.as_strided((1, 300, 1, 32), (0, 1 << 24, 32, 1), 64), cache.as_strided((1, 300, 1, 32), (0, 1 << 24, 32, 1), 96)
    nm.nm_attention_grad(g[:1], q[:1], *far, o, lse, out=out)
    assert all(torch.equal(a, b) for a, b in zip(out, nm.nm_attention_grad(g[:1], q[:1], k[:1], v[:1], *near)))
    far = [cache.as_strided((2, 300, 1, 32), (1 << 31, 32, 32, 1), at) for at in (0, 16384)]
    for f, t in zip(far, (k, v)):
        f.copy_(t)
    assert torch.equal(nm.nm_attention(q, *far, causal=True), nm.nm_attention(q, k, v, causal=True))


def test_refusals():
    import paper_2203_10991_amd as nm
    q, k, v, g = (t.to(DEV) for t in inputs(2, 10, 12, 4, 2, 32, BF16))
    o, lse = nm.nm_attention(q, k, v, want_lse=True)
    bad = [lambda: nm.nm_attention(q, k[:1], v[:1]), lambda: nm.nm_attention(q, k, v[:, :5]), lambda: nm.nm_attention(q.cpu(), k, v), lambda: nm.nm_attention(q[0], k, v),
           lambda: nm.nm_attention(q, k, v, k_lens=torch.ones(3, dtype=torch.int32, device=DEV)), lambda: nm.nm_attention(q, k, v, k_lens=torch.ones(2, dtype=torch.int32)),
           lambda: nm.nm_attention_grad(g, q, k, v, o, lse[..., :3]), lambda: nm.nm_attention_grad(g, q, k, v, o, lse[0]), lambda: nm.nm_attention_grad(g, q, k, v, o, lse[:5]), lambda: nm.nm_attention_grad(g[:, :3], q, k, v, o, lse),
           lambda: nm.nm_attention_grad(g, q, k, v, o, lse, out=(q[:, :3], k, v))]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    for call in (lambda: nm.nm_attention(q, k.float(), v), lambda: nm.nm_attention(q.half(), k.half(), v.half())):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: nm.nm_attention(q[..., :12], k[..., :12], v[..., :12]), lambda: nm.nm_attention(q[:, :, :3], k, v), lambda: nm.nm_attention(q, k, v, scale=0.0),
                 lambda: nm.nm_attention(q, k, v, scale=-1.0), lambda: nm.nm_attention_grad(g, q, k, v, o, lse, out=(torch.empty_like(q), k, torch.empty_like(v))),
                 lambda: nm.nm_attention_grad(g, q, k, v, o, lse, out=(torch.empty_like(q), torch.empty_like(k), torch.empty_like(v[:1]).expand(2, -1, -1, -1)))):
        with pytest.raises(nm.NmError):
            call()
