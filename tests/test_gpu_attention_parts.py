"""nm_attention's and nm_attention_grad's tensors as parts of others: what the forward pass leaves cut as the other tensors are."""
import pytest
import torch

from attention_reference import check, inputs, reference
from gpu_util import DEV

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def _cut(name, at):
    """of q, k, v, g, o and lse: sequences 1 and 2 of 3, the second half of the heads, or queries 40 to 139"""
    if name == "sequences":
        return [t[1:] for t in at[:5]] + [at[5][:, 1:]]
    if name == "heads":
        q, k, v, g, o, lse = at
        return [q[:, :, 4:], k[:, :, 2:], v[:, :, 2:], g[:, :, 4:], o[:, :, 4:], lse[:, :, 4:]]
    q, k, v, g, o, lse = at
    return [q[:, 40:140], k, v, g[:, 40:140], o[:, 40:140], lse[..., 40:140]]


@pytest.mark.parametrize("dtype,D", [(BF16, 64), (BF16, 24), (BF16, 128), (F32, 64)])
@pytest.mark.parametrize("name", ["sequences", "heads", "queries"])
def test_gradients_of_a_cut(name, dtype, D):
    """Gradients of a part of a batch, from what the whole batch's forward pass left, as a view and as a copy.  Scores of a deviation of ten, where a bf16 o alone makes delta too coarse: two
    roundings of at most 2^-8, 0.58 of that in the mean, are 0.32 % of a gradient's 2-norm (binary32: far less)"""
    import paper_2203_10991_amd as nm
    B, T, H, K = 3, 160, 8, 4
    q, k, v, g = inputs(B, T, T, H, K, D, dtype, seed=21, spread=10.0)
    scale = D ** -0.5
    dev = [t.to(DEV) for t in (q, k, v, g)]
    o, lse = nm.nm_attention(*dev[:3], scale=scale, want_lse=True)
    part = _cut(name, [*dev, o, lse])
    at = [t.cpu() for t in part[:4]]
    want = reference(*at, False, scale)
    for stats in (part[5], part[5].contiguous(), part[5].clone()):
        got = nm.nm_attention_grad(part[3], *part[:3], part[4], stats, scale=scale)
        for which, a in zip(("dq", "dk", "dv"), got):
            check(which, a, want[which])
            w = want[which][0]
            assert float((a.cpu().double() - w).norm() / w.norm()) < 0.0032, which


def test_parts_joined():
    """what two calls left, put together along sequences, heads and queries, is what one call leaves"""
    import paper_2203_10991_amd as nm
    q, k, v, _ = (t.to(DEV) for t in inputs(2, 300, 300, 8, 8, 64, BF16, seed=22))
    whole = nm.nm_attention(q, k, v, want_lse=True)[1]
    for dim, cut in ((1, lambda t: (t[:1], t[1:])), (2, lambda t: (t[:, :, :4], t[:, :, 4:]))):
        parts = [nm.nm_attention(*p, want_lse=True)[1] for p in zip(*(cut(t) for t in (q, k, v)))]
        assert torch.equal(torch.cat(parts, dim).view(torch.int32), whole.view(torch.int32))
    parts = [nm.nm_attention(p, k, v, want_lse=True)[1] for p in (q[:, :128], q[:, 128:])]
    assert torch.equal(torch.cat(parts, 3).view(torch.int32), whole.view(torch.int32))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("order", [(0, 1, 2), (1, 0, 2), (0, 2, 1), (2, 0, 1), (1, 2, 0), (2, 1, 0)])
def test_gradients_into_parts_of_one_tensor(order, dtype):
    """dq, dk and dv as heads of one tensor whose sequences, tokens and heads lie in any order; what is between them stays as it was"""
    import paper_2203_10991_amd as nm
    B, T, H, K, D = 3, 70, 4, 2, 32
    q, k, v, g = (t.to(DEV) for t in inputs(B, T, T, H, K, D, dtype, seed=23))
    o, lse = nm.nm_attention(q, k, v, causal=True, want_lse=True)
    want = nm.nm_attention_grad(g, q, k, v, o, lse, causal=True)
    sizes, back = (B, T, H + 2 * K + 1), [order.index(i) for i in range(3)]
    held = torch.full((*(sizes[i] for i in order), D), 7.0, dtype=dtype, device=DEV).permute(*back, 3)
    assert held.shape == (*sizes, D)
    out = held[:, :, :H], held[:, :, H + 1:H + 1 + K], held[:, :, H + 1 + K:]
    nm.nm_attention_grad(g, q, k, v, o, lse, causal=True, out=out)
    assert all(torch.equal(a, b) for a, b in zip(out, want)) and bool((held[:, :, H] == 7).all())
    with pytest.raises(nm.NmError):
        nm.nm_attention_grad(g, q, k, v, o, lse, causal=True, out=(out[0], out[1], held[:, :, H + K:-1]))


def test_heads_turned_into_other_parts():
    """rotary positions of one part of a sequence-first tensor into another"""
    import paper_2203_10991_amd as nm
    held = torch.randn(11, 3, 6, 32, device=DEV).transpose(0, 1)
    freqs = nm.rotary_freqs(32, device=DEV)
    kept = held.clone()
    nm.nm_rotary(held[:, :, :3], freqs, out=held[:, :, 3:])
    assert torch.equal(held[:, :, :3], kept[:, :, :3]) and torch.equal(held[:, :, 3:], nm.nm_rotary(kept[:, :, :3], freqs))
