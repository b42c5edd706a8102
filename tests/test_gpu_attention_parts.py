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
