"""Binary32 tensors in nm_attention, which go through the matrix instructions as three bf16 terms a value: what the products leave out, and the largest values."""
import pytest
import torch

from gpu_util import DEV

pytestmark = pytest.mark.gpu

E32 = 2.0 ** -24                  # half a step of binary32


@pytest.mark.parametrize("D", [8, 16])
@pytest.mark.parametrize("x", [1 + 2.0 ** -7 - 2.0 ** -23, 1 + 2.0 ** -8 + 2.0 ** -16 - 2.0 ** -23, 2 - 2.0 ** -23, 1 + 2.0 ** -8])
def test_scores_of_equal_products(x, D):
    """One key: lse is the score, D x^2, times the binary32 forms of log2(e) and ln 2 (their product is off from one by what it is).  Terms rounded to nearest leave out 2^-24 of a
    product at most; D <= 16 products are one matrix instruction for each pair of terms, of whose six roundings the last two are of the score's size (two more are allowed to the instruction's own
    sum); the product with log2(e) and that with ln 2 round once each: 1 + 4 + 2 half steps.  Terms cut off leave out up to 8, on every product of the first value here"""
    import paper_2203_10991_amd as nm
    q = torch.full((1, 1, 1, D), x, device=DEV)
    _, lse = nm.nm_attention(q, q, q, scale=1.0, want_lse=True)
    log2e, ln2 = (float(torch.tensor(c, dtype=torch.float32)) for c in (1.44269504088896340736, 0.69314718055994530942))
    want = D * x * x * log2e * ln2
    assert abs(float(lse[0]) - want) <= 7 * E32 * want


def test_values_come_through_whole():
    """one key: o is v bit for bit, up to the largest binary32 numbers, whose nearest bf16 number would be an infinity"""
    import paper_2203_10991_amd as nm
    gen = torch.Generator().manual_seed(32)
    v = torch.randn(4, 1, 1, 128, generator=gen) * torch.exp2(torch.randint(-80, 120, (4, 1, 1, 128), generator=gen).float())
    most = torch.finfo(torch.float32).max
    v[0, 0, 0, :8] = torch.tensor([most, -most, 3.3895314e38, 3.3962e38, -3.3961775e38, 3.4e38, 1.0, -1.0])
    q = torch.ones(4, 1, 1, 128)
    o = nm.nm_attention(q.to(DEV), q.to(DEV), v.to(DEV))
    assert torch.equal(o.cpu(), v)
