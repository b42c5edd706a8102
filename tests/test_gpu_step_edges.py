"""The 8-bit integer products and their roundings at their limits."""
import numpy as np
import pytest
import torch

from gpu_util import DEV

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


@pytest.mark.parametrize("T", [3, 200])
@pytest.mark.parametrize("a,b,I", [(-128, -128, 131071), (-128, 127, 131072), (127, -128, 131072), (127, 127, 131072)])
def test_largest_sums(T, a, b, I):
    """What the 32-bit sums hold: -128 on one side at every length, on both up to 131071"""
    import paper_2203_10991_amd as nm
    xq, wq = torch.full((T, 131072), a, dtype=torch.int8, device=DEV)[:, :I], torch.full((300, 131072), b, dtype=torch.int8, device=DEV)[:, :I]
    y = nm.nm_gemm_i8(xq, torch.ones(T, device=DEV), wq, torch.ones(300, device=DEV), out_dtype=F32)
    assert bool((y == float(np.float32(a * b * I))).all())


def test_rounding_of_more_rows_than_a_grid_has_workgroups():
    """A workgroup to a row: 2^24 rows and more are 2^32 threads, which one dimension of a grid does not hold"""
    import paper_2203_10991_amd as nm
    R, C = (1 << 24) + 7, 1032
    x = torch.zeros(R, C, dtype=BF16, device=DEV)
    for at in (0, (1 << 23) - 3, (1 << 24) - 3, R - 6):
        x[at:at + 6] = torch.randn(6, C, device=DEV).to(BF16)
    q, s = nm.nm_quant_i8(x)
    for at in (0, (1 << 23) - 3, (1 << 24) - 3, R - 6):
        want, ws = nm.nm_quant_i8(x[at:at + 6])
        assert torch.equal(q[at:at + 6], want) and torch.equal(s[at:at + 6], ws) and bool((ws > 0).all())
    assert int((s > 0).sum()) == 6 + 6 + 10                                 # (the last two groups overlap)
    del x, q, s
    torch.cuda.empty_cache()
