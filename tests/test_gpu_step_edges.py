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
