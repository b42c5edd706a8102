"""Launches of a thread to a piece that would be 2^32 threads and more, which a dimension of a grid does not hold, are refused: cut to what is left modulo 2^32 they would leave
outputs unwritten without an error."""
import gc

import pytest
import torch

from gpu_util import DEV

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def memory():
    torch.cuda.empty_cache()
    yield
    gc.collect()
    torch.cuda.empty_cache()


def _status(call):
    import paper_2203_10991_amd as nm
    try:
        call()
    except nm.NmError as e:                                  # (its traceback holds the tensors: the status alone leaves)
        return e.status
    return 0


def test_prune_4of8_of_2_35_elements():
    import paper_2203_10991_amd as nm
    assert _status(lambda: nm.mvue_prune_4of8_approx(torch.empty((1 << 20) + 16, 1 << 15, dtype=torch.bfloat16, device=DEV))) == 8


def test_cast_of_2_36_elements():
    import paper_2203_10991_amd as nm
    record = torch.ones(4, device=DEV)
    assert _status(lambda: nm.nm_cast_e4m3(torch.empty((1 << 21) + 16, 1 << 15, dtype=torch.bfloat16, device=DEV), record)) == 8
