"""What the objects over the serving operators refuse before they reach the library (no GPU needed)."""
import pytest
import torch

import paper_2407_02891_amd as bcq
from paper_2407_02891_amd import binding as B


def _refused(call):
    with pytest.raises(bcq.BcqError) as e:
        call()
    assert e.value.status == B.BCQ_ERR_INVALID_ARG


@pytest.mark.parametrize("device", ["cpu", "meta"])
def test_tensors_that_are_not_on_a_gpu(device):
    """Their addresses mean nothing to a kernel."""
    k, v = (torch.zeros((2, 1, 16, 64), dtype=torch.float16, device=device) for _ in range(2))
    _refused(lambda: bcq.PagedCache(k, v))
    _refused(lambda: bcq.PagedCache.empty(2, 16, 1, 64, device=device))
    A, Bm = (torch.zeros(s, dtype=torch.bfloat16, device=device) for s in ((1, 8, 64), (1, 40, 8)))
    _refused(lambda: bcq.Adapters(A, Bm))
    _refused(lambda: bcq.Adapters(A, Bm, torch.ones(1, device=device), torch.ones(1, dtype=torch.int32, device=device)))
