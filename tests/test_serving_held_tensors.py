"""Tensors that an object holds and a program has put others in the place of: a call looks at them as at its arguments, for their sizes are in the descriptor that the
object was made with (no GPU needed: all of it is refused before anything is launched)."""
import ctypes

import pytest
import torch

import paper_2407_02891_amd as bcq
from paper_2407_02891_amd import binding as B, serving


def _refused(call, what):
    with pytest.raises(bcq.BcqError, match=what) as e:
        call()
    assert e.value.status == B.BCQ_ERR_INVALID_ARG


@pytest.mark.parametrize("other", [lambda t: t[:, :3].contiguous(), lambda t: t[:2], lambda t: torch.cat([t, t]), lambda t: t.long(), lambda t: t.float(), lambda t: t[:, :, None],
                                   lambda t: t.flatten(), lambda t: torch.zeros((4, 3), dtype=torch.int32).t(), lambda t: torch.zeros((3, 8), dtype=torch.int32)[:, ::2]])
def test_pages_of_a_table(other):
    pages, i = torch.zeros((3, 4), dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    desc = B.PageTableDesc(16, 10, 3, 4)
    free, count = torch.zeros(10, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    _refused(lambda: serving._load().step(ctypes.addressof(desc), other(pages), i, None, free, count, i.clone(), i.clone(), 5, False, None, bcq.PageTable.STEP, 0), "pages:")
