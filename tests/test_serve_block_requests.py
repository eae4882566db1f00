"""The bookkeeping of serve_block (no GPU needed)."""
import pytest

import paper_2407_02891_amd as bcq
from paper_2407_02891_amd import binding as B
from paper_2407_02891_amd.serve_block import Requests


def test_requests_stay_in_their_own_pages():
    r = Requests(2, 40, 16, [0, -1], device="cpu")        # three pages each, 48 tokens
    batch = r.take([47, 10])
    own = [set(range(0, 48)), set(range(48, 96))]
    assert set(batch["slots"][:47].tolist()) <= own[0] and set(batch["slots"][47:].tolist()) <= own[1]
    for new in ([2, 0], [0, 39]):
        with pytest.raises(bcq.BcqError) as e:
            r.take(new)
        assert e.value.status == B.BCQ_ERR_INVALID_ARG
    assert r.length == [47, 10]                           # (nothing was taken)
    batch = r.take([1, 1])
    assert batch["slots"].tolist() == [47, 58] and batch["kv_len"].tolist() == [48, 11]
    with pytest.raises(bcq.BcqError):
        r.advance(batch)
    assert batch["slots"].tolist() == [47, 58] and r.length == [48, 11]
