"""Calls of attention with shared prefixes beyond what one launch takes (no GPU needed: refused before the first)."""
import pytest

import paper_2407_02891_amd as bcq
from paper_2407_02891_amd import binding as B
from tests.test_step_abi import OK, shared


def _cache(head_dim, kv_heads):
    return dict(head_dim=head_dim, kv_heads=kv_heads, slot_stride=head_dim, head_stride=16 * head_dim, page_stride=16 * head_dim * kv_heads)


# the join has a thread for four elements of a row, heads padded to 64, 128 or 256
@pytest.mark.parametrize("head_dim,kv_heads,q_heads,most", [(256, 16, 128, 2 ** 19), (136, 16, 128, 2 ** 19), (128, 32, 1024, 2 ** 17), (72, 32, 1024, 2 ** 17), (64, 8, 1024, 2 ** 18), (8, 8, 1024, 2 ** 18)])
def test_more_threads_than_a_launch_counts(head_dim, kv_heads, q_heads, most):
    """Was an error of the last of three launches, behind all of the work."""
    cache, ld = _cache(head_dim, kv_heads), q_heads * head_dim
    assert shared(cache, tokens=most, q_heads=q_heads, ld_q=ld, ld_out=ld) == B.BCQ_ERR_UNSUPPORTED
    desc = B.Cache(0, kv_heads, head_dim, 16, 100, *(cache[n] for n in ("page_stride", "head_stride", "slot_stride")))
    assert bcq.attend_shared_workspace_bytes(desc, most, 2, 1, q_heads, 10, 1) == 0
    fits = most - 1024                                     # (refused for its workspace alone)
    assert shared(cache, tokens=fits, q_heads=q_heads, ld_q=ld, ld_out=ld, workspace=OK + 8) == B.BCQ_ERR_WORKSPACE
    assert bcq.attend_shared_workspace_bytes(desc, fits, 2, 1, q_heads, 10, 1) > 0
