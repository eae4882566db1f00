"""Workspaces of the serving operators (no GPU needed): what a call takes in one launch needs none."""
import paper_2407_02891_amd as bcq
from paper_2407_02891_amd import binding as B


def _cache(kv_heads=8, head_dim=128, page=16):
    return B.Cache(B.BCQ_F16, kv_heads, head_dim, page, 1000, kv_heads * page * head_dim, page * head_dim, head_dim)


def test_attend_in_one_launch_needs_none():
    for requests, pages in ((1, 1), (1, 63), (16, 63), (64, 96)):
        assert bcq.attend_workspace_bytes(_cache(), requests, requests, 64, pages, 1) == 0, (requests, pages)
    for requests, pages in ((1, 8192), (64, 500)):
        assert bcq.attend_workspace_bytes(_cache(), requests, requests, 64, pages, 1) > 0, (requests, pages)


def test_attend_of_mixed_calls_needs_what_their_chunks_need():
    assert bcq.attend_workspace_bytes(_cache(), 500, 9, 64, 1, 400) == 0        # (tiles of 16 keys are not cut)
    few, more = (bcq.attend_workspace_bytes(_cache(1, 64), 140, n, 1, 80, 130) for n in (2, 9))
    assert few == more > 0                                                       # the same rows in as many parts
