"""Attention again with tables of pages far longer than the requests need: what a call may have to read decides how it is split, so the
same requests take other ways through the kernels."""
import pytest
import torch

from tests import test_gpu_serving as serving
from tests.test_gpu_serving import (test_attend_chunks, test_attend_flat_and_sharp_softmax, test_attend_hidden_keys_have_no_part_whatever_they_hold,  # noqa: F401
                                    test_attend_many_query_heads_share_one, test_attend_many_requests, test_attend_rows_that_see_nothing,
                                    test_attend_scores_that_grow_and_fall_along_the_keys, test_attend_single_tokens_at_every_edge_of_a_tile,
                                    test_attend_strides_of_the_cache_and_of_the_rows)

pytestmark = pytest.mark.gpu


class LongTables(serving.Batch):
    def __init__(self, new, kv, q_heads, kv_heads, D, page, *args, **kw):
        super().__init__(new, kv, q_heads, kv_heads, D, page, *args, **kw)
        wide = torch.zeros((len(kv), 9000 // page + 3 + self.pages.shape[1]), dtype=torch.int32, device="cuda")
        wide[:, : self.pages.shape[1]] = self.pages
        self.pages = wide


@pytest.fixture(autouse=True)
def long_tables(monkeypatch):
    monkeypatch.setattr(serving, "Batch", LongTables)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_attend_caches_larger_than_the_last_level(dtype, D):
    """Pools of more than 128 MiB, of which the requests have a little: single tokens, and a chunk that one tile holds."""
    spare = (80 << 20) // (4 * D * 16 * 2)
    for new in ([1] * 7, [20, 3]):
        kv = [1300, 2, 700, 33, 64, 95, 1][: len(new)] if len(new) == 7 else [2100, 40]
        LongTables(new, kv, 8, 4, D, 16, dtype, seed=D, spare_pages=spare).check()
