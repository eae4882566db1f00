"""Attention with shared prefixes where the lines are long: more tiles than the first launch keeps the sums of in LDS, and more requests than it has threads."""
import numpy as np
import pytest
import torch

from tests.test_gpu_attend_shared import Shared

pytestmark = pytest.mark.gpu


def _slots(new, groups, group):
    """Places for tiles, of the groups' rows and of the requests': what the line's kernel lays out."""
    rows = sum(new) * group
    return 2 * (rows // 128 + 1) + len(groups) + len(new)


def _lengths(new, groups, seed, most=60, short=()):
    rng = np.random.default_rng(seed)
    of = [s for n, s in groups for _ in range(n)]
    of += [0] * (len(new) - len(of))
    kv = [s + n + int(e) for s, n, e in zip(of, new, rng.integers(0, most, len(new)))]
    for r in short:                                        # fewer keys than are shared
        kv[r] = max(new[r], of[r] // 3)
    return kv


GROUPS = [(700, 90), (1, 40), (500, 131), (0, 17), (250, 65)]


@pytest.mark.parametrize("window", [0, 70, 1])
@pytest.mark.parametrize("short", [(), (3, 250, 699, 702, 1203, 1449)])
def test_more_requests_than_threads(window, short):
    new = [1] * 1500                                       # the last 49 are in no group
    assert _slots(new, GROUPS, 2) > 1024 and len(new) > 1024
    b = Shared(new, _lengths(new, GROUPS, 1, short=short), GROUPS, 4, 2, 64, 64, "f16", seed=2)
    b.check(True, window)


@pytest.mark.parametrize("window", [0, 100])
def test_some_with_drafts_some_without_new_tokens(window):
    rng = np.random.default_rng(3)
    new = [int(n) for n in rng.choice([0, 1, 1, 2, 6, 20], 1400)]
    groups = [(60, 75)] * 20 + [(1, 64)] * 70
    assert _slots(new, groups, 2) > 1024
    b = Shared(new, _lengths(new, groups, 4, short=(61, 130, 500)), groups, 2, 1, 32, 64, "bf16", before=3, seed=5)
    first = b.run(True, window)
    assert all(torch.equal(first, b.run(True, window)) for _ in range(3))
    b.check(True, window)


@pytest.mark.parametrize("q_heads,D,window", [(8, 64, 0), (16, 32, 0), (8, 64, 50), (8, 256, 0)])
def test_few_requests_with_many_rows(q_heads, D, window):
    """Chunks: tiles of shared keys by the hundred for one group, whose rows are of several requests."""
    new = [700, 33, 512, 1, 900, 655, 16, 1027, 3, 1200, 300, 901, 800, 650, 750, 500]
    groups = [(9, 100), (5, 129)]
    if q_heads == 16:
        new, groups = new[:10], [(6, 100), (4, 129)]
    assert _slots(new, groups, q_heads) > 1024
    kv = _lengths(new, groups, 6, short=(2,))
    Shared(new, kv, groups, q_heads, 1, D, 64, "bf16", seed=7).check(True, window)


def test_more_tiles_than_the_first_launch_has_room_for():
    new = [200 + 37 * i % 211 for i in range(16)]
    groups = [(10, 64), (6, 100)]
    assert _slots(new, groups, 20) > 1024
    Shared(new, _lengths(new, groups, 8, most=9), groups, 20, 1, 32, 64, "f16", seed=9).check()
    Shared(new, _lengths(new, groups, 8, most=9), groups, 20, 1, 32, 64, "f16", seed=9).check(True, 40)
