"""Calls of the serving operators at the edges of what they take: strides, single rows, magnitudes and contents that the ordinary cases
do not have.  Bounds are those of the plain forms in serving_util."""
import math

import pytest
import torch

import paper_2407_02891_amd as bcq
from tests.serving_util import assert_close, attend_ref
from tests.test_gpu_serving import DT, _gen, _ints

pytestmark = pytest.mark.gpu


def _interleaved_cache(pages, page, kv_heads, D, slot_stride, dtype, seed):
    """k and v as views of tensors whose slots are slot_stride elements apart (a layer of a cache that keeps all layers of a slot together)."""
    caches = []
    for i in range(2):
        whole = torch.full((pages, page, slot_stride), math.nan, dtype=dtype, device="cuda")
        view = whole[:, :, : kv_heads * D].unflatten(2, (kv_heads, D)).transpose(1, 2)
        view.copy_(torch.randn(view.shape, device="cuda", generator=_gen(seed + i)))
        caches.append(view)
    return caches


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("new,D,kv", [(40, 128, 20011), (40, 128, 13200), (9, 64, 26300), (300, 256, 13111), (1, 128, 20011)])
def test_attend_keys_times_slot_stride_beyond_32_bits(dtype, new, D, kv):
    """A long request over a cache whose slots are far apart; its few pages come again and again, so that the memory stays small."""
    page, heads, stride = 16, 2, 163840
    assert (kv - 1) * stride > 2 ** 31
    k, v = _interleaved_cache(5, page, heads, D, stride, DT[dtype], seed=D)
    table = torch.randint(0, 5, (1, -(-kv // page) + 1), device="cuda", generator=_gen(1), dtype=torch.int32)
    q = torch.randn((new, 4 * D), device="cuda", generator=_gen(2)).to(DT[dtype])
    got = bcq.PagedCache(k, v).attend(q, _ints([0, new]), _ints([kv]), table, new)
    ref, bound, _ = attend_ref(q, k, v, _ints([0, new]), _ints([kv]), table, 4, D ** -0.5, True, 0)
    assert_close(got, ref, bound)
