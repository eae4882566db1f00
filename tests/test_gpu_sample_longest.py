"""Rows of the most logits that a draw takes, most or all of them alike: the list of entries that 16-bit counters could not hold is full to its last place."""
import math

import pytest
import torch

import paper_2407_02891_amd as bcq
from paper_2407_02891_amd import binding as B
from tests.step_util import assert_drawn

pytestmark = pytest.mark.gpu
V = B.BCQ_MAX_VOCAB


def _draw(x, u, **settings):
    rows = x.shape[0]
    put = lambda name, dtype: torch.full((rows,), settings[name], dtype=dtype, device="cuda") if name in settings else None  # noqa: E731
    token, p = bcq.Sampler(torch.ones(rows, device="cuda"), put("top_k", torch.int32), put("top_p", torch.float32), put("min_p", torch.float32)).draw(x, u.cuda())
    return token.tolist(), p.cpu()


def _row(fill, dtype, offset):
    """A row that begins `offset` elements behind 16 bytes."""
    x = torch.empty(V + 16, dtype=dtype, device="cuda")
    x.fill_(math.inf)
    x = x[offset:offset + V]
    x.copy_(fill)
    return x[None]


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("offset", [0, 1, 7])
@pytest.mark.parametrize("values", [(0.0, -0.0), (-0.0, -0.0), (-2.5, -2.5), (3.0, 3.0)], ids=str)
def test_all_alike(values, offset, dtype):
    """Weights of one: the token is where the number points, the shares are whole numbers of entries."""
    fill = torch.tensor(values, device="cuda").repeat(V // 2).to(dtype)
    x = _row(fill, dtype, offset)
    for i in (0, 1, 32767, 32768, V // 3, V - 2, V - 1):
        token, p = _draw(x, torch.tensor([(2 * i + 1) / (2 * V)]))            # (24 bits: exact)
        assert token == [i] and float(p) == 1 / V
    one = torch.ones(1)
    assert _draw(x, one)[0] == [V - 1]                                        # the last number there is
    assert _draw(x, one, top_k=V // 2 + 5)[0] == [V // 2 + 4]
    assert _draw(x, one, top_k=V - 1)[0] == [V - 2]
    assert _draw(x, one, top_p=0.25)[0] == [V // 4 - 1]
    assert _draw(x, one, min_p=1.0)[0] == [V - 1]


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("nothing", [math.nan, -math.nan, -math.inf], ids=["nan", "negative nan", "-inf"])
def test_nearly_all_without_a_part(nothing, dtype):
    fill = torch.full((V,), nothing, device="cuda").to(dtype)
    if nothing != nothing:
        bits = fill.view(torch.int16)
        bits.copy_(torch.full_like(bits, (0x7fff if math.copysign(1.0, nothing) > 0 else -1)))
        assert bool(fill.isnan().all())
    assert _draw(_row(fill, dtype, 3), torch.tensor([0.5]))[0] == [-1]
    at = [5, 40000, V - 3]
    fill[at] = torch.tensor([1.0, -0.0, 1.0], device="cuda").to(dtype)
    x = _row(fill, dtype, 3)
    weight = [1.0, math.exp(-1.0), 1.0]
    for u, i in ((0.0, 0), (0.4, 0), (0.45, 2), (0.8, 2), (0.9, 1)):         # the ones in the order of the index, then zero
        token, p = _draw(x, torch.tensor([u]))
        assert token == [at[i]] and abs(float(p) - weight[i] / sum(weight)) <= 2.0 ** -23 * float(p)


def test_two_values_shuffled():
    g = torch.Generator(device="cuda").manual_seed(2)
    pick = torch.rand(V, device="cuda", generator=g) < 0.5
    x = torch.stack([torch.where(pick, a, b) for a, b in ((1.5, -1.5), (-0.0, 0.0), (-3.0, -3.5))]).to(torch.float16)
    u = torch.tensor([0.3, 0.7, 0.999])
    T, top_p = torch.tensor([1.0, 0.5, 20.0]), torch.tensor([0.97, 0.5, 0.9])
    token, p = bcq.Sampler(T.cuda(), None, top_p.cuda()).draw(x, u.cuda())
    assert_drawn(token, p, x.cpu(), T, None, top_p, None, u)
