"""What a decoder refuses before it launches anything (no GPU needed: stand-ins for the parts that would)."""
from types import SimpleNamespace

import pytest
import torch

import paper_2407_02891_amd as bcq
from paper_2407_02891_amd import binding as B
from paper_2407_02891_amd.serve_block import Decoder

VOCABULARY, HIDDEN, PAGE = 50, 128, 16


class Table:
    def __init__(self, requests, width, pool):
        self.pages, self.page_size, self.device = torch.zeros((requests, width), dtype=torch.int32), PAGE, torch.device("cpu")
        self.held, self.free, self.free_count = torch.zeros(requests, dtype=torch.int32), torch.arange(pool, dtype=torch.int32), torch.tensor([pool], dtype=torch.int32)

    def step(self, *args, **kw):
        raise RuntimeError("a step is made")


def _parts(requests=2):
    layer = lambda M, N: SimpleNamespace(desc=SimpleNamespace(M=M, N=N))  # noqa: E731
    cache = SimpleNamespace(desc=SimpleNamespace(page_size=PAGE, num_pages=20), head_dim=64)
    block = SimpleNamespace(cache=cache, cos_sin=torch.zeros((8 * PAGE, 64)), qkv=layer(3 * HIDDEN, HIDDEN), o=layer(HIDDEN, HIDDEN))
    return dict(block=block, embedding=torch.zeros((VOCABULARY, HIDDEN), dtype=torch.float16), head=layer(VOCABULARY, HIDDEN), table=Table(requests, 8, 20),
                sampler=SimpleNamespace(temperature=torch.ones(requests)), adapter=0)


@pytest.mark.parametrize("shared,own", [([1, VOCABULARY], [[1], [2]]), ([-1], [[1], [2]]), ([], [[1], [VOCABULARY]]), ([1] * 20, [[3, 4, -2], [2]]), ([1] * 40 + [2 ** 40], [[1], [2]]),
                                        ([0], [[0], [-2 ** 70]])])
def test_ids_that_are_not_the_embeddings(shared, own):
    """An index of the device's beyond the embedding ends the process's use of it, and a negative one counts from its end."""
    decoder = Decoder(**_parts())
    with pytest.raises(bcq.BcqError, match="Decoder.prompt .ids") as e:
        decoder.prompt(shared, own, torch.full((2,), 0.5))
    assert e.value.status == B.BCQ_ERR_INVALID_ARG


@pytest.mark.parametrize("shared,own", [([], [[0], [VOCABULARY - 1]]), ([0, VOCABULARY - 1], [[0], [1]]), ([7] * 33, [[1, 2], [VOCABULARY - 1]])])
def test_the_first_and_the_last_id(shared, own):
    with pytest.raises(RuntimeError, match="a step is made"):
        Decoder(**_parts()).prompt(shared, own, torch.full((2,), 0.5))


@pytest.mark.parametrize("change", [dict(embedding=torch.zeros((VOCABULARY, HIDDEN))), dict(embedding=torch.zeros((VOCABULARY, HIDDEN), dtype=torch.bfloat16)),
                                    dict(embedding=torch.zeros((VOCABULARY, HIDDEN + 128), dtype=torch.float16)),
                                    dict(embedding=torch.zeros((VOCABULARY, HIDDEN // 2), dtype=torch.float16)),
                                    dict(head=SimpleNamespace(desc=SimpleNamespace(M=VOCABULARY, N=HIDDEN // 2))),
                                    dict(head=SimpleNamespace(desc=SimpleNamespace(M=VOCABULARY, N=2 * HIDDEN)))])
def test_an_embedding_or_a_head_of_another_type_or_width(change):
    """The products take an address and a row stride: another type was read as binary16, and a wider row's end was left out."""
    Decoder(**_parts())
    with pytest.raises(bcq.BcqError, match="Decoder") as e:
        Decoder(**dict(_parts(), **change))
    assert e.value.status == B.BCQ_ERR_INVALID_ARG
