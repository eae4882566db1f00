"""The operators of a step together, as a server uses them: pages handed out, rotation with the append, attention with a shared prompt, projections and a
head, and the draw, each request against the whole computed in 64 bits."""
import numpy as np
import pytest
import torch

from paper_2407_02891_amd import BcqError, PageTable, Sampler
from paper_2407_02891_amd.serve_block import Decoder, random_block, random_head
from tests.step_util import assert_drawn
from tests.test_gpu_serve_block import ADAPTERS, D, HIDDEN, HKV, HQ, PAGE, RANK, SHARE, _dense, _reference

pytestmark = pytest.mark.gpu

VOCABULARY = 1000


class Recorded:
    """A sampler that keeps what it was given and what it drew."""

    def __init__(self, sampler):
        self.sampler, self.temperature, self.calls = sampler, sampler.temperature, []

    def draw(self, logits, uniform):
        token, probability = self.sampler.draw(logits, uniform)
        self.calls.append((logits.clone(), uniform.clone(), token, probability))
        return token, probability


def _decoder(requests, width, pool, seed=3, adapter=1):
    block, weights = random_block(HIDDEN, HQ, HKV, D, 3, pool, PAGE, width * PAGE, ADAPTERS, RANK, seed=seed)
    embedding, head, dense = random_head(HIDDEN, VOCABULARY, 2, seed=seed + 1)
    g = torch.Generator(device="cuda").manual_seed(seed + 2)
    settings = [torch.rand(requests, device="cuda", generator=g) + 0.3, torch.randint(0, 60, (requests,), device="cuda", generator=g, dtype=torch.int32),
                torch.rand(requests, device="cuda", generator=g) * 0.5 + 0.5, torch.rand(requests, device="cuda", generator=g) * 0.1]
    decoder = Decoder(block, embedding, head, PageTable.empty(requests, width, pool, PAGE), Recorded(Sampler(*settings)), adapter)
    return decoder, weights, dense, settings


def _owned(decoder):
    """Every page of the pool is free, one request's or the prompt's."""
    t = decoder.table
    held, fixed, count = t.held.tolist(), decoder.fixed.tolist(), int(t.free_count)
    mine = [p for r, row in enumerate(t.pages.tolist()) for p in row[fixed[r]:held[r]]]
    every = t.free.tolist()[:count] + mine + t.pages[0].tolist()[:fixed[0]]
    assert sorted(every) == list(range(t.free.shape[0]))


@pytest.mark.parametrize("shared,own,adapter", [(37, (1, 9, 4), 0), (64, (70, 1, 3, 33, 16), 1), (5, (2, 40), -1), (0, (20,), 1)])
def test_against_64_bits(shared, own, adapter):
    steps, g = 5, torch.Generator().manual_seed(shared)
    longest = shared + max(own) + steps
    decoder, weights, dense, settings = _decoder(len(own), -(-longest // PAGE), 64, adapter=adapter)
    ids = torch.randint(0, VOCABULARY, (longest + sum(own),), generator=g).tolist()
    prompt, starts = ids[:shared], [ids[shared + sum(own[:r]):shared + sum(own[:r + 1])] for r in range(len(own))]
    tokens, uniform = [], torch.rand((steps, len(own)), generator=g).cuda()
    for i in range(steps):
        decoder.prompt(prompt, starts, uniform[0]) if i == 0 else decoder.step(uniform[i])
        tokens.append(decoder.token.tolist())
        _owned(decoder)
    for logits, u, token, probability in decoder.sampler.calls:
        assert_drawn(token, probability, logits, *settings, u)
    W = _dense(*dense)
    grow = np.linalg.norm(W, 2)
    for r, start in enumerate(starts):
        sequence = prompt + start + [t[r] for t in tokens[:-1]]
        z = _reference(decoder.block, weights, decoder.embedding[sequence].cpu().double().numpy(), adapter)[-steps:]
        for i in range(steps):
            # the rows' own bound through the head, whose products round once more (2^-11 an element, and its sums as much again)
            off = np.linalg.norm(decoder.sampler.calls[i][0][r].cpu().double().numpy() - z[i] @ W.T)
            assert off <= grow * SHARE * np.linalg.norm(z[i]) + 2.0 ** -10 * np.linalg.norm(z[i] @ W.T), (r, i, off)


def test_a_replayed_step_is_the_eager_one():
    own = (3, 15, 30, 8)
    decoder, _, _, _ = _decoder(4, 8, 40)
    ids = list(range(200))
    uniform = torch.rand(4, device="cuda")
    decoder.prompt(ids[:50], [ids[60:60 + n] for n in own], uniform)
    decoder.sampler = decoder.sampler.sampler
    decoder.step(uniform)
    state = [decoder.cached, decoder.fresh, decoder.token, decoder.probability, decoder.table.pages, decoder.table.held, decoder.table.free,
             decoder.table.free_count, decoder.block.cache.k, decoder.block.cache.v]
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        decoder.step(uniform)
    before, numbers = [t.clone() for t in state], torch.rand((20, 4), device="cuda")
    runs = []
    for make in (graph.replay, lambda: decoder.step(uniform)):
        for t, was in zip(state, before):
            t.copy_(was)
        seen = []
        for i in range(20):
            uniform.copy_(numbers[i])
            if i == 9:
                decoder.leave(2)
            make()
            seen.append((decoder.token.tolist(), decoder.probability.tolist(), decoder.table.held.tolist(), decoder.cached.tolist()))
            _owned(decoder)
        runs.append(seen)
    assert runs[0] == runs[1]
    assert len({tuple(s[0]) for s in runs[0]}) > 10 and runs[0][-1][2][2] == 50 // PAGE and runs[0][-1][3][2] == 0


def test_who_lacks_a_page_waits():
    # two pages of the prompt and one of each request: none is free when they fill
    decoder, _, _, _ = _decoder(3, 4, 5)
    ids = list(range(64))
    uniform = torch.full((3,), 0.5, device="cuda")
    decoder.prompt(ids[:32], [ids[40:54], ids[40:50], ids[40:53]], uniform)
    for _ in range(2):
        decoder.step(uniform)
    assert decoder.cached.tolist() == [48, 44, 47] and int(decoder.table.free_count) == 0
    token = decoder.token.tolist()
    decoder.step(uniform)                                  # the first request's page is full
    assert decoder.plan["lack"].tolist() == [1, 0, 0] and decoder.cached.tolist() == [48, 45, 48]
    assert decoder.token[0] == token[0]
    held_back = decoder.token[0].item()
    decoder.leave(2)
    decoder.step(uniform)
    assert decoder.plan["lack"].tolist() == [0, 0, 0] and decoder.cached.tolist() == [49, 46, 0] and decoder.table.held.tolist() == [4, 3, 2]
    _owned(decoder)
    # as if it had never waited
    other, _, _, _ = _decoder(3, 4, 12)
    other.prompt(ids[:32], [ids[40:54], ids[40:50], ids[40:53]], uniform)
    for _ in range(2):
        other.step(uniform)
    assert other.token.tolist() == token and other.token[0] == held_back
    other.step(uniform)
    assert other.token[0] == decoder.token[0]


@pytest.mark.parametrize("shared,own,message", [(16, [[1], []], "one id"), (65, [[1], [2]], "fit"), (32, [[1] * 33, [2]], "fit"), (80, [[1], [2]], "fit"),
                                                (0, [[1] * 48, [2] * 33], "fit")])
def test_prompts_that_do_not_fit(shared, own, message):
    decoder, _, _, _ = _decoder(2, 4, 5)
    with pytest.raises(BcqError, match=message):
        decoder.prompt(list(range(shared)), own, torch.full((2,), 0.5, device="cuda"))
    assert int(decoder.table.free_count) == 5
    decoder.prompt(list(range(34)), [[1], [2]], torch.full((2,), 0.5, device="cuda"))
    with pytest.raises(BcqError, match="begun"):
        decoder.prompt([], [[1], [2]], torch.full((2,), 0.5, device="cuda"))


def test_parts_that_do_not_belong_together():
    d, _, _, settings = _decoder(2, 4, 5)
    table = lambda width=4, pool=5, page=PAGE, requests=2: PageTable.empty(requests, width, pool, page)  # noqa: E731
    other = Sampler(*(t[:1].contiguous() for t in settings))
    for parts in ((d.embedding, d.head, table(page=2 * PAGE), d.sampler.sampler), (d.embedding, d.head, table(pool=6), d.sampler.sampler),
                  (d.embedding, d.head, table(width=5), d.sampler.sampler), (d.embedding[:-1], d.head, table(), d.sampler.sampler), (d.embedding, d.head, table(), other),
                  (d.embedding, d.head, table(requests=3), d.sampler.sampler)):
        with pytest.raises(BcqError, match="Decoder"):
            Decoder(d.block, *parts, 0)
    Decoder(d.block, d.embedding, d.head, table(width=3, pool=4), d.sampler.sampler, 0)
