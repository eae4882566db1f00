"""The table of pages and the batch's rows from the lengths, against the plain form, request by request."""
import random

import pytest
import torch

import paper_2407_02891_amd as bcq
from tests.step_util import plan_ref

pytestmark = pytest.mark.gpu
STEP = ("q_start", "kv_len", "lack", "held", "free_count", "positions", "slots", "owner")


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


class Pool:
    """A table on the GPU and the same as lists."""

    def __init__(self, requests, max_pages, num_pages, page, seed):
        rng = random.Random(seed)
        self.page, self.max_pages, self.num_pages = page, max_pages, num_pages
        self.free = list(range(num_pages))
        rng.shuffle(self.free)
        self.pages = [[-1] * max_pages for _ in range(requests)]
        self.held, self.count = [0] * requests, num_pages
        self.table = bcq.PageTable(torch.full((requests, max_pages), -1, dtype=torch.int32, device="cuda"), _ints([0] * requests), _ints(self.free),
                                   _ints([num_pages]), page)

    def step(self, cached, fresh, tokens, fixed=None, **kw):
        args = (self.page, self.num_pages, self.max_pages, self.pages, self.held, self.free, self.count, cached, fresh, tokens, fixed)
        ref = plan_ref(*args)
        got = self.table.step(_ints(cached), _ints(fresh), tokens, fixed=None if fixed is None else _ints(fixed), **kw)
        for n in STEP:
            assert got[n].tolist() == ref[n], n
        assert self.table.pages.tolist() == ref["pages"] and self.table.free.tolist() == ref["free"]
        self.pages, self.free = ref["pages"], ref["free"]
        if not kw.get("trial"):
            self.held, self.count = ref["held"], ref["free_count"][0]
            assert self.table.held.tolist() == self.held and self.table.free_count.tolist() == [self.count]
        return ref, got


@pytest.mark.parametrize("requests,page,max_pages", [(1, 16, 9), (2, 1, 40), (7, 8, 20), (64, 16, 12), (65, 32, 6), (1023, 16, 5), (1024, 4, 8), (1025, 16, 5), (2100, 16, 4)])
def test_many_steps(requests, page, max_pages):
    """Requests that grow by tokens, drafts that are rejected, ends and beginnings; pages run out now and then; what the table holds is the pool's, once."""
    rng = random.Random(requests)
    pool = Pool(requests, max_pages, max(3, requests * max_pages // 12), page, requests)
    length = [0] * requests
    short = 0
    for turn in range(8):
        cached, fresh = [], []
        for r in range(requests):
            n = rng.choice([0, 1, 1, 1, 5, rng.randrange(0, max_pages * page + 2) if rng.random() < 0.3 else 1])
            keep = 0 if rng.random() < 0.15 else max(0, length[r] - rng.choice([0, 0, 0, 3]))
            cached.append(keep)
            fresh.append(n)
        tokens = sum(fresh) + rng.choice([0, 1, 70, -sum(fresh) // 3])
        ref, _ = pool.step(cached, fresh, tokens)
        short += sum(v > 0 for v in ref["lack"])
        length = [ref["kv_len"][r] if ref["lack"][r] == 0 else length[r] for r in range(requests)]
        used = [p for r in range(requests) for p in pool.pages[r][:pool.held[r]]] + pool.free[:pool.count]
        assert sorted(used) == list(range(pool.num_pages))
    assert requests < 64 or short > 0  # (some do lack pages)


@pytest.mark.parametrize("tokens", [0, 1, 63, 4095, 4096, 4097, 9000])
def test_rows_of_the_batch(tokens):
    """Batches of one launch and of two, rows that nobody has, rows that do not reach."""
    pool = Pool(5, 600, 2500, 16, 1)
    pool.step([0] * 5, [1000, 0, 2500, 7, 4000], tokens)
    pool.step([0] * 5, [0, 0, 0, 0, 0], tokens)


def test_prompt_that_others_have_too():
    """The first pages of the rows are not taken and not given back."""
    pool = Pool(6, 30, 100, 8, 2)
    pool.step([0] * 6, [40, 0, 0, 0, 0, 0], 40)
    prefix = pool.pages[0][:5]
    for r in range(1, 6):
        pool.pages[r][:5] = prefix
        pool.held[r] = 5
    pool.table.pages[1:, :5] = _ints(prefix)
    pool.table.held[1:] = 5
    fixed = [0, 5, 5, 5, 5, 9]
    pool.step([40] * 6, [1, 3, 9, 0, 30, 1], 50, fixed)
    pool.step([41, 43, 0, 0, 60, 41], [1, 1, 0, 0, 1, 1], 8, fixed)
    ref, _ = pool.step([0] * 6, [0] * 6, 8, fixed)
    assert ref["held"] == [0, 5, 5, 5, 5, 6] and ref["free_count"] == [99]  # (the last holds six, so its nine are six)


def test_pages_that_run_out_to_the_last():
    """Exactly as many as there are; one too few: the first that lacks keeps later ones waiting, those that need none go on."""
    pool = Pool(4, 8, 10, 4, 3)
    ref, _ = pool.step([0] * 4, [16, 12, 8, 4], 40)
    assert ref["lack"] == [0] * 4 and ref["free_count"] == [0]
    ref, _ = pool.step([16, 12, 8, 4], [1, 0, 1, 0], 40)
    assert ref["lack"] == [1, 0, 1, 0] and ref["kv_len"] == [0, 12, 0, 4]
    ref, _ = pool.step([16, 12, 0, 4], [1, 1, 0, 1], 40)  # what one gives back the others take in the same step
    assert ref["lack"] == [0, 0, 0, 1] and ref["free_count"] == [0]


def test_a_trial_moves_nothing():
    pool = Pool(3, 8, 20, 4, 4)
    pool.step([0] * 3, [5, 9, 1], 20)
    before = pool.table.held.tolist(), pool.table.free_count.tolist(), [row[:h] for row, h in zip(pool.pages, pool.held)], pool.free[:pool.count]
    for _ in range(2):
        _, got = pool.step([5, 9, 1], [9, 9, 90], 60, trial=True)
    assert got["held"].data_ptr() != pool.table.held.data_ptr()
    assert before == (pool.table.held.tolist(), pool.table.free_count.tolist(), [row[:h] for row, h in zip(pool.pages, pool.held)], pool.free[:pool.count])
    _, again = pool.step([5, 9, 1], [9, 9, 90], 60, trial=True, out=got)
    assert again is got


def test_numbers_that_make_no_sense():
    """Whatever the arrays hold, nothing outside them is read or written, and sensible requests beside them get what they should."""
    low, high = -2 ** 31, 2 ** 31 - 1
    pool = Pool(8, 6, 30, 8, 5)
    pool.step([0, low, high, 3, -5, 0, high, 0], [4, 1, 1, high, 2, -7, high, low], 20)
    pool.table.held.copy_(_ints([low, 99, high, 0, 1, 2, 3, 0]))
    pool.held = [low, 99, high, 0, 1, 2, 3, 0]
    pool.table.free_count.fill_(12)
    pool.count = 12
    pool.step([1] * 8, [1] * 8, 20, fixed=[high, low, 3, 3, 3, 3, 3, 3])
    for count in (low, -1, high):
        pool.table.free_count.fill_(count)
        pool.table.step(_ints([1] * 8), _ints([9] * 8), 100, trial=True)
    pool.table.pages.fill_(high)  # page numbers that are none: slots outside the cache
    pool.table.held.fill_(6)
    got = pool.table.step(_ints([1] * 8), _ints([1] * 8), 16, trial=True)
    assert got["slots"].tolist() == [-1] * 16 and got["positions"].tolist() == [1] * 8 + [0] * 8
    torch.cuda.synchronize()


def test_no_requests():
    table = bcq.PageTable.empty(0, 4, 10, 16)
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    for tokens in (0, 5, 5000):
        got = table.step(none, none, tokens)
        assert got["q_start"].tolist() == [0] and got["slots"].tolist() == [-1] * tokens and got["owner"].tolist() == [-1] * tokens


def test_a_graph_of_steps():
    """A captured step of single tokens, replayed while the lengths advance in place, is the eager steps."""
    pools = [Pool(20, 10, 120, 4, 6) for _ in range(2)]
    for p in pools:
        p.step([0] * 20, list(range(1, 21)), 300)
    cached, one = _ints(list(range(1, 21))), _ints([1] * 20)
    out = pools[1].table.step(cached, torch.zeros_like(one), 24)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pools[1].table.step(cached, one, 24, out=out)
    length = list(range(1, 21))
    for turn in range(6):
        graph.replay()
        ref, got = pools[0].step(length, [1] * 20, 24)
        torch.cuda.synchronize()
        for n in STEP:
            assert out[n].tolist() == ref[n], (turn, n)
        assert [r[:h] for r, h in zip(pools[1].table.pages.tolist(), ref["held"])] == [r[:h] for r, h in zip(ref["pages"], ref["held"])]
        cached += 1
        length = [n + 1 for n in length]


def test_the_lengths_of_an_earlier_step():
    """kv_len of one step as `cached` of the next: with other tensors for what that writes; the same ones are refused, for they would be read after they are written."""
    pool = Pool(5, 8, 30, 16, 3)
    new = [5, 40, 0, 17, 30]
    _, first = pool.step([0] * 5, new, 100)
    with pytest.raises(bcq.BcqError):
        pool.table.step(first["kv_len"], _ints([1] * 5), 100, out=first)
    with pytest.raises(bcq.BcqError):
        pool.table.step(_ints(new), first["lack"], 100, out=first)
    with pytest.raises(bcq.BcqError):
        pool.table.step(_ints(new), pool.table.held, 100)
    with pytest.raises(bcq.BcqError):
        pool.table.step(_ints(new), _ints(new), 100, out=dict(first, slots=first["positions"]))
    args = (16, 30, 8, pool.pages, pool.held, pool.free, pool.count, new, [1] * 5, 100)
    got = pool.table.step(first["kv_len"], _ints([1] * 5), 100)
    ref = plan_ref(*args)
    for n in STEP:
        assert got[n].tolist() == ref[n], n


def test_refusals():
    """Shapes, types and places that do not fit are refused before anything runs."""
    table = bcq.PageTable.empty(3, 4, 10, 16)
    i = torch.zeros(3, dtype=torch.int32, device="cuda")
    step = table.step(i, i, 5)
    trial = table.step(i, i, 5, trial=True)
    for call in (lambda: table.step(i[:2], i, 5), lambda: table.step(i, i.long(), 5), lambda: table.step(i.cpu(), i, 5), lambda: table.step(i, i, -1),
                 lambda: table.step(i, i, 1 << 32), lambda: table.step(i, i, 5, fixed=i[:1]), lambda: table.step(i, i, 6, out=step), lambda: table.step(i, i, 5, out={}),
                 lambda: table.step(i, i, 5, out=trial), lambda: table.step(i, i, 5, out=step, trial=True), lambda: table.step(i, i, 5, out=i), lambda: table.step(None, i, 5)):
        with pytest.raises(bcq.BcqError):
            call()
    for args in ((table.pages.float(), i, i, i[:1]), (table.pages, i[:2], i, i[:1]), (table.pages, i, i.cpu(), i[:1]), (table.pages, i, i, i), (table.pages.t(), i, i, i[:1])):
        with pytest.raises(bcq.BcqError):
            bcq.PageTable(*args, 16)
    with pytest.raises(bcq.BcqError):
        bcq.PageTable(table.pages, i, i, i[:1], 24).step(i, i, 5)
