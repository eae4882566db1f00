"""Argument checks of the table of pages and of the draw: all before any launch, so none of this needs a GPU."""
import ctypes
import math

import pytest
import torch

import paper_2407_02891_amd as bcq
from paper_2407_02891_amd import binding as B

OK = 0x1000


def plan(t=(), **kw):
    d = dict(page_size=16, num_pages=1000, requests=8, max_pages=40)
    d.update(t)
    a = dict(pages=0, held=1, fixed=2, free=3, free_count=4, cached=5, fresh=6, tokens=8, q_start=7, kv_len=8, lack=9, held_out=1, count_out=4, positions=10,
             slots=11, owner=12)
    at = {n: OK + 0x10000 * i for n, i in a.items() if n != "tokens"}
    a.update(at)
    a.update({n: at[v[0]] + v[1] if isinstance(v, tuple) else v for n, v in kw.items()})
    return bcq.lib().bcq_plan(ctypes.byref(B.PageTableDesc(*d.values())), *a.values(), None)


def sample(**kw):
    a = dict(dtype=0, rows=4, vocab=100, logits=OK, ld=100, temperature=OK, top_k=OK, top_p=OK, min_p=OK, uniform=OK, token=OK, probability=OK)
    a.update(kw)
    return bcq.lib().bcq_sample(*a.values(), None)


@pytest.mark.parametrize("kw", [dict(tokens=-1)] + [{n: v} for n in ("pages", "held", "free", "free_count", "cached", "fresh", "q_start", "kv_len", "lack", "held_out",
                                                                  "count_out", "positions", "slots", "owner") for v in (None, OK + 2)] + [dict(fixed=OK + 1)])
def test_plan_refuses(kw):
    assert plan(**kw) == B.BCQ_ERR_INVALID_ARG


@pytest.mark.parametrize("a,b", [("kv_len", "cached"), ("kv_len", "fresh"), ("lack", "fixed"), ("pages", "held"), ("pages", "free"), ("q_start", "kv_len"), ("positions", "slots"),
                                 ("owner", "positions"), ("free", "free_count"), ("held_out", "cached"), ("count_out", "held"), ("held_out", "count_out"),
                                 ("owner", "fresh")])
@pytest.mark.parametrize("by", [0, 28, -28])
def test_plan_refuses_what_overlaps(a, b, by):
    if by == 28 and b in ("free_count", "count_out") or by == -28 and a == "count_out":
        by = 0                                             # (one number: its only overlap)
    assert plan(**{a: (b, by)}) == B.BCQ_ERR_INVALID_ARG


def test_plan_refuses_counts_that_begin_in_the_midst():
    assert plan(held_out=("held", 4)) == plan(held_out=("held", -4)) == B.BCQ_ERR_INVALID_ARG


@pytest.mark.parametrize("t", [dict(page_size=0), dict(page_size=-4), dict(num_pages=0), dict(requests=-1), dict(max_pages=0)])
def test_plan_refuses_tables(t):
    assert plan(t) == B.BCQ_ERR_INVALID_ARG
    assert bcq.lib().bcq_plan(None, *[OK] * 7, 8, *[OK] * 8, None) == B.BCQ_ERR_INVALID_ARG


@pytest.mark.parametrize("t,kw", [(dict(page_size=24), {}), (dict(page_size=1 << 17), {}), (dict(num_pages=1 << 28), {}), (dict(max_pages=1 << 27), {}),
                                  (dict(requests=(1 << 20) + 1), {}), (dict(requests=1 << 20, max_pages=1 << 12), {}), ({}, dict(tokens=(1 << 20) + 1))])
def test_plan_limits(t, kw):
    assert plan(t, **kw) == B.BCQ_ERR_UNSUPPORTED


@pytest.mark.parametrize("kw", [dict(dtype=2), dict(dtype=-1), dict(rows=-1), dict(vocab=0), dict(vocab=-5), dict(ld=99), dict(logits=None), dict(temperature=None),
                                dict(uniform=None), dict(token=None), dict(logits=OK + 1), dict(temperature=OK + 2), dict(top_k=OK + 1), dict(top_p=OK + 2),
                                dict(min_p=OK + 3), dict(uniform=OK + 2), dict(token=OK + 2), dict(probability=OK + 2)])
def test_sample_refuses(kw):
    assert sample(**kw) == B.BCQ_ERR_INVALID_ARG


def test_sample_limits():
    assert sample(rows=(1 << 20) + 1) == B.BCQ_ERR_UNSUPPORTED
    assert sample(vocab=B.BCQ_MAX_VOCAB + 1, ld=1 << 40) == B.BCQ_ERR_UNSUPPORTED
    assert sample(rows=0, logits=None, token=None) == B.BCQ_OK   # nothing to do


def _refused(call):
    with pytest.raises(bcq.BcqError) as e:
        call()
    assert e.value.status == B.BCQ_ERR_INVALID_ARG


@pytest.mark.parametrize("device", ["cpu", "meta"])
def test_tensors_that_are_not_on_a_gpu(device):
    pages, held = torch.zeros((2, 4), dtype=torch.int32, device=device), torch.zeros(2, dtype=torch.int32, device=device)
    _refused(lambda: bcq.PageTable(pages, held, held, held[:1], 16))
    _refused(lambda: bcq.PageTable.empty(2, 4, 8, 16, device=device))
    _refused(lambda: bcq.Sampler(torch.ones(2, device=device)))


def test_objects_refuse():
    i = torch.zeros(2, dtype=torch.int32)
    _refused(lambda: bcq.PageTable(i, i, i, i[:1], 16))
    _refused(lambda: bcq.PageTable(torch.zeros((4, 2), dtype=torch.int32).t(), i, i, i[:1], 16))
    _refused(lambda: bcq.Sampler(torch.ones(2, dtype=torch.float64)))
    _refused(lambda: bcq.Sampler(torch.ones((2, 1))))


def shared(c=(), **kw):
    f = dict(dtype=0, kv_heads=8, head_dim=128, page_size=16, num_pages=100, page_stride=16384, head_stride=2048, slot_stride=128)
    f.update(c)
    a = dict(k=OK, v=OK, tokens=4, requests=2, groups=1, q_heads=64, q=OK, ld_q=8192, q_start=OK, kv_len=OK, pages=OK, max_pages=10, max_new=2, group_start=OK,
             shared_len=OK, max_shared=100, scale=0.1, causal=1, window=0, out=OK, ld_out=8192, workspace=OK)
    a.update(kw)
    return bcq.lib().bcq_attend_shared(ctypes.byref(B.Cache(*f.values())), *a.values(), None)


@pytest.mark.parametrize("kw", [dict(tokens=-1), dict(requests=-1), dict(groups=-1), dict(q_heads=0), dict(q_heads=60), dict(max_new=0), dict(max_pages=0),
                                dict(max_shared=-1), dict(scale=0.0), dict(scale=math.nan), dict(scale=math.inf), dict(causal=2), dict(window=-1),
                                dict(causal=0, window=5), dict(ld_q=8184), dict(ld_q=8196), dict(ld_out=8184), dict(k=None), dict(v=None), dict(q=None),
                                dict(q_start=None), dict(kv_len=None), dict(pages=None), dict(out=None), dict(group_start=None), dict(shared_len=None),
                                dict(k=OK + 8), dict(q=OK + 8), dict(out=OK + 2), dict(pages=OK + 2), dict(group_start=OK + 2), dict(shared_len=OK + 1)])
def test_attend_shared_refuses(kw):
    assert shared(**kw) == B.BCQ_ERR_INVALID_ARG


def test_attend_shared_limits():
    assert shared(dict(head_dim=264, slot_stride=264)) == shared(dict(page_size=24)) == B.BCQ_ERR_UNSUPPORTED
    assert shared(dict(kv_heads=0)) == shared(dict(head_stride=4)) == B.BCQ_ERR_INVALID_ARG
    assert shared(tokens=(1 << 20) + 1) == shared(groups=(1 << 20) + 1) == shared(max_pages=1 << 28) == B.BCQ_ERR_UNSUPPORTED
    assert shared(tokens=1 << 20, max_pages=1 << 20) == B.BCQ_ERR_UNSUPPORTED     # blocks of all tiles
    assert shared(workspace=None) == shared(workspace=OK + 8) == B.BCQ_ERR_WORKSPACE
    assert shared(tokens=0, q=None) == shared(requests=0, q=None) == B.BCQ_OK     # nothing to do
    cache = B.Cache(0, 8, 128, 16, 100, 16384, 2048, 128)
    assert bcq.attend_shared_workspace_bytes(cache, 4, 2, 1, 64, 10, 2) > 0
    assert bcq.attend_shared_workspace_bytes(cache, 0, 2, 1, 64, 10, 2) == bcq.attend_shared_workspace_bytes(cache, 4, 2, -1, 64, 10, 2) == 0
