"""Attention of requests that share their first keys, against the plain form in 64 bits over requests that each have them: what the others' own rows of pages
say of the shared keys is NaN or no page at all."""
import math

import numpy as np
import pytest
import torch

import paper_2407_02891_amd as bcq
from tests.serving_util import assert_close, attend_ref
from tests.test_gpu_serving import DT, Batch, _ints

pytestmark = pytest.mark.gpu


class Shared(Batch):
    """groups: (number of requests, shared keys) one after the other; requests behind the last are in none."""

    def __init__(self, new, kv, groups, q_heads, kv_heads, D, page, dtype, before=0, **kw):
        super().__init__(new, kv, q_heads, kv_heads, D, page, dtype, **kw)
        self.start, self.shared = list(np.cumsum([before] + [n for n, _ in groups])), [s for _, s in groups]
        self.group_start, self.shared_len = _ints(self.start), _ints(self.shared)
        # the plain form's caches hold the shared keys in every request's own pages
        self.ref_k, self.ref_v, self.ref_pages = self.k.clone(), self.v.clone(), self.pages.clone()
        for c, (n, s) in enumerate(groups):
            first = self.start[c]
            for r in range(first + 1, first + n):
                j = torch.arange(min(s, kv[r]), device="cuda")
                if not len(j):
                    continue
                mine, its = self.pages[r].long()[j // page], self.pages[first].long()[j // page]
                for mut, ref in ((self.k, self.ref_k), (self.v, self.ref_v)):
                    ref[mine, :, j % page] = ref[its, :, j % page]
                    mut[mine, :, j % page] = math.nan
                self.pages[r, : s // page] = -1 if r % 2 else 1 << 30  # whole pages of them: not looked at

    def run(self, causal=True, window=0, scale=None, out=None, max_new=None, max_shared=None):
        return self.cache.attend_shared(self.q, self.q_start, self.kv_len, self.pages, max_new or max(self.new), self.group_start, self.shared_len,
                                        max(self.shared) if max_shared is None else max_shared, scale=scale, causal=causal, window=window, out=out)

    def reference(self, causal=True, window=0, scale=None, max_new=None):
        return attend_ref(self.q, self.ref_k, self.ref_v, self.q_start, self.kv_len, self.ref_pages, self.q_heads,
                          self.k.shape[3] ** -0.5 if scale is None else scale, causal, window, max_new)

    def check(self, causal=True, window=0, scale=None, what=""):
        got = self.run(causal, window, scale)
        torch.cuda.synchronize()
        ref, bound, written = self.reference(causal, window, scale)
        assert bool(written.all())
        assert_close(got, ref, bound, what)


HEADS = [(8, 1, 128, 16), (4, 4, 64, 32), (6, 2, 80, 8), (2, 2, 256, 64), (5, 1, 96, 1), (3, 3, 8, 2), (16, 1, 128, 128), (4, 2, 136, 16)]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("q_heads,kv_heads,D,page", HEADS)
def test_single_tokens(q_heads, kv_heads, D, page, dtype):
    """One group; shared keys that end inside a page and a block, own keys of every edge of a tile."""
    own = [1, 2, 15, 16, 17, 31, 33, 63, 64, 65, 130, 200]
    Shared([1] * len(own), [333 + n for n in own], [(len(own), 333)], q_heads, kv_heads, D, page, dtype, seed=D).check()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("shared", [0, 1, 15, 16, 31, 32, 33, 63, 64, 65, 127, 128, 129, 1000])
def test_every_length_of_what_is_shared(shared, dtype):
    Shared([1, 1, 1], [shared + 1, shared + 40, shared + 64], [(3, shared)], 4, 2, 64, 16, dtype).check(what=shared)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("q_heads,kv_heads,D,page", [(8, 1, 128, 16), (4, 4, 64, 32), (5, 1, 96, 4), (2, 1, 256, 16)])
@pytest.mark.parametrize("causal,window", [(True, 0), (True, 1), (True, 7), (True, 90), (True, 5000), (False, 0)])
def test_groups_and_chunks(q_heads, kv_heads, D, page, causal, window, dtype):
    """Groups of different sizes and lengths, drafts and chunks, requests in front of the groups and behind them, a group of one and one of none."""
    new = [1, 2, 3, 5, 1, 17, 33, 1, 1, 70, 2]
    kv = [40, 150, 190, 161, 151, 117, 133, 116, 1, 270, 77]
    Shared(new, kv, [(4, 145), (0, 50), (3, 100), (1, 200)], q_heads, kv_heads, D, page, dtype, before=1, seed=page).check(causal, window)


@pytest.mark.parametrize("requests,groups,shared", [(300, 1, 70), (130, 40, 33), (65, 65, 20), (257, 3, 700)])
def test_many_requests(requests, groups, shared):
    """Several tiles of rows over the same keys, tiles that hold the ends of requests, no new tokens in some."""
    rng = np.random.default_rng(requests)
    ends = [g * requests // groups for g in range(groups + 1)]
    sizes = [(b - a, int(shared + rng.integers(0, 20))) for a, b in zip(ends, ends[1:])]
    of = [s for n, s in sizes for _ in range(n)]
    for new, dtype in (([1] * requests, "f16"), ([int(n) for n in rng.choice([0, 1, 1, 2, 9], requests)], "bf16")):
        kv = [s + n + int(e) for s, n, e in zip(of, new, rng.integers(0, 60, requests))]
        Shared(new, kv, sizes, 4, 2, 64, 16, dtype).check()


@pytest.mark.parametrize("new", [1, 4])
@pytest.mark.parametrize("q_heads,kv_heads", [(71, 1), (64, 1), (40, 2), (33, 1), (150, 1)])
def test_many_query_heads_share_one(q_heads, kv_heads, new):
    Shared([new] * 4, [100 + new, 177, 500, 101 + new], [(4, 100)], q_heads, kv_heads, 64, 16, "f16").check()


@pytest.mark.parametrize("window", [1, 60, 301, 640, 1100, 5000])
@pytest.mark.parametrize("D,dtype", [(64, "bf16"), (128, "f16"), (256, "bf16")])
def test_windows_that_begin_behind_shared_keys(D, dtype, window):
    # of a group's tiles each begins where the first of its rows does, some have nothing left; by lines laid out in the workgroups and, with many requests, before them
    own = [1, 300, 640, 64, 900, 2, 30, 31]
    Shared([1] * len(own), [1000 + n for n in own], [(len(own), 1000)], 64, 1, D, 16, dtype).check(True, window)
    new = [3, 1, 1, 40] * 40
    kv = [700 + n + (37 * i) % 900 for i, n in enumerate(new)]
    Shared(new, kv, [(90, 700), (70, 513)], 8, 2, D, 16, dtype).check(True, window)


@pytest.mark.parametrize("q_heads,kv_heads,D", [(300, 300, 64), (514, 257, 32), (300, 300, 256), (130, 130, 128), (1000, 500, 64)])
def test_heads_that_fill_the_chip(q_heads, kv_heads, D):
    Shared([1, 1, 1], [150, 90, 60], [(2, 80)], q_heads, kv_heads, D, 16, "bf16").check()
    Shared([1, 20, 2], [150, 100, 60], [(3, 50)], q_heads, kv_heads, D, 16, "f16").check()


@pytest.mark.parametrize("new", [1, 6])
def test_long_prefix_is_split(new):
    Shared([new] * 5, [20011 + n for n in (7, 300, 64, 2000, 6)], [(5, 20011)], 4, 1, 128, 32, "f16").check()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("causal", [True, False])
def test_rows_that_see_little_or_nothing(causal, dtype):
    """Requests with fewer keys than are shared, with none, with new tokens among the shared keys or before the first."""
    new, kv = [1, 0, 5, 2, 40, 1, 3, 4], [100, 150, 3, 0, 33, 101, 80, 82]
    b = Shared(new, kv, [(8, 80)], 8, 2, 64, 16, dtype)
    b.check(causal)
    out = b.run(causal)
    assert bool((out[6:8] == 0).all())
    if causal:
        assert bool((out[1:3] == 0).all()) and not bool((out[3] == 0).any())
    Shared([2, 2], [0, 0], [(2, 0)], 2, 2, 128, 16, dtype).check(causal)


def test_the_first_request_may_have_fewer_keys_than_are_shared():
    """Its row of pages holds what is shared all the same."""
    b = Shared([1, 1, 2], [150, 190, 170], [(3, 140)], 4, 2, 64, 16, "f16")
    b.kv_len[0] = 30
    b.check()


def test_max_shared_bounds_what_is_shared():
    """Keys behind it are each request's own."""
    b = Shared([1, 3, 1], [90, 100, 110], [(3, 50)], 4, 2, 64, 16, "f16")
    b.shared_len.fill_(80)
    for r in (1, 2):  # 50 .. 79: the requests' own
        j = torch.arange(50, 80, device="cuda")
        assert bool(b.k[b.ref_pages[r].long()[j // 16], 0, j % 16].isfinite().all())
    got = b.run(max_shared=50)
    ref, bound, _ = b.reference()
    assert_close(got, ref, bound)
    plain = Shared([1, 3, 1], [90, 100, 110], [(3, 0)], 4, 2, 64, 16, "f16")
    plain.shared_len.fill_(60)
    got = plain.run(max_shared=0)
    ref, bound, _ = plain.reference()
    assert_close(got, ref, bound)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_strides_and_rows_of_nobody(dtype):
    for new in ([1, 1, 1, 1], [1, 70, 9, 2]):
        b = Shared(new, [120, 190, 133, 118], [(4, 101)], 6, 3, 64, 16, dtype, slots_first=True, gap=24)
        T = sum(new)
        wide = torch.full((T + 3, 6 * 64 + 8), 7.0, dtype=DT[dtype], device="cuda")
        q = torch.full((T + 3, 6 * 64 + 16), math.nan, dtype=DT[dtype], device="cuda")
        q[:T, :6 * 64] = b.q
        rows = b.q
        b.q = q[:, :6 * 64]
        out = b.run(out=wide[:, : 6 * 64])
        b.q = rows
        ref, bound, _ = b.reference()
        assert_close(out[:T], ref, bound)
        assert bool((wide[:, 6 * 64:] == 7.0).all()) and bool((wide[T:] == 7.0).all())


def test_more_new_tokens_than_promised_are_left_alone():
    b = Shared([1, 3, 1], [90, 91, 92], [(3, 66)], 4, 2, 64, 16, "f16")
    out = torch.full((5, 4 * 64), 7.0, dtype=torch.float16, device="cuda")
    b.run(out=out, max_new=2)
    ref, bound, written = b.reference(max_new=2)
    assert written.tolist() == [True, True, True, False, True]
    assert_close(out[written.cuda()], ref[written], bound[written])
    assert bool((out[3] == 7.0).all())


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("D,page,gain,window", [(64, 16, 1.0, 0), (128, 16, 40.0, 0), (256, 32, 1.0, 150), (80, 8, 8.0, 0)])
def test_infinities_and_nan(D, page, gain, window, dtype):
    """Among hidden keys and values they have no part; among those that a row sees, shared or its own, an infinity is one of the result and a NaN a NaN."""
    b = Shared([1, 3, 1, 40, 1], [400, 420, 431, 460, 401], [(4, 390)], 4, 2, D, page, dtype, gain=gain, seed=3)
    for cache in (b.v, b.ref_v):
        for r, j, value in ((0, 7, math.inf), (0, 389, -math.inf), (1, 419, math.nan), (2, 395, math.inf), (3, 459, -math.inf), (3, 430, math.inf)):
            for t in ([0] if j >= 390 or cache is b.v else [0, 1, 2, 3]):  # a shared one: in everybody's pages of the plain form
                row = r if j >= 390 else t
                table = b.pages if j >= 390 or cache is b.v else b.ref_pages
                cache[int(table[row, j // page]), 0, j % page, (r + j % 2)::3] = value
    b.check(window=window)


def test_agrees_with_attention_of_every_request_for_itself():
    """The same rows of pages for all that is shared: both operators, each within its bound of the same numbers."""
    b = Shared([1, 2, 1, 1], [700, 650, 640, 641], [(4, 600)], 8, 2, 128, 16, "bf16")
    one = bcq.PagedCache(b.ref_k, b.ref_v).attend(b.q, b.q_start, b.kv_len, b.ref_pages, 2)
    ref, bound, _ = b.reference()
    assert_close(one, ref, bound)
    assert_close(b.run(), ref, bound)


def test_offsets_beyond_32_bits():
    """The cache's last pages lie more than 2^32 bytes, and 2^31 elements, behind its first."""
    pages, page, kv_heads, D = 2 ** 31 // (16 * 2 * 128) + 40, 16, 2, 128
    k, v = (torch.empty((pages, kv_heads, page, D), dtype=torch.float16, device="cuda") for _ in range(2))
    for c, s in ((k, 1), (v, 2)):
        c[-20:] = torch.randn((20, kv_heads, page, D), device="cuda", generator=torch.Generator(device="cuda").manual_seed(s)).half()
    q = torch.randn((3, 4 * D), device="cuda").half()
    table = torch.tensor([[0, 1, 2, 3, 4, 5], [0, 1, 2, 6, 7, 8], [0, 1, 2, 9, 19, 18]], dtype=torch.int32, device="cuda")
    got = bcq.PagedCache(k, v).attend_shared(q, _ints([0, 1, 2, 3]), _ints([90, 60, 95]), table + pages - 20, 1, _ints([0, 3]), _ints([48]), 48)
    ref, bound, _ = attend_ref(q, k[-20:], v[-20:], _ints([0, 1, 2, 3]), _ints([90, 60, 95]), table, 4, D ** -0.5, True, 0)
    assert_close(got, ref, bound)


def test_index_arrays_are_bounded():
    """Numbers outside their ranges give some result, from inside the buffers: the call returns, and sensible requests beside them are right."""
    low, high = -2 ** 31, 2 ** 31 - 1
    b = Shared([1, 1, 1, 20], [90, 85, 60, 70], [(2, 80)], 4, 2, 64, 16, "f16")
    good = b.run()
    b.pages[2] = torch.tensor([-5, 1 << 30, low, high, 99, 7, -1, 8][: b.pages.shape[1]], dtype=torch.int32, device="cuda")
    b.kv_len[2] = 1 << 30
    got = b.run()
    assert torch.equal(got[:2], good[:2])
    b.kv_len[2] = 60
    for start, lengths in (([low, high], [high]), ([1, 0], [80]), ([0, 9], [low]), ([high, low], [80]), ([-3, 2], [high]), ([3, 1], [50])):
        b.group_start, b.shared_len = _ints(start), _ints(lengths)
        for most in (high, 80, 0):
            b.run(max_shared=most)
    b.group_start, b.shared_len = _ints([0, 3, 1, 4, 2]), _ints([40, 10, 70, 33])
    b.run(max_shared=200)
    b.q_start.copy_(_ints([-7, -1, 5, 2, 1 << 30]))
    b.run(max_shared=200)
    torch.cuda.synchronize()


@pytest.mark.parametrize("new,kv", [([1] * 6, [700, 633, 601, 2000, 664, 640]), ([3, 100, 1, 2], [900, 750, 5000, 603])])
def test_repeats_bit_for_bit_on_any_stream_and_in_graphs(new, kv):
    """Two graphs that are replayed one after the other share no workspace; lengths that change between replays."""
    b = Shared(new, kv, [(len(new) - 1, 600)], 8, 2, 128, 16, "bf16")
    first = b.run().clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = [b.run() for _ in range(3)]
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(first, o) for o in other)
    outs, graphs = [torch.empty_like(first) for _ in range(2)], []
    for out in outs:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            b.run(out=out)
        graphs.append(graph)
    for turn in range(4):
        b.shared_len.fill_(600 - 100 * (turn % 2))
        if turn % 2:  # (what is not shared is each one's own then, which holds the same)
            b.pages.copy_(b.ref_pages)
            b.k.copy_(b.ref_k)
            b.v.copy_(b.ref_v)
        want = b.run().clone()
        for out, graph in zip(outs, graphs):
            out.zero_()
            graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(out, want) for out in outs)
        ref, bound, _ = b.reference()
        assert_close(outs[0], ref, bound)


def test_nothing_to_do():
    b = Shared([1], [5], [(1, 3)], 4, 2, 64, 16, "f16")
    none = _ints([])
    assert b.cache.attend_shared(b.q[:0], _ints([0]), none, b.pages[:0], 1, _ints([0]), none, 5).shape == (0, 256)
    got = b.cache.attend_shared(b.q, b.q_start, b.kv_len, b.pages, 1, _ints([0]), none, 0)  # no groups
    ref, bound, _ = b.reference()
    assert_close(got, ref, bound)


def test_refusals():
    b = Shared([1, 1], [40, 50], [(2, 30)], 4, 2, 64, 16, "f16")
    f, a = b.cache.attend_shared, [b.q, b.q_start, b.kv_len, b.pages, 1, b.group_start, b.shared_len, 30]
    f(*a)
    for i, bad in ((0, b.q.float()), (0, b.q[0]), (1, b.q_start[:2]), (2, b.kv_len.long()), (3, b.pages.long()), (3, b.pages.t()), (4, 0), (4, 1 << 40), (5, b.group_start[:1]),
                   (5, b.group_start.cpu()), (6, b.shared_len.long()), (6, None), (6, b.pages), (7, -1), (7, 1 << 32)):
        with pytest.raises(bcq.BcqError):
            f(*[bad if j == i else x for j, x in enumerate(a)])
    for kw in (dict(scale=-1.0), dict(window=-1), dict(window=5, causal=False), dict(out=b.q.float()), dict(out=b.q[:1])):
        with pytest.raises(bcq.BcqError):
            f(*a, **kw)
