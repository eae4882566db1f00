"""The serving operators (attention over the paged cache, norm with rotation and append, low-rank adapters) against plain forms in 64
bits, at the sizes, masks, strides and contents where they can go wrong."""
import math

import numpy as np
import pytest
import torch

import paper_2407_02891_amd as bcq
from paper_2407_02891_amd import binding as B
from tests.serving_util import assert_close, attend_ref, lora_ref, rotate_ref

pytestmark = pytest.mark.gpu
DT = {"f16": torch.float16, "bf16": torch.bfloat16}


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


class Batch:
    """Requests with the given new tokens and keys; pages in any order; whatever no request owns is NaN."""

    def __init__(self, new, kv, q_heads, kv_heads, D, page, dtype, seed=0, slots_first=False, spare_pages=3, gain=1.0, gap=0):
        g = _gen(seed)
        dtype = DT[dtype]
        self.new, self.kv, self.q_heads = new, kv, q_heads
        counts = [-(-n // page) for n in kv]
        pool, width = sum(counts) + spare_pages, max(max(counts), 1) + 1
        shape = (pool, page, kv_heads, D) if slots_first else (pool, kv_heads, page, D)
        self.k, self.v = (torch.full(shape, math.nan, dtype=dtype, device="cuda") for _ in range(2))
        if slots_first:
            self.k, self.v = self.k.transpose(1, 2), self.v.transpose(1, 2)
        order = np.random.default_rng(seed).permutation(pool)
        table = np.full((len(kv), width), 0, np.int32)
        at = 0
        for r, c in enumerate(counts):
            table[r, :c] = order[at:at + c]
            at += c
            for j in range(c):
                used = min(page, kv[r] - j * page)
                for cache in (self.k, self.v):
                    cache[int(table[r, j]), :, :used] = torch.randn((kv_heads, used, D), device="cuda", generator=g).to(dtype)
        self.pages = torch.from_numpy(table).cuda()
        self.q_start = _ints([0] + list(np.cumsum(new)))
        self.kv_len = _ints(kv)
        T = sum(new)
        wide = torch.full((T, q_heads * D + gap), math.nan, dtype=dtype, device="cuda")
        self.q = wide[:, : q_heads * D]
        self.q.copy_(torch.randn((T, q_heads * D), device="cuda", generator=g) * gain)
        self.cache = bcq.PagedCache(self.k, self.v)

    def run(self, causal=True, window=0, scale=None, out=None, max_new=None):
        return self.cache.attend(self.q, self.q_start, self.kv_len, self.pages, max_new or max(self.new), scale=scale, causal=causal, window=window, out=out)

    def check(self, causal=True, window=0, scale=None, what=""):
        D = self.k.shape[3]
        got = self.run(causal, window, scale)
        torch.cuda.synchronize()
        ref, bound, written = attend_ref(self.q, self.k, self.v, self.q_start, self.kv_len, self.pages, self.q_heads,
                                         D ** -0.5 if scale is None else scale, causal, window)
        assert bool(written.all())
        assert_close(got, ref, bound, what)


EDGES = [1, 2, 7, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 300, 511, 1000]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("q_heads,kv_heads,D,page", [(8, 1, 128, 16), (4, 4, 64, 8), (6, 2, 80, 32), (5, 1, 96, 1), (2, 2, 256, 64), (16, 1, 128, 128),
                                                     (3, 3, 8, 2), (4, 2, 136, 16), (4, 1, 72, 256)])
def test_attend_single_tokens_at_every_edge_of_a_tile(dtype, q_heads, kv_heads, D, page):
    Batch([1] * len(EDGES), EDGES, q_heads, kv_heads, D, page, dtype, seed=D).check()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("q_heads,kv_heads,D,page", [(8, 1, 128, 16), (4, 4, 64, 32), (5, 1, 96, 4), (2, 1, 256, 16)])
@pytest.mark.parametrize("causal,window", [(True, 0), (True, 1), (True, 7), (True, 64), (True, 5000), (False, 0)])
def test_attend_chunks(dtype, q_heads, kv_heads, D, page, causal, window):
    Batch([1, 2, 3, 5, 16, 17, 33, 70, 130], [1, 2, 40, 64, 16, 100, 333, 70, 259], q_heads, kv_heads, D, page, dtype, seed=page).check(causal, window)


@pytest.mark.parametrize("new", [1, 4])
@pytest.mark.parametrize("q_heads,kv_heads", [(71, 1), (64, 1), (40, 2), (33, 1), (48, 3)])
def test_attend_many_query_heads_share_one(q_heads, kv_heads, new):
    Batch([new, new, new], [new, 77, 500], q_heads, kv_heads, 64, 16, "f16").check()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("causal", [True, False])
def test_attend_rows_that_see_nothing(dtype, causal):
    # no keys at all; no new tokens; fewer keys than new tokens (the first of them see none)
    b = Batch([1, 0, 5, 2, 40, 1], [0, 50, 3, 0, 33, 65], 8, 2, 64, 16, dtype)
    b.check(causal)
    out = b.run(causal)
    assert bool((out[0] == 0).all()) and bool((out[6:8] == 0).all())
    if causal:
        assert bool((out[1:3] == 0).all()) and not bool((out[3] == 0).any())
    Batch([3], [0], 2, 2, 128, 16, dtype).check(causal)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("poison", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("new,D,window", [(6, 64, 0), (6, 128, 9), (90, 128, 0), (90, 64, 21), (200, 256, 50)])
def test_attend_hidden_keys_have_no_part_whatever_they_hold(dtype, poison, new, D, window):
    """The last new token's key and value, and with a window the first keys of the request, are not finite: rows that do not see them do
    not feel them, rows that do give what the formula gives."""
    n = 231
    b = Batch([new, 1], [n, 40], 4, 2, D, 16, dtype)
    for j in [n - 1, n - 1 - new // 2] + ([0, n - new - window + 3] if window else []):
        at, off = int(b.pages[0, j // 16]), j % 16
        b.k[at, 0, off] = poison
        b.k[at, 1, off, 5] = poison
        b.v[at, :, off, ::3] = poison
    got = b.run(window=window).double().cpu()
    ref, bound, _ = attend_ref(b.q, b.k, b.v, b.q_start, b.kv_len, b.pages, 4, D ** -0.5, True, window)
    fine = ref.isfinite()
    assert bool(fine.any()) and not bool(fine.all())
    assert bool(got[fine].isfinite().all())
    assert float(((got - ref).abs() - bound)[fine].max()) <= 0
    assert not bool(got[~fine].isfinite().any())


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("gain", [0.0, 30.0, 1000.0])
def test_attend_flat_and_sharp_softmax(dtype, gain):
    Batch([1, 2, 60], [777, 300, 600], 8, 2, 128, 16, dtype, gain=gain).check()


def test_attend_scores_that_grow_and_fall_along_the_keys():
    """Running maxima that change at every block, and one that never does after the first."""
    for sign in (1.0, -1.0):
        b = Batch([1, 1, 40], [900, 64, 500], 2, 1, 64, 16, "f16")
        for r, n in enumerate(b.kv):
            for j in range(n):
                b.k[int(b.pages[r, j // 16]), :, j % 16] = sign * 0.02 * j
        b.q.fill_(1.0)
        b.check()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_attend_strides_of_the_cache_and_of_the_rows(dtype):
    for new in ([1, 1, 1], [1, 70, 9]):
        b = Batch(new, [100, 170, 33], 6, 3, 64, 16, dtype, slots_first=True, gap=24)
        wide = torch.full((sum(new), 6 * 64 + 8), 7.0, dtype=DT[dtype], device="cuda")
        out = b.run(out=wide[:, : 6 * 64])
        ref, bound, _ = attend_ref(b.q, b.k, b.v, b.q_start, b.kv_len, b.pages, 6, 0.125, True, 0)
        assert_close(out, ref, bound)
        assert bool((wide[:, 6 * 64:] == 7.0).all())


@pytest.mark.parametrize("requests", [65, 130, 300])
def test_attend_many_requests(requests):
    rng = np.random.default_rng(requests)
    Batch([1] * requests, [int(n) for n in rng.integers(1, 90, requests)], 4, 2, 64, 16, "f16").check()
    new = [int(n) for n in rng.choice([0, 1, 1, 2, 20], requests)]
    Batch(new, [n + int(e) for n, e in zip(new, rng.integers(0, 60, requests))], 4, 2, 64, 16, "bf16").check()


@pytest.mark.parametrize("new", [1, 5, 40])
def test_attend_long_contexts_are_split(new):
    Batch([new, new], [20011, 3001], 4, 1, 128, 32, "f16").check()


def test_attend_offsets_beyond_32_bits():
    """The cache's last pages lie more than 2^32 bytes, and 2^31 elements, behind its first."""
    pages, page, kv_heads, D = 2 ** 31 // (16 * 2 * 128) + 40, 16, 2, 128
    k, v = (torch.empty((pages, kv_heads, page, D), dtype=torch.float16, device="cuda") for _ in range(2))
    assert k[pages - 20].storage_offset() > 2 ** 31
    for new in (1, 50):
        n = 20 * page - 3
        for c, s in ((k, 1), (v, 2)):
            c[-20:] = torch.randn((20, kv_heads, page, D), device="cuda", generator=_gen(s)).half()
        cache = bcq.PagedCache(k, v)
        q = torch.randn((new, 4 * D), device="cuda", generator=_gen(3)).half()
        table = torch.arange(pages - 20, pages, dtype=torch.int32, device="cuda")[None].contiguous()
        got = cache.attend(q, _ints([0, new]), _ints([n]), table, new)
        ref, bound, _ = attend_ref(q, k[-20:], v[-20:], _ints([0, new]), _ints([n]), table - (pages - 20), 4, D ** -0.5, True, 0)
        assert_close(got, ref, bound)
    # and the append
    qkv = torch.randn((3, 8 * D), device="cuda", generator=_gen(4)).half()
    slots = _ints([pages * page - 1, pages * page - page, 5])
    cache.rotate(qkv, _ints([0, 0, 0]), None, slots)
    assert torch.equal(k[-1, :, -1], qkv[0].view(8, D)[4:6]) and torch.equal(v[-1, :, 0], qkv[1].view(8, D)[6:])
    assert torch.equal(k[0, :, 5], qkv[2].view(8, D)[4:6])


def test_attend_more_new_tokens_than_promised_are_left_alone():
    b = Batch([1, 3, 1], [40, 41, 42], 4, 2, 64, 16, "f16")
    out = torch.full((5, 4 * 64), 7.0, dtype=torch.float16, device="cuda")
    b.run(out=out, max_new=2)
    ref, bound, written = attend_ref(b.q, b.k, b.v, b.q_start, b.kv_len, b.pages, 4, 0.125, True, 0, max_new=2)
    assert written.tolist() == [True, True, True, False, True]
    assert_close(out[written.cuda()], ref[written], bound[written])
    assert bool((out[3] == 7.0).all())


def test_attend_index_arrays_are_bounded():
    """Numbers outside their ranges give some result, from inside the buffers: the call returns and other requests' rows are right."""
    b = Batch([1, 1, 40], [50, 60, 70], 4, 2, 64, 16, "f16")
    b.pages[1] = torch.tensor([-5, 1 << 30, -(1 << 31), (1 << 31) - 1, 99, 7][: b.pages.shape[1]], dtype=torch.int32, device="cuda")
    b.kv_len[1] = 1 << 30
    out = b.run()
    torch.cuda.synchronize()
    ref, bound, _ = attend_ref(b.q[:1], b.k, b.v, _ints([0, 1]), b.kv_len[:1], b.pages[:1], 4, 0.125, True, 0)
    assert_close(out[:1], ref, bound)
    b.kv_len[1] = -3
    b.q_start[3] = 1 << 30
    b.run()
    b.q_start.copy_(_ints([-7, -1, 5, 2]))
    b.run()
    torch.cuda.synchronize()


@pytest.mark.parametrize("new,kv", [([1] * 5, [700, 33, 1, 2000, 64]), ([3, 100, 1], [900, 300, 5000])])
def test_attend_repeats_bit_for_bit_on_any_stream_and_in_graphs(new, kv):
    b = Batch(new, kv, 8, 2, 128, 16, "bf16")
    first = b.run().clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = [b.run() for _ in range(3)]
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(first, o) for o in other)
    out = torch.empty_like(first)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.run(out=out)
    for _ in range(4):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, first)
        assert torch.equal(b.run(), first)


def test_attend_nothing_to_do():
    b = Batch([1], [5], 4, 2, 64, 16, "f16")
    empty = b.cache.attend(b.q[:0], _ints([0]), _ints([]), b.pages[:0], 1)
    assert empty.shape == (0, 256)


# ------------------------------------------------------------------------------------------------


def _rotate_case(T, q_heads, kv_heads, D, rot, interleaved, norm, dtype, page=16, seed=0, gap=0, slots_first=False):
    g = _gen(seed)
    dt = DT[dtype]
    wide = torch.randn((T, (q_heads + 2 * kv_heads) * D + gap), device="cuda", generator=g).to(dt)
    qkv = wide[:, : (q_heads + 2 * kv_heads) * D]
    pool = -(-T // page) + 2
    shape = (pool, page, kv_heads, D) if slots_first else (pool, kv_heads, page, D)
    k, v = (torch.full(shape, 5.0, dtype=dt, device="cuda") for _ in range(2))
    if slots_first:
        k, v = k.transpose(1, 2), v.transpose(1, 2)
    slots = torch.from_numpy(np.random.default_rng(seed).permutation(pool * page)[:T].astype(np.int32)).cuda()
    if T > 2:
        slots[T // 2] = -1
    most = 5000
    positions = torch.randint(0, most, (T,), device="cuda", generator=g, dtype=torch.int32)
    table = None
    if rot:
        angle = torch.arange(most, device="cuda", dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(0, rot, 2, device="cuda", dtype=torch.float64) / rot)
        table = torch.cat([angle.cos(), angle.sin()], 1).float()
    weights = [(1 + 0.3 * torch.randn(D, device="cuda", generator=g)).to(dt) if norm & bit else None for bit in (1, 2)]
    return qkv, k, v, slots, positions, table, weights


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("D,rot", [(128, 128), (128, 64), (64, 64), (80, 80), (80, 20), (96, 24), (256, 256), (8, 8), (72, 6), (128, 0), (248, 250 // 2 * 2 - 4)])
def test_rotate(D, rot, interleaved, dtype):
    for T, norm, q_heads, kv_heads in ((1, 3, 8, 2), (37, 3, 5, 5), (37, 0, 3, 1), (9, 1, 2, 2), (9, 2, 2, 1)):
        qkv, k, v, slots, positions, table, (wq, wk) = _rotate_case(T, q_heads, kv_heads, D, rot, interleaved, norm, dtype, seed=T + D)
        cache = bcq.PagedCache(k, v)
        before = qkv.clone()
        q = cache.rotate(qkv, positions, table, slots, wq, wk, eps=1e-6, interleaved=interleaved)
        ref, bound = rotate_ref(before, q_heads, kv_heads, D, positions, table, wq, wk, 1e-6, interleaved)
        assert_close(q.view(T, q_heads, D), ref[:, :q_heads], bound[:, :q_heads], f"q T={T} norm={norm}")
        flat_k, flat_v = (c.transpose(1, 2).reshape(-1, kv_heads, D) for c in (k, v))
        here = (slots >= 0).cpu()
        assert_close(flat_k[slots[here.cuda()].long()], ref[here][:, q_heads:q_heads + kv_heads], bound[here][:, q_heads:q_heads + kv_heads], "k")
        assert torch.equal(flat_v[slots[here.cuda()].long()].cpu(), before[here.cuda()].view(-1, q_heads + 2 * kv_heads, D)[:, q_heads + kv_heads:].cpu())
        rest = torch.ones(flat_k.shape[0], dtype=torch.bool, device="cuda")
        rest[slots[here.cuda()].long()] = False
        assert bool((flat_k[rest] == 5.0).all()) and bool((flat_v[rest] == 5.0).all())
        assert torch.equal(qkv, before)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("interleaved", [False, True])
def test_rotate_in_place_with_gaps_and_slots_first(dtype, interleaved):
    T, Hq, Hkv, D = 33, 6, 3, 64
    qkv, k, v, slots, positions, table, (wq, wk) = _rotate_case(T, Hq, Hkv, D, 64, interleaved, 3, dtype, gap=16, slots_first=True)
    before = qkv.clone()
    cache = bcq.PagedCache(k, v)
    q = cache.rotate(qkv, positions, table, slots, wq, wk, interleaved=interleaved, out=qkv[:, : Hq * D])
    ref, bound = rotate_ref(before, Hq, Hkv, D, positions, table, wq, wk, 1e-6, interleaved)
    assert_close(q.reshape(T, Hq, D), ref[:, :Hq], bound[:, :Hq])
    assert torch.equal(qkv[:, Hq * D:], before[:, Hq * D:])
    ok = slots >= 0
    s = slots[ok].long()
    assert_close(k[s // 16, :, s % 16], ref[ok.cpu()][:, Hq:Hq + Hkv], bound[ok.cpu()][:, Hq:Hq + Hkv])


def test_rotate_numbers_outside_their_ranges():
    """Positions are bounded, slots outside the cache are not stored; zeros, and values whose squares pass binary16, have finite norms."""
    T, D = 6, 64
    qkv, k, v, slots, positions, table, (wq, wk) = _rotate_case(T, 2, 1, D, 64, False, 3, "f16")
    qkv[0] = 0
    qkv[1] = 60000.0
    positions.copy_(_ints([-1, 5000, 1 << 30, -(1 << 31), 4999, 0]))
    slots.copy_(_ints([-1, k.shape[0] * 16, (1 << 31) - 1, -(1 << 31), 3, 4]))
    q = bcq.PagedCache(k, v).rotate(qkv, positions, table, slots, wq, wk)
    ref, bound = rotate_ref(qkv, 2, 1, D, positions, table, wq, wk, 1e-6, False)
    assert_close(q.view(T, 2, D), ref[:, :2], bound[:, :2])
    flat = k.transpose(1, 2).reshape(-1, 1, D)
    assert_close(flat[3:5], ref[4:, 2:3], bound[4:, 2:3])
    assert int((flat != 5.0).any(-1).sum()) == 2
    assert bcq.PagedCache(k, v).rotate(qkv[:0], positions[:0], table, slots[:0]).shape == (0, 2 * D)


# ------------------------------------------------------------------------------------------------


def _lora_case(T, N, M, C, width, dtype, seed=0, ranks=None, bare=True, strides=(0, 0)):
    g = _gen(seed)
    dt = DT[dtype]
    A = (torch.randn((C, width, N), device="cuda", generator=g) * N ** -0.5).to(dt)
    Bm = (torch.randn((C, M, width), device="cuda", generator=g) * width ** -0.5).to(dt)
    rank = None
    if ranks is not None:
        rank = _ints([ranks[c % len(ranks)] for c in range(C)])
        for c in range(C):
            A[c, int(rank[c]):] = math.nan
            Bm[c, :, int(rank[c]):] = math.inf
    scale = torch.empty(C, device="cuda").uniform_(-2, 2, generator=g)
    X = torch.randn((T, N + strides[0]), device="cuda", generator=g).to(dt)[:, :N]
    base = torch.randn((T, M + strides[1]), device="cuda", generator=g).to(dt)[:, :M]
    adapter = torch.randint(-1 if bare else 0, C, (T,), device="cuda", generator=g, dtype=torch.int32)
    return X, A, Bm, scale, rank, adapter, base


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("T,N,M,C,width", [(1, 64, 64, 1, 8), (1, 8, 1, 1, 8), (3, 264, 100, 2, 16), (17, 1000, 333, 3, 24), (64, 512, 512, 64, 16), (65, 2056, 130, 5, 40),
                                           (100, 768, 768, 2, 64), (40, 1536, 257, 1, 128), (200, 520, 1025, 7, 136), (33, 4096, 1024, 4, 256), (300, 72, 40, 300, 8),
                                           (2, 16392, 64, 2, 16), (5, 64, 8200, 2, 32)])
def test_lora(dtype, T, N, M, C, width):
    for ranks in (None, [width, 1, width - 3, 0, 5]):
        X, A, Bm, scale, rank, adapter, base = _lora_case(T, N, M, C, width, dtype, seed=T, ranks=ranks)
        got = bcq.Adapters(A, Bm, scale, rank).add(X, adapter, base)
        ref, bound = lora_ref(X, A, Bm, scale, rank, adapter, base)
        assert_close(got, ref, bound, f"ranks {ranks}")


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("T,N,M,C,width", [(1100, 264, 333, 3, 64), (520, 136, 1025, 5, 128), (4200, 72, 130, 2, 16), (2200, 520, 192, 30, 32), (1400, 1032, 64, 1, 56),
                                           (1030, 96, 640, 4, 72)])
def test_lora_many_tokens(dtype, T, N, M, C, width):
    """Enough tokens of an adapter that v is turned into operands in a launch of its own; sorted by adapter, in runs, and mixed."""
    for ranks, runs in ((None, True), ([width, 1, width - 3, 0, 9], False)):
        X, A, Bm, scale, rank, adapter, base = _lora_case(T, N, M, C, width, dtype, seed=T, ranks=ranks)
        if runs:
            adapter = adapter.sort().values.contiguous()
        got = bcq.Adapters(A, Bm, scale, rank).add(X, adapter, base)
        ref, bound = lora_ref(X, A, Bm, scale, rank, adapter, base)
        assert_close(got, ref, bound, f"ranks {ranks}")
        assert bcq.Adapters(A, Bm, scale, rank).add(X, adapter, base, out=base) is base
        assert torch.equal(base, got)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("N,M,width", [(8192, 1300, 16), (520, 513, 40), (4104, 5000, 24), (16, 140000, 8), (1032, 511, 120), (8, 1, 256), (16384, 700, 8), (20000, 64, 16)])
def test_lora_one_token(dtype, N, M, width):
    """Adapters of every rank, numbers of none, into another tensor and in place."""
    X, A, Bm, scale, rank, _, base = _lora_case(1, N, M, 6, width, dtype, seed=N, ranks=[width, 1, width - 3, 0, min(9, width), width - 7])
    adapters = bcq.Adapters(A, Bm, scale, rank)
    for a in (0, 1, 2, 3, 4, 5, -1, 6):
        adapter = _ints([a])
        ref, bound = lora_ref(X, A, Bm, scale, rank, adapter, base)
        assert_close(adapters.add(X, adapter, base), ref, bound, f"adapter {a}")
        own = base.clone()
        adapters.add(X, adapter, own, out=own)
        assert_close(own, ref, bound, f"adapter {a} in place")


def test_lora_very_many_adapters():
    """More adapters than the sorting launch counts in LDS."""
    X, A, Bm, scale, rank, adapter, base = _lora_case(900, 64, 40, 5000, 8, "f16", bare=True)
    got = bcq.Adapters(A, Bm, scale).add(X, adapter, base)
    ref, bound = lora_ref(X, A, Bm, scale, None, adapter, base)
    assert_close(got, ref, bound)


@pytest.mark.parametrize("T", [5, 150])
def test_lora_in_place_with_strides_and_defaults(T):
    X, A, Bm, _, _, adapter, base = _lora_case(T, 256, 200, 3, 16, "f16", strides=(24, 7))
    ref, bound = lora_ref(X, A, Bm, None, None, adapter, base)
    got = bcq.Adapters(A, Bm).add(X, adapter, base, out=base)
    assert got.data_ptr() == base.data_ptr()
    assert_close(base, ref, bound)
    X, A, Bm, scale, rank, adapter, base = _lora_case(T, 256, 200, 3, 16, "bf16", strides=(8, 8))
    wide = torch.full((T, 216), 7.0, dtype=torch.bfloat16, device="cuda")
    bcq.Adapters(A, Bm, scale).add(X, adapter, base, out=wide[:, :200])
    ref, bound = lora_ref(X, A, Bm, scale, None, adapter, base)
    assert_close(wide[:, :200], ref, bound)
    assert bool((wide[:, 200:] == 7.0).all())


def test_lora_ids_outside_the_range_leave_the_base():
    X, A, Bm, scale, rank, adapter, base = _lora_case(70, 128, 96, 2, 8, "f16")
    adapter[::3] = 2
    adapter[1::9] = -(1 << 31)
    adapter[2::9] = (1 << 31) - 1
    got = bcq.Adapters(A, Bm, scale).add(X, adapter, base)
    ref, bound = lora_ref(X, A, Bm, scale, None, adapter, base)
    assert_close(got, ref, bound)
    assert torch.equal(got[::3], base[::3])
    assert bcq.Adapters(A, Bm, scale).add(X[:0], adapter[:0], base[:0]).shape == (0, 96)


@pytest.mark.parametrize("T", [4, 200, 4200])
def test_lora_wide_ranges_of_activations(T):
    """A x beyond binary16, and tokens whose A x differ by 2^20 beside each other."""
    X, A, Bm, scale, rank, adapter, base = _lora_case(T, 512, 96, 2, 16, "f16", bare=False)
    X[::2] *= 300.0
    A[0] *= 100.0
    Bm *= 1e-3
    X[1::2] *= 1e-3
    got = bcq.Adapters(A, Bm, scale).add(X, adapter, base)
    ref, bound = lora_ref(X, A, Bm, scale, None, adapter, base)
    assert_close(got, ref, bound)


@pytest.mark.parametrize("T,M", [(6, 512), (200, 1024), (2100, 320)])
def test_lora_repeats_bit_for_bit_on_any_stream_and_in_graphs(T, M):
    X, A, Bm, scale, rank, adapter, base = _lora_case(T, 2048, M, 4, 32, "f16", ranks=[32, 7])
    ad = bcq.Adapters(A, Bm, scale, rank)
    first = ad.add(X, adapter, base).clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = [ad.add(X, adapter, base) for _ in range(3)]
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(first, o) for o in other)
    out = torch.empty_like(first)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ad.add(X, adapter, base, out=out)
    for _ in range(4):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, first) and torch.equal(ad.add(X, adapter, base), first)


def test_lora_offsets_beyond_32_bits():
    C, width, N, M = 70, 256, 131072, 64                     # A holds more than 2^31 elements
    A = torch.empty((C, width, N), dtype=torch.float16, device="cuda")
    A[-2:] = (torch.randn((2, width, N), device="cuda", generator=_gen(1)) * N ** -0.5).half()
    assert A[-1].storage_offset() > 2 ** 31
    Bm = (torch.randn((C, M, width), device="cuda", generator=_gen(2)) * width ** -0.5).half()
    X, base = torch.randn((3, N), device="cuda", generator=_gen(3)).half(), torch.randn((3, M), device="cuda", generator=_gen(4)).half()
    adapter = _ints([C - 1, C - 2, C - 1])
    got = bcq.Adapters(A, Bm).add(X, adapter, base)
    ref, bound = lora_ref(X, A[-2:], Bm[-2:], None, None, adapter - (C - 2), base)
    assert_close(got, ref, bound)


# ------------------------------------------------------------------------------------------------


def test_objects_refuse_what_does_not_fit():
    b = Batch([1, 1], [5, 6], 4, 2, 64, 16, "f16")
    c = b.cache

    def refused(f, status=B.BCQ_ERR_INVALID_ARG):
        with pytest.raises(bcq.BcqError) as e:
            f()
        assert e.value.status == status

    refused(lambda: bcq.PagedCache(b.k.float(), b.v.float()))
    refused(lambda: bcq.PagedCache(b.k, b.v[:, :, :8]))
    refused(lambda: bcq.PagedCache(b.k.transpose(2, 3), b.v.transpose(2, 3)))
    refused(lambda: c.attend(b.q.bfloat16(), b.q_start, b.kv_len, b.pages, 1))
    refused(lambda: c.attend(b.q[:, :-8], b.q_start, b.kv_len, b.pages, 1))
    refused(lambda: c.attend(b.q, b.q_start[:-1], b.kv_len, b.pages, 1))
    refused(lambda: c.attend(b.q, b.q_start.long(), b.kv_len, b.pages, 1))
    refused(lambda: c.attend(b.q, b.q_start, b.kv_len, b.pages.t(), 1))
    refused(lambda: c.attend(b.q[:, : 3 * 64], b.q_start, b.kv_len, b.pages, 1))          # three query heads over two
    refused(lambda: c.attend(b.q, b.q_start, b.kv_len, b.pages, 0))
    refused(lambda: c.attend(b.q, b.q_start, b.kv_len, b.pages, 1, scale=0.0))
    refused(lambda: c.attend(b.q, b.q_start, b.kv_len, b.pages, 1, causal=False, window=3))
    refused(lambda: c.attend(b.q, b.q_start, b.kv_len, b.pages, 1, out=torch.empty_like(b.q)[:1]))
    three = torch.empty((2, 1, 3, 64), dtype=torch.float16, device="cuda")
    refused(lambda: bcq.PagedCache(three, three).attend(b.q, b.q_start, b.kv_len, b.pages, 1), B.BCQ_ERR_UNSUPPORTED)
    qkv = torch.zeros((2, 8 * 64), dtype=torch.float16, device="cuda")
    at = _ints([0, 1])
    table = torch.zeros((9, 64), device="cuda")
    refused(lambda: c.rotate(qkv[:, :-1], at, table, at))
    refused(lambda: c.rotate(qkv[:, : 4 * 64], at, table, at))                            # no q head left
    refused(lambda: c.rotate(qkv, at[:1], table, at))
    refused(lambda: c.rotate(qkv, at, table[:, :63].contiguous(), at))
    refused(lambda: c.rotate(qkv, at, torch.zeros((9, 66), device="cuda"), at))
    refused(lambda: c.rotate(qkv, at, table.double(), at))
    refused(lambda: c.rotate(qkv, at, table, at, q_weight=torch.zeros(63, dtype=torch.float16, device="cuda")))
    refused(lambda: c.rotate(qkv, at, table, at, eps=-1.0))
    A, Bm = torch.zeros((2, 8, 64), dtype=torch.float16, device="cuda"), torch.zeros((2, 40, 8), dtype=torch.float16, device="cuda")
    X, base = torch.zeros((2, 64), dtype=torch.float16, device="cuda"), torch.zeros((2, 40), dtype=torch.float16, device="cuda")
    ad = bcq.Adapters(A, Bm)
    refused(lambda: bcq.Adapters(A, Bm[:, :, :4].contiguous()))
    refused(lambda: bcq.Adapters(A, Bm, torch.zeros(3, device="cuda")))
    refused(lambda: ad.add(X[:, :56], at, base))
    refused(lambda: ad.add(X, at, base[:1]))
    refused(lambda: ad.add(X, at.long(), base))
    refused(lambda: ad.add(X, at, base.bfloat16()))
    refused(lambda: ad.add(X.expand(2, 64)[:1].expand(2, 64), at, base))                  # rows of stride 0
    odd = bcq.Adapters(A[:, :4].contiguous(), Bm[:, :, :4].contiguous())
    refused(lambda: odd.add(X, at, base))
