"""Calls of the serving operators at the edges of what they take: strides, single rows, magnitudes and contents that the ordinary cases
do not have.  Bounds are those of the plain forms in serving_util."""
import math

import pytest
import torch

import paper_2407_02891_amd as bcq
from tests.serving_util import assert_close, attend_ref, lora_ref, rotate_ref
from tests.test_gpu_serving import DT, Batch, _gen, _ints, _lora_case, _rotate_case

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


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("q_heads,kv_heads,D,gap", [(64, 8, 128, 0), (3, 1, 80, 8), (5, 5, 256, 0)])
def test_rotate_one_token_in_place(q_heads, kv_heads, D, gap, interleaved, dtype):
    qkv, k, v, slots, positions, table, (wq, wk) = _rotate_case(1, q_heads, kv_heads, D, D, interleaved, 3, dtype, gap=gap)
    before = qkv.clone()
    q = bcq.PagedCache(k, v).rotate(qkv, positions, table, slots, wq, wk, interleaved=interleaved, out=qkv[:, : q_heads * D])
    assert q.data_ptr() == qkv.data_ptr()
    ref, bound = rotate_ref(before, q_heads, kv_heads, D, positions, table, wq, wk, 1e-6, interleaved)
    assert_close(q.view(1, q_heads, D), ref[:, :q_heads], bound[:, :q_heads])
    assert torch.equal(qkv[:, q_heads * D:], before[:, q_heads * D:])
    at = int(slots[0])
    assert_close(k[at // 16, :, at % 16][None], ref[:, q_heads:q_heads + kv_heads], bound[:, q_heads:q_heads + kv_heads])
    assert torch.equal(v[at // 16, :, at % 16], before.view(-1, D)[q_heads + kv_heads:])


def test_lora_one_row_in_place_whatever_its_strides():
    """Through the C entry points' binding: a lone row may be named with two strides."""
    from paper_2407_02891_amd import binding as B
    A, Bm = (torch.randn(s, device="cuda", generator=_gen(1)).half() * 0.1 for s in ((2, 8, 64), (2, 40, 8)))
    X, base = torch.randn((1, 64), device="cuda", generator=_gen(2)).half(), torch.randn((1, 40), device="cuda", generator=_gen(3)).half()
    ids = _ints([1])
    want = bcq.Adapters(A, Bm).add(X, ids, base)
    desc = B.AdaptersDesc(B.BCQ_F16, 2, 8, 40, 64)
    scratch = torch.empty(bcq.lora_workspace_bytes(desc, 1) + 16, dtype=torch.uint8, device="cuda")
    bcq.lora(desc, A, Bm, None, None, 1, ids, X, 64, base, 40, base, 96, scratch)
    assert torch.equal(base, want)


@pytest.mark.skipif(torch.cuda.device_count() < 2, reason="needs two GPUs")
def test_objects_of_a_device_that_is_not_the_current_one():
    """The same calls with everything on the second device, while the first is the current one."""
    first = Batch([1, 40], [300, 70], 4, 2, 64, 16, "f16")
    want = first.run()
    there = "cuda:1"
    cache = bcq.PagedCache(first.k.to(there), first.v.to(there))
    got = cache.attend(first.q.to(there), first.q_start.to(there), first.kv_len.to(there), first.pages.to(there), 40)
    assert torch.cuda.current_device() == 0 and got.device == torch.device(there)
    assert torch.equal(got.cpu(), want.cpu())
    X, A, Bm, scale, rank, adapter, base = _lora_case(200, 256, 200, 3, 16, "f16")
    want = bcq.Adapters(A, Bm, scale).add(X, adapter, base)
    got = bcq.Adapters(A.to(there), Bm.to(there), scale.to(there)).add(X.to(there), adapter.to(there), base.to(there))
    assert torch.equal(got.cpu(), want.cpu())


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("new", [1, 20, 140])
@pytest.mark.parametrize("kv,nats", [(1000, 13.0), (1000, 14.0), (131073, 16.0), (131073, 18.0)])
def test_attend_small_weights_beside_a_key_of_no_value(kv, nats, new, dtype):
    """The first key has nearly all the weight and a value of zero, so the small weights are the result."""
    D, page = 64, 16
    if kv > 1000 and new > 20:
        new, kv = 140, 16385
    dt = DT[dtype]
    pages = -(-kv // page)
    k = torch.zeros((pages, 1, page, D), dtype=dt, device="cuda")
    v = (1 + 0.1 * torch.randn((pages, 1, page, D), device="cuda", generator=_gen(kv))).to(dt)
    k[0, 0, 0] = nats / 8
    v[0, 0, 0] = 0
    q = torch.ones((new, D), dtype=dt, device="cuda")
    table = torch.arange(pages, dtype=torch.int32, device="cuda")[None]
    # (with a table far longer than the keys too: the keys are cut otherwise)
    for wide in (table, torch.cat([table, table.new_zeros((1, 3 * 131072 // page))], 1)):
        got = bcq.PagedCache(k, v).attend(q, _ints([0, new]), _ints([kv]), wide.contiguous(), new)
        ref, bound, _ = attend_ref(q, k, v, _ints([0, new]), _ints([kv]), table, 1, D ** -0.5, True, 0)
        assert_close(got, ref, bound)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("q_heads,kv_heads,D,page", [(4, 2, 64, 16), (4, 2, 128, 16), (2, 2, 256, 32), (4, 2, 80, 8)])
@pytest.mark.parametrize("gain", [1.0, 8.0, 40.0])
def test_attend_infinities_that_are_seen(gain, q_heads, kv_heads, D, page, dtype):
    """An infinity among the values is one of every row that sees it, however little weight its key has and wherever it lies; a NaN, and infinities of both signs, are NaN."""
    for long_table in (False, True):
        b = Batch([1, 3, 70, 150, 1], [700, 500, 300, 650, 2100], q_heads, kv_heads, D, page, dtype, seed=D, gain=gain)
        if long_table:
            b.pages = torch.cat([b.pages, b.pages.new_zeros((5, 20000 // page))], 1).contiguous()
        for r, j, value in ((0, 3, math.inf), (0, 400, -math.inf), (1, 130, math.inf), (1, 498, -math.inf), (2, 64, -math.inf), (2, 260, math.nan), (3, 40, math.inf),
                            (3, 600, math.inf), (4, 1000, -math.inf)):
            b.v[int(b.pages[r, j // page]), 0, j % page, (r + j % 2)::3] = value
        b.check(what=f"long table {long_table}")
        b.check(window=100, what=f"window, long table {long_table}")


@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 5, 2 ** 30 + 1, 2 ** 30])
def test_attend_windows_longer_than_anything(window):
    """No window at all, also where there are more new tokens than keys."""
    for new, kv in (([1, 3, 16], [400, 2, 9]), ([200, 1, 70], [100, 50, 300])):
        b = Batch(new, kv, 2, 2, 64, 16, "f16")
        b.check(window=window)
        assert torch.equal(b.run(window=window), b.run())


def test_attend_in_one_launch_takes_no_workspace():
    b = Batch([1, 2, 1], [600, 33, 1], 8, 2, 128, 16, "f16")
    out = torch.empty_like(b.q)
    assert bcq.attend_workspace_bytes(b.cache.desc, 4, 3, 8, b.pages.shape[1], 2) == 0
    bcq.attend(b.cache.desc, b.k, b.v, 4, 3, 8, b.q, b.q.stride(0), b.q_start, b.kv_len, b.pages, b.pages.shape[1], 2, 128 ** -0.5, True, 0, out, out.stride(0), None)
    assert torch.equal(out, b.run())


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("T,N,M,C,width", [(1, 64, 200, 2, 16), (1, 16384, 100, 2, 64), (5, 264, 130, 2, 24), (64, 512, 100, 3, 8), (300, 136, 333, 3, 40), (1100, 264, 200, 2, 64),
                                           (4200, 72, 130, 2, 16)])
def test_lora_infinities_among_the_weights(T, N, M, C, width, dtype):
    """An infinity in an adapter's B is one of the outputs it belongs to, for tokens of that adapter; a NaN, and infinities of both signs there, are NaN."""
    X, A, Bm, scale, rank, adapter, base = _lora_case(T, N, M, C, width, dtype, seed=T, ranks=[width, width - 3])
    for m, j, value in ((3, 0, math.inf), (7, 4, -math.inf), (64, 2, math.inf), (64, 3, math.inf), (90, 1, math.nan), (M - 1, 4, math.inf)):
        Bm[0, m, j] = value
    adapter[0] = 0
    ref, bound = lora_ref(X, A, Bm, scale, rank, adapter, base)
    assert bool(ref.isinf().any()) and bool(ref.isnan().any())
    assert_close(bcq.Adapters(A, Bm, scale, rank).add(X, adapter, base), ref, bound)
