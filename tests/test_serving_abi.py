"""Argument checks of the serving operators: all before any launch, so none of this needs a GPU."""
import ctypes
import math

import pytest

import paper_2407_02891_amd as bcq
from paper_2407_02891_amd import binding as B

OK = 0x1000
HUGE = 1 << 40


def cache(**kw):
    f = dict(dtype=0, kv_heads=8, head_dim=128, page_size=16, num_pages=100, page_stride=16384, head_stride=2048, slot_stride=128)
    f.update(kw)
    return B.Cache(*f.values())


def rotate(c, **kw):
    a = dict(tokens=4, q_heads=64, qkv=OK, ld_qkv=10240, positions=OK, cos_sin=OK, max_position=100, rot_dim=128, interleaved=0, q_weight=OK, k_weight=OK,
             eps=1e-6, q_out=OK, ld_q=8192, slots=OK, k=OK, v=OK)
    a.update(kw)
    return bcq.lib().bcq_rotate(ctypes.byref(c) if c else None, *a.values(), None)


def attend(c, **kw):
    a = dict(k=OK, v=OK, tokens=4, requests=2, q_heads=64, q=OK, ld_q=8192, q_start=OK, kv_len=OK, pages=OK, max_pages=10, max_new=2, scale=0.1, causal=1,
             window=0, out=OK, ld_out=8192, workspace=OK)
    a.update(kw)
    return bcq.lib().bcq_attend(ctypes.byref(c) if c else None, *a.values(), None)


def lora(d, **kw):
    a = dict(A=OK, B=OK, rank=OK, scale=OK, tokens=3, adapter=OK, X=OK, ldx=4096, base=OK, ld_base=1024, Y=OK, ldy=1024, workspace=OK)
    a.update(kw)
    return bcq.lib().bcq_lora(ctypes.byref(d) if d else None, *a.values(), None)


INVALID_CACHES = [dict(dtype=2), dict(dtype=-1), dict(kv_heads=0), dict(head_dim=0), dict(page_size=0), dict(num_pages=0), dict(page_stride=-8),
                  dict(head_stride=4), dict(slot_stride=120), dict(slot_stride=129)]
UNSUPPORTED_CACHES = [dict(head_dim=264, slot_stride=264), dict(head_dim=100, slot_stride=104), dict(page_size=24), dict(page_size=1 << 17),
                      dict(slot_stride=1 << 28), dict(num_pages=1 << 30)]


@pytest.mark.parametrize("call", [rotate, attend])
def test_caches(call):
    assert call(None) == B.BCQ_ERR_INVALID_ARG
    for kw in INVALID_CACHES:
        assert call(cache(**kw)) == B.BCQ_ERR_INVALID_ARG, kw
    for kw in UNSUPPORTED_CACHES:
        assert call(cache(**kw)) == B.BCQ_ERR_UNSUPPORTED, kw


@pytest.mark.parametrize("kw", [dict(tokens=-1), dict(q_heads=0), dict(rot_dim=-2), dict(rot_dim=63), dict(rot_dim=130), dict(max_position=0), dict(interleaved=2),
                                dict(eps=-1e-6), dict(eps=math.nan), dict(eps=math.inf), dict(ld_qkv=10232), dict(ld_qkv=10244), dict(ld_q=8184),
                                dict(qkv=None), dict(positions=None), dict(cos_sin=None), dict(rot_dim=0), dict(q_out=None), dict(slots=None), dict(k=None),
                                dict(v=None), dict(qkv=OK + 2), dict(q_out=OK + 8), dict(k=OK + 2), dict(v=OK + 2), dict(q_weight=OK + 2), dict(k_weight=OK + 8),
                                dict(cos_sin=OK + 2), dict(positions=OK + 2), dict(slots=OK + 1)])
def test_rotate_refuses(kw):
    assert rotate(cache(), **kw) == B.BCQ_ERR_INVALID_ARG      # (q_out is qkv here, so ld_q has to be ld_qkv: refused too)
    kw = {"q_out": 2 * OK, **kw}
    assert rotate(cache(), **kw) == B.BCQ_ERR_INVALID_ARG


def test_rotate_limits():
    assert rotate(cache()) == B.BCQ_ERR_INVALID_ARG             # q_out is qkv with another row stride
    assert rotate(cache(), tokens=1 << 21) == B.BCQ_ERR_UNSUPPORTED
    assert rotate(cache(), q_heads=2000, ld_qkv=HUGE, ld_q=HUGE) == B.BCQ_ERR_UNSUPPORTED
    assert rotate(cache(), tokens=0, qkv=None) == B.BCQ_OK       # nothing to do


@pytest.mark.parametrize("kw", [dict(tokens=-1), dict(requests=-1), dict(q_heads=0), dict(q_heads=60), dict(max_new=0), dict(max_pages=0), dict(scale=0.0),
                                dict(scale=-1.0), dict(scale=math.nan), dict(scale=math.inf), dict(causal=2), dict(window=-1), dict(causal=0, window=5),
                                dict(ld_q=8184), dict(ld_q=8196), dict(ld_out=8184), dict(k=None), dict(v=None), dict(q=None), dict(q_start=None),
                                dict(kv_len=None), dict(pages=None), dict(out=None), dict(k=OK + 8), dict(v=OK + 8), dict(q=OK + 8), dict(out=OK + 2),
                                dict(q_start=OK + 2), dict(kv_len=OK + 2), dict(pages=OK + 2)])
def test_attend_refuses(kw):
    assert attend(cache(), **kw) == B.BCQ_ERR_INVALID_ARG


def test_attend_limits_and_workspace():
    assert attend(cache(), tokens=1 << 21) == B.BCQ_ERR_UNSUPPORTED
    assert attend(cache(kv_heads=1), q_heads=1025, ld_q=HUGE, ld_out=HUGE) == B.BCQ_ERR_UNSUPPORTED
    assert attend(cache(), max_pages=1 << 27) == B.BCQ_ERR_UNSUPPORTED
    assert attend(cache(), tokens=0, q=None) == B.BCQ_OK
    assert attend(cache(), requests=0, q=None) == B.BCQ_OK
    c = cache()
    assert bcq.attend_workspace_bytes(c, 0, 4, 64, 10, 1) == 0
    assert bcq.attend_workspace_bytes(c, 4, 4, 60, 10, 1) == 0
    if bcq.attend_workspace_bytes(c, 4, 2, 64, 10, 2):
        assert attend(c, workspace=None) == B.BCQ_ERR_WORKSPACE
        assert attend(c, workspace=OK + 4) == B.BCQ_ERR_WORKSPACE


@pytest.mark.parametrize("kw,status", [(dict(dtype=3), 1), (dict(count=0), 1), (dict(max_rank=0), 1), (dict(max_rank=12), 1), (dict(M=0), 1), (dict(N=0), 1),
                                       (dict(N=4092), 1), (dict(max_rank=264), 2), (dict(M=1 << 25), 2), (dict(N=1 << 25), 2)])
def test_adapters(kw, status):
    f = dict(dtype=1, count=2, max_rank=16, M=1024, N=4096)
    f.update(kw)
    d = B.AdaptersDesc(*f.values())
    assert lora(d, ldx=HUGE, ld_base=HUGE, ldy=HUGE) == status
    assert bcq.lora_workspace_bytes(d, 4) == 0


@pytest.mark.parametrize("kw", [dict(tokens=-1), dict(ldx=4088), dict(ldx=4100), dict(ld_base=1023), dict(ldy=1023), dict(A=None), dict(B=None), dict(adapter=None),
                                dict(X=None), dict(base=None), dict(Y=None), dict(A=OK + 8), dict(B=OK + 8), dict(X=OK + 8), dict(base=OK + 1), dict(Y=OK + 1),
                                dict(rank=OK + 2), dict(scale=OK + 2), dict(adapter=OK + 2), dict(ldy=1032)])
def test_lora_refuses(kw):
    assert lora(B.AdaptersDesc(0, 2, 16, 1024, 4096), **kw) == B.BCQ_ERR_INVALID_ARG


def test_lora_limits_and_workspace():
    d = B.AdaptersDesc(0, 2, 16, 1024, 4096)
    assert lora(None) == B.BCQ_ERR_INVALID_ARG
    assert lora(d, tokens=1 << 21) == B.BCQ_ERR_UNSUPPORTED
    assert lora(d, tokens=0, X=None) == B.BCQ_OK
    assert bcq.lora_workspace_bytes(d, 0) == 0
    if bcq.lora_workspace_bytes(d, 3):
        assert lora(d, workspace=None) == B.BCQ_ERR_WORKSPACE
        assert lora(d, workspace=OK + 4) == B.BCQ_ERR_WORKSPACE


def test_exports():
    for name in ("PagedCache", "Adapters", "attend", "rotate", "lora"):
        assert hasattr(bcq, name)
