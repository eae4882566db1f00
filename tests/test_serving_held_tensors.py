"""What native calls look at beside their arguments.  Tensors that an object holds and a program has put others in the place of: a call looks at them as at its arguments, for their sizes are in the descriptor that the
object was made with (no GPU needed: all of it is refused before anything is launched)."""
import ctypes

import pytest
import torch

import paper_2407_02891_amd as bcq
from paper_2407_02891_amd import binding as B, serving


def _refused(call, what):
    with pytest.raises(bcq.BcqError, match=what) as e:
        call()
    assert e.value.status == B.BCQ_ERR_INVALID_ARG


@pytest.mark.parametrize("other", [lambda t: t[:, :3].contiguous(), lambda t: t[:2], lambda t: torch.cat([t, t]), lambda t: t.long(), lambda t: t.float(), lambda t: t[:, :, None],
                                   lambda t: t.flatten(), lambda t: torch.zeros((4, 3), dtype=torch.int32).t(), lambda t: torch.zeros((3, 8), dtype=torch.int32)[:, ::2]])
def test_pages_of_a_table(other):
    pages, i = torch.zeros((3, 4), dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    desc = B.PageTableDesc(16, 10, 3, 4)
    free, count = torch.zeros(10, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    _refused(lambda: serving._load().step(ctypes.addressof(desc), other(pages), i, None, free, count, i.clone(), i.clone(), 5, False, None, bcq.PageTable.STEP, 0), "pages:")


def test_a_result_that_cannot_be_named():
    """An error of Python's on the way to a step's dict ends the call there, before the step is made."""
    class Name(str):
        asked = 0

        def __hash__(self):
            Name.asked += 1
            raise MemoryError("no dict")

    pages, i = torch.zeros((3, 4), dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    desc = B.PageTableDesc(16, 10, 3, 4)
    free, count = torch.zeros(10, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    with pytest.raises(MemoryError, match="no dict"):
        serving._load().step(ctypes.addressof(desc), pages, i, None, free, count, i.clone(), i.clone(), 5, False, None, tuple(Name(n) for n in bcq.PageTable.STEP), 0)
    assert Name.asked == 1


def _ids(*v):
    return torch.tensor(v, dtype=torch.int32)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("other", [lambda t: t[:4], lambda t: t[:, :1], lambda t: t[:, :, :8].contiguous(), lambda t: t[..., :32], lambda t: t.float(), lambda t: t.view(torch.int16),
                                   lambda t: t.transpose(1, 2).contiguous().transpose(1, 2), lambda t: t.flatten(1), lambda t: torch.cat([t, t])[::2],
                                   lambda t: t.to(torch.float16 if t.dtype == torch.bfloat16 else torch.bfloat16)])
def test_keys_and_values_of_a_cache(other, dtype):
    good = torch.zeros((5, 2, 16, 64), dtype=dtype)
    desc = B.Cache(B.BCQ_F16 if dtype == torch.float16 else B.BCQ_BF16, 2, 64, 16, 5, *good.stride()[:3])
    at, native = ctypes.addressof(desc), serving._load()
    for k, v in ((other(good), good), (good, other(good)), (other(good), other(good))):
        x, q = torch.zeros((1, 6 * 64), dtype=k.dtype), torch.zeros((1, 2 * 64), dtype=k.dtype)
        one = _ids(0), _ids(0)
        _refused(lambda: native.rotate(at, k, v, x, one[0], None, one[1], None, None, 1e-6, False, None, 0), "k, v:")
        _refused(lambda: native.attend(at, k, v, q, _ids(0, 1), _ids(1), _ids(0)[:, None], 1, 1.0, True, 0, None, 0), "k, v:")
        _refused(lambda: native.attend_shared(at, k, v, q, _ids(0, 1), _ids(1), _ids(0)[:, None], 1, _ids(0, 1), _ids(1), 1, 1.0, True, 0, None, 0), "k, v:")


def test_a_lone_page_or_slot_has_any_stride():
    """Looked at no further than what a kernel multiplies by (what is refused behind it is a tensor that is missing)."""
    for shape, stride in (((1, 2, 16, 64), (7, 1024, 64, 1)), ((5, 1, 1, 64), (64, 8, 8, 1)), ((5, 2, 16, 8), (256, 128, 8, 1))):
        k = torch.zeros(5 * 2 * 16 * 64, dtype=torch.float16).as_strided(shape, stride)
        made = [n if size > 1 else shape[3] for n, size in zip(stride, shape)]
        desc = B.Cache(B.BCQ_F16, shape[1], shape[3], shape[2], shape[0], *made[:3])
        q = torch.zeros((1, shape[1] * shape[3]), dtype=torch.float16)
        _refused(lambda: serving._load().attend(ctypes.addressof(desc), k, k, q, _ids(0, 1), None, _ids(0)[:, None], 1, 1.0, True, 0, None, 0), "kv_len:")


@pytest.mark.parametrize("other", [lambda t: t[:2], lambda t: t[:, :, :-8].contiguous(), lambda t: t[:, :8].contiguous(), lambda t: t.float(), lambda t: t.bfloat16(),
                                   lambda t: t.transpose(1, 2).contiguous().transpose(1, 2), lambda t: t.flatten(1), lambda t: torch.cat([t, t])])
def test_factors_of_adapters(other):
    A, Bm = torch.zeros((3, 16, 64), dtype=torch.float16), torch.zeros((3, 40, 16), dtype=torch.float16)
    desc = B.AdaptersDesc(B.BCQ_F16, 3, 16, 40, 64)
    for a, b in ((other(A), Bm), (A, other(Bm)), (other(A), other(Bm))):
        X, base = torch.zeros((1, 64), dtype=a.dtype), torch.zeros((1, 40), dtype=a.dtype)
        _refused(lambda: serving._load().add(ctypes.addressof(desc), a, b, None, None, X, _ids(0), base, None, 0), "A, B:")
