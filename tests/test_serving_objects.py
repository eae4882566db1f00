"""What the objects over the serving operators refuse before they reach the library (no GPU needed)."""
import subprocess
import sys

import pytest
import torch

import paper_2407_02891_amd as bcq
from paper_2407_02891_amd import binding as B


def _refused(call):
    with pytest.raises(bcq.BcqError) as e:
        call()
    assert e.value.status == B.BCQ_ERR_INVALID_ARG


@pytest.mark.parametrize("device", ["cpu", "meta"])
def test_tensors_that_are_not_on_a_gpu(device):
    """Their addresses mean nothing to a kernel."""
    k, v = (torch.zeros((2, 1, 16, 64), dtype=torch.float16, device=device) for _ in range(2))
    _refused(lambda: bcq.PagedCache(k, v))
    _refused(lambda: bcq.PagedCache.empty(2, 16, 1, 64, device=device))
    A, Bm = (torch.zeros(s, dtype=torch.bfloat16, device=device) for s in ((1, 8, 64), (1, 40, 8)))
    _refused(lambda: bcq.Adapters(A, Bm))
    _refused(lambda: bcq.Adapters(A, Bm, torch.ones(1, device=device), torch.ones(1, dtype=torch.int32, device=device)))


@pytest.mark.parametrize("call", ["rotate(at, k, k, x, ids, None, ids, None, None, 1e-6, False, None, 0)",
                                  "attend(at, k, k, x, ids, ids, ids[:, None], 1, 1.0, True, 0, None, 0)"])
def test_heads_without_elements(call):
    """Refused, where rows were divided by them (in a process of its own, which that ended)."""
    code = f"""
import ctypes, torch
import paper_2407_02891_amd as bcq
from paper_2407_02891_amd import binding as B, serving
desc = B.Cache(B.BCQ_F16, 1, 0, 16, 2, 16, 16, 8)
at, k = ctypes.addressof(desc), torch.zeros((2, 1, 16, 0), dtype=torch.float16)
x, ids = torch.zeros((1, 0), dtype=torch.float16), torch.zeros(1, dtype=torch.int32)
try:
    serving._load().{call}
except bcq.BcqError as e:
    print("refused", e.status)
"""
    done = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=120)
    assert (done.returncode, done.stdout.strip()) == (0, f"refused {B.BCQ_ERR_INVALID_ARG}"), done


def test_the_package_needs_no_torch():
    """Importing it and calling the C ABI through it leaves torch alone, as it did before there were objects over tensors."""
    code = """
import sys
import paper_2407_02891_amd as bcq
assert bcq.packed_bytes(bcq.Desc(64, 128, 2, 128)) > 0 and "PagedCache" in dir(bcq)
assert "torch" not in sys.modules
assert bcq.PagedCache.__name__ == "PagedCache" and bcq.Adapters.__name__ == "Adapters" and "torch" in sys.modules
"""
    done = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=120)
    assert done.returncode == 0, done.stderr


@pytest.mark.parametrize("order", ["bcq.lib(); import torch", "import torch; bcq.lib()"])
def test_one_hip_runtime_whatever_is_loaded_first(order):
    """Streams of torch's mean nothing to a second HIP runtime."""
    code = f"""
import paper_2407_02891_amd as bcq
{order}
print(len({{l.split()[-1] for l in open("/proc/self/maps") if "libamdhip64" in l}}))
"""
    done = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=120)
    assert (done.returncode, done.stdout.strip()) == (0, "1"), done
