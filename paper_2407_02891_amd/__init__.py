"""MI355X-native binary-coding GEMV (inference path of GPTQT, arXiv 2407.02891).

Thin Python binding over the C ABI in include/bcq.h; see `binding`.
"""
from .binding import (  # noqa: F401
    AdaptersDesc, BcqError, Cache, PageTableDesc, attend, attend_shared, attend_shared_workspace_bytes, attend_workspace_bytes, lora, lora_workspace_bytes, plan, rotate, sample, Desc, PackedLayer, from_linear, from_linear_rows, gemm_skinny, gemv, gemv_noalloc, lib, pack, pack_rows, packed_bytes, quant_factor, quant_factor_workspace_bytes, quant_gptq, quant_hessian, quant_search, quant_workspace_bytes,
    read_probe, set_option, status_string, unpack, workspace_bytes, workspace_init,
)

_OBJECTS = ("Adapters", "PageTable", "PagedCache", "Sampler")


def __getattr__(name):
    """The objects over torch tensors come with their first use: the C ABI's binding needs no torch."""
    if name in _OBJECTS:
        from . import serving
        globals().update({n: getattr(serving, n) for n in _OBJECTS})
        return globals()[name]
    raise AttributeError(f"module {__name__!r} has no attribute {name!r}")


def __dir__():
    return sorted({*globals(), *_OBJECTS})
