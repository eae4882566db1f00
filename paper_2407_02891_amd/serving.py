"""Objects over the serving operators of include/bcq.h: a paged key/value cache that is appended to and attended, the adapters of
many requests beside a shared projection, the table of a cache's pages from one step to the next, and the drawing of tokens from logits.  They hold tensors and descriptors and call the C entry points on torch's current stream (no
arithmetic here).  Scratch memory comes from torch's allocator for each call, so calls on different streams share none of it; tensors
that another stream wrote or will free follow torch's usual rules (wait_stream, record_stream).

A call of a few tokens is over on the GPU in 3 to 10 us.  Its checks and allocations, 9 to 14 us in Python, are native code for that reason
(csrc/bcq_torch.cpp, built as _serving.so); there is no other path."""
import ctypes

import torch

from . import binding as B

_DTYPES = {torch.float16: B.BCQ_F16, torch.bfloat16: B.BCQ_BF16}
_native = None


def _load():
    """_serving.so, bound to libbcq.so.  Raises if either is not built."""
    global _native
    if _native is None:
        lib = B.lib()
        try:
            from . import _serving
        except ImportError as e:
            raise RuntimeError("paper_2407_02891_amd/_serving.so is missing: run `python __graft_entry__.py build` (there is no fallback path)") from e
        _serving.bind(lib._handle, B.BcqError)
        _native = _serving
    return _native


def _need(ok, where, what):
    if not ok:
        raise B.BcqError(B.BCQ_ERR_INVALID_ARG, f"{where} ({what})")


class PagedCache:
    """Keys and values in pages: k and v [pages][kv_heads][page_size][head_dim], binary16 or bfloat16, any strides with contiguous
    head_dim (a transposed view of [pages][page_size][kv_heads][head_dim] too)."""

    def __init__(self, k, v):
        where = "PagedCache"
        _need(k.dim() == 4 and k.dtype in _DTYPES, where, "k: [pages][kv_heads][page_size][head_dim] of float16 or bfloat16")
        _need(k.is_cuda, where, f"k: on a GPU, not on {k.device}")
        strides = [[n if size > 1 else t.shape[3] for n, size in zip(t.stride(), t.shape)] for t in (k, v)]  # (of a lone page or slot: nothing)
        _need(v.shape == k.shape and v.dtype == k.dtype and strides[0] == strides[1] and v.device == k.device, where,
              "v: shape, strides, type and device of k")
        _need(k.stride(3) == 1 or k.shape[3] == 1, where, "head_dim contiguous")
        self.k, self.v = k, v
        self.dtype, self.device = k.dtype, k.device
        pages, self.kv_heads, self.page_size, self.head_dim = k.shape
        self.desc = B.Cache(_DTYPES[k.dtype], self.kv_heads, self.head_dim, self.page_size, pages, *strides[0][:3])
        self._desc, self._index, self._native = ctypes.addressof(self.desc), k.get_device(), _load()

    @classmethod
    def empty(cls, pages, page_size, kv_heads, head_dim, dtype=torch.float16, device="cuda"):
        """A cache of its own, pages heads-major: a head's slots of a page are one contiguous run."""
        return cls(*(torch.empty((pages, kv_heads, page_size, head_dim), dtype=dtype, device=device) for _ in range(2)))

    def rotate(self, qkv, positions, cos_sin, slots, q_weight=None, k_weight=None, eps=1e-6, interleaved=False, out=None):
        """bcq_rotate: norms of q and k heads (those whose weight is given), rotation, k and v into `slots`.  qkv: [tokens][(q_heads +
        2 kv_heads) * head_dim]; cos_sin [positions][rot_dim] binary32 or None (no rotation); positions, slots int32 [tokens].  Returns q
        [tokens][q_heads * head_dim] (`out`, which may be qkv[:, :q_heads * head_dim])."""
        return self._native.rotate(self._desc, self.k, self.v, qkv, positions, cos_sin, slots, q_weight, k_weight, eps, interleaved, out,
                                   B.raw_stream(self._index))

    def attend(self, q, q_start, kv_len, pages, max_new, scale=None, causal=True, window=0, out=None):
        """bcq_attend: q [tokens][q_heads * head_dim] (request r's rows are q_start[r] .. q_start[r+1] - 1, at most max_new of them)
        over the kv_len[r] keys that the pages of row r hold.  q_start, kv_len, pages int32.  scale: head_dim ** -0.5 if None.  Returns
        [tokens][q_heads * head_dim] (`out`)."""
        return self._native.attend(self._desc, self.k, self.v, q, q_start, kv_len, pages, max_new, self.head_dim ** -0.5 if scale is None else scale,
                                   causal, window, out, B.raw_stream(self._index))

    def attend_shared(self, q, q_start, kv_len, pages, max_new, group_start, shared_len, max_shared, scale=None, causal=True, window=0, out=None):
        """bcq_attend_shared: attend, for requests of which group c, group_start[c] .. group_start[c+1] - 1, share their first shared_len[c] keys (at most max_shared):
        those are taken from the first one's pages and read once.  group_start int32 [groups + 1], shared_len int32 [groups].  Single tokens gain where that saves some 16000 keys or
        more ((requests - 1) * shared_len) of prefixes of 2048 and more; for chunks, and for less, attend with the pages in every row is faster."""
        return self._native.attend_shared(self._desc, self.k, self.v, q, q_start, kv_len, pages, max_new, group_start, shared_len, max_shared,
                                          self.head_dim ** -0.5 if scale is None else scale, causal, window, out, B.raw_stream(self._index))


class Adapters:
    """Low-rank adapters of one projection: A [count][max_rank][N], B [count][M][max_rank] contiguous, binary16 or bfloat16; scale
    float32 [count] or None (1), rank int32 [count] or None (max_rank)."""

    def __init__(self, A, B_, scale=None, rank=None):
        where = "Adapters"
        _need(A.dim() == 3 and A.dtype in _DTYPES and A.is_contiguous(), where, "A: contiguous [count][max_rank][N] of float16 or bfloat16")
        _need(A.is_cuda, where, f"A: on a GPU, not on {A.device}")
        count, width, N = A.shape
        _need(B_.dim() == 3 and B_.shape[0] == count and B_.shape[2] == width and B_.dtype == A.dtype and B_.is_contiguous() and B_.device == A.device,
              where, "B: contiguous [count][M][max_rank] of A's type")
        for name, t, dtype in (("scale", scale, torch.float32), ("rank", rank, torch.int32)):
            _need(t is None or (t.shape == (count,) and t.dtype == dtype and t.is_contiguous() and t.device == A.device), where,
                  f"{name}: contiguous {dtype} [count]")
        self.A, self.B, self.scale, self.rank = A, B_, scale, rank
        self.dtype, self.device = A.dtype, A.device
        self.M, self.N = B_.shape[1], N
        self.desc = B.AdaptersDesc(_DTYPES[A.dtype], count, width, self.M, N)
        self._desc, self._index, self._native = ctypes.addressof(self.desc), A.get_device(), _load()
        self._rank, self._scale = B._ptr(rank), B._ptr(scale)

    def add(self, X, adapter, base, out=None):
        """bcq_lora: base + scale * B (A X) by the adapter of each row (int32 [tokens]; any number outside 0 .. count - 1: none).  `out` may
        be base."""
        return self._native.add(self._desc, self.A, self.B, self._rank, self._scale, X, adapter, base, out, B.raw_stream(self._index))


class PageTable:
    """Which pages of a pool each request has: pages int32 [requests][max_pages] (the first held[r] of row r are the request's), the stack of free ones
    (int32 [pages of the pool], the first free_count[0] of them), held int32 [requests], free_count int32 [1]."""

    STEP = ("q_start", "kv_len", "lack", "held", "free_count", "positions", "slots", "owner")

    def __init__(self, pages, held, free, free_count, page_size):
        where = "PageTable"
        _need(pages.dim() == 2 and pages.dtype == torch.int32 and pages.is_contiguous(), where, "pages: contiguous int32 [requests][max_pages]")
        _need(pages.is_cuda, where, f"pages: on a GPU, not on {pages.device}")
        for name, t, n in (("held", held, pages.shape[0]), ("free", free, None), ("free_count", free_count, 1)):
            _need(t.dim() == 1 and t.dtype == torch.int32 and t.is_contiguous() and t.device == pages.device and (n is None or t.shape[0] == n), where,
                  f"{name}: contiguous int32 [{'pages of the pool' if n is None else n}] on {pages.device}")
        self.pages, self.held, self.free, self.free_count, self.page_size, self.device = pages, held, free, free_count, int(page_size), pages.device
        self.desc = B.PageTableDesc(self.page_size, free.shape[0], *pages.shape)
        self._desc, self._index, self._native = ctypes.addressof(self.desc), pages.get_device(), _load()

    @classmethod
    def empty(cls, requests, max_pages, num_pages, page_size, device="cuda"):
        """All pages of the pool free, none held; page 0 is taken first."""
        return cls(torch.zeros((requests, max_pages), dtype=torch.int32, device=device), torch.zeros(requests, dtype=torch.int32, device=device),
                   torch.arange(num_pages - 1, -1, -1, dtype=torch.int32, device=device), torch.full((1,), num_pages, dtype=torch.int32, device=device), page_size)

    def step(self, cached, fresh, tokens, fixed=None, out=None, trial=False):
        """bcq_plan: cached[r] tokens of request r are in the cache, fresh[r] more come with a batch of `tokens` rows (int32 [requests]); the first fixed[r] pages of a
        row are not its own.  Returns a dict of q_start, kv_len, lack, held, free_count, positions, slots, owner (`out`: one that an earlier step returned, whose
        tensors are written again: none of them may be cached, fresh or fixed).  held and free_count are the table's own and move with the step.  With `trial` they stay, and those that the step would leave are
        tensors of their own: what a step would take and who would lack pages, before it is made (entries of `pages` behind held, and of `free` behind free_count,
        are scratch)."""
        return self._native.step(self._desc, self.pages, self.held, fixed, self.free, self.free_count, cached, fresh, tokens, trial, out, self.STEP,
                                 B.raw_stream(self._index))


class Sampler:
    """Settings of the rows of a batch: temperature float32 [rows] (not above 0: the largest logit), top_k int32 (0: all), top_p (1: all) and min_p (0: all)
    float32 [rows], or None."""

    def __init__(self, temperature, top_k=None, top_p=None, min_p=None):
        where = "Sampler"
        _need(temperature.dim() == 1 and temperature.dtype == torch.float32 and temperature.is_contiguous(), where, "temperature: contiguous float32 [rows]")
        _need(temperature.is_cuda, where, f"temperature: on a GPU, not on {temperature.device}")
        for name, t, dtype in (("top_k", top_k, torch.int32), ("top_p", top_p, torch.float32), ("min_p", min_p, torch.float32)):
            _need(t is None or (t.shape == temperature.shape and t.dtype == dtype and t.is_contiguous() and t.device == temperature.device), where,
                  f"{name}: contiguous {dtype} [rows] on {temperature.device}")
        self.temperature, self.top_k, self.top_p, self.min_p = temperature, top_k, top_p, min_p
        self._index, self._native = temperature.get_device(), _load()

    def draw(self, logits, uniform, out=None):
        """bcq_sample: logits [rows][vocabulary] float16 or bfloat16, uniform float32 [rows] in 0 .. 1.  Returns (tokens int32 [rows], -1 where a row has nothing to
        draw from; their probabilities among what the filters keep, float32 [rows]), `out`."""
        return self._native.draw(self.temperature, self.top_k, self.top_p, self.min_p, logits, uniform, out, B.raw_stream(self._index))
