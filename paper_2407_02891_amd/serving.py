"""Objects over the serving operators of include/bcq.h: a paged key/value cache that is appended to and attended, and the adapters of
many requests beside a shared projection.  They hold tensors and descriptors, check shapes and types, and forward to the C entry
points on torch's current stream (no arithmetic here).  Scratch memory comes from torch's allocator for each call, so calls on
different streams share none of it; tensors that another stream wrote or will free follow torch's usual rules (wait_stream,
record_stream)."""
import torch

from . import binding as B

_DTYPES = {torch.float16: B.BCQ_F16, torch.bfloat16: B.BCQ_BF16}


def _need(ok, where, what):
    if not ok:
        raise B.BcqError(B.BCQ_ERR_INVALID_ARG, f"{where} ({what})")


def _ints(where, name, t, shape, device):
    _need(t.dtype == torch.int32 and t.shape == shape and t.is_contiguous() and t.device == device, where,
          f"{name}: contiguous int32 of shape {tuple(shape)} on {device}")


def _rows(where, name, t, cols, dtype, device):
    """A matrix of `cols` columns whose rows are contiguous."""
    _need(t.dim() == 2 and t.shape[1] == cols and t.dtype == dtype and t.device == device and (t.stride(1) == 1 or cols == 1), where,
          f"{name}: [rows][{cols}] {dtype} on {device}, rows contiguous")
    return t.stride(0) if t.shape[0] > 1 else cols  # (the stride of a lone row means nothing)


class PagedCache:
    """Keys and values in pages: k and v [pages][kv_heads][page_size][head_dim], binary16 or bfloat16, any strides with contiguous
    head_dim (a transposed view of [pages][page_size][kv_heads][head_dim] too)."""

    def __init__(self, k, v):
        _need(k.dim() == 4 and k.dtype in _DTYPES, "PagedCache", "k: [pages][kv_heads][page_size][head_dim] of float16 or bfloat16")
        strides = [[n if size > 1 else t.shape[3] for n, size in zip(t.stride(), t.shape)] for t in (k, v)]  # (of a lone page or slot: nothing)
        _need(v.shape == k.shape and v.dtype == k.dtype and strides[0] == strides[1] and v.device == k.device, "PagedCache",
              "v: shape, strides, type and device of k")
        _need(k.stride(3) == 1 or k.shape[3] == 1, "PagedCache", "head_dim contiguous")
        self.k, self.v = k, v
        self.dtype, self.device = k.dtype, k.device
        pages, self.kv_heads, self.page_size, self.head_dim = k.shape
        self.desc = B.Cache(_DTYPES[k.dtype], self.kv_heads, self.head_dim, self.page_size, pages, *strides[0][:3])

    @classmethod
    def empty(cls, pages, page_size, kv_heads, head_dim, dtype=torch.float16, device="cuda"):
        """A cache of its own, pages heads-major: a head's slots of a page are one contiguous run."""
        return cls(*(torch.empty((pages, kv_heads, page_size, head_dim), dtype=dtype, device=device) for _ in range(2)))

    def rotate(self, qkv, positions, cos_sin, slots, q_weight=None, k_weight=None, eps=1e-6, interleaved=False, out=None):
        """bcq_rotate: norms of q and k heads (those whose weight is given), rotation, k and v into `slots`.  qkv: [tokens][(q_heads +
        2 kv_heads) * head_dim]; cos_sin [positions][rot_dim] binary32 or None (no rotation).  Returns q [tokens][q_heads * head_dim]
        (`out`, which may be qkv[:, :q_heads * head_dim])."""
        where = "PagedCache.rotate"
        D = self.head_dim
        _need(qkv.dim() == 2 and qkv.shape[1] % D == 0, where, "qkv: [tokens][heads * head_dim]")
        T, q_heads = qkv.shape[0], qkv.shape[1] // D - 2 * self.kv_heads
        _need(q_heads >= 1, where, "qkv: at least one q head before the k and v heads")
        ld = _rows(where, "qkv", qkv, qkv.shape[1], self.dtype, self.device)
        _ints(where, "positions", positions, (T,), self.device)
        _ints(where, "slots", slots, (T,), self.device)
        most, rot = 1, 0
        if cos_sin is not None:
            _need(cos_sin.dim() == 2 and cos_sin.dtype == torch.float32 and cos_sin.is_contiguous() and cos_sin.device == self.device, where,
                  "cos_sin: contiguous float32 [positions][rot_dim]")
            most, rot = cos_sin.shape
        for name, w in (("q_weight", q_weight), ("k_weight", k_weight)):
            _need(w is None or (w.shape == (D,) and w.dtype == self.dtype and w.is_contiguous() and w.device == self.device), where,
                  f"{name}: contiguous [head_dim] of the cache's type")
        if out is None:
            out = torch.empty((T, q_heads * D), dtype=self.dtype, device=self.device)
        _need(out.shape[0] == T, where, "out: a row per token")
        ld_q = _rows(where, "out", out, q_heads * D, self.dtype, self.device)
        B.rotate(self.desc, T, q_heads, qkv, ld, positions, cos_sin, most, rot, interleaved, q_weight, k_weight, eps, out, ld_q, slots,
                 self.k, self.v)
        return out

    def attend(self, q, q_start, kv_len, pages, max_new, scale=None, causal=True, window=0, out=None):
        """bcq_attend: q [tokens][q_heads * head_dim] (request r's rows are q_start[r] .. q_start[r+1] - 1, at most max_new of them)
        over the kv_len[r] keys that the pages of row r hold.  Returns [tokens][q_heads * head_dim] (`out`)."""
        where = "PagedCache.attend"
        D = self.head_dim
        _need(q.dim() == 2 and q.shape[1] % D == 0, where, "q: [tokens][q_heads * head_dim]")
        T, R, q_heads = q.shape[0], kv_len.numel(), q.shape[1] // D
        ld = _rows(where, "q", q, q.shape[1], self.dtype, self.device)
        _ints(where, "q_start", q_start, (R + 1,), self.device)
        _ints(where, "kv_len", kv_len, (R,), self.device)
        _need(pages.dim() == 2, where, "pages: [requests][max_pages]")
        _ints(where, "pages", pages, (R, pages.shape[1]), self.device)
        if out is None:
            out = torch.empty((T, q_heads * D), dtype=self.dtype, device=self.device)
        _need(out.shape[0] == T, where, "out: a row per token")
        ld_out = _rows(where, "out", out, q_heads * D, self.dtype, self.device)
        nbytes = B.attend_workspace_bytes(self.desc, T, R, q_heads, pages.shape[1], max_new)
        ws = torch.empty(nbytes, dtype=torch.uint8, device=self.device) if nbytes else None
        B.attend(self.desc, self.k, self.v, T, R, q_heads, q, ld, q_start, kv_len, pages, pages.shape[1], max_new,
                 D ** -0.5 if scale is None else scale, causal, window, out, ld_out, ws)
        return out


class Adapters:
    """Low-rank adapters of one projection: A [count][max_rank][N], B [count][M][max_rank] contiguous, binary16 or bfloat16; scale
    float32 [count] or None (1), rank int32 [count] or None (max_rank)."""

    def __init__(self, A, B_, scale=None, rank=None):
        where = "Adapters"
        _need(A.dim() == 3 and A.dtype in _DTYPES and A.is_contiguous(), where, "A: contiguous [count][max_rank][N] of float16 or bfloat16")
        count, width, N = A.shape
        _need(B_.dim() == 3 and B_.shape[0] == count and B_.shape[2] == width and B_.dtype == A.dtype and B_.is_contiguous() and B_.device == A.device,
              where, "B: contiguous [count][M][max_rank] of A's type")
        _need(scale is None or (scale.shape == (count,) and scale.dtype == torch.float32 and scale.is_contiguous() and scale.device == A.device),
              where, "scale: contiguous float32 [count]")
        if rank is not None:
            _ints(where, "rank", rank, (count,), A.device)
        self.A, self.B, self.scale, self.rank = A, B_, scale, rank
        self.dtype, self.device = A.dtype, A.device
        self.M, self.N = B_.shape[1], N
        self.desc = B.AdaptersDesc(_DTYPES[A.dtype], count, width, self.M, N)

    def add(self, X, adapter, base, out=None):
        """bcq_lora: base + scale * B (A X) by the adapter of each row (any number outside 0 .. count - 1: none).  `out` may be base."""
        where = "Adapters.add"
        _need(X.dim() == 2, where, "X: [tokens][N]")
        T = X.shape[0]
        ldx = _rows(where, "X", X, self.N, self.dtype, self.device)
        _ints(where, "adapter", adapter, (T,), self.device)
        _need(base.shape[0] == T, where, "base: a row per token")
        ld_base = _rows(where, "base", base, self.M, self.dtype, self.device)
        if out is None:
            out = torch.empty((T, self.M), dtype=self.dtype, device=self.device)
        _need(out.shape[0] == T, where, "out: a row per token")
        ldy = _rows(where, "out", out, self.M, self.dtype, self.device)
        nbytes = B.lora_workspace_bytes(self.desc, T)
        ws = torch.empty(nbytes, dtype=torch.uint8, device=self.device) if nbytes else None
        B.lora(self.desc, self.A, self.B, self.rank, self.scale, T, adapter, X, ldx, base, ld_base, out, ldy, ws)
        return out
