"""ctypes binding of libbcq.so: same names as the C entry points, argument
marshalling only.  Tensors are torch CUDA(ROCm) tensors used as device memory;
the stream is torch's current stream unless one is given.  There is no CPU
fallback: if the library is missing, loading raises."""
import ctypes
import importlib.util
import os
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libbcq.so")

BCQ_OK, BCQ_ERR_INVALID_ARG, BCQ_ERR_UNSUPPORTED, BCQ_ERR_WORKSPACE, BCQ_ERR_HIP, BCQ_ERR_SCRATCH_LIMIT = range(6)
BCQ_NOALLOC_MAX_ROWS = 131072
BCQ_LAYOUT_VERSION = 2
BCQ_MAX_BATCH = 64

EXPORTS = ["bcq_packed_bytes", "bcq_workspace_bytes", "bcq_workspace_init", "bcq_pack",
           "bcq_pack_rows", "bcq_from_linear", "bcq_quant_workspace_bytes", "bcq_quant_hessian", "bcq_quant_factor_workspace_bytes", "bcq_quant_factor", "bcq_quant_search",
           "bcq_quant_gptq", "bcq_from_linear_rows", "bcq_unpack", "bcq_gemv", "bcq_gemv_noalloc", "bcq_gemm_skinny", "bcq_read_probe_sink_bytes",
           "bcq_read_probe", "bcq_set_option", "bcq_status_string",
           "bcq_rotate", "bcq_attend_workspace_bytes", "bcq_attend", "bcq_lora_workspace_bytes", "bcq_lora",
           "bcq_attend_shared_workspace_bytes", "bcq_attend_shared", "bcq_plan", "bcq_sample"]

BCQ_F16, BCQ_BF16 = range(2)
BCQ_MAX_HEAD_DIM = 256
BCQ_MAX_RANK = 256
BCQ_MAX_VOCAB = 1 << 22


class Desc(ctypes.Structure):
    """struct bcq_desc"""
    _fields_ = [("M", ctypes.c_int32), ("N", ctypes.c_int32), ("q", ctypes.c_int32),
                ("group", ctypes.c_int32), ("has_offset", ctypes.c_int32),
                ("layout_version", ctypes.c_int32)]


class Cache(ctypes.Structure):
    """struct bcq_cache"""
    _fields_ = [("dtype", ctypes.c_int32), ("kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("page_size", ctypes.c_int32), ("num_pages", ctypes.c_int32),
                ("page_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64), ("slot_stride", ctypes.c_int64)]


class AdaptersDesc(ctypes.Structure):
    """struct bcq_adapters"""
    _fields_ = [("dtype", ctypes.c_int32), ("count", ctypes.c_int32), ("max_rank", ctypes.c_int32),
                ("M", ctypes.c_int32), ("N", ctypes.c_int32)]


class PageTableDesc(ctypes.Structure):
    """struct bcq_page_table"""
    _fields_ = [("page_size", ctypes.c_int32), ("num_pages", ctypes.c_int32), ("requests", ctypes.c_int32), ("max_pages", ctypes.c_int32)]


class BcqError(RuntimeError):
    def __init__(self, status, where):
        self.status = int(status)
        super().__init__(f"{where}: {status_string(status)} (status {int(status)})")


_lib = None


def _share_torch_runtime():
    """torch brings a HIP runtime of its own, and a process with two of them cannot pass streams from one to the other.  The first that is loaded
    serves both, so where torch is installed but not imported yet, its runtime is loaded before the library (without torch: ROCm's)."""
    if "torch" in sys.modules:
        return
    spec = importlib.util.find_spec("torch")
    if spec is not None and spec.origin:
        runtime = os.path.join(os.path.dirname(spec.origin), "lib", "libamdhip64.so")
        if os.path.exists(runtime):
            ctypes.CDLL(runtime)


def lib():
    """Load libbcq.so (built in-tree by build.py).  Raises if it is not there."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: run `python __graft_entry__.py build` "
                               "(there is no fallback path)")
        _share_torch_runtime()
        L = ctypes.CDLL(LIB_PATH)
        vp, i32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
        dp = ctypes.POINTER(Desc)
        L.bcq_packed_bytes.restype, L.bcq_packed_bytes.argtypes = sz, [dp]
        L.bcq_workspace_bytes.restype, L.bcq_workspace_bytes.argtypes = sz, [dp, i32]
        L.bcq_workspace_init.restype, L.bcq_workspace_init.argtypes = i32, [vp, sz, vp]
        L.bcq_pack.restype, L.bcq_pack.argtypes = i32, [dp, vp, vp, vp, vp, vp]
        L.bcq_pack_rows.restype, L.bcq_pack_rows.argtypes = i32, [dp, i32, i32, vp, vp, vp, vp, vp]
        L.bcq_from_linear.restype = i32
        L.bcq_from_linear.argtypes = [i32, i32, i32, i32, i32, ctypes.POINTER(ctypes.c_int32), vp, vp, vp, vp, vp, vp, vp]
        L.bcq_quant_workspace_bytes.restype, L.bcq_quant_workspace_bytes.argtypes = sz, [i32, i32]
        L.bcq_quant_hessian.restype, L.bcq_quant_hessian.argtypes = i32, [i32, i32, vp, vp, vp]
        L.bcq_quant_factor_workspace_bytes.restype, L.bcq_quant_factor_workspace_bytes.argtypes = sz, [i32]
        L.bcq_quant_factor.restype = i32
        L.bcq_quant_factor.argtypes = [i32, ctypes.c_float, vp, vp, vp, vp]
        L.bcq_quant_search.restype = i32
        L.bcq_quant_search.argtypes = [i32, i32, i32, i32, i32, vp, vp, vp, vp, vp, vp, vp, vp]
        L.bcq_quant_gptq.restype = i32
        L.bcq_quant_gptq.argtypes = [i32, i32, i32, i32, vp, vp, vp, vp, vp, vp, vp, vp]
        L.bcq_from_linear_rows.restype = i32
        L.bcq_from_linear_rows.argtypes = [i32, i32, i32, i32, vp, vp, vp, vp, vp, vp, vp, vp]
        L.bcq_unpack.restype, L.bcq_unpack.argtypes = i32, [dp, vp, vp, vp, vp, vp]
        L.bcq_gemv.restype, L.bcq_gemv.argtypes = i32, [dp, vp, vp, vp, vp, vp]
        L.bcq_gemv_noalloc.restype, L.bcq_gemv_noalloc.argtypes = i32, [dp, vp, vp, vp, vp]
        L.bcq_gemm_skinny.restype = i32
        L.bcq_gemm_skinny.argtypes = [dp, vp, vp, i32, vp, i32, i32, vp, vp]
        L.bcq_read_probe_sink_bytes.restype, L.bcq_read_probe_sink_bytes.argtypes = sz, []
        L.bcq_read_probe.restype, L.bcq_read_probe.argtypes = i32, [vp, sz, vp, vp]
        L.bcq_set_option.restype, L.bcq_set_option.argtypes = i32, [ctypes.c_char_p, i32]
        cp, ap, i64, f32 = ctypes.POINTER(Cache), ctypes.POINTER(AdaptersDesc), ctypes.c_int64, ctypes.c_float
        L.bcq_rotate.restype = i32
        L.bcq_rotate.argtypes = [cp, i32, i32, vp, i64, vp, vp, i32, i32, i32, vp, vp, f32, vp, i64, vp, vp, vp, vp]
        L.bcq_attend_workspace_bytes.restype, L.bcq_attend_workspace_bytes.argtypes = sz, [cp, i32, i32, i32, i32, i32]
        L.bcq_attend.restype = i32
        L.bcq_attend.argtypes = [cp, vp, vp, i32, i32, i32, vp, i64, vp, vp, vp, i32, i32, f32, i32, i32, vp, i64, vp, vp]
        L.bcq_lora_workspace_bytes.restype, L.bcq_lora_workspace_bytes.argtypes = sz, [ap, i32]
        L.bcq_attend_shared_workspace_bytes.restype, L.bcq_attend_shared_workspace_bytes.argtypes = sz, [cp] + [i32] * 6
        L.bcq_attend_shared.restype = i32
        L.bcq_attend_shared.argtypes = [cp, vp, vp, i32, i32, i32, i32, vp, i64, vp, vp, vp, i32, i32, vp, vp, i32, f32, i32, i32, vp, i64, vp, vp]
        L.bcq_plan.restype, L.bcq_plan.argtypes = i32, [ctypes.POINTER(PageTableDesc)] + [vp] * 7 + [i32] + [vp] * 9
        L.bcq_sample.restype, L.bcq_sample.argtypes = i32, [i32, i32, i32, vp, i64] + [vp] * 8
        L.bcq_lora.restype, L.bcq_lora.argtypes = i32, [ap, vp, vp, vp, vp, i32, vp, vp, i64, vp, i64, vp, i64, vp, vp]
        L.bcq_status_string.restype, L.bcq_status_string.argtypes = ctypes.c_char_p, [i32]
        _lib = L
    return _lib


def status_string(status):
    return lib().bcq_status_string(int(status)).decode()


def _check(status, where):
    if status != BCQ_OK:
        raise BcqError(status, where)


def _ptr(t):
    """Device pointer of a tensor (or a raw int / None)."""
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


def _stream(stream):
    """hipStream_t of `stream`, of torch's current stream if it is None.  The current one is asked for as a number:
    torch.cuda.current_stream() builds an object around it, 2.8 us of the 7.1 to 7.5 us an eager GEMV call on 1024 x 8192
    took from Python (0.3 us this way: 4.6 to 5.1 us on different cards; in a graph or from C nothing changes)."""
    if stream is None:
        import torch
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        if raw is not None:
            return raw(torch.cuda.current_device())
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


_current_raw_stream = None


def raw_stream(device_index):
    """hipStream_t of torch's current stream of a device, as a number (see _stream)."""
    global _current_raw_stream
    if _current_raw_stream is None:
        import torch
        _current_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda i: torch.cuda.current_stream(i).cuda_stream)
    return _current_raw_stream(device_index)


def packed_bytes(desc):
    return int(lib().bcq_packed_bytes(ctypes.byref(desc)))


def workspace_bytes(desc, batch=1):
    return int(lib().bcq_workspace_bytes(ctypes.byref(desc), int(batch)))


def workspace_init(workspace, nbytes=None, stream=None):
    if nbytes is None:
        nbytes = workspace.numel() * workspace.element_size()
    _check(lib().bcq_workspace_init(_ptr(workspace), nbytes, _stream(stream)), "bcq_workspace_init")


def pack(desc, codes, alpha, offset, packed, stream=None):
    _check(lib().bcq_pack(ctypes.byref(desc), _ptr(codes), _ptr(alpha), _ptr(offset), _ptr(packed),
                          _stream(stream)), "bcq_pack")


def pack_rows(desc, row_begin, rows, codes, alpha, offset, packed, stream=None):
    _check(lib().bcq_pack_rows(ctypes.byref(desc), int(row_begin), int(rows), _ptr(codes), _ptr(alpha),
                               _ptr(offset), _ptr(packed), _stream(stream)), "bcq_pack_rows")


def from_linear(M, N, group, n_bits, q, class_of_plane, w_int, S, qbias, codes, alpha, offset, stream=None):
    """class_of_plane: sequence of n_bits ints (host); the rest are device tensors."""
    labels = (ctypes.c_int32 * len(class_of_plane))(*[int(c) for c in class_of_plane])
    _check(lib().bcq_from_linear(int(M), int(N), int(group), int(n_bits), int(q), labels, _ptr(w_int), _ptr(S),
                                 _ptr(qbias), _ptr(codes), _ptr(alpha), _ptr(offset), _stream(stream)),
           "bcq_from_linear")


def quant_workspace_bytes(M, N):
    return int(lib().bcq_quant_workspace_bytes(int(M), int(N)))


def quant_hessian(N, T, X, H, stream=None):
    _check(lib().bcq_quant_hessian(int(N), int(T), _ptr(X), _ptr(H), _stream(stream)), "bcq_quant_hessian")


def quant_factor_workspace_bytes(N):
    return int(lib().bcq_quant_factor_workspace_bytes(int(N)))


def quant_factor(N, damp, H, U, workspace, stream=None):
    _check(lib().bcq_quant_factor(int(N), float(damp), _ptr(H), _ptr(U), _ptr(workspace), _stream(stream)),
           "bcq_quant_factor")


def quant_search(M, N, n_bits, q, grid, W, H, S, qbias, class_of_plane, err, workspace, stream=None):
    _check(lib().bcq_quant_search(int(M), int(N), int(n_bits), int(q), int(grid), _ptr(W), _ptr(H), _ptr(S),
                                  _ptr(qbias), _ptr(class_of_plane), _ptr(err), _ptr(workspace), _stream(stream)),
           "bcq_quant_search")


def quant_gptq(M, N, n_bits, q, W, U, S, qbias, class_of_plane, w_int, workspace, stream=None):
    _check(lib().bcq_quant_gptq(int(M), int(N), int(n_bits), int(q), _ptr(W), _ptr(U), _ptr(S), _ptr(qbias),
                                _ptr(class_of_plane), _ptr(w_int), _ptr(workspace), _stream(stream)), "bcq_quant_gptq")


def from_linear_rows(M, N, n_bits, q, class_of_plane, w_int, S, qbias, codes, alpha, offset, stream=None):
    _check(lib().bcq_from_linear_rows(int(M), int(N), int(n_bits), int(q), _ptr(class_of_plane), _ptr(w_int), _ptr(S),
                                      _ptr(qbias), _ptr(codes), _ptr(alpha), _ptr(offset), _stream(stream)),
           "bcq_from_linear_rows")


def unpack(desc, packed, codes, alpha, offset, stream=None):
    _check(lib().bcq_unpack(ctypes.byref(desc), _ptr(packed), _ptr(codes), _ptr(alpha), _ptr(offset),
                            _stream(stream)), "bcq_unpack")


def gemv(desc, packed, x, y, workspace, stream=None):
    _check(lib().bcq_gemv(ctypes.byref(desc), _ptr(packed), _ptr(x), _ptr(y), _ptr(workspace),
                          _stream(stream)), "bcq_gemv")


def gemv_noalloc(desc, packed, x, y, stream=None):
    _check(lib().bcq_gemv_noalloc(ctypes.byref(desc), _ptr(packed), _ptr(x), _ptr(y), _stream(stream)),
           "bcq_gemv_noalloc")


def gemm_skinny(desc, packed, X, ldx, Y, ldy, batch, workspace, stream=None):
    _check(lib().bcq_gemm_skinny(ctypes.byref(desc), _ptr(packed), _ptr(X), int(ldx), _ptr(Y), int(ldy),
                                 int(batch), _ptr(workspace), _stream(stream)), "bcq_gemm_skinny")


def read_probe(buf, nbytes, sink, stream=None):
    _check(lib().bcq_read_probe(_ptr(buf), int(nbytes), _ptr(sink), _stream(stream)), "bcq_read_probe")


def read_probe_sink_bytes():
    return int(lib().bcq_read_probe_sink_bytes())


def rotate(cache, tokens, q_heads, qkv, ld_qkv, positions, cos_sin, max_position, rot_dim, interleaved, q_weight, k_weight,
           eps, q_out, ld_q, slots, k_cache, v_cache, stream=None):
    _check(lib().bcq_rotate(ctypes.byref(cache), tokens, q_heads, _ptr(qkv), ld_qkv, _ptr(positions), _ptr(cos_sin),
                            max_position, rot_dim, 1 if interleaved else 0, _ptr(q_weight), _ptr(k_weight), eps, _ptr(q_out),
                            ld_q, _ptr(slots), _ptr(k_cache), _ptr(v_cache), _stream(stream)), "bcq_rotate")


def attend_workspace_bytes(cache, tokens, requests, q_heads, max_pages, max_new):
    return int(lib().bcq_attend_workspace_bytes(ctypes.byref(cache), tokens, requests, q_heads, max_pages, max_new))


def attend(cache, k_cache, v_cache, tokens, requests, q_heads, q, ld_q, q_start, kv_len, pages, max_pages, max_new, scale,
           causal, window, out, ld_out, workspace, stream=None):
    _check(lib().bcq_attend(ctypes.byref(cache), _ptr(k_cache), _ptr(v_cache), tokens, requests, q_heads, _ptr(q), ld_q,
                            _ptr(q_start), _ptr(kv_len), _ptr(pages), max_pages, max_new, scale, 1 if causal else 0, window,
                            _ptr(out), ld_out, _ptr(workspace), _stream(stream)), "bcq_attend")


def attend_shared_workspace_bytes(cache, tokens, requests, groups, q_heads, max_pages, max_new):
    return int(lib().bcq_attend_shared_workspace_bytes(ctypes.byref(cache), tokens, requests, groups, q_heads, max_pages, max_new))


def attend_shared(cache, k_cache, v_cache, tokens, requests, groups, q_heads, q, ld_q, q_start, kv_len, pages, max_pages, max_new, group_start, shared_len,
                  max_shared, scale, causal, window, out, ld_out, workspace, stream=None):
    _check(lib().bcq_attend_shared(ctypes.byref(cache), _ptr(k_cache), _ptr(v_cache), tokens, requests, groups, q_heads, _ptr(q), ld_q, _ptr(q_start),
                                   _ptr(kv_len), _ptr(pages), max_pages, max_new, _ptr(group_start), _ptr(shared_len), max_shared, scale, 1 if causal else 0,
                                   window, _ptr(out), ld_out, _ptr(workspace), _stream(stream)), "bcq_attend_shared")


def lora_workspace_bytes(desc, tokens):
    return int(lib().bcq_lora_workspace_bytes(ctypes.byref(desc), tokens))


def lora(desc, A, B, rank, scale, tokens, adapter, X, ldx, base, ld_base, Y, ldy, workspace, stream=None):
    _check(lib().bcq_lora(ctypes.byref(desc), _ptr(A), _ptr(B), _ptr(rank), _ptr(scale), tokens, _ptr(adapter), _ptr(X), ldx,
                          _ptr(base), ld_base, _ptr(Y), ldy, _ptr(workspace), _stream(stream)), "bcq_lora")


def plan(table, pages, held, fixed, free_pages, free_count, cached, fresh, tokens, q_start, kv_len, lack, held_out, free_count_out, positions, slots, owner,
         stream=None):
    _check(lib().bcq_plan(ctypes.byref(table), _ptr(pages), _ptr(held), _ptr(fixed), _ptr(free_pages), _ptr(free_count), _ptr(cached), _ptr(fresh), tokens,
                          _ptr(q_start), _ptr(kv_len), _ptr(lack), _ptr(held_out), _ptr(free_count_out), _ptr(positions), _ptr(slots), _ptr(owner),
                          _stream(stream)), "bcq_plan")


def sample(dtype, rows, vocab, logits, ld, temperature, top_k, top_p, min_p, uniform, token, probability, stream=None):
    _check(lib().bcq_sample(dtype, rows, vocab, _ptr(logits), ld, _ptr(temperature), _ptr(top_k), _ptr(top_p), _ptr(min_p), _ptr(uniform), _ptr(token),
                            _ptr(probability), _stream(stream)), "bcq_sample")


def set_option(name, value):
    _check(lib().bcq_set_option(name.encode(), int(value)), "bcq_set_option")


class PackedLayer:
    """Device buffers of one packed layer: holds torch allocations and the
    descriptor, and forwards to the C entry points (no arithmetic here)."""

    def __init__(self, M, N, q, group=128, has_offset=False, max_batch=1, device="cuda"):
        import torch
        self.desc = Desc(M, N, q, group, 1 if has_offset else 0, 0)
        nbytes = packed_bytes(self.desc)
        if nbytes == 0:
            raise BcqError(BCQ_ERR_UNSUPPORTED, "bcq_packed_bytes")
        self.device = device
        self.packed = torch.empty(nbytes, dtype=torch.uint8, device=device)
        self.max_batch = max_batch
        ws = workspace_bytes(self.desc, max_batch)
        self.workspace = torch.empty(max(ws, 16), dtype=torch.uint8, device=device)
        self.workspace_bytes = ws
        workspace_init(self.workspace, self.workspace.numel())

    def pack_from(self, codes, alpha, offset):
        """codes uint8 [M][N], alpha fp16 [M][G][q], offset fp16 [M][G] or None (device tensors)."""
        pack(self.desc, codes, alpha, offset, self.packed)
        return self

    def pack_rows_from(self, row_begin, codes, alpha, offset):
        """Rows [row_begin, row_begin + codes.shape[0]) from tensors that hold only those rows."""
        pack_rows(self.desc, row_begin, codes.shape[0], codes, alpha, offset, self.packed)
        return self

    def gemv(self, x, y=None):
        import torch
        if y is None:
            y = torch.empty(self.desc.M, dtype=torch.float16, device=self.device)
        gemv(self.desc, self.packed, x, y, self.workspace if self.workspace_bytes else None)
        return y

    def gemm_skinny(self, X, Y=None):
        import torch
        batch = X.shape[0]
        if not 1 <= batch <= BCQ_MAX_BATCH:
            raise BcqError(BCQ_ERR_INVALID_ARG, "PackedLayer.gemm_skinny (batch outside 1..%d)" % BCQ_MAX_BATCH)
        if batch > self.max_batch:   # the workspace holds max_batch accumulators per row
            raise BcqError(BCQ_ERR_WORKSPACE, "PackedLayer.gemm_skinny (batch %d > max_batch %d)" % (batch, self.max_batch))
        if Y is None:
            Y = torch.empty((batch, self.desc.M), dtype=torch.float16, device=self.device)
        gemm_skinny(self.desc, self.packed, X, X.stride(0), Y, Y.stride(0), batch,
                    self.workspace if self.workspace_bytes else None)
        return Y
