"""Plain 64-bit forms of the serving operators (CPU, float64, loops over requests, heads and tokens) with the error that a correct
implementation may have beside them, element by element.

u is half a unit in the last place of the result's type (2^-11 binary16, 2^-8 bfloat16), w = 2^-24 that of binary32.  What is
rounded to 16 bits on the way is stated at each bound; every sum of n terms in binary32 is off by at most n w times the sum of the
terms' magnitudes, in whatever order it is formed."""
import math

import torch

U = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float16: 2.0 ** -25, torch.bfloat16: 0.0}   # half the distance of subnormal results
W = 2.0 ** -24


def assert_close(got, ref, bound, what=""):
    got = got.double().cpu()
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    assert torch.equal(torch.isnan(got), torch.isnan(ref)), f"{what}: NaN in other places"
    assert torch.equal(got.isinf() & (got > 0), ref.isinf() & (ref > 0)) and torch.equal(got.isinf() & (got < 0), ref.isinf() & (ref < 0)), \
        f"{what}: infinities in other places"
    fine = ref.isfinite()
    over = ((got - ref).abs() - bound)[fine]
    assert over.numel() == 0 or float(over.max()) <= 0, \
        f"{what}: off by {float((got - ref).abs()[fine].max()):.3g}, {int((over > 0).sum())} of {over.numel()} elements beyond their bound"


def rotate_ref(qkv, q_heads, kv_heads, D, positions, cos_sin, q_weight, k_weight, eps, interleaved):
    """(rows [tokens][heads][D] in float64, bound), v heads as they are.  The norm sums D squares, divides and multiplies (D + 6 roundings
    of the value), the rotation adds two products of it."""
    T = qkv.shape[0]
    x = qkv.double().cpu().view(T, q_heads + 2 * kv_heads, D)
    out, size = x.clone(), x.abs()
    for lo, hi, weight in ((0, q_heads, q_weight), (q_heads, q_heads + kv_heads, k_weight)):
        n = x[:, lo:hi]
        if weight is not None:
            n = n / (n.square().mean(-1, keepdim=True) + eps).sqrt() * weight.double().cpu()
        out[:, lo:hi], size[:, lo:hi] = n, n.abs()
        if cos_sin is None:
            continue
        rot = cos_sin.shape[1]
        first = torch.arange(0, rot, 2) if interleaved else torch.arange(rot // 2)
        second = first + (1 if interleaved else rot // 2)
        turn = cos_sin.double().cpu()[positions.long().cpu().clamp(0, cos_sin.shape[0] - 1)][:, None]
        c, z = turn[..., : rot // 2], turn[..., rot // 2:]
        a, b = n[..., first], n[..., second]
        out[:, lo:hi][..., first], out[:, lo:hi][..., second] = a * c - b * z, b * c + a * z
        both = (a * c).abs() + (b * z).abs(), (b * c).abs() + (a * z).abs()
        size[:, lo:hi][..., first], size[:, lo:hi][..., second] = both
    bound = U[qkv.dtype] * out.abs() + (D + 10) * W * 2 * size + TINY[qkv.dtype]
    bound[:, q_heads + kv_heads:] = 0
    return out, bound


def attend_ref(q, k, v, q_start, kv_len, pages, q_heads, scale, causal, window, max_new=None):
    """(out [tokens][q_heads * D] in float64, bound).  A weight is rounded to 16 bits at most once (relative u); scores are sums of D products,
    so a weight is off by a factor of 1 + 2 ds, ds the error of a score; sums over the keys.  Rows that no request has are NaN (`missing`)."""
    page, D, kv_heads = k.shape[2], k.shape[3], k.shape[1]
    T, G = q.shape[0], q_heads // kv_heads
    qs, lens, table = q_start.tolist(), kv_len.tolist(), pages.cpu().long()
    qq = q.double().cpu().view(T, q_heads, D)
    kk, vv = k.cpu(), v.cpu()
    out = torch.full((T, q_heads, D), math.nan, dtype=torch.float64)
    bound = torch.zeros_like(out)
    written = torch.zeros(T, dtype=torch.bool)
    u = U[q.dtype]
    for r, L in enumerate(lens):
        n = qs[r + 1] - qs[r]
        key = torch.arange(L)
        at = table[r][key // page] if L else key
        for h in range(kv_heads):
            K, V = kk[at, h, key % page].double(), vv[at, h, key % page].double()
            for i in range(n if max_new is None else min(n, max_new)):
                t, p = qs[r] + i, L - n + i
                end = min(L, p + 1) if causal else L
                begin = max(0, p + 1 - window) if window else 0
                written[t] = True
                rows = slice(h * G, h * G + G)
                if begin >= end:
                    out[t, rows] = 0.0
                    continue
                s = qq[t, rows] @ K[begin:end].T * scale
                size = qq[t, rows].abs() @ K[begin:end].abs().T * scale
                weight = torch.softmax(s, dim=1)
                y = weight @ V[begin:end]
                mean = weight @ V[begin:end].abs()
                ds = (D + 4) * W * size.max(dim=1, keepdim=True).values + 4 * W * s.abs().max(dim=1, keepdim=True).values + 4 * W
                out[t, rows] = y
                bound[t, rows] = u * y.abs() + (u + 4 * ds + (2 * (end - begin) + 64) * W) * mean + TINY[q.dtype]
    return out.view(T, -1), bound.view(T, -1), written


def lora_ref(X, A, B, scale, rank, adapter, base):
    """(Y in float64, bound).  A x is a sum of N products; held to 2^-21 of the largest value of its token at least; then a sum of rank
    products, one addition to the base."""
    C, width, N = A.shape
    y = base.double().cpu().clone()
    bound = U[base.dtype] * y.abs() + TINY[base.dtype]
    for t, a in enumerate(adapter.tolist()):
        if not 0 <= a < C:
            bound[t] = 0
            continue
        n = min(max(int(rank[a]), 0), width) if rank is not None else width
        s = float(scale[a]) if scale is not None else 1.0
        Aa, Ba, x = A[a, :n].double().cpu(), B[a, :, :n].double().cpu(), X[t].double().cpu()
        v = Aa @ x
        dv = N * W * (Aa.abs() @ x.abs()) + (2.0 ** -21 * v.abs().max() if n else 0.0)
        delta = s * (Ba @ v)
        size = abs(s) * (Ba.abs() @ v.abs())
        extra = abs(s) * (Ba.abs() @ dv) + (n + 4) * W * size + 2 * W * y[t].abs()
        y[t] += delta
        bound[t] = U[base.dtype] * y[t].abs() + 2 * extra + TINY[base.dtype]
    return y, bound
