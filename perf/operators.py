"""Operators of a serving step between the stacked q/k/v projection and the output projection, as cases that can be timed and compared.

* attend: attention of new tokens (one per request, a few, or a chunk) over a paged key/value cache;
* rotate: norms of q and k per head, position rotation, append of k and v to the pages, in one pass;
* lora: low-rank adapters of many requests beside a shared projection.

`listed()` holds the cases, `draw(rng)` gives more of the same ranges, `prepare` makes the inputs on the GPU from a seed, `run` is one
pass: the plain form in elementary torch operations in 32 bits, or with `own` the library's entry points.  `exact` is the definition in 64
bits and `work` what a pass cannot do without.
"""
import math

import torch

own = False

# ------------------------------------------------------------------------------------------------
# the cases
# ------------------------------------------------------------------------------------------------


def listed():
    return [
        # One user's next token over a short context, heads of a Llama-2-70B-shaped block: latency.
        _attend("attend_one_1000", 1, (1, 1), (1000, 1000), 64, 8),
        # Sixty-four users' next tokens, contexts of very different lengths: the ordinary decode step.
        _attend("attend_decode_64", 64, (1, 1), (200, 8000), 64, 8),
        # Two users of an OPT-66B-shaped block, a key/value head for every query head.
        _attend("attend_decode_72_heads", 2, (1, 1), (12345, 16411), 72, 72, dtype="bf16", page=64),
        # Five drafted tokens verified over a long document.
        _attend("attend_draft_131077", 1, (5, 5), (131077, 131077), 64, 8, page=32),
        # A chunk of a long prompt, OPT-30B-shaped heads: the largest amount of arithmetic.
        _attend("attend_chunk_2048", 1, (2048, 2048), (8192, 8192), 56, 56, dtype="bf16"),
        # Chunks and single tokens of several users together, small heads, sliding window, ragged lengths.
        _attend("attend_mixed_window", 9, (1, 211), (3, 1531), 12, 12, head_dim=64, dtype="bf16", page=32, window=500),
        # The rotation for one user's next token: latency.
        _rotate("rotate_one", 1, 64, 8),
        # A batch of prompt chunks, OPT-30B-shaped heads, half of each head rotated, neighbouring pairs.
        _rotate("rotate_chunk_4096", 4096, 56, 56, rot=64, interleaved=True, dtype="bf16"),
        # One user's adapter beside the stacked q/k/v projection of a Llama-2-70B-shaped block: latency.
        _lora("lora_one", 1, 8192, 10240, 1, (16, 16)),
        # Sixty-four users' next tokens with thirty-two adapters, the same projection.
        _lora("lora_decode_64", 64, 8192, 10240, 32, (16, 16)),
        # Ragged sizes, ranks that differ, an odd number of users, some without an adapter.
        _lora("lora_ragged_27", 27, 7232, 5000, 9, (5, 40), bare=5),
        # Prompt chunks of four users beside the widest projection of an OPT-30B-shaped block.
        _lora("lora_chunk_2048", 2048, 7168, 28672, 4, (64, 64), dtype="bf16"),
    ]


def _attend(name, requests, new, kv, q_heads, kv_heads, head_dim=128, dtype="f16", page=16, causal=True, window=0):
    c = {"kind": "attend", "requests": requests, "new_lo": new[0], "new_hi": new[1], "kv_lo": kv[0], "kv_hi": kv[1],
         "q_heads": q_heads, "kv_heads": kv_heads, "head_dim": head_dim, "dtype": dtype, "page": page, "causal": causal, "window": window}
    return dict(c, name=name) if name else c


def _rotate(name, tokens, q_heads, kv_heads, head_dim=128, rot=128, interleaved=False, norm=True, dtype="f16", page=16):
    c = {"kind": "rotate", "tokens": tokens, "q_heads": q_heads, "kv_heads": kv_heads, "head_dim": head_dim, "rot": rot,
         "interleaved": interleaved, "norm": norm, "dtype": dtype, "page": page}
    return dict(c, name=name) if name else c


def _lora(name, tokens, N, M, adapters, rank, bare=0, dtype="f16"):
    """`bare`: every bare-th token has no adapter (0: all have one)."""
    c = {"kind": "lora", "tokens": tokens, "N": N, "M": M, "adapters": adapters, "rank_lo": rank[0], "rank_hi": rank[1], "bare": bare, "dtype": dtype}
    return dict(c, name=name) if name else c


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi, step=1):
    """A size of the range, none of them 3072."""
    n = max(1, _log_uniform(rng, lo, hi) // step) * step
    return n if n != 3072 else n + step


_HEADS = [(64, 8), (64, 8), (56, 56), (72, 72), (12, 12), (32, 32), (32, 4), (8, 1), (40, 8), (15, 5)]


def draw(rng):
    kind = rng.choice(["attend", "attend", "attend", "rotate", "lora", "lora"])
    dtype = rng.choice(["f16", "bf16"])
    q_heads, kv_heads = rng.choice(_HEADS)
    head_dim = rng.choice([128, 128, 128, 64, 64, 80, 96, 256])
    page = rng.choice([16, 16, 8, 32, 64, 128])
    if kind == "rotate":
        rot = rng.choice([head_dim, head_dim, head_dim // 2, head_dim // 4])
        return _rotate(None, _size(rng, 1, 4096), q_heads, kv_heads, head_dim, rot, rng.random() < 0.4, rng.random() < 0.8, dtype, page)
    if kind == "lora":
        while True:
            adapters = _size(rng, 1, 64)
            hi = _size(rng, 4, 128)
            c = _lora(None, _size(rng, 1, 2048), _size(rng, 768, 28672, 8), _size(rng, 512, 36864), adapters, (rng.randrange(1, hi + 1), hi),
                      rng.choice([0, 0, 3, 7]), dtype)
            # the plain form multiplies by all adapters at once
            if adapters * hi * (c["N"] + c["M"]) <= 5e7 and c["tokens"] * (c["N"] + c["M"]) * max(64, hi) <= 2048 * 35840 * 64:
                return c
    while True:
        requests = _size(rng, 1, 96)
        kv = _size(rng, 16, 131072)
        new = rng.choice([1, 1, 1, _size(rng, 2, 16), _size(rng, 16, 2048)])
        if new > kv or requests * q_heads * new * kv * 4 > 4e9 or requests * kv * kv_heads * head_dim * 4 > 1.2e9:
            continue
        causal = rng.random() < 0.9
        return _attend(None, requests, (rng.choice([1, new]), new), (max(new, kv // rng.choice([1, 2, 16])), kv), q_heads, kv_heads, head_dim,
                       dtype, page, causal, rng.choice([0, 0, 0, _size(rng, 16, 4096)]) if causal else 0)


# ------------------------------------------------------------------------------------------------
# sizes that follow from a case alone
# ------------------------------------------------------------------------------------------------


def _spread(lo, hi, i):
    """The i-th of numbers spread over lo..hi, beginning with hi."""
    return hi - int(((i * 0.6180339887498949) % 1.0) * (hi - lo + 1)) if hi > lo else hi


def _lengths(case):
    """(new tokens, keys) of each request; a request has at least as many keys as new tokens."""
    new = [_spread(case["new_lo"], case["new_hi"], i) for i in range(case["requests"])]
    return new, [max(n, _spread(case["kv_lo"], case["kv_hi"], 3 * i)) for i, n in enumerate(new)]


def _adapter_of(case):
    bare = case["bare"]
    return [-1 if bare and t % bare == bare - 1 else (t * case["adapters"]) // case["tokens"] if case["tokens"] > 64 else (t * 7) % case["adapters"]
            for t in range(case["tokens"])]


def _ranks(case):
    return [_spread(case["rank_lo"], case["rank_hi"], i) for i in range(case["adapters"])]


def work(case):
    if case["kind"] == "rotate":
        n = case["tokens"] * (case["q_heads"] + 2 * case["kv_heads"]) * case["head_dim"]
        return {"bytes": 4 * n + case["tokens"] * (4 * case["rot"] + 8), "flops": 10 * n}
    if case["kind"] == "lora":
        ranks, of = _ranks(case), _adapter_of(case)
        N, M, T = case["N"], case["M"], case["tokens"]
        return {"bytes": 2 * (T * N + 2 * T * M) + 4 * T + 2 * (N + M) * sum(ranks[a] for a in set(of) if a >= 0),
                "flops": 2 * (N + M) * sum(ranks[a] for a in of if a >= 0)}
    new, kv = _lengths(case)
    Hq, Hkv, D, window = case["q_heads"], case["kv_heads"], case["head_dim"], case["window"]
    pairs = seen = 0
    for n, L in zip(new, kv):
        first = L - n  # position of the first new token
        if not case["causal"]:
            pairs, seen = pairs + n * L, seen + L
            continue
        pairs += sum(min(p + 1, window) if window else p + 1 for p in range(first, L))
        seen += L - max(0, first + 1 - window) if window else L
    return {"bytes": 4 * seen * Hkv * D + 4 * sum(new) * Hq * D, "flops": 4 * D * Hq * pairs}


# ------------------------------------------------------------------------------------------------
# inputs, from the seed alone
# ------------------------------------------------------------------------------------------------

_DTYPE = {"f16": torch.float16, "bf16": torch.bfloat16}


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _randn(shape, dtype, g):
    return torch.randn(shape, device="cuda", generator=g, dtype=dtype)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    g, dtype = _gen(seed), _DTYPE[case["dtype"]]
    return {"attend": _prepare_attend, "rotate": _prepare_rotate, "lora": _prepare_lora}[case["kind"]](case, g, dtype)


def _prepare_attend(case, g, dtype):
    """Normed and rotated queries and keys (entries of unit variance, query heads of different sharpness), pages in any order; the pages
    that no request has, and the slots behind a request's last key, hold what other requests left there."""
    new, kv = _lengths(case)
    Hq, Hkv, D, page = case["q_heads"], case["kv_heads"], case["head_dim"], case["page"]
    pages = [-(-L // page) for L in kv]
    pool, width = sum(pages) + 3, max(pages) + 2
    k, v = (_randn((pool, Hkv, page, D), dtype, g) for _ in range(2))
    order = torch.randperm(pool, device="cuda", generator=g).int()
    count = _ints(pages)
    first = count.cumsum(0) - count
    column = torch.arange(width, device="cuda")
    table = torch.where(column < count[:, None], order[(first[:, None] + column).clamp(max=pool - 1).long()], 0).int()
    q = _randn((sum(new), Hq, D), dtype, g) * torch.empty((Hq, 1), device="cuda").uniform_(0.5, 3.0, generator=g).to(dtype)
    start = torch.cat([_ints([0]), _ints(new).cumsum(0).int()])
    return {"case": case, "q": q.view(sum(new), Hq * D), "k": k, "v": v, "q_start": start, "kv_len": _ints(kv), "pages": table, "max_new": max(new),
            "scale": D ** -0.5}


def _prepare_rotate(case, g, dtype):
    """What the stacked projection left, norm weights near one, the table of cosines and sines that a program makes once, tokens of
    consecutive positions in pages of any order."""
    T, Hq, Hkv, D, page, rot = (case[n] for n in ("tokens", "q_heads", "kv_heads", "head_dim", "page", "rot"))
    qkv = _randn((T, (Hq + 2 * Hkv) * D), dtype, g)
    weights = [(1 + 0.2 * _randn((D,), torch.float32, g)).to(dtype) if case["norm"] else None for _ in range(2)]
    longest = T + 1000
    angle = torch.arange(longest, device="cuda", dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(0, rot, 2, device="cuda", dtype=torch.float64) / rot)
    table = torch.cat([angle.cos(), angle.sin()], dim=1).float()
    pool = -(-T // page) + 3
    order = torch.randperm(pool, device="cuda", generator=g)
    t = torch.arange(T, device="cuda")
    slots = (order[t // page] * page + t % page).int()
    position = (t + torch.randint(0, 1000, (1,), device="cuda", generator=g)).int()
    k, v = (_randn((pool, Hkv, page, D), dtype, g) for _ in range(2))
    return {"case": case, "qkv": qkv, "q_weight": weights[0], "k_weight": weights[1], "table": table, "slots": slots, "position": position, "k": k, "v": v,
            "eps": 1e-6}


def _prepare_lora(case, g, dtype):
    """Adapters whose update is a few tenths of the projection's output; rows of an adapter behind its own rank hold another's weights."""
    T, N, M, C = case["tokens"], case["N"], case["M"], case["adapters"]
    ranks = _ranks(case)
    width = -(-max(ranks) // 8) * 8
    A = _randn((C, width, N), dtype, g) * N ** -0.5
    B = _randn((C, M, width), dtype, g) * max(ranks) ** -0.5
    scale = torch.empty(C, device="cuda").uniform_(0.2, 0.6, generator=g)
    return {"case": case, "X": _randn((T, N), dtype, g), "base": _randn((T, M), dtype, g), "A": A, "B": B, "scale": scale, "rank": _ints(ranks),
            "adapter": _ints(_adapter_of(case))}


# ------------------------------------------------------------------------------------------------
# one pass
# ------------------------------------------------------------------------------------------------


def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"attend": _own_attend, "rotate": _own_rotate, "lora": _own_lora}[kind](state)
    return {"attend": _plain_attend, "rotate": _plain_rotate, "lora": _plain_lora}[kind](state)


def _handle(state, make):
    """The object that a program keeps beside its cache or its adapters (it holds them and nothing that follows from their values)."""
    if "handle" not in state:
        state["handle"] = make()
    return state["handle"]


def _own_attend(s):
    import paper_2407_02891_amd as bcq
    cache = _handle(s, lambda: bcq.PagedCache(s["k"], s["v"]))
    return cache.attend(s["q"], s["q_start"], s["kv_len"], s["pages"], s["max_new"], scale=s["scale"], causal=s["case"]["causal"], window=s["case"]["window"])


def _own_rotate(s):
    import paper_2407_02891_amd as bcq
    cache = _handle(s, lambda: bcq.PagedCache(s["k"], s["v"]))
    q = cache.rotate(s["qkv"], s["position"], s["table"], s["slots"], s["q_weight"], s["k_weight"], eps=s["eps"], interleaved=s["case"]["interleaved"])
    return {"q": q, "k": s["k"], "v": s["v"]}


def _own_lora(s):
    import paper_2407_02891_amd as bcq
    adapters = _handle(s, lambda: bcq.Adapters(s["A"], s["B"], s["scale"], s["rank"]))
    return adapters.add(s["X"], s["adapter"], s["base"])


def _plain_attend(s):
    case, start, kv_len = s["case"], s["q_start"].long(), s["kv_len"].long()
    Hq, Hkv, D, n, R = case["q_heads"], case["kv_heads"], case["head_dim"], s["max_new"], case["requests"]
    G, T = Hq // Hkv, s["q"].shape[0]
    here = torch.arange(n, device="cuda")
    rows = (start[:-1, None] + here).clamp(max=T - 1)
    Q = s["q"].float()[rows].view(R, n, Hkv, G, D).permute(0, 2, 3, 1, 4).reshape(R, Hkv, G * n, D)
    pages = s["pages"].long()
    K, V = (c[pages].permute(0, 2, 1, 3, 4).reshape(R, Hkv, -1, D).float() for c in (s["k"], s["v"]))
    L = K.shape[2]
    key, position = torch.arange(L, device="cuda"), (kv_len - (start[1:] - start[:-1]))[:, None] + here
    see = (key < kv_len[:, None, None]).expand(R, n, L)
    if case["causal"]:
        see = see & (key <= position[:, :, None])
    if case["window"]:
        see = see & (key > position[:, :, None] - case["window"])
    score = (torch.matmul(Q, K.transpose(2, 3)).view(R, Hkv, G, n, L) * s["scale"]).masked_fill_(~see[:, None, None], -math.inf)
    weight = score.sub_(score.amax(dim=4, keepdim=True).clamp(min=-1e30)).exp_()
    total = weight.sum(dim=4, keepdim=True)
    out = torch.matmul(weight.view(R, Hkv, G * n, L), V).view(R, Hkv, G, n, D) / total.clamp(min=1e-30)
    token = torch.arange(T, device="cuda")
    request = torch.searchsorted(start[1:].contiguous(), token, right=True)
    return out.permute(0, 3, 1, 2, 4).reshape(R, n, Hq * D)[request, token - start[request]].to(s["q"].dtype)


def _plain_rotate(s):
    case, dtype = s["case"], s["qkv"].dtype
    T, Hq, Hkv, D, page, rot = (case[n] for n in ("tokens", "q_heads", "kv_heads", "head_dim", "page", "rot"))
    x = s["qkv"].view(T, Hq + 2 * Hkv, D)
    qk = x[:, : Hq + Hkv].float()
    if case["norm"]:
        w = torch.cat([s["q_weight"].float().expand(Hq, D), s["k_weight"].float().expand(Hkv, D)])
        qk = qk * torch.rsqrt((qk * qk).mean(dim=2, keepdim=True) + s["eps"]) * w
    turn = s["table"][s["position"].long()][:, None]
    cos, sin = turn[..., : rot // 2], turn[..., rot // 2 :]
    a, b = (qk[..., 0:rot:2], qk[..., 1:rot:2]) if case["interleaved"] else (qk[..., : rot // 2], qk[..., rot // 2 : rot])
    a, b = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([a, b], dim=3).flatten(2) if case["interleaved"] else torch.cat([a, b], dim=2)
    qk = torch.cat([turned, qk[..., rot:]], dim=2).to(dtype)
    at, offset = s["slots"].long() // page, s["slots"].long() % page
    s["k"][at, :, offset] = qk[:, Hq:]
    s["v"][at, :, offset] = x[:, Hq + Hkv :]
    return {"q": qk[:, :Hq].reshape(T, Hq * D), "k": s["k"], "v": s["v"]}


def _plain_lora(s):
    case = s["case"]
    C, width, N = s["A"].shape
    v = torch.matmul(s["X"].float(), s["A"].float().view(C * width, N).t()).view(-1, C, width)
    keep = (s["adapter"][:, None] == torch.arange(C, device="cuda"))[:, :, None] & (torch.arange(width, device="cuda") < s["rank"][:, None])
    v = torch.where(keep, v * s["scale"][:, None], 0.0).view(-1, C * width)
    return (s["base"].float() + torch.matmul(v, s["B"].float().permute(0, 2, 1).reshape(C * width, case["M"]))).to(s["base"].dtype)


# ------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ------------------------------------------------------------------------------------------------


def exact(case, seed):
    s = prepare(case, seed)

    def attend():
        new, kv = _lengths(case)
        Hq, Hkv, D, page, window = case["q_heads"], case["kv_heads"], case["head_dim"], case["page"], case["window"]
        G, t0 = Hq // Hkv, 0
        out = torch.zeros((sum(new), Hq, D), dtype=torch.float64, device="cuda")
        q = s["q"].view(-1, Hq, D)
        for r, (n, L) in enumerate(zip(new, kv)):
            used = s["pages"][r, : -(-L // page)].long()
            position, key = torch.arange(L - n, L, device="cuda")[:, None], torch.arange(L, device="cuda")
            hidden = torch.zeros((n, L), dtype=torch.bool, device="cuda")
            if case["causal"]:
                hidden |= key > position
            if window:
                hidden |= key <= position - window
            for h in range(Hkv):
                K, V = (c[used, h].reshape(-1, D)[:L].double() for c in (s["k"], s["v"]))
                for head in range(h * G, h * G + G):
                    score = (q[t0 : t0 + n, head].double() @ K.t()) * s["scale"]
                    score[hidden] = -math.inf
                    out[t0 : t0 + n, head] = torch.softmax(score, dim=1) @ V
            t0 += n
        return out.view(-1, Hq * D)

    def rotate():
        T, Hq, Hkv, D, page, rot = (case[n] for n in ("tokens", "q_heads", "kv_heads", "head_dim", "page", "rot"))
        x = s["qkv"].double().view(T, Hq + 2 * Hkv, D)
        out = x.clone()
        for first, heads, weight in ((0, Hq, s["q_weight"]), (Hq, Hkv, s["k_weight"])):
            part = x[:, first : first + heads]
            if case["norm"]:
                part = part / (part.square().mean(dim=-1, keepdim=True) + s["eps"]).sqrt() * weight.double()
            spun = part.clone()
            for i in range(rot // 2):
                at = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + rot // 2)
                c = s["table"][s["position"].long(), i].double()[:, None]
                z = s["table"][s["position"].long(), i + rot // 2].double()[:, None]
                spun[..., at[0]] = part[..., at[0]] * c - part[..., at[1]] * z
                spun[..., at[1]] = part[..., at[1]] * c + part[..., at[0]] * z
            out[:, first : first + heads] = spun
        caches = []
        for cache, first in ((s["k"], Hq), (s["v"], Hq + Hkv)):
            pool = cache.shape[0]
            flat = cache.double().transpose(1, 2).reshape(pool * page, Hkv, D)
            flat[s["slots"].long()] = out[:, first : first + Hkv]
            caches.append(flat.view(pool, page, Hkv, D).transpose(1, 2).contiguous())
        return {"q": out[:, :Hq].reshape(T, Hq * D), "k": caches[0], "v": caches[1]}

    def lora():
        of, ranks = torch.tensor(_adapter_of(case), device="cuda"), _ranks(case)
        y = s["base"].double()
        for a in sorted(set(_adapter_of(case)) - {-1}):
            rows = (of == a).nonzero()[:, 0]
            v = s["X"][rows].double() @ s["A"][a, : ranks[a]].double().t()
            y[rows] += s["scale"][a].double() * (v @ s["B"][a, :, : ranks[a]].double().t())
        return y

    return {"attend": attend, "rotate": rotate, "lora": lora}[case["kind"]]()
