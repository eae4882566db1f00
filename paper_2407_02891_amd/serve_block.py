"""The attention half of a decoder block as a server runs it, for requests of mixed lengths: the stacked q/k/v projection in the binary
coding, each request's low-rank adapter beside it, norm and rotation of q and k with the append to a paged cache, attention over the
pages, and the output projection with its adapter.  Everything runs in the library's kernels on torch's current stream; `step` allocates
from torch alone, so a step of single tokens can be captured in a graph and replayed while `positions`, `slots` and `kv_len` are advanced
in place.

Run as a module for timings with random weights (prompts as one chunk, then single tokens, eagerly and as a replayed graph):
    python -m paper_2407_02891_amd.serve_block --requests 16 --prompt 100 --tokens 16
"""
import argparse
import json
import time

import torch

from . import binding as B
from .serving import Adapters, PagedCache


def product(layer, X):
    """layer applied to any number of rows, BCQ_MAX_BATCH a call."""
    out = torch.empty((X.shape[0], layer.desc.M), dtype=torch.float16, device=X.device)
    for at in range(0, X.shape[0], B.BCQ_MAX_BATCH):
        layer.gemm_skinny(X[at:at + B.BCQ_MAX_BATCH], out[at:at + B.BCQ_MAX_BATCH])
    return out


def rotation_table(positions, rot_dim, base=10000.0, device="cuda"):
    """Cosines and sines of position * base^(-2i / rot_dim), binary32 [positions][rot_dim], as PagedCache.rotate takes them."""
    t = torch.arange(positions, dtype=torch.float64, device=device)
    angle = t[:, None] * base ** (-torch.arange(0, rot_dim, 2, dtype=torch.float64, device=device) / rot_dim)
    return torch.cat([angle.cos(), angle.sin()], dim=1).float()


class Requests:
    """Who is where: requests of up to `longest` tokens own a run of pages each (a server would hand pages out as they fill).  `take(new)`
    returns what a step of new[r] tokens of each request needs, `advance` moves single-token tensors one token on, in place."""

    def __init__(self, count, longest, page_size, adapter, device="cuda"):
        self.page_size, self.width = page_size, -(-longest // page_size)
        self.pages = torch.arange(count * self.width, dtype=torch.int32, device=device).view(count, self.width)
        self.length = [0] * count
        self.adapter = adapter  # of each request, any number outside the adapters': none
        self.device = device

    def _room(self, new):
        for r, n in enumerate(new):
            if self.length[r] + n > self.width * self.page_size:
                raise B.BcqError(B.BCQ_ERR_INVALID_ARG, f"Requests (request {r}: {self.length[r]} tokens and {n} more do not fit its {self.width} pages)")

    def take(self, new):
        self._room(new)
        positions, slots, owner = [], [], []
        for r, n in enumerate(new):
            at = range(self.length[r], self.length[r] + n)
            positions += at
            slots += [(r * self.width + j // self.page_size) * self.page_size + j % self.page_size for j in at]
            owner += [self.adapter[r]] * n
            self.length[r] += n
        ints = [positions, slots, owner, self.length, [0] + torch.tensor(new).cumsum(0).tolist()]
        positions, slots, owner, kv_len, q_start = (torch.tensor(v, dtype=torch.int32, device=self.device) for v in ints)
        return dict(positions=positions, slots=slots, adapter=owner, kv_len=kv_len, q_start=q_start, pages=self.pages, max_new=max(new))

    def advance(self, batch):
        """The next single token of every request (pages of a request are neighbours here, so slots advance by one)."""
        self._room([1] * len(self.length))
        for name in ("positions", "slots", "kv_len"):
            batch[name].add_(1)
        self.length = [n + 1 for n in self.length]


class AttentionBlock:
    def __init__(self, qkv, o, q_heads, cache, cos_sin, q_weight=None, k_weight=None, qkv_adapters=None, o_adapters=None, eps=1e-6):
        """qkv, o: PackedLayer of (q_heads + 2 kv_heads) * head_dim by hidden and of hidden by q_heads * head_dim, packed for batches of up to
        BCQ_MAX_BATCH; cache: PagedCache; cos_sin: rotation_table; q_weight, k_weight: of the norms, or None; adapters: Adapters or None."""
        self.qkv, self.o, self.q_heads, self.cache, self.cos_sin, self.eps = qkv, o, q_heads, cache, cos_sin, eps
        self.q_weight, self.k_weight, self.qkv_adapters, self.o_adapters = q_weight, k_weight, qkv_adapters, o_adapters

    def step(self, X, positions, slots, adapter, kv_len, q_start, pages, max_new):
        """X [tokens][hidden] binary16 -> [tokens][hidden]; the tokens' keys and values are in the cache afterwards."""
        y = product(self.qkv, X)
        if self.qkv_adapters is not None:
            self.qkv_adapters.add(X, adapter, y, out=y)
        q = self.cache.rotate(y, positions, self.cos_sin, slots, self.q_weight, self.k_weight, eps=self.eps,
                              out=y[:, : self.q_heads * self.cache.head_dim])
        a = self.cache.attend(q, q_start, kv_len, pages, max_new)
        z = product(self.o, a)
        if self.o_adapters is not None:
            self.o_adapters.add(a, adapter, z, out=z)
        return z


def random_block(hidden, q_heads, kv_heads, head_dim, planes, pages, page_size, longest, adapters, rank, seed=0):
    """A block of that shape with random weights (of a size that keeps activations near one)."""
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, scale=1.0):
        return (torch.randn(shape, device="cuda", generator=g) * scale).half()

    def layer(M, N):
        codes = torch.randint(0, 1 << planes, (M, N), device="cuda", generator=g, dtype=torch.uint8)
        step = 2.0 ** -torch.arange(planes, device="cuda")
        alpha = ((0.5 + torch.rand((M, N // 128, planes), device="cuda", generator=g)) * step * N ** -0.5).half()
        return B.PackedLayer(M, N, planes, 128, False, max_batch=B.BCQ_MAX_BATCH).pack_from(codes, alpha, None), codes, alpha

    def low_rank(M, N):
        return Adapters(normal(adapters, rank, N, scale=N ** -0.5), normal(adapters, M, rank, scale=rank ** -0.5),
                        torch.full((adapters,), 0.3, device="cuda"))

    wide = (q_heads + 2 * kv_heads) * head_dim
    qkv, o = layer(wide, hidden), layer(hidden, q_heads * head_dim)
    block = AttentionBlock(qkv[0], o[0], q_heads, PagedCache.empty(pages, page_size, kv_heads, head_dim), rotation_table(longest, head_dim),
                           1 + normal(head_dim, scale=0.1), 1 + normal(head_dim, scale=0.1), low_rank(wide, hidden), low_rank(hidden, q_heads * head_dim))
    return block, {"qkv": qkv[1:], "o": o[1:]}


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("hidden", 8192), ("q-heads", 64), ("kv-heads", 8), ("head-dim", 128), ("planes", 3), ("requests", 16), ("prompt", 100),
                        ("tokens", 16), ("page", 16), ("adapters", 4), ("rank", 16)):
        ap.add_argument("--" + name, type=int, default=value)
    a = ap.parse_args()
    longest = a.prompt + a.requests + 2 * a.tokens + 2
    # prompts of different lengths, one adapter more than there are: some requests have none
    requests = Requests(a.requests, longest, a.page, [r % (a.adapters + 1) - 1 for r in range(a.requests)])
    block, _ = random_block(a.hidden, a.q_heads, a.kv_heads, a.head_dim, a.planes, requests.pages.numel(), a.page, longest, a.adapters, a.rank)

    def timed(f):
        torch.cuda.synchronize()
        t0 = time.perf_counter()
        out = f()
        torch.cuda.synchronize()
        return out, (time.perf_counter() - t0) * 1e3

    batch = requests.take([a.prompt + r for r in range(a.requests)])
    X = torch.randn((batch["slots"].numel(), a.hidden), device="cuda").half()
    Z, prompt_ms = timed(lambda: block.step(X, **batch))
    x = Z[batch["q_start"][1:].long() - 1].contiguous()
    batch = requests.take([1] * a.requests)
    block.step(x, **batch)

    def eager():
        for _ in range(a.tokens):
            requests.advance(batch)
            block.step(x, **batch)

    _, eager_ms = timed(eager)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        z = block.step(x, **batch)

    def replayed():
        for _ in range(a.tokens):
            requests.advance(batch)
            graph.replay()

    _, graph_ms = timed(replayed)
    assert bool(z.isfinite().all())
    print(json.dumps({"what": "attention half of a block", "hidden": a.hidden, "requests": a.requests, "prompt_tokens": X.shape[0],
                      "prompt_ms": round(prompt_ms, 3), "token_eager_ms": round(eager_ms / a.tokens, 4), "token_graph_ms": round(graph_ms / a.tokens, 4),
                      "keys_at_end": max(requests.length)}))


if __name__ == "__main__":
    main()
