"""The attention half of a decoder block as a server runs it, for requests of mixed lengths: the stacked q/k/v projection in the binary
coding, each request's low-rank adapter beside it, norm and rotation of q and k with the append to a paged cache, attention over the
pages, and the output projection with its adapter.  Everything runs in the library's kernels on torch's current stream; `step` allocates
from torch alone, so a step of single tokens can be captured in a graph and replayed while `positions`, `slots` and `kv_len` are advanced
in place.  `Decoder` puts it between an embedding and a head, hands pages out as requests grow, reads a prompt that they share once and draws
their tokens, all on the device.

Run as a module for timings with random weights (prompts as one chunk, then single tokens, eagerly and as a replayed graph; with --shared, then
drawn tokens of requests that begin with a prompt of so many):
    python -m paper_2407_02891_amd.serve_block --requests 16 --prompt 100 --tokens 16 --shared 1000
"""
import argparse
import json
import time

import torch

from . import binding as B
from .serving import Adapters, PagedCache, PageTable, Sampler


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

    def step(self, X, positions, slots, adapter, kv_len, q_start, pages, max_new, shared=None):
        """X [tokens][hidden] binary16 -> [tokens][hidden]; the tokens' keys and values are in the cache afterwards.  shared: (group_start, shared_len,
        max_shared) of PagedCache.attend_shared, or None."""
        y = product(self.qkv, X)
        if self.qkv_adapters is not None:
            self.qkv_adapters.add(X, adapter, y, out=y)
        q = self.cache.rotate(y, positions, self.cos_sin, slots, self.q_weight, self.k_weight, eps=self.eps,
                              out=y[:, : self.q_heads * self.cache.head_dim])
        if shared is None:
            a = self.cache.attend(q, q_start, kv_len, pages, max_new)
        else:
            a = self.cache.attend_shared(q, q_start, kv_len, pages, max_new, *shared)
        z = product(self.o, a)
        if self.o_adapters is not None:
            self.o_adapters.add(a, adapter, z, out=z)
        return z


class Decoder:
    """Requests that begin with one prompt and go on by themselves, a drawn token at a time.  The prompt's whole pages stand in every request's row of
    the table and are attended to as shared keys; the pages behind them are taken as the requests grow and given back by those that `leave`."""

    def __init__(self, block, embedding, head, table, sampler, adapter):
        """block: AttentionBlock; embedding [vocabulary][hidden] binary16; head: PackedLayer of vocabulary by hidden; table: PageTable with nothing held,
        over the block's cache; sampler: Sampler, a row per request; adapter: of all requests (keys that are shared depend on it), any number outside
        the adapters': none."""
        cache, longest = block.cache, table.pages.shape[1] * table.page_size
        for holds, why in ((table.page_size == cache.desc.page_size and table.free.shape[0] <= cache.desc.num_pages, "a table of other pages than the cache's"),
                           (block.cos_sin.shape[0] >= longest, f"a rotation table of less than {longest} positions"),
                           (embedding.shape[0] >= head.desc.M, "an embedding of fewer tokens than the head's"),
                           (embedding.dtype == torch.float16 and embedding.shape[1] == block.qkv.desc.N, f"an embedding that is not binary16 of {block.qkv.desc.N} a token"),
                           (head.desc.N == block.o.desc.M, f"a head of other than {block.o.desc.M} inputs"),
                           (sampler.temperature.shape[0] == table.pages.shape[0], "a sampler of another number of rows than requests")):
            if not holds:
                raise B.BcqError(B.BCQ_ERR_INVALID_ARG, f"Decoder ({why})")
        self.block, self.embedding, self.head, self.table, self.sampler, self.adapter = block, embedding, head, table, sampler, adapter
        self.count = table.pages.shape[0]
        self.cached, self.fresh, self.fixed, self.token = (torch.zeros(self.count, dtype=torch.int32, device=table.device) for _ in range(4))
        self.probability = torch.zeros(self.count, device=table.device)
        self.shared, self.plan = None, None

    def _pass(self, ids, plan, max_new):
        """ids of the batch's rows -> the rows that come out of the block."""
        adapter = torch.full_like(plan["owner"], self.adapter)
        return self.block.step(self.embedding[ids], plan["positions"], plan["slots"], adapter, plan["kv_len"], plan["q_start"], self.table.pages, max_new,
                               self.shared)

    def _next(self, z, plan, uniform):
        """Each request's next token from its last row, where it had one and the pages for it; without the pages the step can be made again.  (A token also
        stays where no logit is a number.)"""
        last = (plan["q_start"][1:] - 1).clamp(min=0).long()
        token, probability = self.sampler.draw(product(self.head, z[last]), uniform)
        ready = (plan["lack"] == 0) & (self.fresh > 0) & (token >= 0)
        self.token.copy_(torch.where(ready, token, self.token))
        self.probability.copy_(torch.where(ready, probability, self.probability))
        self.cached.add_(torch.where(plan["lack"] == 0, self.fresh, 0))

    def _take(self, counts):
        """The plan of a batch of so many tokens of each request."""
        self.fresh.copy_(torch.tensor(counts, dtype=torch.int32))
        return self.table.step(self.cached, self.fresh, sum(counts), self.fixed)

    def prompt(self, shared, own, uniform):
        """The ids that all requests begin with, the ids (at least one) that follow in each, and the numbers that their first tokens are drawn with."""
        page, device, where = self.table.page_size, self.table.device, "Decoder.prompt"
        whole = len(shared) // page * page
        rest = [shared[whole:] + ids for ids in own]
        pages = [-(-len(ids) // page) for ids in rest]
        if len(own) != self.count or not all(own):
            raise B.BcqError(B.BCQ_ERR_INVALID_ARG, f"{where} (one id or more of each of the {self.count} requests)")
        if any(ids and not 0 <= min(ids) <= max(ids) < self.embedding.shape[0] for ids in [shared] + own):
            raise B.BcqError(B.BCQ_ERR_INVALID_ARG, f"{where} (ids of 0 to {self.embedding.shape[0] - 1}, the embedding's)")
        if bool((self.cached + self.table.held).any()):
            raise B.BcqError(B.BCQ_ERR_INVALID_ARG, f"{where} (requests that have begun)")
        if whole // page + max(pages) > self.table.pages.shape[1] or whole // page + sum(pages) > int(self.table.free_count):
            raise B.BcqError(B.BCQ_ERR_INVALID_ARG, f"{where} ({whole // page} pages of the shared ids and {pages} of the requests' own do not fit)")
        if whole:
            plan = self._take([whole] + [0] * (self.count - 1))
            self._pass(torch.tensor(shared[:whole], device=device), plan, whole)
            n = whole // page
            self.table.pages[1:, :n] = self.table.pages[0, :n]
            self.table.held.fill_(n)
            self.fixed.fill_(n)
            self.cached.fill_(whole)
            self.shared = (torch.tensor([0, self.count], dtype=torch.int32, device=device), torch.full((1,), whole, dtype=torch.int32, device=device), whole)
        plan = self._take([len(ids) for ids in rest])
        self._next(self._pass(torch.tensor(sum(rest, []), device=device), plan, max(map(len, rest))), plan, uniform)
        self.fresh.fill_(1)

    def step(self, uniform):
        """The keys of each request's token into the cache, and the token after it into `token`: nothing waits for the device, and a captured step can be
        replayed (with other numbers in `uniform`)."""
        plan = self.plan = self.table.step(self.cached, self.fresh, self.count, self.fixed, out=self.plan)
        self._next(self._pass(self.token[plan["owner"].clamp(min=0).long()].long(), plan, 1), plan, uniform)

    def leave(self, request):
        """The request is over: its own pages go back with the next step."""
        self.cached[request] = 0
        self.fresh[request] = 0


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
                        ("tokens", 16), ("page", 16), ("adapters", 4), ("rank", 16), ("shared", 0), ("vocabulary", 32000)):
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
    if a.shared:
        answers(a)


def random_head(hidden, vocabulary, planes, seed=0):
    """An embedding and a head of that size with random weights: (embedding, PackedLayer, (codes, alpha)); logits of rows of size one have size four."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    codes = torch.randint(0, 1 << planes, (vocabulary, hidden), device="cuda", generator=g, dtype=torch.uint8)
    step = 2.0 ** -torch.arange(planes, device="cuda")
    alpha = (4 * (0.5 + torch.rand((vocabulary, hidden // 128, planes), device="cuda", generator=g)) * step * hidden ** -0.5).half()
    head = B.PackedLayer(vocabulary, hidden, planes, 128, False, max_batch=B.BCQ_MAX_BATCH).pack_from(codes, alpha, None)
    return torch.randn((vocabulary, hidden), device="cuda", generator=g).half(), head, (codes, alpha)


def answers(a):
    longest = a.shared + a.prompt + a.requests + 2 * a.tokens + a.page
    width = -(-longest // a.page)
    own = a.requests * (-(-(longest - a.shared) // a.page) + 1)
    block, _ = random_block(a.hidden, a.q_heads, a.kv_heads, a.head_dim, a.planes, width + own, a.page, width * a.page, a.adapters, a.rank)
    embedding, head, _ = random_head(a.hidden, a.vocabulary, a.planes)
    table = PageTable.empty(a.requests, width, width + own, a.page)
    sampler = Sampler(torch.full((a.requests,), 0.8, device="cuda"), torch.full((a.requests,), 50, dtype=torch.int32, device="cuda"),
                      torch.full((a.requests,), 0.95, device="cuda"))
    decoder = Decoder(block, embedding, head, table, sampler, adapter=0)
    ids = torch.randint(0, a.vocabulary, (longest,)).tolist()
    uniform = torch.rand(a.requests, device="cuda")
    decoder.prompt(ids[:a.shared], [ids[: a.prompt + r] for r in range(a.requests)], uniform)

    def timed(f):
        torch.cuda.synchronize()
        t0 = time.perf_counter()
        for _ in range(a.tokens):
            uniform.uniform_()
            f()
        torch.cuda.synchronize()
        return (time.perf_counter() - t0) * 1e3 / a.tokens

    decoder.step(uniform)
    eager_ms = timed(lambda: decoder.step(uniform))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        decoder.step(uniform)
    graph_ms = timed(graph.replay)
    print(json.dumps({"what": "answers that begin alike, block and head", "hidden": a.hidden, "vocabulary": a.vocabulary, "requests": a.requests, "shared": a.shared,
                      "token_eager_ms": round(eager_ms, 4), "token_graph_ms": round(graph_ms, 4), "keys_at_end": int(decoder.cached.max())}))


if __name__ == "__main__":
    main()
