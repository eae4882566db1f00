"""The operators together: a block's attention half, step by step, against the whole computed in 64 bits."""
import numpy as np
import pytest
import torch

from paper_2407_02891_amd import binding as B
from paper_2407_02891_amd.serve_block import Requests, random_block

pytestmark = pytest.mark.gpu

HIDDEN, HQ, HKV, D, PAGE, ADAPTERS, RANK = 512, 8, 2, 64, 16, 2, 16
# Each row passes eight roundings to binary16 (projection, adapter, rotation, attention, projection, adapter; v the first two), 2^-11 each at most
# and relative to its row: 2^-8 if all line up.  The scores |s| <= 4 carry those of q and k, three each and 6 * 2^-11 * 4 < 2^-6 together, into
# the weights.  Sum of both, as a share of the norm of the result.
SHARE = 2.0 ** -6 + 2.0 ** -8


def _dense(codes, alpha):
    bits = codes.cpu().numpy()
    a = np.repeat(alpha.cpu().double().numpy(), codes.shape[1] // alpha.shape[1], axis=1)
    return sum(a[:, :, i] * (2.0 * (bits >> i & 1) - 1.0) for i in range(alpha.shape[2]))


def _reference(block, weights, X, adapter):
    """All tokens of one request at once, float64 on the host."""
    f = lambda t: t.cpu().double().numpy()  # noqa: E731

    def linear(name, adapters, x):
        y = x @ _dense(*weights[name]).T
        if 0 <= adapter < ADAPTERS:
            y = y + 0.3 * (x @ f(adapters.A[adapter]).T) @ f(adapters.B[adapter]).T
        return y

    T = X.shape[0]
    y = linear("qkv", block.qkv_adapters, X).reshape(T, HQ + 2 * HKV, D)
    table = f(block.cos_sin)[:T, None]
    c, s = table[..., : D // 2], table[..., D // 2:]

    def rotate(x, w):
        x = x / np.sqrt((x ** 2).mean(-1, keepdims=True) + block.eps) * f(w)
        a, b = x[..., : D // 2], x[..., D // 2:]
        return np.concatenate([a * c - b * s, b * c + a * s], -1)

    q, k, v = rotate(y[:, :HQ], block.q_weight), rotate(y[:, HQ:HQ + HKV], block.k_weight), y[:, HQ + HKV:]
    out = np.empty((T, HQ, D))
    for h in range(HQ):
        p = q[:, h] @ k[:, h // (HQ // HKV)].T * D ** -0.5
        p[np.triu_indices(T, 1)] = -np.inf
        p = np.exp(p - p.max(1, keepdims=True))
        out[:, h] = p / p.sum(1, keepdims=True) @ v[:, h // (HQ // HKV)]
    return linear("o", block.o_adapters, out.reshape(T, HQ * D))


def test_prompts_then_tokens_and_graph():
    prompts, single = [5, 70, 33], 4
    requests = Requests(3, 96, PAGE, [0, 1, -1])
    block, weights = random_block(HIDDEN, HQ, HKV, D, 3, requests.pages.numel(), PAGE, 96, ADAPTERS, RANK, seed=5)
    g = torch.Generator(device="cuda").manual_seed(1)
    X = [torch.randn((n + single, HIDDEN), device="cuda", generator=g).half() for n in prompts]
    got = [[] for _ in prompts]

    def collect(z, counts):
        for r, part in enumerate(z.split(counts)):
            got[r].append(part)

    # chunks of mixed lengths (one request has none of the second)
    first = [5, 40, 20]
    collect(block.step(torch.cat([x[:n] for x, n in zip(X, first)]), **requests.take(first)), first)
    second = [n - m for n, m in zip(prompts, first)]
    collect(block.step(torch.cat([x[m:n] for x, n, m in zip(X, prompts, first)]), **requests.take(second)), second)
    # single tokens: eager, then replays of one graph with the numbers advanced in place
    batch = requests.take([1] * 3)
    x = torch.stack([x[n] for x, n in zip(X, prompts)])
    collect(block.step(x, **batch), [1] * 3)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        z = block.step(x, **batch)
    for i in range(1, single):
        requests.advance(batch)
        x.copy_(torch.stack([x[n + i] for x, n in zip(X, prompts)]))
        graph.replay()
        again = z.clone()
        assert torch.equal(again, block.step(x, **batch))
        collect(again, [1] * 3)
    for r, n in enumerate(prompts):
        ref = _reference(block, weights, X[r].cpu().double().numpy(), requests.adapter[r])
        have = torch.cat(got[r]).cpu().double().numpy()
        assert have.shape == ref.shape
        for a, b in ((0, n), (n, n + single)):
            share = np.linalg.norm(have[a:b] - ref[a:b], axis=1) / np.linalg.norm(ref[a:b], axis=1)
            assert share.max() <= SHARE, (r, a, share.max())


def test_products_of_more_rows_than_a_call_takes():
    from paper_2407_02891_amd.serve_block import product
    block, _ = random_block(HIDDEN, HQ, HKV, D, 2, 4, PAGE, 16, 1, 8)
    X = torch.randn((2 * B.BCQ_MAX_BATCH + 5, HIDDEN), device="cuda").half()
    Y = product(block.qkv, X)
    assert torch.equal(Y[B.BCQ_MAX_BATCH:2 * B.BCQ_MAX_BATCH], block.qkv.gemm_skinny(X[B.BCQ_MAX_BATCH:2 * B.BCQ_MAX_BATCH]))
    assert torch.equal(Y[-5:], block.qkv.gemm_skinny(X[-5:]))
