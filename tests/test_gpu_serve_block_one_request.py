"""One user alone: a block's attention half with a single request, whose steps are calls of one token."""
import numpy as np
import pytest
import torch

from paper_2407_02891_amd.serve_block import Requests, random_block
from tests.test_gpu_serve_block import ADAPTERS, D, HIDDEN, HKV, HQ, PAGE, RANK, SHARE, _reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("prompt,adapter", [(1, 0), (20, 1), (5, -1)])
def test_one_request(prompt, adapter):
    single = 4
    requests = Requests(1, 48, PAGE, [adapter])
    block, weights = random_block(HIDDEN, HQ, HKV, D, 3, requests.pages.numel(), PAGE, 48, ADAPTERS, RANK, seed=7)
    X = torch.randn((prompt + single, HIDDEN), device="cuda", generator=torch.Generator(device="cuda").manual_seed(3)).half()
    got = [block.step(X[:prompt], **requests.take([prompt]))]
    batch = requests.take([1])
    x = X[prompt:prompt + 1].clone()
    got.append(block.step(x, **batch))
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        z = block.step(x, **batch)
    for i in range(1, single):
        requests.advance(batch)
        x.copy_(X[prompt + i:prompt + i + 1])
        graph.replay()
        again = z.clone()
        assert torch.equal(again, block.step(x, **batch))
        got.append(again)
    ref = _reference(block, weights, X.cpu().double().numpy(), adapter)
    have = torch.cat(got).cpu().double().numpy()
    assert have.shape == ref.shape
    for rows in (slice(0, prompt), slice(prompt, None)):
        share = np.linalg.norm(have[rows] - ref[rows], axis=1) / np.linalg.norm(ref[rows], axis=1)
        assert share.max() <= SHARE, share.max()
