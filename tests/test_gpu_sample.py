"""Drawing tokens from logits against the plain form in 64 bits: every filter alone and together, values that repeat, masks, odd lengths and strides."""
import math

import pytest
import torch

import paper_2407_02891_amd as bcq
from tests.step_util import assert_drawn

pytestmark = pytest.mark.gpu
TYPES = [torch.float16, torch.bfloat16]
F32 = torch.float32


def _settings(rows, seed):
    g = torch.Generator().manual_seed(seed)

    def one_of(values, dtype):
        return torch.tensor(values, dtype=dtype)[torch.randint(0, len(values), (rows,), generator=g)]

    return (one_of([0.0, 0.3, 0.7, 1.0, 1.0, 2.0, 50.0], F32), one_of([0, 0, 1, 2, 7, 50, 10 ** 6], torch.int32), one_of([1.0, 1.0, 0.0, 0.1, 0.5, 0.9, 0.999], F32),
            one_of([0.0, 0.0, 0.01, 0.3, 1.0, 3.0], F32), torch.rand(rows, generator=g))


def _draw(logits, temperature, top_k, top_p, min_p, u, out=None):
    put = lambda t: None if t is None else t.cuda()
    sampler = bcq.Sampler(temperature.cuda(), put(top_k), put(top_p), put(min_p))
    token, p = sampler.draw(logits.cuda() if not logits.is_cuda else logits, u.cuda(), out=out)
    return token.cpu(), p.cpu()


def _check(logits, *settings, what=""):
    token, p = _draw(logits, *settings)
    unsure = assert_drawn(token, p, logits.cpu(), *settings, what=what)
    assert 4 * unsure <= logits.shape[0], what
    return token, p


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,vocab", [(1, 1), (3, 2), (40, 7), (40, 63), (40, 64), (40, 65), (33, 1000), (20, 4097), (9, 8192), (5, 32000), (3, 50259), (2, 65528),
                                        (2, 65529), (3, 70001), (2, 131072), (1, 262144)])
def test_settings_together(rows, vocab, dtype):
    g = torch.Generator().manual_seed(rows * 1000003 + vocab)
    x = (torch.randn((rows, vocab), generator=g) * 2.5).to(dtype)
    _check(x, *_settings(rows, vocab), what=(rows, vocab))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [300, 20000, 150000])
def test_each_filter_alone(vocab, dtype):
    g = torch.Generator().manual_seed(5)
    rows = 8
    x = (torch.randn((rows, vocab), generator=g) * 2).to(dtype)
    T, u = torch.linspace(0.5, 1.5, rows), torch.rand(rows, generator=g)
    _check(x, T, None, None, None, u)
    _check(x, T, torch.tensor([2, 3, 5, 17, 100, 299, 300, 301], dtype=torch.int32), None, None, u)
    _check(x, T, None, torch.linspace(0.05, 0.98, rows), None, u)
    _check(x, T, None, None, torch.tensor([1e-6, 1e-4, 1e-3, 1e-2, 0.05, 0.2, 0.7, 0.99]), u)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [1, 5, 64, 1000, 65528, 65536, 131072, 200001])
def test_equal_logits(vocab, dtype):
    """Weights of one: every border falls on whole numbers, ties go to the lowest index, and counters of one value reach their ends."""
    at = sorted({0, vocab // 7, vocab // 2, vocab - 1})
    rows = len(at)
    x = torch.full((rows, vocab), -1.5, dtype=dtype)
    one = torch.ones(rows)
    # the last u that still belongs to the entry before, and one that belongs to the entry itself
    u = torch.tensor([(i + 0.5) / vocab for i in at])
    token, p = _draw(x, one, None, None, None, u)
    assert token.tolist() == at
    assert torch.allclose(p, one / vocab, rtol=2.0 ** -23, atol=0)
    if vocab >= 4:
        half = vocab // 2
        token, p = _draw(x, one, torch.full((rows,), half, dtype=torch.int32), None, None, one)  # u = 1: the last that is kept
        assert token.tolist() == [half - 1] * rows
        token, p = _draw(x, one, None, torch.full((rows,), 0.5), None, one)
        assert token.tolist() == [(vocab + 1) // 2 - 1] * rows  # those before which less than half stands
        token, p = _draw(x, one, None, None, one, u)
        assert token.tolist() == at


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [257, 40000, 140000])
def test_values_that_repeat(vocab, dtype):
    """A handful of values, entries of each all over the row."""
    g = torch.Generator().manual_seed(vocab)
    rows = 12
    x = torch.tensor([3.0, 2.5, 2.5, 0.0, -0.0, -1.0, -30.0]).to(dtype)[torch.randint(0, 7, (rows, vocab), generator=g)]
    _check(x, *_settings(rows, 3))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [66, 3000, 66000])
def test_masked_logits(vocab, dtype):
    """-infinity, the lowest value of the type and NaN have no part; a row of them has no token; +infinity has all."""
    g = torch.Generator().manual_seed(vocab)
    rows = 14
    x = (torch.randn((rows, vocab), generator=g) * 2).to(dtype)
    hidden = torch.rand((rows, vocab), generator=g) < 0.97
    hidden[:, vocab // 3] = False
    lowest = torch.finfo(dtype).min
    for r, v in enumerate([-math.inf, -math.inf, math.nan, lowest, lowest, -math.inf]):
        x[r] = torch.where(hidden[r], torch.tensor(v, dtype=dtype), x[r])
    x[6] = -math.inf
    x[7] = math.nan
    x[8] = lowest
    x[9, vocab // 2] = math.inf
    x[10, [3, 50, vocab - 1]] = math.inf
    x[11] = -math.inf
    x[11, vocab - 1] = -2.0
    x[12] = -math.inf
    x[12, [0, 1]] = math.nan
    x[13, 7:] = -math.inf
    T, k, p, m, u = _settings(rows, 9)
    T = torch.where(T > 0, T, 1.0)
    token, prob = _check(x, T, k, p, m, u)
    assert token[[6, 7, 12]].tolist() == [-1] * 3 and prob[[6, 7, 12]].tolist() == [0.0] * 3
    assert token[9] == vocab // 2 and token[10] in (3, 50, vocab - 1) and token[11] == vocab - 1
    token, prob = _check(x, torch.zeros(rows), k, p, m, u)  # greedy
    assert token[[6, 7, 12]].tolist() == [-1] * 3 and token[10] == 3


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("counts", [{1.5: 65535}, {1.5: 65536}, {1.5: 65537}, {-1.5: 65536}, {1.5: 65536, -1.5: 65536}, {1.5: 131072, -1.5: 70000}, {0.0: 65536, -0.0: 65536},
                                    {float("nan"): 65536, 2.0: 10}, {-float("inf"): 140000, 0.5: 66000}, {-3.0: 196608}], ids=str)
def test_values_that_fill_a_long_row(counts, dtype):
    # not side by side: in front, behind and shuffled with others, what a counter of 16 bits holds and more
    g = torch.Generator().manual_seed(11)
    filling = torch.cat([torch.full((n,), v) for v, n in counts.items()])
    others = torch.randn(20000, generator=g)
    every = torch.cat([filling, others])
    x = torch.stack([every, every.flip(0), every[torch.randperm(every.shape[0], generator=g)], every[torch.randperm(every.shape[0], generator=g)]]).to(dtype)
    u = torch.rand(4, generator=g)
    _check(x, torch.tensor([1.0, 0.7, 2.0, 1.0]), None, None, None, u, what=counts)
    _check(x, torch.tensor([1.0, 0.7, 2.0, 50.0]), torch.tensor([1000, 65536, 70000, 65540], dtype=torch.int32), torch.tensor([1.0, 0.9, 0.5, 0.99]), None, u, what=counts)


@pytest.mark.parametrize("vocab", [100, 70000])
def test_odd_settings(vocab):
    """Numbers outside their ranges mean what the header says."""
    g = torch.Generator().manual_seed(1)
    x = (torch.randn((10, vocab), generator=g) * 3).half()
    T = torch.tensor([-1.0, math.nan, math.inf, 1e-30, 1e30, 1.0, 1.0, 1.0, 1.0, 1.0])
    k = torch.tensor([0, 0, 0, 0, 0, -5, 2 ** 31 - 1, 0, 0, 0], dtype=torch.int32)
    p = torch.tensor([1.0, 1.0, 1.0, 1.0, 1.0, math.nan, 2.0, -3.0, 1e-20, 1.0])
    m = torch.tensor([0.0] * 5 + [-1.0, math.nan, 0.0, 0.0, math.inf])
    u = torch.tensor([0.3, 0.3, 0.3, 0.3, 0.3, 0.9, 1.0, 0.5, 0.5, 0.7])
    token, prob = _check(x, T, k, torch.nan_to_num(p, nan=1.0), torch.nan_to_num(m, nan=0.0, posinf=5.0), u)
    again, _ = _draw(x, T, k, p, m, u)
    assert torch.equal(token, again)
    best = x.float().argmax(1)
    assert token[[0, 1, 3, 7, 8, 9]].tolist() == best[[0, 1, 3, 7, 8, 9]].tolist()
    for bad, same in ((math.nan, 0.0), (-2.0, 0.0), (7.0, 1.0), (math.inf, 1.0), (-math.inf, 0.0)):
        a = _draw(x, torch.ones(10), None, None, None, torch.full((10,), bad))[0]
        b = _draw(x, torch.ones(10), None, None, None, torch.full((10,), same))[0]
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [1001, 66003])
@pytest.mark.parametrize("offset,more", [(0, 1), (1, 0), (3, 5), (7, 8), (8, 24)])
def test_rows_that_begin_anywhere(vocab, offset, more, dtype):
    """Any stride and any first element; what stands between the rows has no part."""
    rows = 5
    g = torch.Generator().manual_seed(vocab)
    whole = torch.full((rows * (vocab + more) + offset + 16,), math.inf, dtype=dtype)
    view = whole[offset:offset + rows * (vocab + more)].view(rows, vocab + more)
    view[:, :vocab] = (torch.randn((rows, vocab), generator=g) * 2).to(dtype)
    x = whole.cuda()[offset:offset + rows * (vocab + more)].view(rows, vocab + more)[:, :vocab]
    s = _settings(rows, 21)
    token, p = _draw(x, *s)
    assert assert_drawn(token, p, x.cpu(), *s) == 0


@pytest.mark.parametrize("rows,vocab", [(700, 66000), (1500, 40)])
def test_many_rows(rows, vocab):
    """More than the chip has compute units; each row is as it is alone."""
    g = torch.Generator(device="cuda").manual_seed(3)
    x = (torch.randn((rows, vocab), generator=g, device="cuda") * 2).bfloat16()
    s = _settings(rows, 4)
    token, p = _draw(x, *s)
    pick = list(range(0, rows, 61)) + [rows - 1]
    assert assert_drawn(token[pick], p[pick], x[pick].cpu(), *(t[pick] for t in s)) == 0
    one, q = _draw(x[-1:], *(t[-1:] for t in s))
    assert int(one) == int(token[-1]) and float(q) == float(p[-1])


def test_results_that_are_given():
    x = torch.randn((4, 100), device="cuda").half()
    out = torch.full((4,), -7, dtype=torch.int32, device="cuda"), torch.zeros(4, device="cuda")
    sampler = bcq.Sampler(torch.ones(4, device="cuda"))
    got = sampler.draw(x, torch.rand(4, device="cuda"), out=out)
    assert got[0].data_ptr() == out[0].data_ptr() and got[1].data_ptr() == out[1].data_ptr() and int(out[0].min()) >= 0
    none = bcq.Sampler(torch.ones(0, device="cuda")).draw(x[:0], torch.rand(0, device="cuda"))
    assert none[0].shape == (0,)


def test_another_stream_and_a_graph():
    """Captured with settings, logits and numbers that change between replays, eager work in between; two graphs share no workspace."""
    rows, vocab = 6, 70000
    g = torch.Generator(device="cuda").manual_seed(8)
    xs = [(torch.randn((rows, vocab), generator=g, device="cuda") * 2).half() for _ in range(4)]
    us = [torch.rand(rows, generator=g, device="cuda") for _ in range(4)]
    T = torch.linspace(0.0, 1.2, rows, device="cuda")
    sampler = bcq.Sampler(T, None, torch.full((rows,), 0.9, device="cuda"))
    eager = [tuple(t.cpu() for t in sampler.draw(x, u)) for x, u in zip(xs, us)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = sampler.draw(xs[1], us[1])
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got[0].cpu(), eager[1][0])
    places = [(xs[0].clone(), us[0].clone()) for _ in range(2)]
    graphs, outs = [], []
    for x, u in places:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(sampler.draw(x, u))
        graphs.append(graph)
    for i in (1, 2, 3, 1):
        for (x, u), j in zip(places, (i, (i + 1) % 4)):
            x.copy_(xs[j])
            u.copy_(us[j])
        graphs[0].replay()
        graphs[1].replay()
        sampler.draw(xs[0], us[0])
        torch.cuda.synchronize()
        for out, j in zip(outs, (i, (i + 1) % 4)):
            assert torch.equal(out[0].cpu(), eager[j][0]) and torch.equal(out[1].cpu(), eager[j][1])


def test_shares_of_many_draws():
    """Tokens come as often as their weights say: 20000 rows of one distribution, numbers spread evenly."""
    n, vocab = 20000, 50
    x = torch.linspace(-2, 2, vocab).half().expand(n, vocab).contiguous().cuda()
    u = (torch.arange(n, device="cuda") + 0.5) / n
    token, _ = bcq.Sampler(torch.ones(n, device="cuda")).draw(x, u)
    share = torch.bincount(token.long(), minlength=vocab).double().cpu() / n
    expected = torch.softmax(x[0].double().cpu(), 0)
    assert float((share - expected).abs().max()) <= 1.5 / n  # (the numbers of an interval of the u's are its length, up to one at each end)


def test_refusals():
    """Shapes, types and places that do not fit are refused before anything runs."""
    T, x, u = torch.ones(3, device="cuda"), torch.zeros((3, 10), device="cuda").half(), torch.rand(3, device="cuda")
    ok = bcq.Sampler(T)
    for build in (lambda: bcq.Sampler(T, T), lambda: bcq.Sampler(T, None, T[:2]), lambda: bcq.Sampler(T, None, None, T.cpu()), lambda: bcq.Sampler(T.repeat(2)[::2])):
        with pytest.raises(bcq.BcqError):
            build()
    for call in (lambda: ok.draw(x.float(), u), lambda: ok.draw(x[:2], u), lambda: ok.draw(x, u[:2]), lambda: ok.draw(x, u.double()), lambda: ok.draw(x, None),
                 lambda: ok.draw(x.cpu(), u), lambda: ok.draw(x, u.cpu()), lambda: ok.draw(x[0], u), lambda: ok.draw(x.t().contiguous().t(), u),
                 lambda: ok.draw(x, u, out=(u, u)), lambda: ok.draw(x, u, out=u), lambda: ok.draw(x[:, :0], u)):
        with pytest.raises(bcq.BcqError):
            call()
