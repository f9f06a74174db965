"""GPU tests of sampling: the tokens of rows of logits, equal to those of sorted rows in 64 bits."""
import math

import pytest
import torch

from tests.step_util import BF16, FP32, plain_sample

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def binding():
    from paper_2506_16640_amd import binding as b
    return b


def _gpu(kw):
    return {k: None if v is None else v.cuda() for k, v in kw.items()}


def _check(binding, logits, u, label="", strided=None, **kw):
    """Tokens are equal; a logarithm of a probability is rounded once (2^-24 of it), the quotient's error is far below."""
    want, want_lp = plain_sample(logits, u, **kw)
    lp = torch.full((logits.shape[0],), 7.0, device="cuda")
    x = logits.cuda() if strided is None else strided
    got = binding.sample(x, u.cuda(), logprob=lp, **_gpu(kw))
    torch.cuda.synchronize()
    bad = (got.cpu() != want).nonzero()[:, 0].tolist()
    assert not bad, (label, [(r, int(got[r]), int(want[r])) for r in bad[:5]])
    there = want >= 0
    assert (lp.cpu()[~there] == -math.inf).all(), label
    off = (lp.double().cpu() - want_lp).abs()[there]
    assert (off <= 2.0 ** -24 * want_lp.abs()[there] + 1e-9).all(), (label, off.max().item())


def _rows(R, V, dtype=BF16, spread=2.0, seed=0):
    g = torch.Generator().manual_seed(seed)
    return (spread * torch.randn(R, V, generator=g)).to(dtype), torch.rand(R, generator=g)


def _asks(R, seed=0):
    g = torch.Generator().manual_seed(seed + 100)
    pick = lambda v, t: torch.tensor(v)[torch.randint(len(v), (R,), generator=g)].to(t)  # noqa: E731
    return dict(temperature=pick([0.0, 0.05, 0.3, 0.7, 1.0, 1.5, 5.0], FP32), top_k=pick([0, -3, 1, 2, 20, 50, 400, 10 ** 9], torch.int32),
                top_p=pick([1.0, 1.5, 0.1, 0.5, 0.9, 0.99, 0.0, -1.0], FP32), min_p=pick([0.0, -1.0, 0.01, 0.05, 0.3, 1.0, 2.0], FP32))


VOCABS = [1, 2, 7, 63, 64, 65, 1000, 1023, 8191, 8192, 8193, 20011, 40000]


@pytest.mark.parametrize("V", VOCABS)
@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_plain(binding, V, dtype):
    x, u = _rows(12, V, dtype, seed=V)
    _check(binding, x, u, "plain")


@pytest.mark.parametrize("V", VOCABS)
@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("spread", [0.3, 3.0])
def test_mixed(binding, V, dtype, spread):
    R = 60 if V < 10000 else 24
    x, u = _rows(R, V, dtype, spread, seed=V + 1)
    _check(binding, x, u, "mixed", **_asks(R, V))


@pytest.mark.parametrize("which", ["temperature", "top_k", "top_p", "min_p"])
@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_one_filter(binding, which, dtype):
    x, u = _rows(40, 30011, dtype, seed=5)
    _check(binding, x, u, which, **{which: _asks(40, 3)[which]})


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_many_rows_large_slices(binding, dtype):
    """Enough logits that slices are the large ones."""
    x, u = _rows(40, 33000, dtype, seed=6)
    _check(binding, x, u, "large", **_asks(40, 4))


@pytest.mark.parametrize("p", [0.3, 0.9, 0.999, 1.0 - 2.0 ** -24])
@pytest.mark.parametrize("spread", [0.05, 0.7, 8.0])
def test_top_p_that_keeps_much(binding, p, spread):
    """Longer lists of tokens next to the cut than a workgroup holds."""
    x, u = _rows(6, 60000, FP32, spread, seed=7)
    _check(binding, x, u, "flat", top_p=torch.full((6,), p))
    _check(binding, x, u, "flat, hot", top_p=torch.full((6,), p), temperature=torch.tensor([0.5, 1.0, 3.0, 50.0, 1e10, math.inf]))


@pytest.mark.parametrize("k", [1, 2, 5000, 29999, 30000, 30001])
def test_top_k_that_keeps_much(binding, k):
    x, u = _rows(6, 30000, BF16, 2.0, seed=8)
    _check(binding, x, u, "many", top_k=torch.full((6,), k, dtype=torch.int32), top_p=torch.tensor([1.0, 0.99, 0.9, 0.5, 0.999, 1.0]))


@pytest.mark.parametrize("V", [16, 1000, 20000])
@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_equal_logits(binding, V, dtype):
    """All equal, or of few values: of equal ones the first are kept, and sums are whole numbers that meet borders exactly."""
    for values in (1, 2, 5):
        g = torch.Generator().manual_seed(values)
        x = torch.randint(values, (10, V), generator=g).to(dtype) - 1.0
        u = torch.tensor([0.0, 0.25, 0.5, 0.75, 1.0 - 2.0 ** -24, 0.125, 0.3, 0.9, 0.0, 0.5])
        p = torch.tensor([0.5, 0.25, 0.75, 0.5, 0.125, 0.9, 0.1, 0.5, 1.0, 2.0 ** -20])
        _check(binding, x, u, "equal")
        _check(binding, x, u, "equal, top-p", top_p=p)
        _check(binding, x, u, "equal, top-k", top_k=torch.tensor([1, 2, 3, V // 2, V - 1, V, 7, 8, 9, 10], dtype=torch.int32))
        _check(binding, x, u, "equal, both", top_p=p, top_k=torch.tensor([1, 2, 3, V // 2, V - 1, V, 7, 8, 9, 10], dtype=torch.int32))


def test_zeros_of_both_signs_are_equal(binding):
    x = torch.tensor([[-0.0, 0.0, -0.0, 0.0], [0.0, -0.0, 0.0, -1.0]])
    u = torch.tensor([0.0, 0.0])
    _check(binding, x, u, "zeros", temperature=torch.zeros(2))
    _check(binding, x, u, "zeros", top_k=torch.ones(2, dtype=torch.int32))
    _check(binding, x.bfloat16(), torch.tensor([0.9, 0.9]), "zeros", top_k=torch.tensor([2, 2], dtype=torch.int32))


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_values_that_are_not_finite(binding, dtype):
    V = 9000
    x, _ = _rows(12, V, dtype, seed=9)
    inf, nan = math.inf, math.nan
    low = torch.finfo(dtype).min
    x[0] = -inf
    x[1] = nan
    x[2, ::2] = nan
    x[3, ::3] = -inf
    x[4], x[4, 77] = -inf, -3.0
    x[5, [5, 600, 8999]] = inf
    x[6] = inf
    x[7], x[7, :10] = low, 1.0
    x[8] = low
    x[9], x[9, 8000:] = nan, low
    x[10, :8500] = -inf
    x[11], x[11, 0], x[11, 1] = -inf, inf, nan
    for u in (0.0, 0.4, 1.0 - 2.0 ** -24):
        uu = torch.full((12,), u)
        _check(binding, x, uu, "not finite")
        _check(binding, x, uu, "not finite, greedy", temperature=torch.zeros(12))
        for ask in (dict(top_k=torch.full((12,), 4, dtype=torch.int32)), dict(top_p=torch.full((12,), 0.7)), dict(min_p=torch.full((12,), 0.1)),
                    dict(top_k=torch.full((12,), 4000, dtype=torch.int32), top_p=torch.full((12,), 0.7), min_p=torch.full((12,), 0.1),
                         temperature=torch.full((12,), 0.7))):
            _check(binding, x, uu, str(sorted(ask)), **ask)


def test_parameters_and_numbers_out_of_range(binding):
    x, _ = _rows(8, 500, FP32, seed=10)
    nan, inf = math.nan, math.inf
    _check(binding, x, torch.tensor([-1.0, 0.0, 1.0, 2.0, inf, -inf, nan, 0.5]), "uniform")
    u = torch.rand(8, generator=torch.Generator().manual_seed(1))
    want, _ = plain_sample(x, u)
    best, _ = plain_sample(x, u, temperature=torch.zeros(8))
    for t in (-1.0, nan, -inf):
        assert torch.equal(binding.sample(x.cuda(), u.cuda(), temperature=torch.full((8,), t).cuda()).cpu(), best)
    for kw in (dict(top_p=torch.full((8,), nan)), dict(min_p=torch.full((8,), nan)), dict(min_p=torch.full((8,), -inf)), dict(top_p=torch.full((8,), inf)),
               dict(top_k=torch.full((8,), -2 ** 31, dtype=torch.int32))):
        assert torch.equal(binding.sample(x.cuda(), u.cuda(), **_gpu(kw)).cpu(), want)
    _check(binding, x, u, "tiny temperature", temperature=torch.full((8,), 1e-40))
    _check(binding, 1e30 * x, u, "huge logits", top_p=torch.full((8,), 0.9), temperature=torch.full((8,), 3e29))
    _check(binding, 1e-30 * x, u, "tiny logits", top_p=torch.full((8,), 0.9), temperature=torch.full((8,), 3e-31))


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("V,stride,first", [(1001, 1001, 0), (1001, 1003, 1), (8192, 8197, 3), (16384, 16385, 5), (50, 77, 7)])
def test_rows_that_begin_anywhere(binding, dtype, V, stride, first):
    """Rows whose addresses are round for no load; what lies between them is not looked at."""
    R = 9
    x, u = _rows(R, V, dtype, seed=V)
    room = torch.full((first + R * stride + 9,), math.inf, dtype=dtype)
    view = room[first:first + R * stride].view(R, stride)[:, :V]
    view.copy_(x)
    dev = room.cuda()[first:first + R * stride].view(R, stride)[:, :V]
    _check(binding, x, u, "strided", strided=dev, **_asks(R, 9))


def test_every_token_can_be_drawn(binding):
    """The random number in the middle of each token's share of the sum: the token itself."""
    g = torch.Generator().manual_seed(2)
    x = torch.randn(1, 3000, generator=g)
    w = (x[0].double() - x.max().double()).exp()
    mid = (w.cumsum(0) - w / 2) / w.sum()
    u = mid.float()
    # (a share is some 1e-4 wide or less; a number rounded to 24 bits still lies in it)
    inside = ((u.double() - mid).abs() < w / w.sum() / 4).nonzero()[:, 0]
    assert len(inside) > 2500
    got = binding.sample(x.expand(3000, 3000).contiguous().cuda(), u.cuda()).cpu()
    assert torch.equal(got[inside], inside.int())


def test_replay_and_workspace(binding):
    """A captured call: other logits, numbers and parameters on every replay; the workspace's contents do not matter; the same call gives the same tokens."""
    R, V = 20, 30000
    dev = "cuda"
    logits, u = torch.zeros(R, V, dtype=BF16, device=dev), torch.zeros(R, device=dev)
    ask = {k: v.to(dev) for k, v in _asks(R, 1).items()}
    token, lp, ws = torch.zeros(R, dtype=torch.int32, device=dev), torch.zeros(R, device=dev), binding.new_sample_workspace(logits)
    call = lambda: binding.sample(logits, u, token=token, logprob=lp, workspace=ws, **ask)  # noqa: E731
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for i in range(4):
        x, un = _rows(R, V, BF16, 1.0 + i, seed=i)
        a = _asks(R, i)
        logits.copy_(x)
        u.copy_(un)
        for k in ask:
            ask[k].copy_(a[k])
        ws.fill_(255 if i % 2 else 0)
        graph.replay()
        torch.cuda.synchronize()
        want, _ = plain_sample(x, un, **a)
        assert torch.equal(token.cpu(), want)
        first = lp.clone()
        ws.fill_(17)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(token.cpu(), want) and torch.equal(first, lp)


def test_no_rows(binding):
    assert binding.sample(torch.zeros(0, 10, device="cuda"), torch.zeros(0, device="cuda")).shape == (0,)


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_rows_far_apart(binding, dtype):
    """Rows whose offsets need more than 32 bits."""
    gen = torch.Generator().manual_seed(21)
    x = (2 * torch.randn(3, 20000, generator=gen)).to(dtype)
    u, p = torch.rand(3, generator=gen).cuda(), torch.full((3,), 0.9).cuda()
    stride = (1 << 31) // x.element_size() + 8
    far = torch.empty(2 * stride + 20000, dtype=dtype, device="cuda").as_strided((3, 20000), (stride, 1))
    far.copy_(x)
    assert torch.equal(binding.sample(far, u, None, None, p), binding.sample(x.cuda(), u, None, None, p))
