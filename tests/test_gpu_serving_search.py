"""GPU tests of the serving attention's thresholds: general alpha up to 2, scores far from zero, scores far apart."""
import pytest
import torch

from tests.serving_util import BF16, FP32, Problem

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def binding():
    from paper_2506_16640_amd import binding as b
    return b


def _within(p, got, ref, tol, label):
    half = torch.finfo(p.dtype).eps / 2
    err = (got.double().cpu() - ref).abs()
    assert torch.isfinite(got[p.owned().cuda()]).all(), label
    excess = (err - half * ref.abs() - tol)[p.owned()].max().item()
    print(label, "largest error", err[p.owned()].max().item())
    assert excess <= 0.0, (label, "beyond the bound by", excess)


@pytest.mark.parametrize("scale", ["head", "dense", "none"])
@pytest.mark.parametrize("dtype", [FP32, BF16])
@pytest.mark.parametrize("alpha", [1.7, 1.8, 1.9, 1.95, 1.99, 2.0])
def test_alphas_up_to_two(binding, alpha, dtype, scale):
    packed = Problem([(500, 500), (130, 130), (70, 70)], Hq=6, Hkv=3, paged=False, alpha=alpha, dtype=dtype, scale=scale, seed=41)
    paged = Problem([(150, 600), (3, 900), (1, 333)], Hq=4, Hkv=2, alpha=alpha, dtype=dtype, scale=scale, seed=42)
    for p in (packed, paged):
        ref, tol = p.reference()
        for path in (1, 0):
            _within(p, p.run(binding, path=path), ref, tol, "alpha %g %s path %d" % (alpha, scale, path))


@pytest.mark.parametrize("dtype", [FP32, BF16])
@pytest.mark.parametrize("alpha", [1.25, 1.5, 1.7, 1.9, 2.0])
@pytest.mark.parametrize("paged", [True, False])
def test_scores_far_from_zero(binding, paged, alpha, dtype):
    """Products that 32 bits hold exactly, all of them 32768 off: entmax does not change with that, and the result must not lose bits to it.  The
    bound is that of the same problem without the offset (whose scores are as exact)."""
    lens = [(1, 700), (5, 300), (140, 500), (300, 300)] if paged else [(300, 300), (1, 1), (140, 140)]
    p = Problem(lens, dtype=dtype, paged=paged, alpha=alpha, scale="none", seed=43)
    g = torch.Generator().manual_seed(44)
    ints = lambda t: torch.randint(-3, 4, t.shape, generator=g).to(dtype)  # noqa: E731
    keys = p.kc if paged else p.kp
    p.q.copy_(ints(p.q)), keys.copy_(ints(keys))
    p.q[..., 0], keys[..., 0] = 64.0, 0.0
    ref, tol = p.reference()
    keys[..., 0] = 512.0
    for path in (1, 0):
        _within(p, p.run(binding, path=path), ref, tol, "32768 off, alpha %g path %d" % (alpha, path))


@pytest.mark.parametrize("dtype", [FP32, BF16])
@pytest.mark.parametrize("alpha", [1.25, 1.5, 1.7, 2.0])
@pytest.mark.parametrize("paged", [True, False])
def test_scores_far_apart(binding, paged, alpha, dtype):
    """Scores of up to 2^28, 2^20 apart: the largest key alone counts, wholly."""
    lens = [(1, 240), (5, 200), (140, 250), (200, 200)] if paged else [(250, 250), (1, 1), (140, 140)]
    p = Problem(lens, dtype=dtype, paged=paged, alpha=alpha, scale="none", seed=45)
    keys = p.kc if paged else p.kp
    p.q.zero_(), keys.zero_()
    p.q[..., 0] = 2.0 ** 20
    value = lambda j: ((j * 37) % 251).to(dtype)  # noqa: E731  (exact, different for all keys of a sequence)
    ref = torch.zeros(p.T, p.Hq, p.D, dtype=torch.float64)
    for s, (n, L) in enumerate(lens):
        j = torch.arange(L)
        if paged:
            p.kc[p.table[s][j // p.page].long(), :, j % p.page, 0] = value(j)[:, None]
        else:
            p.kp[p.cu[s]:p.cu[s + 1], :, 0] = value(j)[:, None]
        v = p.keys(s)[1].double()
        for t in range(n):
            top = int(value(j[:L - n + t + 1]).double().argmax())
            ref[p.cu[s] + t] = v[:, top].repeat_interleave(p.Hq // p.Hkv, 0)
    for path in (1, 0):
        # (a probability of 1 to a few steps of 2^-24)
        _within(p, p.run(binding, path=path), ref, 2.0 ** -20 * ref.abs(), "far apart, alpha %g path %d" % (alpha, path))
