"""GPU tests of the softmax attention's cap: large caps leave the scores nearly as they are."""
import math

import pytest
import torch

from tests.serving_util import BF16, FP32, Problem
from tests.step_util import softmax_reference
from tests.test_gpu_softmax import TYPES, _run, _within, binding  # noqa: F401

pytestmark = pytest.mark.gpu

LENS = [(1, 700), (3, 900), (9, 300), (150, 400)]  # 16-row tiles, 32-row tiles, prompts


def _bounds(p, cap):
    """The plain form, and bounds without those of step_util.py that grow with the cap: a capped score is off by at most 2^-19 of the uncapped one's products.  Below a
    quarter of the cap the series tanh takes five terms (the sixth is 1e-8 of it) of numbers rounded some ten times, 2^-21 of it; above, 1 - 2 / (1 + exp(2 x)) is off by at
    most 2^-21 of the cap (see step_util.py), and the score is at least tanh(1/4) > 2^-2.04 of that.  As there, an output moves by at most 4 e max |v|, lse by e."""
    ref, ref_l, _, _ = softmax_reference(p, cap)
    _, _, tol, tol_l = softmax_reference(p)
    k = max(float(x) for s in range(len(p.lens)) for x in [p.keys(s)[0].double().abs().amax()])
    most = float(p.q.double().abs().sum(-1).amax()) * k / math.sqrt(p.D)  # (of all rows: more than any sum of products)
    return ref, ref_l, tol + 4 * most * 2.0 ** -19 * p.vc.double().abs().max(), tol_l + most * 2.0 ** -19


@pytest.mark.parametrize("D,dtype", TYPES)
@pytest.mark.parametrize("cap", [50.0, 1e4, 1e6, 1e9, 3e38])
def test_large_caps(binding, D, dtype, cap):  # noqa: F811
    p = Problem(LENS, D=D, dtype=dtype, seed=41, scale="none")
    ref, ref_l, tol, tol_l = _bounds(p, cap)
    lse = torch.zeros(p.Hq, p.T, device="cuda")
    got = _run(binding, p, cap, lse=lse).double().cpu()
    assert torch.isfinite(got).all()
    off = (got - ref).abs() - torch.finfo(dtype).eps / 2 * ref.abs() - tol
    print("beyond the bound by", off.max().item(), "lse", (lse.double().cpu() - ref_l).abs().max().item())
    assert _within(got, ref, tol, dtype)
    assert bool(((lse.double().cpu() - ref_l).abs() <= tol_l).all())


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("bias_mode", [0, 1])
def test_a_cap_beyond_all_scores_is_none(binding, dtype, bias_mode):  # noqa: F811
    """cap 1e9: s / cap is 1e-8 and less, tanh is its argument: within the bounds of the call without a cap."""
    p = Problem(LENS, dtype=dtype, seed=42, slopes=True, bias_mode=bias_mode)
    ref, _, tol, _ = softmax_reference(p)
    assert _within(_run(binding, p, 1e9).double().cpu(), ref, tol, dtype)


@pytest.mark.parametrize("D,dtype", TYPES)
@pytest.mark.parametrize("cap", [1e-3, 1e-38, 1e-44])
def test_tiny_caps(binding, D, dtype, cap):  # noqa: F811
    """Scores of at most 1e-3 in size, also where the queries are zero: the mean of the values, to 2e-3 of the largest."""
    p = Problem(LENS, D=D, dtype=dtype, seed=43, scale="none")
    p.q[::2] = 0.0
    ref, _, tol, _ = softmax_reference(p, cap)
    assert _within(_run(binding, p, cap).double().cpu(), ref, tol, dtype)
