"""GPU tests of sampling at the ends of its arguments' ranges; all of them run on the CPU first (test_sample_emulated.py)."""
import math

import pytest
import torch

from tests.step_util import BF16, FP32
from tests.test_gpu_sample import _check, binding  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("V", [300, 8192, 40001])
def test_selections_of_several_rounds(binding, dtype, V):  # noqa: F811
    """Lists of equal logits, whose selection goes over its bins more than once."""
    g = torch.Generator().manual_seed(V)
    x = torch.randint(3, (40, V), generator=g).to(dtype)
    x[0] = 1.0
    u, p = torch.rand(40, generator=g), torch.rand(40, generator=g)
    k = torch.randint(1, V, (40,), generator=g).to(torch.int32)
    _check(binding, x, u, "top-p", top_p=p)
    _check(binding, x, u, "both", top_p=p, top_k=k)


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("V", [100, 9001, 40001])
def test_min_p_at_very_high_temperatures(binding, dtype, V):  # noqa: F811
    g = torch.Generator().manual_seed(V)
    x, u = (3 * torch.randn(12, V, generator=g)).to(dtype), torch.rand(12, generator=g)
    t = torch.tensor([1e30, 3e35, 3e36, 1e38, 3e38, math.inf] * 2)
    k = torch.randint(1, V, (12,), generator=g).to(torch.int32)
    for f in (1e-30, 0.2, 1.0):
        _check(binding, x, u, "min-p", temperature=t, min_p=torch.full((12,), f))
        _check(binding, x, u, "min-p and top-k", temperature=t, min_p=torch.full((12,), f), top_k=k)
        _check(binding, x, u, "min-p and top-p", temperature=t, min_p=torch.full((12,), f), top_p=torch.full((12,), 0.7))


@pytest.mark.parametrize("V", [300, 20001])
def test_lowest_logits_at_very_high_temperatures(binding, V):  # noqa: F811
    """The lowest finite number is in the bin of the cut: the bin's tokens begin with it."""
    x = torch.randn(12, V, generator=torch.Generator().manual_seed(6))
    x[:, V // 3:] = torch.finfo(FP32).min
    u = torch.linspace(0.01, 0.99, 12)
    for t in (1e38, 2e38, 3e38):
        _check(binding, x, u, "low", temperature=torch.full((12,), t), top_p=torch.tensor([0.9, 0.95, 0.99, 0.999] * 3))
        _check(binding, x, u, "low, top-k", temperature=torch.full((12,), t), top_k=torch.full((12,), V - 50, dtype=torch.int32))


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_random_number_zero(binding, dtype):  # noqa: F811
    """The first token with any probability, however small: those that are 2^-1074 of the largest as well."""
    u = torch.tensor([0.0, 1.0])
    x = torch.full((2, 20000), -800.0)
    x[:, 12000] = 0.0
    for at in (-500.0, -744.0, -744.4, -744.9) if dtype == FP32 else (-500.0, -744.0):
        x[:, 300:900] = at - (1.0 if dtype == FP32 else 4.0)
        x[:, 5000:5300] = at
        x[0, 15000:15600] = at - 4.0
        _check(binding, x.to(dtype), u, "plain %g" % at)
        _check(binding, x.to(dtype), u, "min-p %g" % at, min_p=torch.full((2,), 1e-38))
    x = torch.randn(2, 9000, generator=torch.Generator().manual_seed(7)).to(dtype)
    k = torch.tensor([5, 700], dtype=torch.int32)
    _check(binding, x, u, "top-k", temperature=torch.full((2,), 0.01), top_k=k)
    _check(binding, x, u, "top-k and top-p", temperature=torch.full((2,), 0.01), top_k=k, top_p=torch.tensor([0.9999, 1.0]))


def test_tiny_logits_at_very_high_temperatures(binding):  # noqa: F811
    """Logits times the bins' grid that no float holds: negative ones stay below zero's bin."""
    g = torch.Generator().manual_seed(3)
    u = torch.tensor([0.0, 0.3, 0.7, 0.98])
    for scale, t in ((1e-30, 1e20), (1e-30, 3e38), (1e-38, 1e30), (1.0, 3e38), (1e-44, math.inf), (1.0, math.inf)):
        for V in (700, 9001):
            x, T = scale * torch.randn(4, V, generator=g), torch.full((4,), t)
            x[0, ::7] = 0.0
            x[1, ::9] = -0.0
            _check(binding, x, u, "top-p %g" % scale, temperature=T, top_p=torch.tensor([0.9, 0.99, 1e-30, 0.3]))
            _check(binding, x, u, "top-k %g" % scale, temperature=T, top_k=torch.tensor([3, 400, 20, 699], dtype=torch.int32))
            _check(binding, -x.abs(), u, "negative %g" % scale, temperature=T, top_p=torch.tensor([0.9, 0.99, 1e-30, 0.3]))


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("V", [3, 9001, 40001])
def test_lowest_logits_at_very_low_temperatures(binding, dtype, V):  # noqa: F811
    """Masks of the lowest finite number: exponents that are far beyond the whole numbers of 64-bit floats."""
    g = torch.Generator().manual_seed(V)
    x, u = (3 * torch.randn(12, V, generator=g)).to(dtype), torch.rand(12, generator=g)
    u[0], u[1] = 0.0, 1.0
    x[:, ::2] = torch.finfo(dtype).min
    x[6:, :V - 3] = torch.finfo(dtype).min
    for t in (1e-6, 1e-12, 1e-13, 1e-20, 1e-38, 1e-40, 1e-45):
        t = torch.full((12,), t)
        _check(binding, x, u, "plain", temperature=t)
        _check(binding, x, u, "top-p", temperature=t, top_p=torch.tensor([0.5, 0.9, 0.0] * 4))
        _check(binding, x, u, "top-k, min-p", temperature=t, min_p=torch.tensor([0.0, 0.1, 1.0] * 4), top_k=torch.tensor([5, 0, 4000, 1] * 3, dtype=torch.int32))
