"""Sampling with its kernels run on the CPU, lane by lane, and a workgroup's waves in the orders that depend most on its barriers (tests/emulate)."""
import ctypes
import math
import os
import subprocess

import pytest
import torch

from tests.step_util import BF16, FP32, plain_sample
from tests.test_sanitize_host import ROOT

UNWRITTEN = -12345


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("emulate") / "sample_emulated.so")
    here = os.path.join(ROOT, "tests", "emulate")
    clang = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "llvm", "bin", "clang++")
    subprocess.run([clang, "-x", "c++", "-std=c++17", "-O1", "-fPIC", "-shared", "-w", "-I", here, "-I", os.path.join(ROOT, "include"), "-I",
                    os.path.join(ROOT, "paper_2506_16640_amd", "csrc"), os.path.join(here, "sample_emulated.cc"), "-o", out], check=True)
    lib = ctypes.CDLL(out)
    lib.entmax_sample.argtypes = [ctypes.c_char_p] + [ctypes.c_void_p] * 9 + [ctypes.c_size_t, ctypes.c_void_p]
    lib.entmax_sample_workspace_bytes.restype = ctypes.c_size_t
    lib.emulate_end.restype = ctypes.c_char_p
    return lib


def sample(lib, logits, u, order, temperature=None, top_k=None, top_p=None, min_p=None):
    from paper_2506_16640_amd import binding
    R, V = logits.shape
    p = binding._sample_bytes.pack(R, V, 0 if logits.dtype == BF16 else 1, V)
    token, logprob = torch.full((R,), UNWRITTEN, dtype=torch.int32), torch.full((R,), float(UNWRITTEN))
    # (a place that a read in front of or behind the workspace meets holds NaN)
    need = int(lib.entmax_sample_workspace_bytes(p))
    room = torch.full((need + (2 << 20),), 255, dtype=torch.uint8)
    at = (room.data_ptr() + (1 << 20) + 255) // 256 * 256
    lib.emulate_begin(order)
    rc = lib.entmax_sample(p, logits.data_ptr(), u.data_ptr(), *[None if t is None else t.data_ptr() for t in (temperature, top_k, top_p, min_p)],
                           token.data_ptr(), logprob.data_ptr(), at, need, None)
    assert rc == 0
    error = lib.emulate_end().decode()
    assert not error, error
    return token, logprob


def check(lib, logits, u, label="", orders=(0, 1, 2), **kw):
    want, want_lp = plain_sample(logits, u, **kw)
    for order in orders:
        token, logprob = sample(lib, logits, u, order, **kw)
        assert torch.equal(token, want), (label, order, token.tolist(), want.tolist())
        there = want >= 0
        assert (logprob[~there] == -math.inf).all()
        off = (logprob.double() - want_lp).abs()[there]
        assert (off <= 2.0 ** -24 * want_lp.abs()[there] + 1e-9).all(), (label, order, off.max().item())


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_ordinary_rows(lib, dtype):
    g = torch.Generator().manual_seed(1)
    x = (2 * torch.randn(4, 9001, generator=g)).to(dtype)
    u = torch.rand(4, generator=g)
    check(lib, x, u, "plain", temperature=torch.tensor([1.0, 0.0, 0.3, 5.0]))
    check(lib, x, u, "filters", temperature=torch.tensor([1.0, 0.0, 0.3, 5.0]), top_k=torch.tensor([50, 3, 0, 4000], dtype=torch.int32),
          top_p=torch.tensor([0.9, 0.5, 1.0, 0.99]), min_p=torch.tensor([0.0, 0.0, 0.05, 0.01]))


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("values", [1, 3])
def test_selections_of_several_rounds(lib, dtype, values):
    """Equal logits: the bins of a round hold more tokens than are compared with each other, so that there is another one, in which the first wave clears what
    the last one may not have read."""
    g = torch.Generator().manual_seed(values)
    x = torch.randint(values, (3, 8100), generator=g).to(dtype)
    u = torch.tensor([0.2, 0.6, 0.99])
    check(lib, x, u, "top-p", top_p=torch.tensor([0.5, 0.9, 0.3]))
    check(lib, x, u, "both", top_k=torch.tensor([4000, 7000, 100], dtype=torch.int32), top_p=torch.tensor([0.5, 0.9, 0.99]))


HOT = [3e36, 1e38, 3e38, math.inf]


def test_min_p_at_very_high_temperatures(lib):
    """All tokens are within min-p of the largest: how far below it they may be is more than a float holds."""
    x = 3 * torch.randn(8, 4001, generator=torch.Generator().manual_seed(5))
    u, t = torch.tensor([0.0, 0.3, 0.6, 0.99, 0.1, 0.5, 0.9, 0.2]), torch.tensor(2 * HOT)
    for f in (1e-30, 0.2, 1.0):
        check(lib, x, u, "min-p", orders=(0,), temperature=t, min_p=torch.full((8,), f))
    check(lib, x, u, "min-p and top-k", orders=(0,), temperature=t, min_p=torch.full((8,), 0.2), top_k=torch.tensor([5, 400, 4000, 1] * 2, dtype=torch.int32))
    check(lib, x.bfloat16(), u, "bf16", orders=(0,), temperature=t, min_p=torch.full((8,), 0.2))


def test_lowest_logits_at_very_high_temperatures(lib):
    """The lowest finite number is in the bin of the cut: the bin's tokens begin with it."""
    low = torch.finfo(FP32).min
    x = torch.randn(4, 300, generator=torch.Generator().manual_seed(6))
    x[:, 100:] = low
    u = torch.tensor([0.2, 0.5, 0.8, 0.999])
    for t in (1e38, 2e38, 3e38):
        check(lib, x, u, "low", orders=(0,), temperature=torch.full((4,), t), top_p=torch.tensor([0.9, 0.99, 0.95, 0.999]))


def test_random_number_zero(lib):
    """The first token with any probability, however small: those that are 2^-1074 of the largest as well."""
    u = torch.tensor([0.0, 1.0])
    x = torch.full((2, 20000), -800.0)
    x[:, 12000] = 0.0
    for at in (-500.0, -744.4, -744.9, -745.0, -745.13):
        # (two slices, the first of which holds nothing but these; tokens whose own w is none next to others of their block and slice that have some)
        x[:, 300:900] = at - 1.0
        x[:, 5000:5300] = at
        x[0, 15000:15600] = at - 1.0
        check(lib, x, u, "plain %g" % at, orders=(0,))
        check(lib, x, u, "min-p %g" % at, orders=(0,), min_p=torch.full((2,), 1e-38))
    x = torch.randn(2, 9000, generator=torch.Generator().manual_seed(7))
    k = torch.tensor([5, 700], dtype=torch.int32)
    check(lib, x, u, "top-k", orders=(0,), temperature=torch.full((2,), 0.01), top_k=k)
    check(lib, x, u, "top-k and top-p", orders=(0,), temperature=torch.full((2,), 0.01), top_k=k, top_p=torch.tensor([0.9999, 1.0]))


def test_tiny_logits_at_very_high_temperatures(lib):
    """Logits times the bins' grid that no float holds: negative ones stay below zero's bin."""
    g = torch.Generator().manual_seed(3)
    u = torch.tensor([0.0, 0.3, 0.7, 0.98])
    for scale, t in ((1e-30, 1e20), (1e-30, 3e38), (1e-38, 1e30), (1.0, 3e38), (1e-44, math.inf), (1.0, math.inf)):
        x, t = scale * torch.randn(4, 700, generator=g), torch.full((4,), t)
        x[0, ::7] = 0.0
        x[1, ::9] = -0.0
        check(lib, x, u, "top-p %g" % scale, orders=(0,), temperature=t, top_p=torch.tensor([0.9, 0.99, 1e-30, 0.3]))
        check(lib, x, u, "top-k %g" % scale, orders=(0,), temperature=t, top_k=torch.tensor([3, 400, 20, 699], dtype=torch.int32))
        check(lib, -x.abs(), u, "negative %g" % scale, orders=(0,), temperature=t, top_p=torch.tensor([0.9, 0.99, 1e-30, 0.3]))


def test_lowest_logits_at_very_low_temperatures(lib):
    """Masks of the lowest finite number: exponents that are far beyond the whole numbers of 64-bit floats."""
    g = torch.Generator().manual_seed(8)
    u = torch.tensor([0.0, 0.3, 0.9, 1.0])
    for dtype in (BF16, FP32):
        x = (3 * torch.randn(4, 9001, generator=g)).to(dtype)
        x[:, ::2] = torch.finfo(dtype).min
        x[2:, :8500] = torch.finfo(dtype).min
        for t in (1e-6, 1e-13, 1e-40):
            t = torch.full((4,), t)
            check(lib, x, u, "plain", orders=(0,), temperature=t)
            check(lib, x, u, "filters", orders=(0,), temperature=t, top_p=torch.tensor([0.5, 0.9, 1.0, 0.0]), min_p=torch.tensor([0.0, 0.1, 0.1, 0.0]),
                  top_k=torch.tensor([0, 0, 5, 4000], dtype=torch.int32))
