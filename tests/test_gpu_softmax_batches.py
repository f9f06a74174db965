"""GPU tests of the softmax attention on batches: many sequences, prompts beside single tokens, prompts whose keys are cut into pieces."""
import random

import pytest
import torch

from tests.serving_util import BF16, FP32, Problem
from tests.test_gpu_softmax import TYPES, _check, binding  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("nseq", [191, 192, 384, 385])
@pytest.mark.parametrize("new", [(1, 1), (0, 3)])
@pytest.mark.parametrize("D,dtype", [(64, BF16), (128, FP32)])
def test_many_sequences(binding, nseq, new, D, dtype):  # noqa: F811
    """Lengths of all sequences decide about the pieces, or the bound of the lengths does; most are short, some are long, some empty."""
    rng = random.Random(nseq)
    lens = []
    for s in range(nseq):
        n = rng.randint(*new)
        lens.append((n, max(n, rng.choice([0, 1, 31, 32, 33, 90, 90, rng.randint(1, 300), 1500 if s % 60 == 7 else 40]))))
    _check(binding, Problem(lens, Hq=2, Hkv=2, D=D, dtype=dtype, page=32, seed=70, pad=2), "many")


MIXED = [(1, 700), (90, 300), (0, 0), (1, 1), (5, 260), (8, 513), (9, 40), (12, 333), (16, 1000), (17, 1000), (1, 2000), (40, 1800)]


@pytest.mark.parametrize("D,dtype", TYPES)
@pytest.mark.parametrize("cap", [0.0, 4.0])
@pytest.mark.parametrize("slopes", [False, True])
def test_prompts_beside_single_tokens(binding, D, dtype, cap, slopes):  # noqa: F811
    """4 heads to a key/value head: sequences of 4 to 64 rows beside those of more."""
    _check(binding, Problem(MIXED, Hq=4, Hkv=1, D=D, dtype=dtype, seed=71, pad=1, slopes=slopes), "mixed", cap)


@pytest.mark.parametrize("D,dtype", TYPES)
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("slopes,bias_mode", [(False, 0), (True, 0), (True, 1)])
def test_prompts_in_pieces(binding, D, dtype, causal, slopes, bias_mode):  # noqa: F811
    _check(binding, Problem([(100, 5000), (64, 64), (70, 2601), (33, 1023)], Hq=2, Hkv=1, D=D, dtype=dtype, seed=72, causal=causal, slopes=slopes,
                            bias_mode=bias_mode, page=64), "pieces")


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_prompts_with_sharp_scores(binding, dtype):  # noqa: F811
    """Scores of hundreds: a row's largest goes up again and again, and its sums are scaled anew."""
    _check(binding, Problem([(130, 1400), (1, 1400)], Hq=2, Hkv=1, D=128, dtype=dtype, seed=73, scale="none", q_factor=30.0), "sharp")


def test_holes_in_prompts(binding):  # noqa: F811
    p = Problem([(80, 900), (1, 300), (20, 700)], Hq=4, Hkv=1, D=64, dtype=BF16, seed=74)
    p.table[0, 3:9] = -1
    p.table[0, 40] = p.pages
    p.table[1, 0] = -5
    p.table[2, 30:] = 1 << 30
    _check(binding, p, "holes")


@pytest.mark.parametrize("D,dtype", TYPES)
@pytest.mark.parametrize("what", [-1, -(1 << 31), (1 << 31) - 1])
def test_holes_behind_the_last_key_of_a_block(binding, D, dtype, what):  # noqa: F811
    """A tile's pages that no row of its block sees, though later rows would: nothing is read where they point."""
    p = Problem([(96, 96), (100, 1100)], Hq=4, Hkv=1, D=D, dtype=dtype, seed=75)
    p.table[0, 2:5] = what  # (32 tokens to a block: its first one sees keys 0 .. 31, in a tile of 64)
    p.table[1, 65:67] = what
    _check(binding, p, "holes")


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_pages_behind_four_gigabytes(binding, dtype):  # noqa: F811
    """Bytes of pages whose offsets need more than 32 bits: the same as in a small cache."""
    p = Problem([(1, 900), (70, 300), (12, 77)], Hq=4, Hkv=1, D=64, dtype=dtype, seed=76)
    cu = torch.tensor(p.cu, dtype=torch.int32).cuda()
    kv = torch.tensor([L for _, L in p.lens], dtype=torch.int32).cuda()
    kw = {k: v for k, v in p.gpu_kw().items() if k != "alpha"}
    small = binding.paged_softmax_fwd(p.q.cuda(), p.kc.cuda(), p.vc.cuda(), cu, kv, p.table.cuda(), **kw)
    page = p.page * p.D
    first = (1 << 32) // (2 * page * p.kc.element_size()) - p.pages // 2  # (in the middle of the pages that are used)
    both = torch.empty(first + p.pages, 2, p.page, p.D, dtype=dtype, device="cuda")
    both[first:, :1], both[first:, 1:] = p.kc.cuda(), p.vc.cuda()
    table = torch.where(p.table >= 0, p.table + first, p.table).to(torch.int32).cuda()
    large = binding.paged_softmax_fwd(p.q.cuda(), both[:, :1], both[:, 1:], cu, kv, table, **kw)
    assert torch.equal(small, large)
