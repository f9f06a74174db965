"""GPU tests of the softmax attention where a wave goes through several tiles of its own, and where every tile's scores are far above those of all before."""
import random

import pytest
import torch

from tests.serving_util import BF16, FP32, Problem
from tests.test_gpu_softmax import TYPES, _check, binding  # noqa: F401

pytestmark = pytest.mark.gpu


def tiles_of_a_wave(p):
    """Tiles of 32 keys that a wave of the kernel that splits the keys has, of the longest sequence: the rule of softmax_layout.h (up to 384 sequences)."""
    heads = len(p.lens) * p.Hkv
    many = heads >= 384
    budget, least = (1024, 16) if many else (512 - heads // 2, 4)
    tiles = [-(-L // 32) for n, L in p.lens]
    most = max(least, -(-sum(max(t, 1) for t in tiles) * p.Hkv // budget))
    n = max(1, -(-max(tiles) // most))
    return -(-max(tiles) // n) / (2 if p.dtype == FP32 and p.D == 128 else 4)


def _many(rows, D, dtype, seed, **kw):
    """96 sequences on 4 key/value heads, the pieces of whose keys are of 16 tiles or more; rows: folded rows of a sequence at most."""
    rng = random.Random(seed)
    G = 1 if rows <= 16 else 4
    lens = [(rng.randint(max(1, rows // G // 2), rows // G), rng.choice([470, 500, 511, 512, 1000, 1023])) for _ in range(96)]
    lens[5], lens[6], lens[50] = (1, 1), (2, 33), (0, 600)
    p = Problem(lens, Hq=4 * G, Hkv=4, D=D, dtype=dtype, page=32, seed=seed, pad=1, **kw)
    assert tiles_of_a_wave(p) >= 3
    return p


@pytest.mark.parametrize("D,dtype", TYPES)
@pytest.mark.parametrize("rows", [5, 32, 64])
@pytest.mark.parametrize("cap,slopes,bias_mode", [(0.0, False, 0), (4.0, True, 1)])
def test_several_tiles_of_a_wave(binding, rows, D, dtype, cap, slopes, bias_mode):  # noqa: F811
    _check(binding, _many(rows, D, dtype, 80 + rows, slopes=slopes, bias_mode=bias_mode), "tiles", cap)


@pytest.mark.parametrize("D,dtype", TYPES)
@pytest.mark.parametrize("rows", [16, 64])
def test_several_tiles_with_holes_and_unseen_values(binding, rows, D, dtype):  # noqa: F811
    p = _many(rows, D, dtype, 90 + rows)
    rng = random.Random(rows)
    for s, (n, L) in enumerate(p.lens):
        for e in range(-(-L // p.page)):
            if s % 3 == 0 and rng.random() < 0.2:
                p.table[s, e] = rng.choice([-1, p.pages, 2 ** 31 - 1, -2 ** 31])
    own = torch.zeros(p.pages, p.page, dtype=torch.bool)
    for s, (n, L) in enumerate(p.lens):
        j = torch.arange(L)
        pg = p.table[s][j // p.page].long()
        there = (pg >= 0) & (pg < p.pages)
        own[pg[there], (j % p.page)[there]] = True
    for t in (p.kc, p.vc):
        t.transpose(1, 2)[~own] = float("nan")
    _check(binding, p, "holes")


@pytest.mark.parametrize("D,dtype", TYPES)
@pytest.mark.parametrize("rows", [4, 64])
def test_long_sequences(binding, rows, D, dtype):  # noqa: F811
    """Few sequences of so many keys that all workgroups on the chip have several tiles to a wave."""
    G = 1 if rows == 4 else 4
    p = Problem([(rows // G, 52000), (1, 70), (rows // G, 47001)], Hq=4 * G, Hkv=4, D=D, dtype=dtype, page=128, seed=85, scale="none")
    assert tiles_of_a_wave(p) >= 3
    _check(binding, p, "long")


def _rise(p, step, back):
    """The first feature of the keys rises by `step` (or falls, from the first tile on) with every tile of 32 keys, the queries' is 16."""
    for s, (n, L) in enumerate(p.lens):
        j = torch.arange(L)
        tile = j // 32
        p.kc[p.table[s][j // p.page].long(), :, j % p.page, 0] = (step * (int(tile.max()) - tile if back else tile)).to(p.dtype)[:, None]
    p.q[..., 0] = 16.0


@pytest.mark.parametrize("D,dtype", TYPES)
@pytest.mark.parametrize("rows", [5, 64])
@pytest.mark.parametrize("back", [False, True])
def test_scores_that_rise_with_every_tile(binding, rows, D, dtype, back):  # noqa: F811
    """By more than 24 powers of two a tile, 16 step / sqrt(D) log2(e), so that a wave's sums are scaled down at each of its tiles."""
    p = _many(rows, D, dtype, 95 + rows, scale="none")
    _rise(p, 16.0, back)
    assert 16.0 * 16.0 / D ** 0.5 * 1.44 > 24
    _check(binding, p, "rising")


@pytest.mark.parametrize("D,dtype", TYPES)
@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("slopes", [False, True])
def test_prompts_whose_scores_rise(binding, D, dtype, back, slopes):  # noqa: F811
    """Tiles are gone through from the last keys to the first: whichever way the scores rise, whole and in pieces."""
    p = Problem([(130, 700), (90, 1500), (300, 300)], Hq=4, Hkv=2, D=D, dtype=dtype, page=64, seed=99, scale="none", slopes=slopes)
    _rise(p, 16.0, back)
    _check(binding, p, "rising prompts")


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_prompts_of_many_groups_whose_scores_rise(binding, dtype):  # noqa: F811
    """So many groups of rows that their keys are not cut up."""
    p = Problem([(130, 400)] * 40, Hq=16, Hkv=8, D=64, dtype=dtype, page=64, seed=100, scale="none")
    _rise(p, 16.0, True)
    _check(binding, p, "rising prompts")
