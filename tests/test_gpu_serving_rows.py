"""GPU tests of the serving attention's ways through a row: long sequences shared out by keys, rows with more candidates than the sweep
remembers or an octet holds, groups of many heads, long supports of decode rows."""
import pytest
import torch

from tests.serving_util import BF16, FP32, Problem

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def binding():
    from paper_2506_16640_amd import binding as b
    return b


def _check(binding, p, label, paths=(1, 0)):
    for path in paths:
        got = p.run(binding, path=path)
        torch.cuda.synchronize()
        print(label, "path", path, p.check(got, "%s path %d" % (label, path)))


@pytest.mark.parametrize("alpha", [1.5, 1.25, 2.0, 1.7])
@pytest.mark.parametrize("D,slopes", [(64, False), (64, True), (128, False), (128, True)])
def test_long_sequences(binding, D, slopes, alpha):
    # 3000 and 4200 keys: shares of one block's sweep; 2500: decode rows; 130: none of it
    p = Problem([(150, 3000), (130, 130), (1, 2500), (33, 4200)], D=D, slopes=slopes, alpha=alpha, page=64, seed=31)
    _check(binding, p, "long")


def _plant(p, s, row, heads, keys):
    """The keys of one row of sequence s that its query of the given heads meets with the same, largest score."""
    for h in heads:
        d = torch.zeros(p.D)
        d[(row * 7 + h) % p.D] = 11.0
        p.q[p.cu[s] + row, h] = (2.0 * d).to(p.dtype)
        pg = p.table[s][keys // p.page].long()
        p.kc[pg, h // (p.Hq // p.Hkv), keys % p.page] = d.to(p.dtype)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("count,step,what", [(40, 100, "more groups than an octet holds"), (20, 32, "more than the sweep remembers"), (100, 32, "many"),
                                             (300, 8, "more than a list holds")])
def test_single_rows_with_many_candidates(binding, D, count, step, what):
    """Sparse rows all around one or two that keep `count` keys, `step` apart (32: all of one half of the row's lanes)."""
    p = Problem([(150, 4500), (40, 4300)], D=D, scale="none", delta=8.0, seed=32, page=128)
    _plant(p, 0, 60, [1], 5 + step * torch.arange(count))
    _plant(p, 0, 61, [2], 9 + step * torch.arange(count))
    _plant(p, 1, 7, [0], 3 + step * torch.arange(count))
    _check(binding, p, what)


@pytest.mark.parametrize("Hq,Hkv", [(96, 1), (64, 1), (130, 2)])
def test_groups_of_many_heads(binding, Hq, Hkv):
    # (more heads a group than the kernels that split the keys take rows)
    _check(binding, Problem([(1, 300), (2, 90), (3, 3)], Hq=Hq, Hkv=Hkv, seed=33), "%d heads a group" % (Hq // Hkv))


@pytest.mark.parametrize("alpha", [1.5, 2.0, 1.25])
@pytest.mark.parametrize("D,dtype", [(64, BF16), (128, FP32)])
@pytest.mark.parametrize("planted", [30, 100, 250, 300, 2000])
def test_supports_of_decode_rows(binding, planted, D, dtype, alpha):
    """One wave's, a workgroup's, and those that a third kernel adds up."""
    p = Problem([(1, 9000), (2, 3000)], D=D, dtype=dtype, alpha=alpha, scale="none", delta=8.0, seed=34, page=64)
    _plant(p, 0, 0, [0, 3], torch.linspace(0, 8990, planted).long().unique())
    _plant(p, 1, 1, [2], torch.linspace(0, 2990, min(planted, 1500)).long().unique())
    _check(binding, p, "%d keys kept" % planted)


def test_sequences_longer_than_the_held_scores(binding):
    _check(binding, Problem([(1, 21000), (1, 17)], Hq=2, Hkv=1, scale="dense", seed=35, page=256), "long dense decode row", paths=(0,))


def test_many_decode_rows(binding):
    gen = torch.Generator().manual_seed(36)
    lens = [(int(n), int(L)) for n, L in zip(torch.randint(1, 9, (40,), generator=gen), torch.randint(9, 700, (40,), generator=gen))]
    _check(binding, Problem(lens, Hq=8, Hkv=2, seed=36, logn=1, scale="query"), "40 sequences of a few tokens")
