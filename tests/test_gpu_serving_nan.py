"""GPU test of values that are NaN where only some rows of a tile see them, at every place of a 32-key block: the others are as without them."""
import pytest
import torch

from tests.serving_util import BF16, FP32, Problem

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def binding():
    from paper_2506_16640_amd import binding as b
    return b


@pytest.mark.parametrize("D,dtype", [(64, BF16), (64, FP32), (128, FP32)])
@pytest.mark.parametrize("n,L", [(4, 96), (70, 96)])
def test_nan_at_every_place(binding, D, dtype, n, L):
    # (half of the rows stand in front of the block's last 32 keys; scores that keep most keys, so that the block's products are formed)
    p = Problem([(n, L)], D=D, dtype=dtype, seed=13, scale="dense", Hq=4, Hkv=1)
    ref, tol = p.reference()
    for j in range(64, 96):
        at = (int(p.table[0][j // p.page]), slice(None), j % p.page)
        before = p.vc[at].clone()
        p.vc[at] = float("nan")
        e = slice(0, max(0, j - (L - n)))
        for path in (1, 0):
            got = p.run(binding, path=path).double().cpu()
            excess = ((got - ref).abs() - torch.finfo(dtype).eps / 2 * ref.abs() - tol)[e]
            worst = excess.max().item() if excess.numel() else 0.0
            assert worst <= 0.0 and bool(torch.isfinite(got[e]).all()), (path, j, worst)
        p.vc[at] = before
