"""GPU tests of serving calls without keys: every row is zero."""
import pytest
import torch

from tests.serving_util import BF16, FP32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def binding():
    from paper_2506_16640_amd import binding as b
    return b


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("pages,columns", [(3, 0), (0, 0), (3, 2)])
def test_no_keys(binding, pages, columns, D, dtype):
    cu = torch.tensor([0, 1, 1, 160], dtype=torch.int32).cuda()
    q = torch.randn(162, 4, D, device="cuda").to(dtype)
    cache = torch.full((pages, 2, 16, D), float("nan"), dtype=dtype, device="cuda")
    table = torch.zeros(3, columns, dtype=torch.int32, device="cuda")
    out = torch.full_like(q, 7.0)
    for path in (1, 0):
        out.fill_(7.0)
        binding.paged_attn_fwd(q, cache, cache, cu, torch.zeros(3, dtype=torch.int32, device="cuda"), table, path=path, out=out)
        torch.cuda.synchronize()
        assert (out[:160] == 0.0).all() and (out[160:] == 7.0).all()
