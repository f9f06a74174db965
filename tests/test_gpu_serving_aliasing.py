"""GPU tests of serving calls whose tensors are parts of one: side by side they are as separate ones, on top of each other they are refused."""
import pytest
import torch

from tests.serving_util import BF16, FP32, Problem

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def binding():
    from paper_2506_16640_amd import binding as b
    return b


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("paged", [True, False])
def test_output_beside_the_queries(binding, paged, dtype):
    lens = [(1, 300), (200, 260), (70, 90)] if paged else [(300, 300), (1, 1), (70, 70)]
    p = Problem(lens, Hq=6, Hkv=2, paged=paged, dtype=dtype, scale="none", seed=51)  # (blocks that two kernels work on among them)
    want = p.run(binding)
    p.check(want, "separate")
    both = torch.zeros(p.T, 12, p.D, dtype=dtype, device="cuda")
    cu = torch.tensor(p.cu, dtype=torch.int32).cuda()
    ints = lambda x: torch.tensor(x, dtype=torch.int32).cuda()  # noqa: E731

    def run(out):
        both[:, :6] = p.q.cuda()
        q = both[:, :6]
        if paged:
            return binding.paged_attn_fwd(q, p.kc.cuda(), p.vc.cuda(), cu, ints([L for _, L in lens]), p.table.cuda(), out=out, **p.gpu_kw())
        return binding.packed_attn_fwd(q, p.kp.cuda(), p.vp.cuda(), cu, out=out, **p.gpu_kw())

    assert torch.equal(run(both[:, 6:]), want)
    for out in (both[:, :6], both[:, 1:7]):
        with pytest.raises(binding.EntmaxAttnError):
            run(out)
        assert torch.equal(both[:, :6], p.q.cuda())


def test_output_in_the_cache(binding):
    p = Problem([(3, 40)], seed=52)
    kc, vc = p.kc.cuda(), p.vc.cuda()
    out = kc.view(-1, p.Hq, p.D)[:p.T]
    with pytest.raises(binding.EntmaxAttnError):
        binding.paged_attn_fwd(p.q.cuda(), kc, vc, torch.tensor(p.cu, dtype=torch.int32).cuda(), torch.tensor([40], dtype=torch.int32).cuda(),
                               p.table.cuda(), out=out, **p.gpu_kw())
    assert torch.equal(kc, p.kc.cuda())


def test_caches_in_one_tensor(binding):
    """Keys and values of a page together; a cache whose heads or pages are one and the same is refused."""
    p = Problem([(3, 40), (1, 17), (20, 20)], seed=53)
    gen = torch.Generator().manual_seed(54)
    k, v = (torch.randn(p.T, p.Hkv, p.D, generator=gen).to(BF16).cuda() for _ in range(2))
    cu, kv = torch.tensor(p.cu, dtype=torch.int32).cuda(), torch.tensor([L for _, L in p.lens], dtype=torch.int32).cuda()
    kc, vc = p.kc.cuda(), p.vc.cuda()
    binding.cache_append(k, v, kc, vc, cu, kv, p.table.cuda())
    both = torch.stack([p.kc, p.vc], 1).cuda()
    binding.cache_append(k, v, both[:, 0], both[:, 1], cu, kv, p.table.cuda())
    assert torch.equal(both[:, 0], kc) and torch.equal(both[:, 1], vc)
    for a, b in ((kc, kc), (kc[:, :1].expand(-1, 2, -1, -1), vc), (kc, vc[:1].expand(p.pages, -1, -1, -1)), (both[:, 0], both[:, 0])):
        with pytest.raises(binding.EntmaxAttnError):
            binding.cache_append(k, v, a, b, cu, kv, p.table.cuda())
