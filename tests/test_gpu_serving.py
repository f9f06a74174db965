"""GPU tests of the serving attention (packed sequences with grouped heads, packed or paged keys) against its plain form in 64 bits."""
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
        out = torch.full((p.T, p.Hq, p.D), 7.0, dtype=p.dtype, device="cuda")
        got = p.run(binding, path=path, out=out)
        torch.cuda.synchronize()
        print(label, "path", path, p.check(got, "%s path %d" % (label, path)))
        assert (got[~p.owned().cuda()] == 7.0).all(), label  # rows of nobody stay as they are


# (new tokens, keys) of the sequences
SMALL = [(1, 1), (3, 3), (1, 17), (0, 0), (5, 40), (33, 33), (1, 200)]
LONGER = [(1, 900), (130, 130), (64, 777), (2, 1500), (200, 1031)]


@pytest.mark.parametrize("alpha", [1.5, 2.0, 1.25, 1.7])
@pytest.mark.parametrize("D,dtype", [(64, BF16), (128, BF16), (64, FP32), (128, FP32)])
@pytest.mark.parametrize("lens", [SMALL, LONGER], ids=["small", "longer"])
def test_paged(binding, lens, D, dtype, alpha):
    _check(binding, Problem(lens, D=D, dtype=dtype, alpha=alpha, pad=3, seed=1), "paged")


@pytest.mark.parametrize("D,dtype", [(64, BF16), (128, BF16), (64, FP32), (128, FP32)])
@pytest.mark.parametrize("causal", [True, False])
def test_packed(binding, D, dtype, causal):
    lens = [(n, n) for n in (1, 2, 31, 32, 33, 0, 129, 300, 64)]
    _check(binding, Problem(lens, D=D, dtype=dtype, paged=False, causal=causal, pad=2, seed=2), "packed")


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (3, 3), (6, 2), (8, 1), (12, 4), (10, 2), (16, 2)])
def test_heads(binding, Hq, Hkv):
    _check(binding, Problem([(1, 70), (7, 300), (40, 90)], Hq=Hq, Hkv=Hkv, seed=3), "heads %d %d" % (Hq, Hkv))


@pytest.mark.parametrize("page", [16, 32, 64, 128, 512])
@pytest.mark.parametrize("D", [64, 128])
def test_page_sizes(binding, page, D):
    _check(binding, Problem([(1, page - 1), (1, page), (2, page + 1), (70, 3 * page + 5)], D=D, page=page, seed=4), "page %d" % page)


@pytest.mark.parametrize("scale", ["none", "head", "query", "dense", "signs"])
@pytest.mark.parametrize("logn", [0, 1])
@pytest.mark.parametrize("slopes,bias_mode", [(False, 0), (True, 0), (True, 1)])
def test_scales_and_bias(binding, scale, logn, slopes, bias_mode):
    p = Problem([(1, 1), (1, 600), (9, 350), (150, 150)], scale=scale, logn=logn, slopes=slopes, bias_mode=bias_mode, seed=5, pad=1)
    _check(binding, p, "%s logn %d bias %s %d" % (scale, logn, slopes, bias_mode))


@pytest.mark.parametrize("alpha", [1.5, 2.0, 1.25, 1.1])
@pytest.mark.parametrize("D,dtype", [(64, BF16), (128, BF16), (64, FP32)])
def test_rows_that_keep_most_keys(binding, alpha, D, dtype):
    p = Problem([(1, 2500), (5, 1201), (140, 600), (300, 300)], alpha=alpha, scale="dense", D=D, dtype=dtype, seed=6)
    p.q[p.cu[1]:p.cu[2], :2] = 0.0  # equal scores: every visible key in the support
    _check(binding, p, "dense")


def test_not_causal(binding):
    _check(binding, Problem([(1, 300), (20, 300), (200, 450), (3, 2)], causal=False, seed=7), "not causal")


def test_more_new_tokens_than_keys(binding):
    # the first n - L tokens see no key
    _check(binding, Problem([(5, 2), (200, 30), (4, 0), (70, 69)], seed=8), "rows without keys")


@pytest.mark.parametrize("D,dtype", [(64, BF16), (128, BF16), (64, FP32)])
def test_rows_of_equal_scores(binding, D, dtype):
    p = Problem([(1, 1000), (2, 100), (140, 500)], D=D, dtype=dtype, seed=9, q_factor=0.0)
    _check(binding, p, "equal scores")


@pytest.mark.parametrize("planted", [1, 2, 40, 200])
def test_planted_keys(binding, planted):
    """Rows whose support is exactly the planted keys, all with the same score, spread over the sequence."""
    p = Problem([(1, 3000), (3, 1000), (130, 700)], seed=10, scale="none")
    for s, (n, L) in enumerate(p.lens):
        j = torch.linspace(0, L - n, min(planted, L - n + 1)).long().unique()
        pg = p.table[s][j // p.page].long()
        for hk in range(p.Hkv):
            d = torch.zeros(p.D)
            d[hk] = 12.0
            p.kc[pg, hk, j % p.page] = d.to(p.dtype)
            p.q[p.cu[s]:p.cu[s + 1], hk * 2:hk * 2 + 2] = (3.0 * d / 12.0 * 4).to(p.dtype)
    _check(binding, p, "planted %d" % planted)


def test_large_scores(binding):
    _check(binding, Problem([(1, 500), (9, 900), (150, 400)], q_factor=60.0, seed=11), "large scores")


@pytest.mark.parametrize("paged", [True, False])
@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("what", [float("inf"), float("-inf"), float("nan")])
def test_values_nobody_sees(binding, what, dtype, paged):
    """Infinities and NaN behind a sequence's keys, on nobody's pages, and in keys that later rows alone would see."""
    lens = [(40, 40), (1, 5 if paged else 1), (4, 100 if paged else 4), (150, 150)]
    p = Problem(lens, dtype=dtype, paged=paged, pad=5, seed=12)
    if paged:
        own = torch.zeros(p.pages, p.page, dtype=torch.bool)
        for s, (n, L) in enumerate(lens):
            j = torch.arange(L)
            own[p.table[s][j // p.page].long(), j % p.page] = True
        for t in (p.kc, p.vc):
            t.transpose(1, 2)[~own] = what
    else:
        p.kp[p.cu[-1]:], p.vp[p.cu[-1]:] = what, what
    # the last token's key and value: only the last row sees them, and it is left out of the comparison
    for s, (n, L) in enumerate(lens):
        if n < 2:
            continue
        if paged:
            at = (int(p.table[s][(L - 1) // p.page]), slice(None), (L - 1) % p.page)
            p.kc[at], p.vc[at] = what, what
        else:
            p.kp[p.cu[s + 1] - 1], p.vp[p.cu[s + 1] - 1] = what, what
    ref, tol = p.reference()
    for path in (1, 0):
        got = p.run(binding, path=path).double().cpu()
        for s, (n, L) in enumerate(lens):
            e = slice(p.cu[s], p.cu[s + 1] - (1 if n > 1 else 0))
            err = (got[e] - ref[e]).abs() - torch.finfo(dtype).eps / 2 * ref[e].abs() - tol[e]
            assert torch.isfinite(got[e]).all() and err.max().item() <= 0.0, (path, s, err.max().item())


def test_rows_next_to_infinite_values(binding):
    """A value of infinity that only some rows of a tile see: the others are as without it."""
    lens = [(64, 64), (100, 300)]
    p = Problem(lens, seed=13, scale="dense")
    ref, tol = p.reference()
    for s, (n, L) in enumerate(lens):
        j = L - n // 2  # seen by the second half of the new tokens
        p.vc[int(p.table[s][j // p.page]), :, j % p.page] = float("inf")
    for path in (1, 0):
        got = p.run(binding, path=path).double().cpu()
        for s, (n, L) in enumerate(lens):
            e = slice(p.cu[s], p.cu[s] + n - n // 2)
            err = (got[e] - ref[e]).abs() - 2.0 ** -8 * ref[e].abs() - tol[e]
            assert err.max().item() <= 0.0, (path, s, err.max().item())


@pytest.mark.parametrize("bad", [-1, 2 ** 31 - 1, -2 ** 31, "pages"])
def test_holes(binding, bad):
    """Page numbers that are none: their keys are seen by nobody, and the others as ever."""
    p = Problem([(1, 200), (5, 400), (150, 333), (2, 16), (1, 900)], seed=14)
    bad = p.pages if bad == "pages" else bad
    p.table[0, 3] = bad
    p.table[1, :6] = bad
    p.table[2, 7] = bad
    p.table[2, 20] = bad
    p.table[3, 0] = bad  # all of its keys: zeros
    p.table[4, ::2] = bad
    _check(binding, p, "holes")


def test_arrays_that_lead_out_of_the_tensors(binding):
    """Sequences whose arrays make no sense are left out, and the others are as ever."""
    p = Problem([(3, 50), (4, 60), (5, 70), (6, 80)], seed=15)
    ref, tol = p.reference()
    cu = torch.tensor(p.cu, dtype=torch.int32)
    kv = torch.tensor([L for _, L in p.lens], dtype=torch.int32)
    def run(cu, kv, **kw):
        out = torch.full((p.T, p.Hq, p.D), 7.0, dtype=p.dtype, device="cuda")
        return binding.paged_attn_fwd(p.q.cuda(), p.kc.cuda(), p.vc.cuda(), cu.cuda(), kv.cuda(), p.table.cuda(), out=out, **kw, **p.gpu_kw()).double().cpu()
    def compare(got, rows, left):
        err = (got[rows] - ref[rows]).abs() - 2.0 ** -8 * ref[rows].abs() - tol[rows]
        assert err.max().item() <= 0.0
        assert (got[left] == 7.0).all()
    for path in (1, 0):
        bad = kv.clone()
        bad[1] = -5
        bad[2] = 10 ** 6
        compare(run(cu, bad, path=path), list(range(0, 3)) + list(range(12, 18)), list(range(3, 12)))
        compare(run(cu, kv, path=path, max_new=4), list(range(0, 7)), list(range(7, 18)))
        compare(run(cu, kv, path=path, max_keys=60), list(range(0, 7)), list(range(7, 18)))
        far = cu.clone()
        far[4] = 10 ** 6
        compare(run(far, kv, path=path), list(range(0, 12)), list(range(12, 18)))


def test_strides(binding):
    """Queries as a part of a fused projection, the cache token-major, keys and values with different strides, the output inside another tensor."""
    p = Problem([(1, 300), (6, 90), (140, 200)], Hq=6, Hkv=2, D=64, seed=16)
    fused = torch.randn(p.T, p.Hq + 4, p.D).to(p.dtype).cuda()
    fused[:, :p.Hq] = p.q.cuda()
    q = fused[:, :p.Hq]
    kc = torch.randn(p.pages, p.page, p.Hkv + 1, p.D).to(p.dtype).cuda()
    kc[:, :, :p.Hkv] = p.kc.cuda().transpose(1, 2)
    kc = kc[:, :, :p.Hkv].transpose(1, 2)
    vc = torch.randn(p.Hkv, p.pages, p.page, 2 * p.D).to(p.dtype).cuda()
    vc[..., :p.D] = p.vc.cuda().transpose(0, 1)
    vc = vc[..., :p.D].transpose(0, 1)
    out = torch.full((p.Hq, p.T, 2 * p.D), 7.0, dtype=p.dtype, device="cuda")
    cu, kv = torch.tensor(p.cu, dtype=torch.int32).cuda(), torch.tensor([L for _, L in p.lens], dtype=torch.int32).cuda()
    for path in (1, 0):
        got = binding.paged_attn_fwd(q, kc, vc, cu, kv, p.table.cuda(), path=path, out=out[..., :p.D].transpose(0, 1), **p.gpu_kw())
        p.check(got, "strides")
        assert (out[..., p.D:] == 7.0).all()


def test_rows_in_front(binding):
    _check(binding, Problem([(3, 50), (130, 130)], seed=17, front=5, pad=4), "rows of nobody in front")


def test_many_sequences(binding):
    gen = torch.Generator().manual_seed(18)
    lens = [(int(n), int(n + k)) for n, k in zip(torch.randint(0, 4, (300,), generator=gen), torch.randint(0, 60, (300,), generator=gen))]
    _check(binding, Problem(lens, Hq=2, Hkv=1, seed=18), "300 sequences")
