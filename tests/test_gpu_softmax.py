"""GPU tests of the softmax attention over a paged cache against its plain form in 64 bits."""
import pytest
import torch

from tests.serving_util import BF16, FP32, Problem
from tests.step_util import softmax_reference

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def binding():
    from paper_2506_16640_amd import binding as b
    return b


def _run(binding, p, cap=0.0, out=None, lse=None, **more):
    kw = {k: v for k, v in p.gpu_kw().items() if k != "alpha"}
    cu = torch.tensor(p.cu, dtype=torch.int32).cuda()
    kv = torch.tensor([L for _, L in p.lens], dtype=torch.int32).cuda()
    return binding.paged_softmax_fwd(p.q.cuda(), p.kc.cuda(), p.vc.cuda(), cu, kv, p.table.cuda(), cap=cap, out=out, lse=lse, **kw, **more)


def _within(got, ref, tol, dtype):
    """Half a step of the type and what 32-bit arithmetic may add; NaN is never within."""
    off = (got - ref).abs() - torch.finfo(dtype).eps / 2 * ref.abs() - tol
    return off.numel() == 0 or bool((off <= 0).all())


def _check(binding, p, label, cap=0.0, **more):
    out = torch.full((p.T, p.Hq, p.D), 7.0, dtype=p.dtype, device="cuda")
    lse = torch.full((p.Hq, p.T), 7.0, device="cuda")
    _run(binding, p, cap, out, lse, **more)
    torch.cuda.synchronize()
    ref, ref_l, tol, tol_l = softmax_reference(p, cap)
    own = p.owned()
    assert (out.cpu()[~own] == 7.0).all() and (lse.cpu()[:, ~own] == 7.0).all(), label  # rows of nobody stay as they are
    got, got_l = out.double().cpu()[own], lse.double().cpu()[:, own]
    assert torch.isfinite(got).all(), label
    off = (got - ref[own]).abs()
    excess = off - torch.finfo(p.dtype).eps / 2 * ref[own].abs() - tol[own]
    print(label, "largest error", off.max().item() if off.numel() else 0.0)
    assert off.numel() == 0 or excess.max().item() <= 0.0, (label, excess.max().item(), off.max().item())
    empty = ref_l[:, own] == -float("inf")
    assert (got_l[empty] == -float("inf")).all(), label
    off = (got_l - ref_l[:, own]).abs()[~empty]
    assert off.numel() == 0 or (off - tol_l[:, own][~empty]).max().item() <= 0.0, (label, "lse", off.max().item())


# (new tokens, keys) of the sequences
SMALL = [(1, 1), (3, 3), (1, 17), (0, 0), (5, 40), (33, 33), (1, 200)]
LONGER = [(1, 900), (130, 130), (64, 777), (2, 1500), (200, 1031)]
TYPES = [(64, BF16), (128, BF16), (64, FP32), (128, FP32)]


@pytest.mark.parametrize("D,dtype", TYPES)
@pytest.mark.parametrize("lens", [SMALL, LONGER], ids=["small", "longer"])
@pytest.mark.parametrize("cap", [0.0, 4.0])
def test_lengths(binding, lens, D, dtype, cap):
    _check(binding, Problem(lens, D=D, dtype=dtype, pad=3, seed=21), "lengths", cap)


@pytest.mark.parametrize("D,dtype", TYPES)
@pytest.mark.parametrize("n", [1, 5, 16])
def test_few_rows_many_keys(binding, n, D, dtype):
    """Keys that are cut into pieces: whole ones, ragged ones, a piece of a single key."""
    _check(binding, Problem([(n, 4096), (n, 4097), (n, 255), (n, 256), (n, 257), (n, 5000)], Hq=4, Hkv=2, D=D, dtype=dtype, seed=22, scale="none"), "pieces")


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (3, 3), (6, 2), (8, 1), (12, 4), (10, 2), (16, 2), (40, 1), (66, 1)])
def test_heads(binding, Hq, Hkv):
    _check(binding, Problem([(1, 70), (2, 300), (7, 300), (40, 90)], Hq=Hq, Hkv=Hkv, seed=23), "heads %d %d" % (Hq, Hkv))


@pytest.mark.parametrize("page", [16, 32, 64, 128, 512])
@pytest.mark.parametrize("D,dtype", [(64, BF16), (128, FP32)])
def test_page_sizes(binding, page, D, dtype):
    _check(binding, Problem([(1, page - 1), (1, page), (2, page + 1), (70, 3 * page + 5)], D=D, dtype=dtype, page=page, seed=24), "page %d" % page)


@pytest.mark.parametrize("scale", ["none", "head", "query", "dense", "signs"])
@pytest.mark.parametrize("logn", [0, 1])
@pytest.mark.parametrize("slopes,bias_mode", [(False, 0), (True, 0), (True, 1)])
@pytest.mark.parametrize("cap", [0.0, 3.0])
def test_scales_and_bias(binding, scale, logn, slopes, bias_mode, cap):
    for dtype in (BF16, FP32):
        p = Problem([(1, 1), (1, 600), (9, 350), (150, 150)], scale=scale, logn=logn, slopes=slopes, bias_mode=bias_mode, seed=25, pad=1, dtype=dtype)
        _check(binding, p, "%s logn %d bias %s %d" % (scale, logn, slopes, bias_mode), cap)


def test_not_causal(binding):
    _check(binding, Problem([(1, 300), (20, 300), (200, 450), (3, 2)], causal=False, seed=26), "not causal")


@pytest.mark.parametrize("D,dtype", TYPES)
def test_more_new_tokens_than_keys(binding, D, dtype):
    _check(binding, Problem([(5, 2), (200, 30), (4, 0), (70, 69)], D=D, dtype=dtype, seed=27), "rows without keys")


@pytest.mark.parametrize("D,dtype", TYPES)
def test_large_scores(binding, D, dtype):
    _check(binding, Problem([(1, 500), (9, 900), (150, 400)], D=D, dtype=dtype, q_factor=60.0, seed=28), "large scores")
    _check(binding, Problem([(1, 500), (9, 900), (150, 400)], D=D, dtype=dtype, q_factor=60.0, seed=28), "large scores, capped", 30.0)


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_scores_that_keep_rising(binding, dtype):
    """Every tile brings a larger score than all before: the output so far is scaled down each time."""
    p = Problem([(1, 2000), (3, 1500), (100, 1000)], dtype=dtype, seed=29, scale="none")
    for s, (n, L) in enumerate(p.lens):
        j = torch.arange(L)
        pg = p.table[s][j // p.page].long()
        p.kc[pg, :, j % p.page, 0] = (8.0 * j / L).to(dtype)[:, None]
    p.q[..., 0] = 16.0
    _check(binding, p, "rising")


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("what", [float("inf"), float("-inf"), float("nan")])
def test_values_nobody_sees(binding, what, dtype):
    """Infinities and NaN behind a sequence's keys and on nobody's pages."""
    lens = [(40, 40), (1, 5), (4, 100), (150, 150), (1, 700)]
    p = Problem(lens, dtype=dtype, pad=5, seed=30)
    own = torch.zeros(p.pages, p.page, dtype=torch.bool)
    for s, (n, L) in enumerate(lens):
        j = torch.arange(L)
        own[p.table[s][j // p.page].long(), j % p.page] = True
    for t in (p.kc, p.vc):
        t.transpose(1, 2)[~own] = what
    _check(binding, p, "unseen %s" % what)


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("what", [float("inf"), float("nan")])
@pytest.mark.parametrize("cap", [0.0, 5.0])
def test_values_later_rows_see(binding, what, dtype, cap):
    """A key that only the last rows see holds something that is not finite: the rows before it are as they would be without."""
    for n, L in ((32, 100), (150, 150)):
        p = Problem([(n, L)], dtype=dtype, seed=31, Hq=2, Hkv=1)
        ref, _, tol, _ = softmax_reference(p, cap)
        for j in range(L - 31, L):
            at = (int(p.table[0][j // p.page]), slice(None), j % p.page)
            before = p.kc[at].clone(), p.vc[at].clone()
            p.kc[at], p.vc[at] = what, what
            got = _run(binding, p, cap).double().cpu()
            p.kc[at], p.vc[at] = before
            e = slice(0, j - (L - n))
            assert _within(got[e], ref[e], tol[e], dtype), (n, L, j)


@pytest.mark.parametrize("D,dtype", TYPES)
def test_holes(binding, D, dtype):
    """Pages that are none: their keys are visible to no row, whatever page 0 holds."""
    p = Problem([(1, 900), (5, 300), (150, 400), (2, 20)], D=D, dtype=dtype, seed=32)
    p.table[0, 3] = -1
    p.table[0, 55] = p.pages
    p.table[1, 18] = 2 ** 31 - 1
    p.table[2, ::2] = -5
    p.table[3, :2] = -1
    free = sorted(set(range(p.pages)) - set(p.table[p.table >= 0].tolist()))
    if 0 in free:
        p.kc[0], p.vc[0] = float("nan"), float("nan")
    _check(binding, p, "holes")


def test_strides(binding):
    """Queries, outputs and caches that are slices of larger tensors."""
    p = Problem([(1, 300), (40, 200), (3, 70)], D=64, Hq=4, Hkv=2, seed=33)
    q = torch.zeros(p.T, 6, 192, dtype=BF16, device="cuda")
    q[:, 1:5, 64:128] = p.q.cuda()
    kv = torch.zeros(p.pages, p.page, 2, 2, 64, dtype=BF16, device="cuda")  # [page, token, key or value, head, feature]
    kv[:, :, 0], kv[:, :, 1] = p.kc.cuda().transpose(1, 2), p.vc.cuda().transpose(1, 2)
    out = torch.full((4, p.T, 128), 7.0, dtype=BF16, device="cuda")
    kw = {k: v for k, v in p.gpu_kw().items() if k != "alpha"}
    binding.paged_softmax_fwd(q[:, 1:5, 64:128], kv[:, :, 0].transpose(1, 2), kv[:, :, 1].transpose(1, 2), torch.tensor(p.cu, dtype=torch.int32).cuda(),
                              torch.tensor([L for _, L in p.lens], dtype=torch.int32).cuda(), p.table.cuda(), out=out[..., 64:].transpose(0, 1), **kw)
    ref, _, tol, _ = softmax_reference(p)
    assert (out[..., :64] == 7.0).all()
    assert _within(out[..., 64:].transpose(0, 1).double().cpu(), ref, tol, BF16)


def test_left_out_sequences(binding):
    """Bounds that a sequence passes, lengths that make no sense: its rows are not written, the others are right."""
    p = Problem([(1, 50), (6, 60), (1, 90), (2, 80)], seed=34)
    out = torch.full((p.T, p.Hq, p.D), 7.0, dtype=BF16, device="cuda")
    _run(binding, p, out=out, max_new=4, max_keys=85)
    ref, _, tol, _ = softmax_reference(p)
    got = out.double().cpu()
    for s, there in enumerate((True, False, False, True)):
        e = slice(p.cu[s], p.cu[s + 1])
        if there:
            assert _within(got[e], ref[e], tol[e], BF16)
        else:
            assert (got[e] == 7.0).all()


def test_replay_serves_other_lengths(binding):
    """A captured call on another stream, replayed with other lengths and pages between eager work."""
    problems = [Problem([(1, L1), (3, L2), (70, L3)], seed=35 + i, page=16, spare=60) for i, (L1, L2, L3) in enumerate(((900, 40, 70), (17, 1000, 900), (1, 3, 71)))]
    first = problems[0]
    columns, pages = max(p.table.shape[1] for p in problems), max(p.pages for p in problems)
    dev = "cuda"
    q, out = first.q.to(dev), torch.zeros(first.T, first.Hq, first.D, dtype=BF16, device=dev)
    lse = torch.zeros(first.Hq, first.T, device=dev)
    kc, vc = (torch.zeros(pages, 2, 16, 64, dtype=BF16, device=dev) for _ in range(2))
    table = torch.full((3, columns), -1, dtype=torch.int32, device=dev)
    cu, kv = torch.tensor(first.cu, dtype=torch.int32, device=dev), torch.zeros(3, dtype=torch.int32, device=dev)
    beta, gamma = first.kw["beta"].to(dev), first.kw["gamma"].to(dev)
    ws = binding.new_softmax_workspace(q, kc, table, max_new=70, max_keys=1000)
    call = lambda: binding.paged_softmax_fwd(q, kc, vc, cu, kv, table, max_new=70, max_keys=1000, beta=beta, gamma=gamma, out=out, lse=lse, workspace=ws)  # noqa: E731
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for p in problems + problems[:1]:
        p.kw["beta"], p.kw["gamma"] = first.kw["beta"], first.kw["gamma"]
        q.copy_(p.q)
        kc[:p.pages], vc[:p.pages] = p.kc.to(dev), p.vc.to(dev)
        table.fill_(-1)
        table[:, :p.table.shape[1]] = p.table.to(dev)
        kv.copy_(torch.tensor([L for _, L in p.lens], dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        ref, ref_l, tol, tol_l = softmax_reference(p)
        assert _within(out.double().cpu(), ref, tol, BF16)
        assert bool(((lse.double().cpu() - ref_l).abs() <= tol_l).all())
        eager = torch.empty_like(out)
        binding.paged_softmax_fwd(q, kc, vc, cu, kv, table, max_new=70, max_keys=1000, beta=beta, gamma=gamma, out=eager)
        assert torch.equal(eager, out)


def test_default_arguments(binding):
    p = Problem([(1, 40), (4, 60)], seed=39, scale="none", pad=2)
    got = binding.paged_softmax_fwd(p.q.cuda(), p.kc.cuda(), p.vc.cuda(), torch.tensor(p.cu, dtype=torch.int32).cuda(),
                                    torch.tensor([40, 60], dtype=torch.int32).cuda(), p.table.cuda()).double().cpu()
    ref, _, tol, _ = softmax_reference(p)
    assert _within(got, ref, tol, BF16) and bool((got[-2:] == 0).all())


def test_entmax_approaches_it(binding):
    """The entmax attention's outputs come closer as alpha falls to 1 (the difference shrinks about linearly)."""
    p = Problem([(1, 60), (3, 200)], seed=40, scale="none", dtype=FP32)
    soft = _run(binding, p).double()
    off = []
    for alpha in (1.2, 1.1, 1.05):
        p.kw["alpha"] = alpha
        off.append((p.run(binding).double() - soft).abs().max().item())
    assert off[0] > 1.5 * off[1] > 2.25 * off[2] > 0
