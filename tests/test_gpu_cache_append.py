"""GPU tests of cache_append (new keys and values to their pages, positions rotated on the way) against its plain form in 64 bits, and of
the serving operators together."""
import math

import pytest
import torch

from tests.serving_util import BF16, FP32, Problem

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def binding():
    from paper_2506_16640_amd import binding as b
    return b


def rotate(x, pos, inv_freq, interleaved):
    """x [n, H, D] rotated by its rows' positions, in 64 bits, and the size of the products the result is made of."""
    x = x.double().clone()
    size = x.abs()
    if inv_freq is None:
        return x, torch.zeros_like(size)
    half = inv_freq.shape[0]
    e = torch.arange(half)
    i, j = (2 * e, 2 * e + 1) if interleaved else (e, e + half)
    ang = pos.double()[:, None, None] * inv_freq.double()
    a, b = x[..., i].clone(), x[..., j].clone()
    x[..., i], x[..., j] = a * ang.cos() - b * ang.sin(), b * ang.cos() + a * ang.sin()
    s = torch.zeros_like(size)
    s[..., i] = s[..., j] = a.abs() + b.abs()
    return x, s


class Append:
    def __init__(self, lens, Hq=4, Hkv=2, D=64, dtype=BF16, page=16, rot=None, interleaved=False, pad=0, seed=0, with_q=True, theta=10000.0, front=0):
        self.p = Problem(lens, Hq=Hq, Hkv=Hkv, D=D, dtype=dtype, page=page, pad=pad, seed=seed, front=front)
        g = torch.Generator().manual_seed(seed + 1000)
        self.k, self.v = (torch.randn(self.p.T, Hkv, D, generator=g).to(dtype) for _ in range(2))
        rot = D if rot is None else rot
        self.inv_freq = (theta ** (-torch.arange(0, rot, 2).double() / max(rot, 1))).float() if rot else None
        self.interleaved, self.with_q = interleaved, with_q

    def run(self, binding, q=None, q_out=None, k=None, v=None, kc=None, vc=None, **kw):
        p = self.p
        self.kc = p.kc.cuda() if kc is None else kc
        self.vc = p.vc.cuda() if vc is None else vc
        cu = torch.tensor(p.cu, dtype=torch.int32).cuda()
        kv = torch.tensor([L for _, L in p.lens], dtype=torch.int32).cuda()
        q = p.q.cuda() if q is None else q
        return binding.cache_append(self.k.cuda() if k is None else k, self.v.cuda() if v is None else v, self.kc, self.vc, cu, kv, p.table.cuda(),
                                    q=q if self.with_q else None, q_out=q_out, inv_freq=None if self.inv_freq is None else self.inv_freq.cuda(),
                                    interleaved=self.interleaved)

    def check(self, q_out, before=7.0):
        """Half a step of the type of the value, and 2^-21 of the products it is made of (angle, sine and cosine to 2^-23 each, three roundings)."""
        p = self.p
        half = torch.finfo(p.dtype).eps / 2
        want_k, want_v, size_k = p.kc.double(), p.vc.double(), torch.zeros(p.kc.shape, dtype=torch.float64)
        want_q, size_q = torch.full(p.q.shape, before, dtype=torch.float64), torch.zeros(p.q.shape, dtype=torch.float64)
        for s, (n, L) in enumerate(p.lens):
            if L < n:
                continue
            e = slice(p.cu[s], p.cu[s] + n)
            pos = torch.arange(L - n, L)
            want_q[e], size_q[e] = rotate(p.q[e], pos, self.inv_freq, self.interleaved)
            rk, sk = rotate(self.k[e], pos, self.inv_freq, self.interleaved)
            for t in range(n):
                pg, at = int(p.table[s][int(pos[t]) // p.page]), int(pos[t]) % p.page
                if 0 <= pg < p.pages:
                    want_k[pg, :, at], want_v[pg, :, at], size_k[pg, :, at] = rk[t], self.v[e][t].double(), sk[t]
        def compare(got, want, size):
            got = got.double().cpu()
            err = (got - want).abs() - half * torch.where(size > 0, want.abs(), 0.0) - 2.0 ** -21 * size
            assert err.max().item() <= 0.0, err.max().item()
        compare(self.kc, want_k, size_k)
        assert torch.equal(self.vc.double().cpu(), want_v)  # (values and everything else: the very bits)
        if self.with_q:
            compare(q_out, want_q, size_q)


def _run(binding, a):
    q_out = torch.full(a.p.q.shape, 7.0, dtype=a.p.dtype, device="cuda") if a.with_q else None
    got = a.run(binding, q_out=q_out)
    assert (got is None) == (not a.with_q)
    a.check(got)


LENS = [(1, 1), (3, 3), (1, 17), (0, 0), (5, 40), (33, 33), (1, 200), (70, 1000)]


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("D,dtype,rot", [(64, BF16, 64), (64, BF16, 0), (64, BF16, 16), (128, BF16, 128), (128, BF16, 48), (64, FP32, 64), (64, FP32, 32),
                                         (128, FP32, 128), (128, FP32, 16)])
def test_append(binding, D, dtype, rot, interleaved):
    _run(binding, Append(LENS, D=D, dtype=dtype, rot=rot, interleaved=interleaved, pad=3, seed=1))


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (12, 4), (16, 16), (40, 8), (3, 1)])
@pytest.mark.parametrize("page", [16, 64, 256])
def test_heads_and_pages(binding, Hq, Hkv, page):
    _run(binding, Append(LENS, Hq=Hq, Hkv=Hkv, page=page, seed=2))


def test_without_queries(binding):
    _run(binding, Append(LENS, with_q=False, seed=3))


def test_many_tokens(binding):
    # more tokens than one workgroup each is made for, an odd number of them, rows of nobody in front and behind
    _run(binding, Append([(1200, 1300), (1, 5), (901, 901), (0, 3)], Hq=3, Hkv=1, pad=6, seed=4, front=3))


def test_many_sequences(binding):
    gen = torch.Generator().manual_seed(5)
    lens = [(int(n), int(n + k)) for n, k in zip(torch.randint(0, 3, (300,), generator=gen), torch.randint(0, 60, (300,), generator=gen))]
    _run(binding, Append(lens, Hq=2, Hkv=1, seed=5))


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_far_positions(binding, dtype):
    """Angles of a million turns and more: as good as near ones."""
    p = Append([(3, 1 << 16)], dtype=dtype, page=1 << 14, seed=6, theta=3.0)
    _run(binding, p)
    a = Append([(2, 30)], dtype=dtype, seed=7)
    a.p.table = torch.full((1, 1 << 17), -1, dtype=torch.int32)
    a.p.table[0, -1] = 1
    a.p.lens = [(2, 1 << 21)]  # (positions 2^21 - 2 and 2^21 - 1; every other page is a hole)
    _run(binding, a)


def test_in_place(binding):
    a = Append(LENS, seed=8)
    q = a.p.q.cuda()
    got = a.run(binding, q=q, q_out=q)
    assert got.data_ptr() == q.data_ptr()
    a.check(q)


@pytest.mark.parametrize("bad", [-1, 2 ** 31 - 1, -2 ** 31, "pages"])
def test_holes(binding, bad):
    a = Append([(5, 40), (20, 100), (1, 17)], seed=9)
    bad = a.p.pages if bad == "pages" else bad
    a.p.table[0, 2] = bad
    a.p.table[1, 5] = bad
    a.p.table[2, 1] = bad
    _run(binding, a)


def test_sequences_left_out(binding):
    """Fewer keys than new tokens, more keys than the table holds, rows outside the tensors: nothing is written for them."""
    a = Append([(5, 40), (4, 60), (3, 17), (2, 20)], seed=10)
    p = a.p
    cu = torch.tensor(p.cu, dtype=torch.int32)
    q_out = torch.full(p.q.shape, 7.0, dtype=p.dtype, device="cuda")
    def call(cu, kv):
        a.kc, a.vc = p.kc.cuda(), p.vc.cuda()
        q_out.fill_(7.0)
        binding.cache_append(a.k.cuda(), a.v.cuda(), a.kc, a.vc, cu.cuda(), torch.tensor(kv, dtype=torch.int32).cuda(), p.table.cuda(), q=p.q.cuda(),
                             q_out=q_out, inv_freq=a.inv_freq.cuda())
    lens = list(p.lens)
    call(cu, [4, 10 ** 6, -3, 20])
    p.lens = [(5, 4), (4, 0), (3, 0), (2, 20)]  # (the plain form leaves out those with fewer keys than tokens)
    a.check(q_out)
    far = cu.clone()
    far[4] = 10 ** 6
    call(far, [L for _, L in lens])
    p.lens = lens[:3] + [(2, 0)]
    a.check(q_out)


def test_strides(binding):
    """Queries, keys and values as parts of one fused projection, a token-major cache."""
    a = Append(LENS, Hq=6, Hkv=2, seed=11)
    p = a.p
    fused = torch.zeros(p.T, 10, p.D, dtype=p.dtype, device="cuda")
    fused[:, :6], fused[:, 6:8], fused[:, 8:] = p.q.cuda(), a.k.cuda(), a.v.cuda()
    kc, vc = (t.cuda().transpose(1, 2).contiguous().transpose(1, 2) for t in (p.kc, p.vc))
    got = a.run(binding, q=fused[:, :6], q_out=fused[:, :6], k=fused[:, 6:8], v=fused[:, 8:], kc=kc, vc=vc)
    a.check(got)


# ------------------------------------------------------------------- the operators together

def _serve(binding, p, steps, inv_freq, out, alpha=1.5):
    """The sequences of p (packed) through the cache, steps[s] tokens of sequence s at a time."""
    cu = [0]
    for n, _ in p.lens:
        cu.append(cu[-1] + n)
    page = 16
    per = [(n + page - 1) // page for n, _ in p.lens]
    kc, vc = (torch.full((sum(per), p.Hkv, page, p.D), float("nan"), dtype=p.dtype, device="cuda") for _ in range(2))
    table = torch.full((len(per), max(per)), -1, dtype=torch.int32)
    order = torch.randperm(sum(per), generator=torch.Generator().manual_seed(3)).to(torch.int32)
    at = 0
    for s, n in enumerate(per):
        table[s, :n] = order[at:at + n]
        at += n
    table = table.cuda()
    q, k, v = p.q.cuda(), p.kp.cuda(), p.vp.cuda()
    have = [0] * len(per)
    kw = p.gpu_kw()
    ints = lambda x: torch.tensor(x, dtype=torch.int32).cuda()  # noqa: E731
    while any(h < n for h, (n, _) in zip(have, p.lens)):
        new = [min(st, n - h) for st, h, (n, _) in zip(steps, have, p.lens)]
        rows = torch.cat([torch.arange(c + h, c + h + m) for c, h, m in zip(cu, have, new)]).cuda()
        have = [h + m for h, m in zip(have, new)]
        bounds = [0]
        for m in new:
            bounds.append(bounds[-1] + m)
        rq = binding.cache_append(k[rows], v[rows], kc, vc, ints(bounds), ints(have), table, q=q[rows], inv_freq=inv_freq)
        out[rows] = binding.paged_attn_fwd(rq, kc, vc, ints(bounds), ints(have), table, max_new=max(new), max_keys=max(have), **kw)
    return out


@pytest.mark.parametrize("steps", [[1, 1, 1], [7, 1, 50], [1000, 3, 1000]])
@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_chunks_equal_whole_prompts(binding, steps, dtype):
    """Prompts fed through the cache in pieces give what the packed attention of the rotated prompts gives (n in (ln n)^gamma counts the keys a row sees)."""
    lens = [(60, 60), (9, 9), (150, 150)]
    p = Problem(lens, Hq=6, Hkv=2, dtype=dtype, paged=False, logn=1, slopes=True, seed=20)
    inv_freq = (1000.0 ** (-torch.arange(0, 64, 2).double() / 64)).float().cuda()
    got = _serve(binding, p, steps, inv_freq, torch.zeros(p.T, p.Hq, p.D, dtype=dtype, device="cuda"))
    pos = torch.cat([torch.arange(n) for n, _ in lens])
    p.q = rotate(p.q, pos, inv_freq.cpu(), False)[0].float().to(dtype)
    p.kp = rotate(p.kp, pos, inv_freq.cpu(), False)[0].float().to(dtype)
    whole = p.run(binding)
    p.check(whole, "packed")
    if dtype == BF16:  # (a rotated value next to the middle of two bf16 numbers may go to the other one; fp32 differs by roundings)
        assert (got.double() - whole.double()).abs().max().item() <= 0.1 and (got != whole).double().mean().item() < 0.2
    else:
        assert (got - whole).abs().max().item() <= 1e-3


def test_a_step_in_a_graph(binding):
    """Append and attention captured once and replayed for later steps: lengths, pages, tokens change in place between the replays."""
    B, Hq, Hkv, D, page, most = 5, 6, 2, 64, 16, 40
    gen = torch.Generator().manual_seed(21)
    rnd = lambda *s: torch.randn(*s, generator=gen).to(BF16).cuda()  # noqa: E731
    kc, vc = rnd(B * most, Hkv, page, D), rnd(B * most, Hkv, page, D)
    table = torch.randperm(B * most, generator=gen).to(torch.int32).reshape(B, most).cuda()
    cu = torch.arange(B + 1, dtype=torch.int32).cuda()
    kv = torch.tensor([1, 30, 77, 300, 12], dtype=torch.int32).cuda()
    q, k, v = rnd(B, Hq, D), rnd(B, Hkv, D), rnd(B, Hkv, D)
    beta, gamma = torch.rand(Hq).cuda() + 0.5, torch.rand(Hq).cuda() + 0.5
    inv_freq = (10000.0 ** (-torch.arange(0, D, 2).double() / D)).float().cuda()
    rq, out = torch.zeros_like(q), torch.zeros_like(q)
    ws = binding.new_paged_workspace(q, kc, table, max_new=1)
    kw = dict(max_new=1, beta=beta, gamma=gamma, logn_mode=1)

    def step(kc, vc, rq, out, ws):
        binding.cache_append(k, v, kc, vc, cu, kv, table, q=q, q_out=rq, inv_freq=inv_freq)
        return binding.paged_attn_fwd(rq, kc, vc, cu, kv, table, out=out, workspace=ws, **kw)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(kc, vc, rq, out, ws)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(kc, vc, rq, out, ws)
    torch.cuda.synchronize()
    kc2, vc2 = kc.clone(), vc.clone()
    for it in range(6):
        kv += torch.tensor([1, 1, 40, 1, 0], dtype=torch.int32).cuda()
        q.copy_(rnd(B, Hq, D)), k.copy_(rnd(B, Hkv, D)), v.copy_(rnd(B, Hkv, D))
        if it == 3:  # two sequences exchange their pages
            table[[0, 2]] = table[[2, 0]]
        graph.replay()
        torch.cuda.synchronize()
        want = step(kc2, vc2, torch.zeros_like(q), torch.zeros_like(q), None)
        assert torch.equal(out, want) and torch.equal(kc, kc2) and torch.equal(vc, vc2), it


def test_two_streams(binding):
    """Calls on two streams at once, each with its own workspace, give what they give alone."""
    ps = [Problem([(1, 2000), (150, 700)], seed=22), Problem([(3, 1500), (1, 5), (200, 200)], seed=23, scale="dense")]
    alone = [p.run(binding) for p in ps]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in ps]
    for _ in range(3):
        got = []
        for p, st in zip(ps, streams):
            with torch.cuda.stream(st):
                got.append(p.run(binding))
        torch.cuda.synchronize()
        for a, b in zip(alone, got):
            assert torch.equal(a, b)


def test_same_bits_every_time(binding):
    p = Problem([(1, 3000), (5, 900), (140, 500), (300, 300)], seed=24)
    first = p.run(binding)
    for _ in range(3):
        assert torch.equal(first, p.run(binding))
