"""GPU tests of a serving step's operators together: the plan, the new keys and values into the cache, both kinds of attention, and the next tokens."""
import pytest
import torch

from tests.serving_util import BF16
from tests.step_util import plain_plan, plain_sample, softmax_rows

pytestmark = pytest.mark.gpu

PAGE, PAGES, COLUMNS, HQ, HKV, D, V = 16, 120, 40, 4, 2, 64, 301


@pytest.fixture(scope="module")
def binding():
    from paper_2506_16640_amd import binding as b
    return b


class Server:
    """Places for `nseq` sequences, `rows` rows a step; a model of one layer whose logits are features of its heads' outputs."""

    def __init__(self, binding, nseq, rows, seed, most_new):
        gen = torch.Generator().manual_seed(seed)
        normal = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
        dev = "cuda"
        ints = lambda *s: torch.zeros(*s, dtype=torch.int32, device=dev)  # noqa: E731
        self.binding, self.nseq, self.rows, self.most_new = binding, nseq, rows, most_new
        self.embed = normal(V, HQ + 2 * HKV, D).to(BF16).to(dev)
        self.feature, self.weight = torch.randint(HQ * D, (V,), generator=gen).to(dev), (4 * normal(V)).to(dev)
        self.freq = (10000.0 ** (-torch.arange(D // 2).float() / (D // 2))).to(dev)
        self.kc, self.vc = (torch.zeros(PAGES, HKV, PAGE, D, dtype=BF16, device=dev) for _ in range(2))
        self.new, self.release = ints(nseq), ints(nseq)
        self.table = torch.full((nseq, COLUMNS), -1, dtype=torch.int32, device=dev)
        self.free = torch.randperm(PAGES, generator=gen).to(torch.int32).to(dev)
        self.plan = binding.new_plan(nseq, rows, dev)
        self.plan.free_count.fill_(PAGES)
        self.ids = torch.zeros(rows, dtype=torch.int64, device=dev)
        self.u, self.temperature, self.top_p = torch.zeros(rows, device=dev), torch.full((rows,), 0.8, device=dev), torch.full((rows,), 0.9, device=dev)
        self.top_k = torch.full((rows,), 50, dtype=torch.int32, device=dev)
        self.token, self.logprob = ints(rows), torch.zeros(rows, device=dev)
        self.qr, self.o, self.oe = (torch.zeros(rows, HQ, D, dtype=BF16, device=dev) for _ in range(3))
        self.lse, self.logits = torch.zeros(HQ, rows, device=dev), torch.zeros(rows, V, device=dev)
        bounds = dict(max_new=most_new, max_keys=PAGE * COLUMNS)
        self.bounds = bounds
        self.ws = binding.new_softmax_workspace(self.qr, self.kc, self.table, **bounds)
        self.wse = binding.new_paged_workspace(self.qr, self.kc, self.table, **bounds)
        self.wsl = binding.new_sample_workspace(self.logits)

    def step(self):
        b, p = self.binding, self.plan
        b.cache_plan(self.new, p.kv_len, self.table, self.free, p.free_count, PAGE, p, release=self.release)
        x = self.embed[self.ids]
        self.q, self.k, self.v = x[:, :HQ], x[:, HQ:HQ + HKV], x[:, HQ + HKV:]
        b.cache_append(self.k, self.v, self.kc, self.vc, p.cu_seqlens, p.kv_len, self.table, q=self.q, inv_freq=self.freq, q_out=self.qr)
        b.paged_softmax_fwd(self.qr, self.kc, self.vc, p.cu_seqlens, p.kv_len, self.table, out=self.o, lse=self.lse, workspace=self.ws, **self.bounds)
        b.paged_attn_fwd(self.qr, self.kc, self.vc, p.cu_seqlens, p.kv_len, self.table, alpha=1.5, out=self.oe, workspace=self.wse, **self.bounds)
        self.logits.copy_((self.o + self.oe).float().reshape(self.rows, HQ * D)[:, self.feature] * self.weight)
        b.sample(self.logits, self.u, self.temperature, self.top_k, self.top_p, token=self.token, logprob=self.logprob, workspace=self.wsl)


def _steps(server, run, seed):
    """Prompts, decoding, sequences that end and others in their places; every step against the plain forms."""
    gen = torch.Generator().manual_seed(seed)
    nseq, rows = server.nseq, server.rows
    kv, table, free, count = [0] * nseq, [[-1] * COLUMNS for _ in range(nseq)], server.free.tolist(), PAGES
    cached = {}  # (page, offset) -> the key and value that belong there
    for turn in range(9):
        new, gone = [1 if kv[s] else 0 for s in range(nseq)], [0] * nseq
        if turn in (0, 5):
            new = [int(torch.randint(1, server.most_new + 1, (1,), generator=gen)) if not kv[s] else 1 for s in range(nseq)]
        if turn in (3, 4):
            s = int(torch.randint(nseq, (1,), generator=gen))
            gone[s], new[s] = 1, 0
        if turn == 7:
            new = [0] * nseq
        ids = torch.randint(V, (rows,), generator=gen)
        u = torch.rand(rows, generator=gen)
        server.new.copy_(torch.tensor(new, dtype=torch.int32))
        server.release.copy_(torch.tensor(gone, dtype=torch.int32))
        server.ids.copy_(ids)
        server.u.copy_(u)
        server.o.fill_(7.0)
        server.oe.fill_(0.0)
        run()
        torch.cuda.synchronize()
        cu, count, slots, positions, sequences = plain_plan(new, kv, table, free, count, PAGE, rows, gone)
        p = server.plan
        for name, got, want in (("cu", p.cu_seqlens, cu), ("kv", p.kv_len, kv), ("count", p.free_count, [count]), ("slots", p.slots, slots),
                                ("positions", p.positions, positions), ("sequences", p.sequences, sequences), ("table", server.table, table)):
            assert got.tolist() == want, (turn, name)
        assert server.free.tolist()[:count] == free[:count]
        # the places of the plan are those that the new keys and values went to
        kc, vc = server.kc.cpu(), server.vc.cpu()
        v = server.embed.cpu()[ids][:, HQ + HKV:]
        for r in range(cu[-1]):
            pg, off = divmod(slots[r], PAGE)
            assert torch.equal(vc[pg, :, off], v[r]), (turn, r)
            cached[slots[r]] = (kc[pg, :, off].clone(), vc[pg, :, off].clone())
        qr, o, lse = server.qr.cpu(), server.o.cpu(), server.lse.cpu()
        for s in range(nseq):
            n, L = cu[s + 1] - cu[s], kv[s]
            if n == 0:
                continue
            at = [table[s][j // PAGE] * PAGE + j % PAGE for j in range(L)]
            k, vv = (torch.stack([cached[x][i] for x in at]) for i in range(2))  # (what was put there, in any of the steps)
            for h in range(HQ):
                e = slice(cu[s], cu[s + 1])
                ref, rl, tol, tl = softmax_rows(qr[e, h], k[:, h // 2], vv[:, h // 2], torch.ones(L, dtype=torch.bool), L - n)
                off = (o[e, h].double() - ref).abs() - torch.finfo(BF16).eps / 2 * ref.abs() - tol[:, None]
                assert (off <= 0).all() and ((lse[h, e].double() - rl).abs() <= tl).all(), (turn, s, h)
        assert (o[cu[-1]:] == 7.0).all()
        # the step's own logits, of the rows that there are
        tokens, logs = plain_sample(server.logits.cpu(), u, server.temperature.cpu(), server.top_k.cpu(), server.top_p.cpu())
        assert server.token.tolist()[:cu[-1]] == tokens.tolist()[:cu[-1]], turn
        close = (server.logprob.cpu().double()[:cu[-1]] - logs.double()[:cu[-1]]).abs()
        assert (close <= 1e-6 + 2.0 ** -24 * 20).all()


@pytest.mark.parametrize("nseq,rows,most_new", [(1, 40, 40), (5, 90, 30), (70, 400, 6)])
def test_step_by_step(binding, nseq, rows, most_new):
    server = Server(binding, nseq, rows, 50 + nseq, most_new)
    _steps(server, server.step, 60)


def test_captured_step(binding):
    """The whole step as one graph, captured on another stream and replayed for prompts and single tokens alike, with eager work between the replays."""
    server, other = Server(binding, 5, 90, 70, 30), Server(binding, 5, 90, 71, 30)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        server.step()  # (nobody asks for anything: nothing changes)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        server.step()
    other.new.fill_(1)

    def run():
        other.step()
        graph.replay()
        other.step()
    _steps(server, run, 61)
    torch.cuda.synchronize()
    assert other.plan.kv_len.tolist() == [18] * 5


def test_two_captured_steps_side_by_side(binding):
    """Two graphs with their own workspaces, replayed on two streams at once."""
    servers = [Server(binding, 4, 60, 80 + i, 20) for i in range(2)]
    alone = [Server(binding, 4, 60, 80 + i, 20) for i in range(2)]
    graphs, streams = [], [torch.cuda.Stream() for _ in servers]
    for s in servers:
        s.step()
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            s.step()
    for s, a in zip(servers, alone):
        for x in (s, a):
            x.new.copy_(torch.tensor([3, 1, 5, 2], dtype=torch.int32))
            x.ids.copy_(torch.arange(60) % V)
            x.u.copy_(torch.linspace(0.01, 0.99, 60))
    torch.cuda.synchronize()
    for turn in range(12):
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
        for a in alone:
            a.step()
        torch.cuda.synchronize()
        for s, a in zip(servers, alone):
            n = int(a.plan.cu_seqlens[-1])
            assert n == 11 and torch.equal(s.plan.kv_len, a.plan.kv_len) and torch.equal(s.table, a.table)
            assert torch.equal(s.o[:n], a.o[:n]) and torch.equal(s.lse[:, :n], a.lse[:, :n])
            assert torch.equal(s.token[:n], a.token[:n]) and torch.equal(s.logprob[:n], a.logprob[:n])


def test_calls_follow_the_current_stream(binding):
    """Inputs that a stream's earlier work makes are there when its call runs."""
    s = Server(binding, 4, 60, 90, 20)
    ref = Server(binding, 4, 60, 90, 20)
    for x in (s, ref):
        x.ids.copy_(torch.arange(60) % V)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    busy = torch.zeros(4096, 4096, device="cuda")
    with torch.cuda.stream(side):
        for _ in range(10):
            busy = busy @ busy
        s.new.fill_(7)
        s.u.fill_(0.5)
        s.step()
    side.synchronize()
    ref.new.fill_(7)
    ref.u.fill_(0.5)
    ref.step()
    torch.cuda.synchronize()
    assert torch.equal(s.o[:28], ref.o[:28]) and torch.equal(s.token[:28], ref.token[:28]) and torch.equal(s.plan.slots, ref.plan.slots)
