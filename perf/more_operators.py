"""Workloads of a decode step around the paged key/value cache: the plan that gives new tokens their pages and places, softmax attention
over the cache (the limit alpha -> 1 of the entmax attention, for the heads and models that are compared with it), and sampling of the
next tokens from their logits.

`listed()` are the calls a serving loop makes; `draw(rng)` gives further ones of the same ranges.  A case is a dict, with "op":

  "plan"     pages for the new tokens of nseq sequences from a list of free pages, sequence offsets, lengths, and for every row of the
             step its place in the cache, its position and its sequence.  `prompts` sequences (all if negative) have new_lo .. new_hi new
             tokens, one in three of the others one and the rest none if `sparse`, else all of them one; keys_lo .. keys_hi keys are
             cached before.  `release`: share of the sequences that have ended and give their pages back; `pool`: free pages as a share
             of those that are asked for (below one: the last sequences get none); `rows`: rows of the step, as a share of the tokens
  "softmax"  attention of the new tokens over the cache (their own keys are in it), Hq query heads on Hkv key/value heads.  Lengths as
             above, keys counted with the new ones.  `cap`: scores s become cap tanh(s / cap), 0: as they are; scale, logn, nape: the
             adaptive scale and the distance bias of the entmax attention
  "sample"   tokens from `rows` rows of `vocab` logits.  `filters`: which of temperature (t), top-k (k), top-p (p) and min-p (m) are given;
             `spread`: standard deviation of the logits, `peaks`: tokens of a row that stand out, `banned`: share of the rows in which most
             tokens are -infinity
"""
import math
import random

import torch

own = False


def _plan(nseq, new, keys, prompts=0, sparse=False, release=0.0, pool=1.5, rows=1.0, page=16, seed=1, name=None):
    c = dict(op="plan", nseq=nseq, new_lo=new[0], new_hi=new[1], keys_lo=keys[0], keys_hi=keys[1], prompts=prompts, sparse=sparse,
             release=release, pool=pool, rows=rows, page=page, lens_seed=seed)
    return c if name is None else dict(c, name=name)


def _softmax(nseq, new, keys, Hq, Hkv, d, dtype="bf16", page=16, cap=0.0, scale="head", logn=0, nape=False, bias_mode=0, prompts=-1, causal=True,
             pad=0, seed=1, name=None):
    c = dict(op="softmax", nseq=nseq, new_lo=new[0], new_hi=new[1], keys_lo=keys[0], keys_hi=keys[1], prompts=prompts, sparse=False, Hq=Hq,
             Hkv=Hkv, d=d, dtype=dtype, page=page, cap=cap, scale=scale, logn=logn, nape=nape, bias_mode=bias_mode, causal=causal, pad=pad,
             lens_seed=seed)
    return c if name is None else dict(c, name=name)


def _sample(rows, vocab, dtype="bf16", filters="tkpm", spread=2.0, peaks=20, banned=0.0, seed=1, name=None):
    c = dict(op="sample", rows=rows, vocab=vocab, dtype=dtype, filters=filters, spread=spread, peaks=peaks, banned=banned, lens_seed=seed)
    return c if name is None else dict(c, name=name)


def listed():
    return [
        # a single user's next token: launch latency
        _plan(1, (1, 1), (700, 700), pool=9.0, name="plan_1_token"),
        # a decode step of a busy server, a few sequences have ended
        _plan(256, (1, 1), (100, 8000), release=0.05, page=32, pool=20.0, name="plan_decode_256"),
        # a step that takes in prompts beside the decode steps of many others, until the pages run out
        _plan(3000, (20, 2000), (1, 6000), prompts=400, sparse=True, release=0.02, pool=0.9, rows=1.02, page=16, name="plan_prompts"),
        # a single user's next token
        _softmax(1, (1, 1), (901, 901), 12, 4, 64, name="softmax_1_of_901"),
        # a decode step of a batch, caches of all ages
        _softmax(48, (1, 1), (150, 9000), 16, 2, 128, page=32, scale="none", name="softmax_batch_48"),
        # one new token against long caches
        _softmax(2, (1, 1), (65536, 65536), 16, 4, 128, page=64, name="softmax_1_of_65536"),
        # drafted tokens, capped scores, distance bias on half of the heads, scales from the tokens, in fp32
        _softmax(12, (3, 3), (1000, 6001), 12, 4, 64, dtype="fp32", page=32, cap=30.0, scale="query", logn=1, nape=True, bias_mode=1,
                 name="softmax_3_capped_fp32"),
        # the next chunk of long prompts
        _softmax(4, (700, 700), (2000, 12000), 16, 4, 128, page=64, name="softmax_chunk_700"),
        # a single user's next token: latency
        _sample(1, 50021, filters="tkp", name="sample_1_of_50021"),
        # a batch whose users ask for different things
        _sample(64, 131072, filters="tkpm", banned=0.1, name="sample_64_mixed"),
        # rollouts that follow the model's own distribution
        _sample(256, 32768, dtype="fp32", filters="t", name="sample_256_plain_fp32"),
        # a flat distribution, from which top-p keeps much: early training, high temperatures
        _sample(16, 200003, dtype="fp32", filters="tp", spread=0.7, peaks=0, name="sample_16_flat_fp32"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["plan", "softmax", "softmax", "sample"])
    seed = rng.randint(1, 10 ** 6)
    if op == "plan":
        nseq = _log_int(rng, 1, 3000)
        prompts = rng.choice([0, 0, rng.randint(0, min(nseq, 300))])
        hi = _log_int(rng, 2, 2000)
        return _plan(nseq, (max(1, hi // 30), hi), (1, _log_int(rng, 20, 8000)), prompts=prompts, sparse=rng.random() < 0.5,
                     release=rng.choice([0.0, 0.05, 0.5]), pool=rng.choice([0.5, 0.9, 1.5, 20.0]), rows=rng.choice([1.0, 1.0, 1.3, 0.8]),
                     page=rng.choice([16, 32, 64, 128]), seed=seed)
    if op == "sample":
        vocab = _log_int(rng, 200, 200003)
        rows = _log_int(rng, 1, max(1, min(256, 8 * 2 ** 20 // vocab)))
        return _sample(rows, vocab, rng.choice(["bf16", "bf16", "fp32"]), rng.choice(["", "t", "tk", "tp", "tm", "tkp", "kp", "tkpm", "tkpm"]),
                       spread=rng.uniform(0.5, 4.0), peaks=rng.choice([0, 3, 20]), banned=rng.choice([0.0, 0.0, 0.3]), seed=seed)
    Hq, Hkv, d = rng.choice([(12, 4, 64), (12, 12, 64), (8, 2, 64), (16, 4, 128), (16, 2, 128), (16, 16, 128)])
    dtype = "fp32" if rng.random() < 0.25 else "bf16"
    kw = dict(dtype=dtype, page=rng.choice([16, 32, 64, 128]), cap=rng.choice([0.0, 0.0, 30.0, rng.uniform(5.0, 60.0)]),
              scale=rng.choice(["none", "head", "head", "query"]), logn=rng.choice([0, 1]), nape=rng.random() < 0.3,
              bias_mode=rng.choice([0, 1]), pad=rng.choice([0, 0, 1, 65]), seed=seed)
    kind = rng.choice(["one", "one", "few", "chunk", "mixed"])
    hi = _log_int(rng, 30, 65536)
    lo = max(1, hi // rng.choice([1, 4, 40]))
    if kind in ("one", "few"):
        # keys and values of all sequences: at most those of the longest listed caches
        most = 2 * 65536 * 4 * 128 // (hi * Hkv * d * (2 if dtype == "fp32" else 1))
        hi = hi if most else 16384
        nseq = _log_int(rng, 1, max(1, min(64, most)))
        return _softmax(nseq, (1, 1) if kind == "one" else (1, rng.randint(2, 16)), (min(lo, hi), hi), Hq, Hkv, d, **kw)
    hi = min(hi, 12000 if dtype == "bf16" else 3000) if kind == "chunk" else min(hi, 6000 if dtype == "bf16" else 3000)
    lo = min(lo, hi)
    n = _log_int(rng, 20, 700)
    most = max(1, 2 * 65536 * 4 * 128 // (max(hi, n) * Hkv * d * (2 if dtype == "fp32" else 1)))
    if kind == "chunk":
        nseq = rng.randint(1, max(1, min(4, 1400 // (n * (2 if Hkv * d > 1024 else 1)), most)))
        return _softmax(nseq, (max(1, n // 2), n), (lo, hi), Hq, Hkv, d, causal=rng.random() < 0.85, **kw)
    return _softmax(rng.randint(3, max(3, min(24, most))), (max(1, n // 2), n), (lo, hi), Hq, Hkv, d, prompts=rng.randint(1, 2), **kw)


def _lengths(case):
    """New tokens and keys of every sequence; the keys with the new ones, "plan": before them."""
    rng = random.Random(case["lens_seed"])
    new, keys = [], []
    for s in range(case["nseq"]):
        prompt = case["prompts"] < 0 or s < case["prompts"]
        n = _log_int(rng, case["new_lo"], case["new_hi"]) if prompt else (1 if not case["sparse"] or rng.random() < 0.33 else 0)
        L = _log_int(rng, case["keys_lo"], case["keys_hi"])
        new.append(n)
        keys.append(L if case["op"] == "plan" else max(n, L))
    order = list(range(case["nseq"]))
    rng.shuffle(order)
    return [new[i] for i in order], [keys[i] for i in order]


def _plan_sizes(case):
    """(new, keys, released, rows, pages of a table's row, free pages) of a plan case."""
    new, keys = _lengths(case)
    rng = random.Random(case["lens_seed"] + 1)
    page = case["page"]
    released = [rng.random() < case["release"] for _ in new]
    new = [0 if r else n for n, r in zip(new, released)]  # (a place that has just become free is given away a step later)
    need = sum(-(-(L + n) // page) - -(-L // page) for n, L in zip(new, keys))
    rows = max(1, int(sum(new) * case["rows"]))
    return new, keys, released, rows, max(-(-(L + n) // page) for n, L in zip(new, keys)) + 1, int(need * case["pool"]) + 1


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(int(seed))
    normal = lambda *s: torch.randn(*s, generator=gen, device=dev)  # noqa: E731
    uniform = lambda *s: torch.rand(*s, generator=gen, device=dev)  # noqa: E731
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=dev)  # noqa: E731
    s = {"case": case}

    def tables(keys, columns, extra, page):
        """A table of distinct random pages for the keys, and the pages that are left."""
        per = [-(-k // page) for k in keys]
        perm = torch.randperm(sum(per) + extra, generator=gen, device=dev).to(torch.int32)
        # the entries of sequence i are perm[first[i] : first[i] + per[i]]; those behind them are nobody's
        first, at = [], 0
        for n in per:
            first.append(at)
            at += n
        col = torch.arange(columns, device=dev)[None]
        per_t, first_t = ints(per)[:, None], ints(first)[:, None]
        return torch.where(col < per_t, perm[(first_t + col.clamp(max=max(per))).clamp(max=perm.shape[0] - 1).long()], -1).to(torch.int32), perm[at:]

    if case["op"] == "plan":
        new, keys, released, rows, columns, free = _plan_sizes(case)
        table, spare = tables(keys, columns, free, case["page"])
        pages = sum(-(-k // case["page"]) for k in keys) + free
        s.update(new=ints(new), kv_len=ints(keys), release=ints([int(r) for r in released]), table=table.contiguous(), rows=rows)
        s["free"] = torch.full((pages,), -1, dtype=torch.int32, device=dev)
        s["free"][:free] = spare
        s["count"] = ints([free])
        if own:
            from paper_2506_16640_amd import binding
            s["plan"] = binding.new_plan(len(new), rows, dev)
        return s
    tdt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    if case["op"] == "sample":
        R, V, f = case["rows"], case["vocab"], case["filters"]
        x = normal(R, V) * case["spread"]
        if case["peaks"]:
            at = torch.randint(V, (R, case["peaks"]), generator=gen, device=dev)
            x.scatter_add_(1, at, 3.0 * case["spread"] * uniform(R, case["peaks"]) + 2.0)
        if case["banned"]:  # a grammar that lets through one token in fifty
            x = x.masked_fill((uniform(R, 1) < case["banned"]) & (uniform(R, V) > 0.02), -math.inf)
        s["logits"], s["u"] = x.to(tdt), uniform(R)
        pick = lambda values, t: values[torch.randint(values.shape[0], (R,), generator=gen, device=dev)].to(t).contiguous()  # noqa: E731
        floats = lambda v: torch.tensor(v, device=dev)  # noqa: E731
        mixed = "k" in f  # (users who ask for different things; some for nothing, some for the best token)
        s["kw"] = dict(
            temperature=None if "t" not in f else (pick(floats([0.0, 0.3, 0.7, 1.0, 1.0, 1.3]), torch.float32) if mixed else 0.7 + 0.6 * uniform(R)),
            top_k=pick(ints([0, 1, 20, 40, 50, 1000]), torch.int32) if "k" in f else None,
            top_p=None if "p" not in f else (pick(floats([1.0, 0.5, 0.9, 0.95]), torch.float32) if mixed else 0.9 + 0.09 * uniform(R)),
            min_p=pick(floats([0.0, 0.02, 0.05, 0.1]), torch.float32) if "m" in f else None)
        if own:
            from paper_2506_16640_amd import binding
            s["token"] = torch.zeros(R, dtype=torch.int32, device=dev)
            s["logprob"] = torch.zeros(R, device=dev)
            s["workspace"] = binding.new_sample_workspace(s["logits"])
        return s
    Hq, Hkv, d, page = (case[x] for x in ("Hq", "Hkv", "d", "page"))
    new, keys = _lengths(case)
    T = sum(new) + case["pad"]
    cu = [0]
    for n in new:
        cu.append(cu[-1] + n)
    s.update(new=new, keys=keys, cu_list=cu, cu=ints(cu), kv_len=ints(keys), q=normal(T, Hq, d).to(tdt))
    s["table"], _ = tables(keys, -(-max(keys) // page), 3, page)
    s["table"] = s["table"].contiguous()
    pages = sum(-(-k // page) for k in keys) + 3
    s["kc"], s["vc"] = normal(pages, Hkv, page, d).to(tdt), normal(pages, Hkv, page, d).to(tdt)
    s["out"], s["lse"] = torch.zeros_like(s["q"]), torch.zeros(Hq, T, device=dev)  # (the rows behind the last sequence stay as they are)
    beta = gamma = slopes = None
    if case["scale"] == "head":
        beta, gamma = 0.3 + 0.5 * uniform(Hq), 0.5 + 0.5 * uniform(Hq)
    elif case["scale"] == "query":
        beta, gamma = 0.3 + 0.5 * uniform(Hq, T), 0.5 + 0.5 * uniform(Hq, T)
    if case["nape"]:
        biased = Hq // 2  # every other head, slopes 2^(-k / biased)
        slopes = torch.zeros(Hq, device=dev)
        slopes[1::2] = torch.tensor([2.0 ** (-k / biased) for k in range(1, biased + 1)], device=dev)
    s["kw"] = dict(cap=case["cap"], beta=beta, gamma=gamma, delta=1.0, causal=case["causal"], logn_mode=case["logn"], alibi_slopes=slopes,
                   bias_mode=case["bias_mode"])
    s["most"] = (max(new), max(keys))
    if own:
        from paper_2506_16640_amd import binding
        s["workspace"] = binding.new_softmax_workspace(s["q"], s["kc"], s["table"], max_new=s["most"][0], max_keys=s["most"][1])
    return s


def run(s):
    op = s["case"]["op"]
    if own:
        from paper_2506_16640_amd import binding
        if op == "plan":
            p = binding.cache_plan(s["new"], s["kv_len"], s["table"], s["free"], s["count"], s["case"]["page"], s["plan"], release=s["release"])
            return p.cu_seqlens, p.kv_len, s["table"], s["free"], p.free_count, p.slots, p.positions, p.sequences
        if op == "softmax":
            binding.paged_softmax_fwd(s["q"], s["kc"], s["vc"], s["cu"], s["kv_len"], s["table"], max_new=s["most"][0], max_keys=s["most"][1],
                                      out=s["out"], lse=s["lse"], workspace=s["workspace"], **s["kw"])
            return s["out"], s["lse"]
        binding.sample(s["logits"], s["u"], token=s["token"], logprob=s["logprob"], workspace=s["workspace"], **s["kw"])
        return s["token"], s["logprob"]
    return {"plan": _plain_plan, "softmax": _plain_softmax, "sample": _plain_sample}[op](s)


# ----------------------------------------------------------------- the plain forms

def _plain_plan(s):
    page, table, free, rows = s["case"]["page"], s["table"], s["free"], s["rows"]
    nseq, columns = table.shape
    num_pages = free.shape[0]
    L, new = s["kv_len"].long(), s["new"].long().clamp(min=0)
    # the pages of the sequences that have ended go on top of the free ones, in their order
    gone = s["release"] != 0
    col = torch.arange(columns, device="cuda")
    back = table[gone[:, None] & (col[None] < ((L + page - 1) // page)[:, None]) & (table >= 0) & (table < num_pages)]
    count = s["count"].long()
    free[count + torch.arange(back.shape[0], device="cuda")] = back
    count = count + back.shape[0]
    L = torch.where(gone, 0, L)
    # who gets pages: all before whom, and for whom, they suffice, and whose tokens fit the rows of the step
    new = torch.where(L + new <= columns * page, new, 0)
    have = (L + page - 1) // page
    need = (L + new + page - 1) // page - have
    new = torch.where((need == 0) | (need.cumsum(0) <= count), new, 0)
    new = torch.where(new.cumsum(0) <= rows, new, 0)
    need = (L + new + page - 1) // page - have
    cu = torch.cat([torch.zeros(1, dtype=torch.int64, device="cuda"), new.cumsum(0)])
    # every row's sequence and position; the pages are taken from the top of the free ones
    row = torch.arange(rows, device="cuda")
    seq = (row[:, None] >= cu[None, 1:]).sum(1) if rows * nseq <= 2 ** 24 else torch.bucketize(row, cu[1:], right=True)
    there = seq < nseq
    at = seq.clamp(max=nseq - 1)
    pos = L[at] + row - cu[at]
    first = need.cumsum(0) - need
    where = (pos // page).clamp(0, columns - 1)
    fresh = there & (where >= have[at])
    number = torch.where(fresh, free[(count - 1 - (first[at] + where - have[at])).clamp(0, num_pages - 1)], 0)
    table[at[fresh], where[fresh]] = number[fresh]
    got = table[at, where].long()
    slots = torch.where(there & (got >= 0) & (got < num_pages), got * page + pos % page, -1)
    i32 = lambda x: x.to(torch.int32)  # noqa: E731
    return (i32(cu), i32(L + new), table, free, i32(count - need.sum()), slots, i32(torch.where(there, pos, -1)), i32(torch.where(there, seq, -1)))


def _plain_softmax(s):
    c, kw = s["case"], s["kw"]
    Hq, Hkv, d, page, cap = c["Hq"], c["Hkv"], c["d"], c["page"], kw["cap"]
    G = Hq // Hkv
    for i, (n, L) in enumerate(zip(s["new"], s["keys"])):
        number = s["table"][i, :(L + page - 1) // page].long()
        k, v = (x[number].transpose(0, 1).reshape(Hkv, -1, d)[:, :L].float() for x in (s["kc"], s["vc"]))
        step = max(1, 2 ** 27 // (Hq * L))
        for t0 in range(0, n, step):
            m = min(step, n - t0)
            row = s["cu_list"][i] + t0
            q = s["q"][row:row + m].float().reshape(m, Hkv, G, d).permute(1, 2, 0, 3).reshape(Hkv, G * m, d)
            z = torch.matmul(q, k.transpose(1, 2).contiguous()).reshape(Hkv, G, m, L) / math.sqrt(d)
            pos = torch.arange(L - n + t0, L - n + t0 + m, device="cuda")
            key = torch.arange(L, device="cuda")
            seen = (key[None] <= pos[:, None]) if c["causal"] else torch.ones(m, L, dtype=torch.bool, device="cuda")
            bias = 0.0
            if kw["alibi_slopes"] is not None:
                bias = -kw["alibi_slopes"].reshape(Hkv, G, 1, 1) * (pos[:, None] - key[None]).clamp(min=0).float()
            scale = torch.full((Hkv, G, m, 1), kw["delta"], device="cuda")
            if kw["beta"] is not None:
                b, g = ((x[:, row:row + m] if x.dim() == 2 else x[:, None].expand(-1, m)).reshape(Hkv, G, m, 1) for x in (kw["beta"], kw["gamma"]))
                cnt = seen.sum(1).float() if c["logn"] else torch.full((m,), float(L), device="cuda")
                scale = scale + torch.where(cnt[:, None] > 1, b * torch.log(cnt)[:, None] ** g, torch.zeros_like(b))
            x = scale * (z + bias) if c["bias_mode"] == 0 else scale * z
            x = cap * torch.tanh(x / cap) if cap > 0 else x
            x = x + bias if c["bias_mode"] == 1 else x
            x = x.masked_fill(~seen, -math.inf)
            top = x.amax(-1, keepdim=True)
            p = torch.exp(x - top)
            total = p.sum(-1, keepdim=True)
            o = torch.matmul((p / total).reshape(Hkv, G * m, L), v)
            s["out"][row:row + m] = o.reshape(Hkv, G, m, d).permute(2, 0, 1, 3).reshape(m, Hq, d).to(s["out"].dtype)
            s["lse"][:, row:row + m] = (top + torch.log(total)).reshape(Hq, m)
    return s["out"], s["lse"]


def _plain_sample(s):
    kw = s["kw"]
    x = s["logits"].double()  # (64 bits: which token a number falls on is decided next to borders)
    R, V = x.shape
    column = lambda t, off: torch.full((R, 1), off, dtype=torch.float64, device="cuda") if t is None else t.double()[:, None]  # noqa: E731
    t = column(kw["temperature"], 1.0)
    order = torch.sort(x, dim=1, descending=True, stable=True).indices  # (equal ones: the lowest index first)
    best = order[:, :1]
    top = x.gather(1, best)
    w = torch.exp((x - top) / torch.where(t > 0, t, 1.0))
    ranked = w.gather(1, order)
    rank = torch.arange(V, device="cuda")[None]
    keep = torch.ones(R, V, dtype=torch.bool, device="cuda")
    if kw["top_k"] is not None:
        k = kw["top_k"].long()[:, None]
        keep &= (k <= 0) | (rank < k)
    if kw["top_p"] is not None:
        p = column(kw["top_p"], 1.0)
        before = ranked.cumsum(1) - ranked
        total = (ranked * keep).sum(1, keepdim=True)
        keep &= (p >= 1) | (before < p * total) | (rank == 0)
    if kw["min_p"] is not None:
        keep &= ranked >= column(kw["min_p"], 0.0).clamp(max=1.0)
    kept = torch.zeros_like(keep).scatter(1, order, keep) & (w > 0)
    mass = torch.where(kept, w, 0.0)
    sums = mass.cumsum(1)
    total = sums[:, -1:]
    last = V - 1 - kept.flip(1).long().argmax(1)
    token = torch.minimum((sums <= s["u"].double()[:, None] * total).sum(1), last)[:, None]
    logprob = torch.log(w.gather(1, token) / total)
    greedy = t <= 0
    return torch.where(greedy, best, token)[:, 0].to(torch.int32), torch.where(greedy, 0.0, logprob)[:, 0].float()


# ----------------------------------------------------------------- what cannot be left out

def work(case):
    if case["op"] == "plan":
        new, keys, released, rows, _, _ = _plan_sizes(case)
        page = case["page"]
        need = sum(-(-(L + n) // page) - -(-L // page) for n, L in zip(new, keys))
        back = sum(-(-L // page) for L, r in zip(keys, released) if r)
        # three numbers a sequence in, two out; pages given: out of the list and into the table, given back: the reverse; for every row its
        # place, position and sequence, and the page that its sequence's last one was on
        return {"bytes": 20 * len(new) + 12 + 8 * need + 8 * back + 16 * rows + 4 * sum(1 for n in new if n), "flops": 0.0}
    if case["op"] == "sample":
        eb = 2 if case["dtype"] == "bf16" else 4
        n = case["rows"] * case["vocab"]
        # the logits once, four parameters and a number in, a token and its logarithm out; a difference, a product and an exponential each
        return {"bytes": eb * n + 4 * case["rows"] * (3 + len(case["filters"])), "flops": 4.0 * n}
    new, keys = _lengths(case)
    eb = 2 if case["dtype"] == "bf16" else 4
    Hq, Hkv, d = case["Hq"], case["Hkv"], case["d"]
    T = sum(new)
    pairs = float(Hq) * sum(n * (L - n) + n * (n + 1) / 2.0 if case["causal"] else float(n) * L for n, L in zip(new, keys))
    return {"bytes": eb * d * (2 * Hq * T + 2 * Hkv * sum(keys)) + 4 * Hq * T, "flops": 4.0 * d * pairs}


# ----------------------------------------------------------------- the definitions in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    return {"plan": _exact_plan, "softmax": _exact_softmax, "sample": _exact_sample}[case["op"]](s)


def _exact_plan(s):
    """One sequence after the other, one page after the other."""
    page = s["case"]["page"]
    new, kv, gone, table, free = (s[x].tolist() for x in ("new", "kv_len", "release", "table", "free"))
    rows, room = s["rows"], len(table[0]) * page
    top = s["count"].item()
    for i in range(len(kv)):
        if gone[i]:
            for e in range((kv[i] + page - 1) // page):
                free[top] = table[i][e]
                top += 1
            kv[i] = 0
    cu, slots, positions, sequences = [0], [], [], []
    asked = left = top
    closed = False
    for i, n in enumerate(new):
        if kv[i] + n > room:
            n = 0
        need = sum(1 for p in range(kv[i], kv[i] + n) if p % page == 0)
        asked -= need
        if need and asked < 0:
            n = 0
        closed = closed or len(slots) + n > rows
        if n and closed:
            n = 0
        for p in range(kv[i], kv[i] + n):
            if p % page == 0:
                left -= 1
                table[i][p // page] = free[left]
            slots.append(table[i][p // page] * page + p % page)
            positions.append(p)
            sequences.append(i)
        kv[i] += n
        cu.append(len(slots))
    pad = [-1] * (rows - len(slots))
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    return (ints(cu), ints(kv), ints(table), ints(free), ints([left]), torch.tensor(slots + pad, dtype=torch.int64, device="cuda"),
            ints(positions + pad), ints(sequences + pad))


def _exact_softmax(s):
    case, kw = s["case"], s["kw"]
    new, keys, cu = s["new"], s["keys"], s["cu_list"]
    Hq, Hkv, d, page, cap = (case[x] for x in ("Hq", "Hkv", "d", "page", "cap"))
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["lse"].shape, dtype=torch.float64, device="cuda")
    table = s["table"].cpu()
    for i in range(case["nseq"]):
        n, L = new[i], keys[i]
        pages = table[i, :(L + page - 1) // page].tolist()
        for h in range(Hq):
            hk = h // (Hq // Hkv)
            k, v = (x[pages, hk].reshape(-1, d)[:L].double() for x in (s["kc"], s["vc"]))
            step = max(1, 2 ** 25 // L)
            for t0 in range(0, n, step):
                rows = torch.arange(t0, min(n, t0 + step), device="cuda")
                at = cu[i] + rows
                seen_to = rows + (L - n) if case["causal"] else torch.full_like(rows, L - 1)  # last key of a row
                y = s["q"][at, h].double() @ k.T / d ** 0.5
                slope = 0.0 if kw["alibi_slopes"] is None else float(kw["alibi_slopes"][h])
                dist = ((rows + (L - n))[:, None] - torch.arange(L, device="cuda")[None]).clamp(min=0).double()
                mult = torch.full((len(rows),), float(kw["delta"]), dtype=torch.float64, device="cuda")
                if kw["beta"] is not None:
                    b, g = (x[h, at].double() if x.dim() == 2 else x[h].double() for x in (kw["beta"], kw["gamma"]))
                    count = (seen_to + 1).double() if case["logn"] else torch.full_like(mult, float(L))
                    mult = mult + torch.where(count > 1, b * count.log() ** g, 0.0)
                y = mult[:, None] * (y - slope * dist if case["bias_mode"] == 0 else y)
                if cap > 0:
                    y = cap * (y / cap).tanh()
                if case["bias_mode"] == 1:
                    y = y - slope * dist
                y[torch.arange(L, device="cuda")[None] > seen_to[:, None]] = -math.inf
                total = y.logsumexp(1)
                lse[h, at] = total
                out[at, h] = (y - total[:, None]).exp() @ v
    return out, lse


def _exact_sample(s):
    """Row by row: tokens are taken by falling logit until a filter says enough."""
    R, V = s["logits"].shape
    given = lambda name, off: [off] * R if s["kw"][name] is None else s["kw"][name].tolist()  # noqa: E731
    tokens, logs = [], []
    for r, (t, k, p, m, u) in enumerate(zip(given("temperature", 1.0), given("top_k", 0), given("top_p", 1.0), given("min_p", 0.0), s["u"].tolist())):
        x = s["logits"][r].double()
        if t <= 0:
            tokens.append(int((x == x.max()).nonzero()[0, 0]))
            logs.append(0.0)
            continue
        value, index = torch.sort(-x, stable=True)
        z = (value[0] - value) / t
        n = min(k, V) if k > 0 else V
        prob = z[:n].exp() / z[:n].exp().sum()
        if p < 1:
            n = max(1, int((prob.cumsum(0) - prob < p).sum()))
        if m > 0:
            n = min(n, int((z[:n].exp() >= min(m, 1.0)).sum()))
        n = min(n, int((z > -math.inf).sum()))
        kept, at = index[:n].sort()
        prob = z[:n][at].exp()
        sums = prob.cumsum(0)
        e = min(int((sums <= u * sums[-1]).sum()), n - 1)
        tokens.append(int(kept[e]))
        logs.append(math.log(float(prob[e] / sums[-1])))
    return torch.tensor(tokens, dtype=torch.int32, device="cuda"), torch.tensor(logs, dtype=torch.float64, device="cuda")
