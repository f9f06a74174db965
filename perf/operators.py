"""Workloads of the serving operators: appending to a paged key/value cache, entmax attention of a chunk of new tokens over that
cache, and entmax attention over packed prompts; all with grouped heads (Hq query heads share Hkv key/value heads).

`listed()` are the calls a serving loop makes, from one token of one sequence to prompts of thousands of tokens; `draw(rng)`
gives further ones of the same ranges.  A case is a dict:

  op         "append": rotate the new tokens' queries and keys, write keys and values to their pages; "paged": attention of the
             new tokens over the cache (their own keys are in it); "packed": attention of whole prompts, keys and values packed
             like the queries
  nseq new_lo new_hi keys_lo keys_hi chunks lens_seed
             the lengths: `chunks` sequences (all of them if negative) have new_lo .. new_hi new tokens, the others one; a
             sequence has keys_lo .. keys_hi keys, at least as many as new tokens ("packed": as many)
  pad        rows of Q behind the last sequence's
  Hq Hkv d dtype page alpha causal
  scale      "none": logits / sqrt(d); "head": beta, gamma per head ~ U(0.5, 1.5), delta = 1; "query": the same per token and head;
             "dense": beta per head ~ U(0.5, 1.5), gamma = -1/2, delta = 0 (rows keep most of their keys)
  logn       0: n in (ln n)^gamma is the sequence's number of keys, 1: the number of keys the row sees
  nape       every other head carries the linear distance bias
  rot        features of a head that are rotated (append); interleaved: neighbouring features are a pair, else i and i + rot / 2
"""
import math
import random

import torch

own = False


def _case(op, nseq, new, keys, Hq, Hkv, d, dtype="bf16", page=16, alpha=1.5, causal=True, scale="head", logn=0, nape=False, chunks=-1,
          pad=0, rot=0, interleaved=False, lens_seed=1, name=None):
    c = dict(op=op, nseq=nseq, new_lo=new[0], new_hi=new[1], keys_lo=keys[0], keys_hi=keys[1], chunks=chunks, lens_seed=lens_seed, pad=pad,
             Hq=Hq, Hkv=Hkv, d=d, dtype=dtype, page=page, alpha=alpha, causal=causal, scale=scale, logn=logn, nape=nape, rot=rot,
             interleaved=interleaved)
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # a single user's next token: launch latency
        _case("append", 1, (1, 1), (700, 700), 12, 4, 64, rot=64, name="append_1_token"),
        # one decode step of a batch, caches of all ages
        _case("append", 64, (1, 1), (100, 2000), 16, 4, 128, page=32, rot=128, name="append_decode_64"),
        # prompts of a busy scheduler's step, padded to a bucket of rows; half of the features rotated, in neighbouring pairs
        _case("append", 24, (40, 2000), (40, 2000), 16, 4, 128, page=64, rot=64, interleaved=True, pad=100, name="append_prompts"),
        # a single user's next token in fp32, every head with its own keys
        _case("paged", 1, (1, 1), (1001, 1001), 12, 12, 64, dtype="fp32", name="decode_1_of_1001_fp32"),
        # one decode step of a batch, caches of all ages
        _case("paged", 64, (1, 1), (200, 8192), 16, 2, 128, name="decode_batch_64"),
        # one new token against long caches
        _case("paged", 4, (1, 1), (32768, 32768), 12, 4, 64, page=64, name="decode_1_of_32768_grouped"),
        # a few drafted tokens per sequence, scales from the tokens, half of the heads with the distance bias
        _case("paged", 16, (5, 5), (2500, 7000), 16, 4, 128, page=32, scale="query", logn=1, nape=True, name="decode_5_nape"),
        # a decode step whose rows keep most of their keys
        _case("paged", 8, (1, 1), (8192, 16384), 16, 4, 128, scale="dense", name="decode_dense"),
        # the next chunk of long prompts
        _case("paged", 4, (512, 512), (2000, 16384), 16, 4, 128, page=64, name="chunk_512"),
        # chunks of some prompts among the decode steps of other sequences, longer supports
        _case("paged", 32, (300, 900), (900, 6000), 12, 4, 64, alpha=1.25, chunks=4, pad=37, name="mixed_alpha1.25"),
        # whole prompts of a 12-head model
        _case("packed", 10, (100, 4096), (0, 0), 12, 4, 64, name="packed_prompts"),
        # whole prompts whose logits carry no scale: supports of tens to hundreds of keys
        _case("packed", 6, (300, 2000), (0, 0), 16, 4, 128, scale="none", name="packed_no_scale"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["append", "paged", "paged", "paged", "packed", "packed"])
    Hq, Hkv, d = rng.choice([(12, 4, 64), (12, 12, 64), (8, 2, 64), (16, 4, 128), (16, 2, 128), (16, 16, 128)])
    dtype = "fp32" if rng.random() < 0.2 else "bf16"
    page = rng.choice([16, 32, 64, 128])
    seed = rng.randint(1, 10 ** 6)
    pad = rng.choice([0, 0, 1, 65])
    if op == "append":
        nseq = _log_int(rng, 1, 64)
        hi = _log_int(rng, 1, 2000) if rng.random() < 0.6 else 1
        hi = max(1, min(hi, 20000 // nseq))
        rot = rng.choice([d, d, d // 2, 0])
        return _case("append", nseq, (max(1, hi // 20), hi), (hi, max(hi, 2000)), Hq, Hkv, d, dtype, page, rot=rot,
                     interleaved=rng.random() < 0.5, pad=pad, lens_seed=seed)
    alpha = rng.choice([1.5, 1.5, 1.25, 2.0, 1.7])
    scale = rng.choice(["head", "head", "head", "query", "none", "dense"])
    kw = dict(dtype=dtype, page=page, alpha=alpha, scale=scale, logn=rng.choice([0, 1]), nape=rng.random() < 0.2, pad=pad, lens_seed=seed)
    heavy = 4 if scale in ("none", "dense") or alpha < 1.5 or dtype == "fp32" else 1
    if op == "packed":
        hi = _log_int(rng, 30, 4096 // heavy)
        nseq = rng.randint(1, max(1, min(12, 12000 // (heavy * hi))))
        return _case("packed", nseq, (max(1, hi // 30), hi), (0, 0), Hq, Hkv, d, causal=rng.random() < 0.85, **kw)
    kind = rng.choice(["one", "one", "few", "chunk", "mixed"])
    hi = _log_int(rng, 300, 32768)
    lo = max(1, hi // rng.choice([1, 4, 40]))
    if kind in ("one", "few"):
        nseq = rng.randint(1, max(1, min(64, 64 * 4096 // (hi * Hkv * d // 256))))
        new = (1, 1) if kind == "one" else (1, rng.randint(2, 16))
        return _case("paged", nseq, new, (lo, hi), Hq, Hkv, d, **kw)
    hi = min(hi, 16384 // heavy)
    lo = min(lo, hi)
    n = _log_int(rng, 20, 900)
    if kind == "chunk":
        return _case("paged", rng.randint(1, max(1, min(4, 2000 // (n * heavy)))), (max(1, n // 2), n), (lo, hi), Hq, Hkv, d, **kw)
    return _case("paged", rng.randint(5, 24), (max(1, n // 2), n), (lo, min(hi, 6000)), Hq, Hkv, d, chunks=rng.randint(1, 2), **kw)


def _lengths(case):
    """New tokens and keys of every sequence."""
    rng = random.Random(case["lens_seed"])
    new, keys = [], []
    for s in range(case["nseq"]):
        chunk = case["chunks"] < 0 or s < case["chunks"]
        n = _log_int(rng, case["new_lo"], case["new_hi"]) if chunk else 1
        new.append(n)
        keys.append(n if case["op"] == "packed" else max(n, _log_int(rng, case["keys_lo"], case["keys_hi"])))
    order = list(range(case["nseq"]))
    rng.shuffle(order)  # (chunks and decode steps come in any order)
    return [new[i] for i in order], [keys[i] for i in order]


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(int(seed))
    normal = lambda *s: torch.randn(*s, generator=gen, device=dev)  # noqa: E731
    uniform = lambda *s: 0.5 + torch.rand(*s, generator=gen, device=dev)  # noqa: E731
    tdt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    Hq, Hkv, d, page = (case[x] for x in ("Hq", "Hkv", "d", "page"))
    new, keys = _lengths(case)
    T = sum(new) + case["pad"]
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=dev)  # noqa: E731
    cu = [0]
    for n in new:
        cu.append(cu[-1] + n)
    s = {"case": case, "new": new, "keys": keys, "cu_list": cu, "cu": ints(cu), "kv_len": ints(keys), "q": normal(T, Hq, d).to(tdt)}
    if case["op"] != "packed":
        per = [(k + page - 1) // page for k in keys]
        pages = sum(per) + 3
        s["table"] = torch.zeros(case["nseq"], max(per), dtype=torch.int32, device=dev)
        perm = torch.randperm(pages, generator=gen, device=dev).to(torch.int32)
        at = 0
        for i, n in enumerate(per):
            s["table"][i, :n] = perm[at:at + n]
            at += n
        s["table_list"] = s["table"].long().cpu()
        s["kc"], s["vc"] = normal(pages, Hkv, page, d).to(tdt), normal(pages, Hkv, page, d).to(tdt)
    if case["op"] != "paged":
        s["k"], s["v"] = normal(T, Hkv, d).to(tdt), normal(T, Hkv, d).to(tdt)
    s["out"] = torch.zeros_like(s["q"])  # (the rows behind the last sequence stay as they are)
    if case["op"] == "append":
        rot = case["rot"]
        s["inv_freq"] = (10000.0 ** (-torch.arange(0, rot, 2, device=dev, dtype=torch.float64) / max(rot, 1))).float() if rot else None
        return s
    beta = gamma = slopes = None
    delta = 1.0
    if case["scale"] == "head":
        beta, gamma = uniform(Hq), uniform(Hq)
    elif case["scale"] == "query":
        beta, gamma = uniform(Hq, T), uniform(Hq, T)
    elif case["scale"] == "dense":
        beta, gamma, delta = uniform(Hq), torch.full((Hq,), -0.5, device=dev), 0.0
    if case["nape"]:
        biased = Hq // 2  # every other head, slopes 2^(-k / biased)
        slopes = torch.zeros(Hq, device=dev)
        slopes[1::2] = torch.tensor([2.0 ** (-k / biased) for k in range(1, biased + 1)], device=dev)
    s["kw"] = dict(alpha=case["alpha"], beta=beta, gamma=gamma, delta=delta, causal=case["causal"], logn_mode=case["logn"], alibi_slopes=slopes)
    s["most"] = (max(new), max(keys))
    if own:
        from paper_2506_16640_amd import binding
        if case["op"] == "paged":
            s["workspace"] = binding.new_paged_workspace(s["q"], s["kc"], s["table"], max_new=s["most"][0], max_keys=s["most"][1])
        else:
            s["workspace"] = binding.new_packed_workspace(s["q"], s["k"], s["cu"], max_len=s["most"][0])
    return s


def run(s):
    op = s["case"]["op"]
    if own:
        from paper_2506_16640_amd import binding
        if op == "append":
            c = s["case"]
            binding.cache_append(s["k"], s["v"], s["kc"], s["vc"], s["cu"], s["kv_len"], s["table"], q=s["q"], q_out=s["out"],
                                 inv_freq=s["inv_freq"], interleaved=c["interleaved"])
            return s["out"], s["kc"], s["vc"]
        if op == "paged":
            return binding.paged_attn_fwd(s["q"], s["kc"], s["vc"], s["cu"], s["kv_len"], s["table"], max_new=s["most"][0],
                                          max_keys=s["most"][1], out=s["out"], workspace=s["workspace"], **s["kw"])
        return binding.packed_attn_fwd(s["q"], s["k"], s["v"], s["cu"], max_len=s["most"][0], out=s["out"], workspace=s["workspace"], **s["kw"])
    return _plain_append(s) if op == "append" else _plain_attention(s)


# ----------------------------------------------------------------- the plain form

def _rotate(x, cos, sin, rot, interleaved):
    """x [n, H, d] in fp32, cos and sin [n, rot / 2]."""
    if rot == 0:
        return x
    y = x.clone()
    cos, sin = cos[:, None], sin[:, None]
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if interleaved else (x[..., :rot // 2], x[..., rot // 2:rot])
    ra, rb = a * cos - b * sin, b * cos + a * sin
    if interleaved:
        y[..., 0:rot:2], y[..., 1:rot:2] = ra, rb
    else:
        y[..., :rot // 2], y[..., rot // 2:rot] = ra, rb
    return y


def _plain_append(s):
    c = s["case"]
    rot, page, tdt = c["rot"], c["page"], s["q"].dtype
    for i, (n, L) in enumerate(zip(s["new"], s["keys"])):
        rows = slice(s["cu_list"][i], s["cu_list"][i] + n)
        pos = torch.arange(L - n, L, device="cuda")
        cos = sin = None
        if rot:
            angle = pos.double()[:, None] * s["inv_freq"].double()[None]  # (far positions need the bits)
            cos, sin = angle.cos().float(), angle.sin().float()
        s["out"][rows] = _rotate(s["q"][rows].float(), cos, sin, rot, c["interleaved"]).to(tdt)
        where = s["table"][i, pos // page].long()
        s["kc"][where, :, pos % page] = _rotate(s["k"][rows].float(), cos, sin, rot, c["interleaved"]).to(tdt)
        s["vc"][where, :, pos % page] = s["v"][rows]
    return s["out"], s["kc"], s["vc"]


def _keys_of(s, i, kind):
    """Keys or values of sequence i as [Hkv, L, d]."""
    if s["case"]["op"] == "packed":
        return s[kind][s["cu_list"][i]:s["cu_list"][i + 1]].transpose(0, 1)
    L, page = s["keys"][i], s["case"]["page"]
    pages = s[kind + "c"][s["table"][i, :(L + page - 1) // page].long()]  # [n, Hkv, page, d]
    return pages.transpose(0, 1).reshape(pages.shape[1], -1, pages.shape[3])[:, :L]


def _plain_attention(s):
    c, kw = s["case"], s["kw"]
    Hq, Hkv, d = c["Hq"], c["Hkv"], c["d"]
    G, alpha = Hq // Hkv, c["alpha"]
    r = 1.0 / (alpha - 1.0)
    for i, (n, L) in enumerate(zip(s["new"], s["keys"])):
        k, v = _keys_of(s, i, "k").float(), _keys_of(s, i, "v").float()
        step = max(1, 2 ** 28 // (Hq * L))
        for t0 in range(0, n, step):
            m = min(step, n - t0)
            row = s["cu_list"][i] + t0
            q = s["q"][row:row + m].float().reshape(m, Hkv, G, d).permute(1, 2, 0, 3).reshape(Hkv, G * m, d)
            z = torch.matmul(q, k.transpose(1, 2).contiguous()).reshape(Hkv, G, m, L) / math.sqrt(d)
            pos = torch.arange(L - n + t0, L - n + t0 + m, device="cuda")
            key = torch.arange(L, device="cuda")
            seen = (key[None] <= pos[:, None]) if c["causal"] else torch.ones(m, L, dtype=torch.bool, device="cuda")
            if kw["alibi_slopes"] is not None:
                z = z - kw["alibi_slopes"].reshape(Hkv, G, 1, 1) * (pos[:, None] - key[None]).clamp(min=0).float()
            scale = torch.full((Hkv, G, m, 1), kw["delta"], device="cuda")
            if kw["beta"] is not None:
                b, g = ((x[:, row:row + m] if x.dim() == 2 else x[:, None].expand(-1, m)).reshape(Hkv, G, m, 1) for x in (kw["beta"], kw["gamma"]))
                cnt = seen.sum(1).float() if c["logn"] else torch.full((m,), float(L), device="cuda")
                ln = torch.log(cnt)[:, None]
                scale = scale + torch.where(cnt[:, None] > 1, b * ln ** g, torch.zeros_like(b))
            y = ((alpha - 1.0) * scale * z).masked_fill(~seen, -math.inf)
            tau = y.amax(-1, keepdim=True) - 1.0
            for _ in range(24):  # sum of [y - tau]^r is convex and decreasing: steps from the left rise to where it is 1
                x = (y - tau).clamp(min=0)
                f, g = (x ** r).sum(-1, keepdim=True), torch.where(x > 0, x ** (r - 1.0), torch.zeros_like(x)).sum(-1, keepdim=True)
                tau = tau + ((f - 1.0) / (r * g)).clamp(min=0)
            p = (y - tau).clamp(min=0) ** r
            o = torch.matmul(p.reshape(Hkv, G * m, L), v)
            s["out"][row:row + m] = o.reshape(Hkv, G, m, d).permute(2, 0, 1, 3).reshape(m, Hq, d).to(s["out"].dtype)
    return s["out"]


# ----------------------------------------------------------------- what cannot be left out

def work(case):
    new, keys = _lengths(case)
    eb = 2 if case["dtype"] == "bf16" else 4
    Hq, Hkv, d = case["Hq"], case["Hkv"], case["d"]
    T = sum(new)
    if case["op"] == "append":  # every element in and out; a rotation is six operations a pair
        return {"bytes": 2 * eb * T * (Hq + 2 * Hkv) * d, "flops": 3.0 * T * (Hq + Hkv) * case["rot"]}
    # Q in, O out, K in; the values only where a probability is not zero (about two keys a row; at most every row of V once)
    dense = case["scale"] in ("dense", "none")
    k_rows = Hkv * sum(keys)
    v_rows = k_rows if dense else min(k_rows, 2 * Hq * T)
    pairs = float(Hq) * sum(n * (L - n) + n * (n + 1) / 2.0 if case["causal"] else float(n) * L for n, L in zip(new, keys))
    return {"bytes": eb * d * (2 * Hq * T + k_rows + v_rows), "flops": 2.0 * d * pairs * (2 if dense else 1)}


# ----------------------------------------------------------------- the definition in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    new, keys, cu = s["new"], s["keys"], s["cu_list"]
    Hq, Hkv, d, page = (case[x] for x in ("Hq", "Hkv", "d", "page"))
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    if case["op"] == "append":
        kc, vc = s["kc"].double(), s["vc"].double()
        half = case["rot"] // 2
        first = [2 * e if case["interleaved"] else e for e in range(half)]
        second = [2 * e + 1 if case["interleaved"] else e + half for e in range(half)]
        for i in range(case["nseq"]):
            pos = torch.arange(keys[i] - new[i], keys[i], device="cuda", dtype=torch.float64)
            where = torch.tensor([int(s["table_list"][i, p // page]) for p in range(keys[i] - new[i], keys[i])], device="cuda")
            slot = pos.long() % page
            for src, dst in ((s["q"], None), (s["k"], kc)):
                x = src[cu[i]:cu[i + 1]].double()
                if half:
                    w = torch.polar(torch.ones(1, dtype=torch.float64, device="cuda"), pos[:, None, None] * s["inv_freq"].double())
                    z = torch.complex(x[..., first], x[..., second]) * w
                    x[..., first], x[..., second] = z.real, z.imag
                if dst is None:
                    out[cu[i]:cu[i + 1]] = x
                else:
                    dst[where, :, slot] = x
            vc[where, :, slot] = s["v"][cu[i]:cu[i + 1]].double()
        return out, kc, vc
    kw, alpha = s["kw"], float(case["alpha"])
    r = 1.0 / (alpha - 1.0)
    for i in range(case["nseq"]):
        n, L = new[i], keys[i]
        for h in range(Hq):
            hk = h // (Hq // Hkv)
            if case["op"] == "packed":
                k, v = s["k"][cu[i]:cu[i + 1], hk].double(), s["v"][cu[i]:cu[i + 1], hk].double()
            else:
                pages = s["table_list"][i, :(L + page - 1) // page].tolist()
                k = torch.cat([s["kc"][pages, hk].reshape(-1, d)[:L]]).double()
                v = torch.cat([s["vc"][pages, hk].reshape(-1, d)[:L]]).double()
            step = max(1, 2 ** 26 // L)
            for t0 in range(0, n, step):
                rows = torch.arange(t0, min(n, t0 + step), device="cuda")
                seen_to = rows + (L - n) if case["causal"] else torch.full_like(rows, L - 1)  # last key of a row
                y = s["q"][cu[i] + rows, h].double() @ k.T / d ** 0.5
                dist = (rows + (L - n))[:, None] - torch.arange(L, device="cuda")[None]
                if kw["alibi_slopes"] is not None:
                    y -= float(kw["alibi_slopes"][h]) * dist.clamp(min=0)
                mult = torch.full((len(rows),), float(kw["delta"]), dtype=torch.float64, device="cuda")
                if kw["beta"] is not None:
                    per_row = kw["beta"].dim() == 2
                    b, g = (x[h, cu[i] + rows].double() if per_row else x[h].double() for x in (kw["beta"], kw["gamma"]))
                    count = (seen_to + 1).double() if case["logn"] else torch.full_like(mult, float(L))
                    mult = mult + torch.where(count > 1, b * count.log() ** g, 0.0)
                y *= (alpha - 1.0) * mult[:, None]
                y[torch.arange(L, device="cuda")[None] > seen_to[:, None]] = -math.inf
                hi = y.amax(1, keepdim=True)
                lo = hi - 1.0
                for _ in range(56):  # the mass above the threshold is at least 1 at lo and 0 at hi
                    mid = 0.5 * (lo + hi)
                    over = (y - mid).clamp_(min=0).pow_(r).sum(1, keepdim=True) >= 1.0
                    lo, hi = torch.where(over, mid, lo), torch.where(over, hi, mid)
                out[cu[i] + rows, h] = (y - 0.5 * (lo + hi)).clamp_(min=0).pow_(r) @ v
    return out
