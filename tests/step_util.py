"""Plain forms, on the CPU and in 64 bits or whole numbers, of what a decode step needs around the cache: plan, softmax attention, sampling."""
import math

import torch

BF16, FP32 = torch.bfloat16, torch.float32


# ------------------------------------------------------------------------------------------- plan

def plain_plan(new, kv, table, free, count, page, rows, release=None):
    """One sequence after the other, one token after the other; lists, changed in place: kv, table, free.
    Returns (cu, free count, slots, positions, sequences)."""
    pages, columns = len(free), len(table[0]) if table else 0
    top = min(max(count, 0), pages)
    for s in range(len(new)):
        if release is not None and release[s] != 0:
            for e in range(min(-(-kv[s] // page), columns) if kv[s] > 0 else 0):
                if 0 <= table[s][e] < pages and top < pages:
                    free[top] = table[s][e]
                    top += 1
            kv[s] = 0
    cu, slots, positions, sequences = [0], [], [], []
    asked, tokens, used = 0, 0, 0
    for s in range(len(new)):
        n = max(new[s], 0)
        if kv[s] < 0 or kv[s] + n > columns * page:
            n = 0
        need = -(-(kv[s] + n) // page) - -(-kv[s] // page) if n else 0
        asked += need
        if need and asked > top:
            n = 0
        tokens += n
        if tokens > rows:
            n = 0
        for pos in range(kv[s], kv[s] + n):
            if pos % page == 0:
                used += 1
                table[s][pos // page] = free[top - used]
            pg = table[s][pos // page]
            slots.append(pg * page + pos % page if 0 <= pg < pages else -1)
            positions.append(pos)
            sequences.append(s)
        kv[s] += n
        cu.append(len(slots))
    pad = [-1] * (rows - len(slots))
    return cu, top - used, slots + pad, positions + pad, sequences + pad


# ------------------------------------------------------------------------------------------- softmax

def softmax_rows(q, k, v, ok, pos0, beta=None, gamma=None, slope=0.0, delta=1.0, causal=True, logn_mode=0, bias_mode=0, cap=0.0, split=True):
    """Rows of one head in 64 bits: o, lse, and bounds of what arithmetic in 32 bits may add to either.
    A score is a sum of D products: with A the sum of their absolute values (times the scale), 32-bit sums and the factors are off by at most
    d = (D + 16) 2^-24 A (fp32: sums of sixteen products and a tree of three levels, 32 2^-24 A); a cap adds 2^-21 of itself.  exp2 and its argument, a difference of scores of at most S in size, 2^-22 (S + 2).
    A row's sum, and its output before it is divided, are added up in runs of a wave's keys and then tile by tile: (n / 8 + 64) 2^-24.
    bf16: probabilities enter the product as the sum of two bf16 numbers, 2^-16.  With e all of these, p is off by a factor of 1 +- 2 e and the output
    by at most 2 e sum_j p_j |v_j - o| <= 4 e max |v|; lse by e."""
    q, k, v = q.double(), k.double(), v.double()
    n, D = q.shape
    L = k.shape[0]
    if L == 0 or n == 0:
        return torch.zeros(n, D, dtype=torch.float64), torch.full((n,), -math.inf, dtype=torch.float64), torch.zeros(n).double(), torch.zeros(n).double()
    pos, key = pos0 + torch.arange(n), torch.arange(L)
    seen = ok[None].expand(n, L).clone()
    if causal:
        seen &= key[None] <= pos[:, None]
    kz = torch.nan_to_num(torch.where(ok[:, None], k, 0.0), 0.0, 0.0, 0.0)
    z = q @ kz.T / math.sqrt(D)
    size = q.abs() @ kz.abs().T / math.sqrt(D)
    dist = (pos[:, None] - key[None]).clamp(min=0).double()
    count = (torch.minimum(pos + 1, torch.tensor(L)).clamp(min=0) if causal else torch.full((n,), L)) if logn_mode else torch.full((n,), L)
    mult = torch.full((n,), float(delta), dtype=torch.float64)
    if beta is not None:
        mult = mult + torch.where(count > 1, beta.double() * torch.log(count.double().clamp(min=2)) ** gamma.double(), 0.0)
    m = mult[:, None]
    bias = -slope * dist
    s = m * (z + bias) if bias_mode == 0 else m * z
    if cap > 0:
        s = cap * torch.tanh(s / cap)
    if bias_mode == 1:
        s = s + torch.where(m != 0, bias, 0.0)  # (a row of scale 0 has no bias)
    s = torch.where(seen, s, -math.inf)
    lse = torch.logsumexp(s, 1)
    live = lse > -math.inf
    p = torch.where(live[:, None], (s - torch.where(live, lse, 0.0)[:, None]).exp(), 0.0)
    vz = torch.nan_to_num(torch.where(ok[:, None], v, 0.0), 0.0, 0.0, 0.0)
    A = torch.where(seen, m.abs() * (size + slope * dist), 0.0)
    near = torch.where(seen & (p > 1e-12), A, 0.0).amax(1)  # (of the keys that count)
    S = torch.where(seen & (p > 1e-12), s.abs(), 0.0).amax(1)
    e = (D + 16 if split else 32) * 2.0 ** -24 * near + 2.0 ** -22 * (2 * S + 2) + (L / 8 + 64) * 2.0 ** -24 + (2.0 ** -16 if split else 0.0) + cap * 2.0 ** -21
    return p @ vz, lse, 4 * e * vz.abs().max(), e + 2.0 ** -22 * torch.where(live, lse, 0.0).abs()


def softmax_reference(p, cap=0.0):
    """out [T,Hq,D], lse [Hq,T] of a Problem of tests/serving_util.py in 64 bits, and their bounds (its alpha does not matter)."""
    out, lse = torch.zeros(p.T, p.Hq, p.D, dtype=torch.float64), torch.zeros(p.Hq, p.T, dtype=torch.float64)
    tol, tol_lse = torch.zeros(p.T, p.Hq, 1, dtype=torch.float64), torch.zeros(p.Hq, p.T, dtype=torch.float64)
    for s, (n, L) in enumerate(p.lens):
        k, v, ok = p.keys(s)
        e = slice(p.cu[s], p.cu[s] + n)
        for h in range(p.Hq):
            pick = lambda x: None if x is None else (x[h, e] if x.dim() == 2 else x[h])  # noqa: E731
            o, l, t, tl = softmax_rows(p.q[e, h], k[h // (p.Hq // p.Hkv)], v[h // (p.Hq // p.Hkv)], ok, L - n, beta=pick(p.kw["beta"]),
                                       gamma=pick(p.kw["gamma"]), slope=0.0 if p.kw["alibi_slopes"] is None else float(p.kw["alibi_slopes"][h]),
                                       cap=cap, split=p.dtype == BF16, **{x: p.kw[x] for x in ("delta", "causal", "logn_mode", "bias_mode")})
            out[e, h], lse[h, e], tol[e, h, 0], tol_lse[h, e] = o, l, t, tl
    return out, lse, tol, tol_lse


# ------------------------------------------------------------------------------------------- sampling

def plain_sample(logits, u, temperature=None, top_k=None, top_p=None, min_p=None):
    """Tokens and log probabilities of the rows, from their sorted logits."""
    tokens, logs = [], []
    R, V = logits.shape
    at = lambda t, r, off: off if t is None else float(t[r])  # noqa: E731
    for r in range(R):
        x = torch.nan_to_num(logits[r].double(), -math.inf, math.inf, -math.inf)
        t, k, p, m = at(temperature, r, 1.0), int(at(top_k, r, 0)), at(top_p, r, 1.0), at(min_p, r, 0.0)
        un = min(max(float(u[r]), 0.0), 1.0) if not math.isnan(float(u[r])) else 0.0
        order = torch.sort(x, descending=True, stable=True).indices
        top = x[order[0]]
        if top == -math.inf:
            tokens.append(-1)
            logs.append(-math.inf)
            continue
        if not t > 0:
            tokens.append(int(order[0]))
            logs.append(0.0)
            continue
        if top == math.inf:
            w = (x == top).double()
        else:
            w = torch.where(x > -math.inf, (x - top) / t if t < math.inf else torch.zeros_like(x), -math.inf).exp()
        ranked = w[order]
        n = V if k <= 0 else min(k, V)
        if p < 1.0:
            before = ranked[:n].cumsum(0) - ranked[:n]
            n = max(1, int((before < max(p, 0.0) * ranked[:n].sum()).sum()))
        if m > 0.0:
            n = min(n, int((ranked >= min(m, 1.0)).sum()))
        kept = torch.zeros(V, dtype=torch.bool)
        kept[order[:n]] = True
        kept &= w > 0
        index = kept.nonzero()[:, 0]
        sums = w[index].cumsum(0)
        e = min(int((sums <= un * sums[-1]).sum()), len(index) - 1)
        tokens.append(int(index[e]))
        logs.append(math.log(float(w[index[e]] / sums[-1])))
    return torch.tensor(tokens, dtype=torch.int32), torch.tensor(logs, dtype=torch.float64)
