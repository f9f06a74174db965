"""Plain 64-bit forms of the serving operators (packed sequences, paged cache) on the CPU, and problems for them."""
import math

import torch

BF16, FP32 = torch.bfloat16, torch.float32


class Problem:
    """Sequences (new tokens, keys) with random contents; the cache as [pages, Hkv, page, D], the keys of sequence s also as k[s], v[s]."""

    def __init__(self, lens, Hq=4, Hkv=2, D=64, dtype=BF16, page=16, seed=0, pad=0, paged=True, scale="head", alpha=1.5, causal=True, logn=0,
                 slopes=False, bias_mode=0, delta=1.0, q_factor=1.0, spare=2, front=0):
        g = torch.Generator().manual_seed(seed)
        self.lens, self.Hq, self.Hkv, self.D, self.dtype, self.page, self.paged = lens, Hq, Hkv, D, dtype, page, paged
        normal = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
        uniform = lambda *s: 0.5 + torch.rand(*s, generator=g)  # noqa: E731
        self.cu = [front]
        for n, _ in lens:
            self.cu.append(self.cu[-1] + n)
        self.T = self.cu[-1] + pad
        self.q = (q_factor * normal(self.T, Hq, D)).to(dtype)
        if paged:
            per = [(L + page - 1) // page for _, L in lens]
            self.pages = sum(per) + spare
            self.kc, self.vc = (normal(self.pages, Hkv, page, D).to(dtype) for _ in range(2))
            perm = torch.randperm(self.pages, generator=g).to(torch.int32)
            self.table = torch.full((len(lens), max(per + [1])), -7, dtype=torch.int32)  # (entries behind the last page are nobody's)
            at = 0
            for s, n in enumerate(per):
                self.table[s, :n] = perm[at:at + n]
                at += n
        else:
            self.kp, self.vp = (normal(self.T, Hkv, D).to(dtype) for _ in range(2))
        beta = gamma = None
        if scale == "head":
            beta, gamma = uniform(Hq), uniform(Hq)
        elif scale == "query":
            beta, gamma = uniform(Hq, self.T), uniform(Hq, self.T)
        elif scale == "dense":
            beta, gamma, delta = uniform(Hq), torch.full((Hq,), -0.5), 0.0
        elif scale == "signs":  # negative, zero and ordinary multipliers
            beta, gamma, delta = torch.tensor([-0.8, 0.0, 0.5, 1.0]).repeat(Hq)[:Hq], torch.ones(Hq), 0.0
        sl = None
        if slopes:
            sl = torch.zeros(Hq)
            sl[::2] = torch.tensor([2.0 ** -(k + 1) for k in range((Hq + 1) // 2)])
        self.kw = dict(alpha=alpha, beta=beta, gamma=gamma, delta=delta, causal=causal, logn_mode=logn, alibi_slopes=sl, bias_mode=bias_mode)

    def keys(self, s):
        """K, V of sequence s [Hkv, L, D] and which keys exist (are on a page)."""
        n, L = self.lens[s]
        if not self.paged:
            e = slice(self.cu[s], self.cu[s] + n)
            return self.kp[e].transpose(0, 1), self.vp[e].transpose(0, 1), torch.ones(L, dtype=torch.bool)
        j = torch.arange(L)
        pg = self.table[s][j // self.page].long()
        ok = (pg >= 0) & (pg < self.pages)
        at = pg.clamp(0, self.pages - 1)
        return self.kc[at, :, j % self.page].transpose(0, 1), self.vc[at, :, j % self.page].transpose(0, 1), ok

    def reference(self):
        """out [T, Hq, D] in 64 bits and a bound of what arithmetic in 32 bits may add to it."""
        out = torch.zeros(self.T, self.Hq, self.D, dtype=torch.float64)
        tol = torch.zeros(self.T, self.Hq, 1, dtype=torch.float64)
        for s, (n, L) in enumerate(self.lens):
            k, v, ok = self.keys(s)
            for h in range(self.Hq):
                e = slice(self.cu[s], self.cu[s] + n)
                per_row = self.kw["beta"] is not None and self.kw["beta"].dim() == 2
                o, t = plain_rows(self.q[e, h], k[h // (self.Hq // self.Hkv)], v[h // (self.Hq // self.Hkv)], ok, L - n,
                                  beta=None if self.kw["beta"] is None else (self.kw["beta"][h, e] if per_row else self.kw["beta"][h]),
                                  gamma=None if self.kw["gamma"] is None else (self.kw["gamma"][h, e] if per_row else self.kw["gamma"][h]),
                                  slope=0.0 if self.kw["alibi_slopes"] is None else float(self.kw["alibi_slopes"][h]),
                                  **{x: self.kw[x] for x in ("alpha", "delta", "causal", "logn_mode", "bias_mode")})
                out[e, h], tol[e, h, 0] = o, t
        return out, tol

    def owned(self):
        m = torch.zeros(self.T, dtype=torch.bool)
        for s in range(len(self.lens)):
            m[self.cu[s]:self.cu[s + 1]] = True
        return m

    def gpu_kw(self):
        return {k: v.cuda() if torch.is_tensor(v) else v for k, v in self.kw.items()}

    def run(self, binding, path=0, out=None, **kw):
        cu = torch.tensor(self.cu, dtype=torch.int32).cuda()
        kw = dict(self.gpu_kw(), path=path, out=out, **kw)
        if not self.paged:
            return binding.packed_attn_fwd(self.q.cuda(), self.kp.cuda(), self.vp.cuda(), cu, **kw)
        kv_len = torch.tensor([L for _, L in self.lens], dtype=torch.int32).cuda()
        return binding.paged_attn_fwd(self.q.cuda(), self.kc.cuda(), self.vc.cuda(), cu, kv_len, self.table.cuda(), **kw)

    def check(self, got, label=""):
        """|got - ref| within half a step of the type (of the value) and what 32-bit arithmetic may add."""
        ref, tol = self.reference()
        own = self.owned()
        got = got.double().cpu()
        half = torch.finfo(self.dtype).eps / 2
        assert torch.isfinite(got[own]).all(), label
        excess = ((got - ref).abs() - half * ref.abs() - tol)[own]
        worst = ((got - ref).abs()[own]).max().item() if own.any() else 0.0
        assert excess.numel() == 0 or excess.max().item() <= 0.0, (label, "beyond the bound by", excess.max().item(), "largest error", worst)
        return worst


def plain_rows(q, k, v, ok, pos0, beta=None, gamma=None, slope=0.0, alpha=1.5, delta=1.0, causal=True, logn_mode=0, bias_mode=0):
    """Rows of one head in 64 bits: o, and a bound of the effect of 32-bit scores and thresholds.
    A score y = (alpha-1) s of size |y| carries the errors of a sum of D products and of its factor, under 2^-20 |y| together, and the
    threshold search stops within 2e-6 max(1, |tau|): delta = 2^-19 max(1, |y|) in all.  The weight x^r of a key changes by r x^(r-1) delta
    (x: how far the key is above the threshold), and by delta^r where x is zero, so the output by at most
    delta * sum_j r (x_j + delta)^(r-1) max |v|, over the keys with x_j > -delta."""
    q, k, v = q.double(), k.double(), v.double()
    n, D = q.shape
    L = k.shape[0]
    r = 1.0 / (alpha - 1.0)
    if L == 0 or n == 0:
        return torch.zeros(n, D, dtype=torch.float64), torch.zeros(n, dtype=torch.float64)
    pos = pos0 + torch.arange(n)
    key = torch.arange(L)
    seen = ok[None].expand(n, L).clone()
    if causal:
        seen &= key[None] <= pos[:, None]
    k = torch.where(ok[:, None], k, 0.0)
    z = torch.where(seen, q @ torch.nan_to_num(k, 0.0, 0.0, 0.0).T / math.sqrt(D), 0.0)
    dist = (pos[:, None] - key[None]).clamp(min=0).double()
    count = (torch.minimum(pos + 1, torch.tensor(L)).clamp(min=0) if causal else torch.full((n,), L)) if logn_mode else torch.full((n,), L)
    mult = torch.full((n,), float(delta), dtype=torch.float64)
    if beta is not None:
        mult = mult + torch.where(count > 1, beta.double() * torch.log(count.double().clamp(min=2)) ** gamma.double(), 0.0)
    if bias_mode == 0:
        s = mult[:, None] * (z - slope * dist)
    else:
        s = mult[:, None] * z - torch.where(mult[:, None] != 0, slope, 0.0) * dist
    y = torch.where(seen, (alpha - 1.0) * s, -math.inf)
    top = y.amax(1, keepdim=True)
    live = top > -math.inf
    lo = torch.where(live, top, 0.0) - 1.0
    hi = lo + 1.0
    for _ in range(60):
        mid = 0.5 * (lo + hi)
        over = ((y - mid).clamp(min=0) ** r).sum(1, keepdim=True) >= 1.0
        lo, hi = torch.where(over, mid, lo), torch.where(over, hi, mid)
    tau = 0.5 * (lo + hi)
    p = torch.where(live, (y - tau).clamp(min=0) ** r, 0.0)
    vz = torch.nan_to_num(torch.where(ok[:, None], v, 0.0), 0.0, 0.0, 0.0)
    o = p @ vz
    size = torch.where(seen & (y > tau - 1.0), y.abs(), 0.0).amax(1)  # (the scores that can matter)
    d = 2.0 ** -19 * size.clamp(min=1.0)
    near = torch.where(seen & (y > tau - d[:, None]), (y - tau).clamp(min=0) + d[:, None], 0.0)
    g = torch.where(near > 0, r * near ** (r - 1.0), 0.0)
    return o, d * g.sum(1) * vz.abs().max()
