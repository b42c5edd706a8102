"""Attention and its gradients from their definition in binary64 on the CPU, with bounds on what a kernel in binary32 with bf16 or binary32 operands may be off by."""
import math

import torch

E32 = 2.0 ** -24                  # half a step of binary32


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def inputs(B, Tq, Tk, H, K, D, dtype, seed=0, spread=1.0):
    gen = torch.Generator().manual_seed(seed)
    new = lambda *s: torch.randn(*s, generator=gen)                          # noqa: E731
    return [(spread * new(B, Tq, H, D)).to(dtype), new(B, Tk, K, D).to(dtype), new(B, Tk, K, D).to(dtype), new(B, Tq, H, D).to(dtype)]


def seen(n, m, causal):
    """[n x m]: which keys a query sees, the last query the last key"""
    i, j = torch.arange(n)[:, None], torch.arange(m)[None]
    return j <= i + m - n if causal else torch.ones(n, m, dtype=torch.bool)


def reference(q, k, v, g, causal, scale, q_lens=None, k_lens=None):
    """{name: (value, bound)} of o, lse, dq, dk, dv.  Rounding errors are taken at their largest and added up:
    a score: D products and sums in binary32, the product with scale log2(e), the subtraction before the exponential (2 roundings of the larger part); the exponential 2 steps;
    P as an operand: one rounding to the operands' type; sums of n terms: n half steps of the sum of magnitudes (in any order); a result: one rounding."""
    B, Tq, H, D = q.shape
    Tk, K = k.shape[1], k.shape[2]
    G, u = H // K, half_step(q.dtype)
    ut = u if q.dtype != torch.float32 else 0.0                              # P and dS as operands (binary32 operands take them as they are)
    zero = lambda *s: torch.zeros(*s, dtype=torch.float64)                   # noqa: E731
    val = dict(o=zero(B, Tq, H, D), lse=torch.full((B, H, Tq), -math.inf, dtype=torch.float64), dq=zero(B, Tq, H, D), dk=zero(B, Tk, K, D), dv=zero(B, Tk, K, D))
    err = dict(o=zero(B, Tq, H, D), lse=zero(B, H, Tq), dq=zero(B, Tq, H, D), dk=zero(B, Tk, K, D), dv=zero(B, Tk, K, D))
    for b in range(B):
        n = Tq if q_lens is None else min(max(int(q_lens[b]), 0), Tq)
        m = Tk if k_lens is None else min(max(int(k_lens[b]), 0), Tk)
        if n == 0 or m == 0:
            continue
        see = seen(n, m, causal)
        some = see.any(1)
        for h in range(H):
            Q, KK, V, GG = (t.double() for t in (q[b, :n, h], k[b, :m, h // G], v[b, :m, h // G], g[b, :n, h]))
            GG = torch.where(some[:, None], GG, 0.0)                         # (what a query that sees nothing brings does not count)
            s = (Q @ KK.t() * scale).masked_fill(~see, -math.inf)
            lse = torch.logsumexp(s, 1)
            base = torch.where(some, lse, 0.0)
            P = torch.exp(s - base[:, None])
            fin = torch.where(see, s, 0.0)
            es = (D + 4) * E32 * scale * (Q.abs() @ KK.abs().t()) + 4 * E32 * (fin.abs() + base.abs()[:, None])
            es = torch.where(see, es, 0.0)
            top = es.amax(1, keepdim=True)
            # P, up to a factor of a row that its sum has too: 2 steps of the exponential, and what moving the maximum multiplies (1 rounding and exponential each; at most
            # one in 8 binary orders: 40 are more than the scores here go through)
            eP = es + top + (m + 4 + 4 * 40) * E32
            o = P @ V
            # (P as rounded in the product, and in the sum that it is divided by)
            eo = (P * (eP + 2 * ut * (1 + 2 * ut))) @ V.abs() + (m + 4) * E32 * (P @ V.abs()) + u * o.abs()
            elr = top[:, 0] + (m + 4 + 4 * 40) * E32 + 4 * E32 * (base.abs() + 64)    # (lse = (m + log2 of the sum) ln 2: m and the logarithm are below 64 + |lse|)
            dP = GG @ V.t()
            delta = (GG * o).sum(1, keepdim=True)
            dS = P * (dP - delta)
            edP = (D + 2) * E32 * (GG.abs() @ V.abs().t())
            ed = (GG.abs() * eo).sum(1, keepdim=True) + (D + 2) * E32 * (GG * o).abs().sum(1, keepdim=True)
            eP2 = es + elr[:, None] + 8 * E32
            edS = dS.abs() * (eP2 + ut + 2 * E32) + P * (edP + ed + E32 * (dP.abs() + delta.abs()))
            put = lambda name, where, x, e: (val[name].__setitem__(where, val[name][where] + x), err[name].__setitem__(where, err[name][where] + e))   # noqa: E731
            put("o", (b, slice(n), h), o, eo)
            val["lse"][b, h, :n] = lse
            err["lse"][b, h, :n] = torch.where(some, elr, 0.0)
            put("dq", (b, slice(n), h), scale * dS @ KK, scale * (edS @ KK.abs() + (m + 3) * E32 * (dS.abs() @ KK.abs())))
            put("dk", (b, slice(m), h // G), scale * dS.t() @ Q, scale * (edS.t() @ Q.abs() + (n * G + 20) * E32 * (dS.abs().t() @ Q.abs())))
            put("dv", (b, slice(m), h // G), P.t() @ GG, (P * (eP2 + ut)).t() @ GG.abs() + (n * G + 20) * E32 * (P.t() @ GG.abs()))
    for name in ("dq", "dk", "dv"):
        err[name] = err[name] + u * (val[name].abs() + err[name])
    err["o"] = err["o"] * (1 + u)
    return {name: (val[name], err[name] + 1e-30) for name in val}


def check(name, got, want):
    value, bound = want
    got = got.cpu().double()
    off = (got - value).abs()
    bad = ~((off <= bound) | (got == value))
    assert not bool(bad.any()), (f"{name}: {int(bad.sum())} of {bad.numel()} beyond the bound, the first at {tuple(bad.nonzero()[0].tolist())}: "
                                 f"{got[bad][0].item():.9g} for {value[bad][0].item():.9g}, bound {bound[bad][0].item():.3g}; largest ratio {(off / bound)[~got.isnan()].max().item():.3g}")
