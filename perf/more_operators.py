"""Performance cases of the operators between a transformer block's linear layers: layer norm, rotary positions, attention, each with its gradient.

A case is a dict of plain values.  `listed()` names the ones that are always timed, `draw(rng)` gives further cases of the
same families over their whole range of sizes, `prepare` makes what a program holds before the call, `run` is one pass,
`work` the bytes and operations one pass cannot do without, `exact` the results in 64 bits.  Where `own` is false `run`
computes the operators in elementary torch operations in 32 bits; where it is true it calls the package.

Families
  norm      y = (x - mean) / sqrt(variance + eps) * w + b over the rows of x; in training the gradients of x, w and b too
  rotary    pairs of each head's first elements turned by position times frequency; in training the gradient turned back too
  attend    softmax(scale q k^T + mask) v for each head, query heads in groups that share keys and values, causal or not (the last query sees the
            last key), sequences of a batch shorter than its tensors; in training the gradients of q, k and v too
"""
from __future__ import annotations

import math

import torch

own = False

DEVICE = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"bf16": 2, "f32": 4}
EPS = 1e-5
CHUNK = 1 << 30                 # scores that the plain form holds at a time


def _norm(name, tokens, width, dtype="bf16", params="f32", train=True):
    return {"name": name, "family": "norm", "tokens": tokens, "width": width, "dtype": dtype, "params": params, "train": train}


def _rotary(name, batch, length, heads, head, part=None, interleaved=False, dtype="bf16", first=0, train=True):
    return {"name": name, "family": "rotary", "batch": batch, "length": length, "heads": heads, "head": head, "part": part or head,
            "interleaved": interleaved, "dtype": dtype, "first": first, "train": train}


def _attend(name, batch, queries, keys, heads, kv_heads, head, causal=True, ragged=False, dtype="bf16", train=True):
    return {"name": name, "family": "attend", "batch": batch, "queries": queries, "keys": keys, "heads": heads, "kv_heads": kv_heads, "head": head,
            "causal": causal, "ragged": ragged, "dtype": dtype, "train": train}


def listed():
    return [
        # the next token of one sequence, served: the latency of a call
        _norm("norm_token", 1, 1024, train=False),
        # 8 images of 197 positions, odd width, binary32 tensors
        _norm("norm_ragged", 8 * 197, 1001, dtype="f32"),
        # 32 x 512 tokens of a transformer with hidden 1024
        _norm("norm_train", 16384, 1024, params="bf16"),
        # 32768 tokens of the large decoder, hidden 8192
        _norm("norm_large", 32768, 8192),
        # queries and keys of the next tokens of 8 sequences, far into a long context
        _rotary("rotary_tokens", 8, 1, 20, 64, first=100000, train=False),
        # part of each head, neighbours as pairs, binary32, an odd length
        _rotary("rotary_ragged", 3, 1333, 7, 80, part=32, interleaved=True, dtype="f32"),
        # queries and keys of 32768 tokens of the large decoder, 64 + 8 heads of 128
        _rotary("rotary_large", 4, 8192, 72, 128),
        # 8 images of 197 positions, 12 heads of 64, binary32: every query sees every key
        _attend("attend_images", 8, 197, 197, 12, 12, 64, causal=False, dtype="f32"),
        # 32 x 512 tokens of a transformer with hidden 1024
        _attend("attend_train", 32, 512, 512, 16, 16, 64),
        # a padded batch of odd lengths, heads of 80 that share one head of keys and values
        _attend("attend_padded", 6, 1333, 1333, 12, 1, 80, ragged=True),
        # one token each of 16 sequences of different lengths over their caches of up to 8192 keys
        _attend("attend_decode", 16, 1, 8192, 64, 8, 128, ragged=True, train=False),
        # the large decoder's attention: 64 heads of 128 over 8 of keys and values, 2 x 8192 tokens
        _attend("attend_large", 2, 8192, 8192, 64, 8, 128),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    family = rng.choice(["norm", "norm", "rotary", "rotary", "attend", "attend", "attend", "attend"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if family == "norm":
        while True:
            T, C = _log_int(rng, 1, 32768), _log_int(rng, 32, 16384)
            if T * C * SIZE[dtype] <= 32768 * 8192 * 2:
                break
        c = _norm("", T, C, dtype=dtype, params=rng.choice(["f32", dtype]), train=rng.random() < 0.7)
    elif family == "rotary":
        while True:
            B, T, H, D = _log_int(rng, 1, 32), _log_int(rng, 1, 8192), _log_int(rng, 1, 80), 8 * _log_int(rng, 4, 16)
            if B * T * H * D * SIZE[dtype] <= 32768 * 72 * 128 * 2:
                break
        c = _rotary("", B, T, H, D, part=rng.choice([D, D, 2 * rng.randint(4, D // 2)]), interleaved=rng.random() < 0.5, dtype=dtype,
                    first=rng.choice([0, 0, rng.randrange(1 << 20)]), train=rng.random() < 0.6)
    else:
        while True:
            B, T, K, G, D = _log_int(rng, 1, 64), _log_int(rng, 16, 8192), _log_int(rng, 1, 32), rng.choice([1, 1, 2, 4, 7, 8]), 8 * _log_int(rng, 4, 16)
            train = rng.random() < 0.6
            tq = T if train else rng.choice([1, 1, T, _log_int(rng, 1, T)])
            c = _attend("", B, tq, T, K * G, K, D, causal=rng.random() < 0.7, ragged=rng.random() < 0.4, dtype=dtype, train=train)
            # (binary32 has a fraction of the rate)
            if K * G <= 64 and B * T * K * D <= 1 << 28 and work(c)["flops"] * (8 if dtype == "f32" else 1) <= 2 * 7 * 64 * 8192 * 8192 * 128:
                break
    c.pop("name", None)
    return c


# ---- inputs

def _generator(seed):
    return torch.Generator(device=DEVICE).manual_seed(int(seed) % (1 << 62))


def _lengths(case):
    """(queries, keys) of each sequence: from all of the tensor down to about half of it where they are ragged."""
    B, Tq, Tk = case["batch"], case["queries"], case["keys"]
    if not case["ragged"]:
        return [(Tq, Tk)] * B
    keys = [Tk - (b * Tk) // (2 * B) for b in range(B)]
    return [(n if Tq == Tk else min(Tq, n), n) for n in keys]


def _frequencies(case):
    r = case["part"]
    return torch.tensor([10000.0 ** (-2 * j / r) for j in range(r // 2)], dtype=torch.float64, device=DEVICE)


def prepare(case, seed):
    gen, family, dtype = _generator(seed), case["family"], DTYPES[case["dtype"]]
    new = lambda *shape: torch.randn(shape, generator=gen, device=DEVICE)        # noqa: E731
    s = {"case": case}
    if family == "norm":
        T, C, params = case["tokens"], case["width"], DTYPES[case["params"]]
        # channels differ in size and have means of their own, as in a residual stream
        s["x"] = (new(T, C) * new(C).mul_(0.5).exp_() + 0.3 * new(C)).to(dtype)
        s["w"], s["b"] = (1 + 0.2 * new(C)).to(params), (0.1 * new(C)).to(params)
        if case["train"]:
            s["g"] = (new(T, C) * new(T, 1).exp_() * 1e-3).to(dtype)
    elif family == "rotary":
        shape = (case["batch"], case["length"], case["heads"], case["head"])
        s["x"] = new(*shape).to(dtype)
        s["freqs"] = _frequencies(case)
        s["positions"] = torch.arange(case["length"], device=DEVICE) + torch.randint(case["first"] + 1, (case["batch"], 1), generator=gen, device=DEVICE)
        if case["train"]:
            s["g"] = (new(*shape) * 1e-3).to(dtype)
    else:
        B, Tq, Tk, H, K, D = (case[k] for k in ("batch", "queries", "keys", "heads", "kv_heads", "head"))
        # scores of a few units: heads that look at single keys and heads that look at many
        s["q"] = (new(B, Tq, H, D) * new(H, 1).mul_(0.5).exp_()).to(dtype)
        s["k"], s["v"] = new(B, Tk, K, D).to(dtype), new(B, Tk, K, D).to(dtype)
        s["scale"] = D ** -0.5
        lens = _lengths(case)
        s["q_lens"] = torch.tensor([a for a, _ in lens], dtype=torch.int32, device=DEVICE) if case["ragged"] else None
        s["k_lens"] = torch.tensor([n for _, n in lens], dtype=torch.int32, device=DEVICE) if case["ragged"] else None
        if case["train"]:
            s["g"] = (new(B, Tq, H, D) * 1e-3).to(dtype)
    return s


# ---- plain forms

def _norm_plain(s):
    x, w = s["x"].float(), s["w"].float()
    mean = x.sum(1, keepdim=True) / x.shape[1]
    d = x - mean
    rstd = 1 / torch.sqrt((d * d).sum(1, keepdim=True) / x.shape[1] + EPS)
    hat = d * rstd
    y = (hat * w + s["b"].float()).to(s["x"].dtype)
    if not s["case"]["train"]:
        return y
    g = s["g"].float()
    u = g * w
    dx = (u - u.sum(1, keepdim=True) / x.shape[1] - hat * ((u * hat).sum(1, keepdim=True) / x.shape[1])) * rstd
    return y, dx.to(s["x"].dtype), (g * hat).sum(0).to(s["w"].dtype), g.sum(0).to(s["b"].dtype)


def _turn(s, x, sign):
    case = s["case"]
    r = case["part"]
    angle = s["positions"].double()[:, :, None, None] * s["freqs"]            # far positions: in 64 bits
    c, sn = torch.cos(angle).float(), (torch.sin(angle) * sign).float()
    y = x.float()
    if case["interleaved"]:
        a, b = y[..., 0:r:2], y[..., 1:r:2]
        turned = torch.stack((a * c - b * sn, a * sn + b * c), -1).flatten(-2)
    else:
        a, b = y[..., :r // 2], y[..., r // 2:r]
        turned = torch.cat((a * c - b * sn, a * sn + b * c), -1)
    return torch.cat((turned, y[..., r:]), -1).to(x.dtype)


def _attend_plain(s):
    case = s["case"]
    B, Tq, Tk, H, K, D = (case[k] for k in ("batch", "queries", "keys", "heads", "kv_heads", "head"))
    G, scale, dtype = H // K, s["scale"], s["q"].dtype
    by_head = lambda t, n: t.float().view(B, -1, K, n, D).permute(0, 2, 3, 1, 4).reshape(B * K, -1, D)       # noqa: E731  [B K, n T, D]
    q, k, v = by_head(s["q"], G), by_head(s["k"], 1), by_head(s["v"], 1)
    g = by_head(s["g"], G) if case["train"] else None
    i, j = torch.arange(Tq, device=DEVICE)[:, None], torch.arange(Tk, device=DEVICE)[None]
    nq = s["q_lens"] if s["q_lens"] is not None else torch.full((B,), Tq, device=DEVICE)
    nk = s["k_lens"] if s["k_lens"] is not None else torch.full((B,), Tk, device=DEVICE)
    some = max(1, CHUNK // (G * Tq * Tk))                                      # heads of keys at a time
    out = [torch.empty_like(q)] + ([torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)] if case["train"] else [])
    for at in range(0, B * K, some):
        part = slice(at, min(at + some, B * K))
        batch = torch.arange(part.start, part.stop, device=DEVICE) // K
        n, m = nq[batch].view(-1, 1, 1, 1), nk[batch].view(-1, 1, 1, 1)
        seen = (i < n) & (j < m)
        if case["causal"]:
            seen = seen & (j - i <= m - n)
        p = (q[part] @ k[part].transpose(1, 2) * scale).view(-1, G, Tq, Tk).masked_fill_(~seen, -math.inf)
        top = p.amax(-1, keepdim=True)
        p = (p - torch.where(top == -math.inf, 0, top)).exp_()
        total = p.sum(-1, keepdim=True)
        p = (p / torch.where(total == 0, 1, total)).view(-1, G * Tq, Tk)       # a row that sees nothing: zeros
        o = p @ v[part]
        out[0][part] = o
        if case["train"]:
            out[3][part] = p.transpose(1, 2) @ g[part]
            ds = p * (g[part] @ v[part].transpose(1, 2) - (g[part] * o).sum(-1, keepdim=True)) * scale
            out[1][part] = ds @ k[part]
            out[2][part] = ds.transpose(1, 2) @ q[part]
    back = lambda t, n: t.view(B, K, n, -1, D).permute(0, 3, 1, 2, 4).reshape(B, -1, K * n, D).to(dtype)     # noqa: E731
    if not case["train"]:
        return back(out[0], G)
    return back(out[0], G), back(out[1], G), back(out[2], 1), back(out[3], 1)


def run(s):
    case, family = s["case"], s["case"]["family"]
    if own:
        import paper_2203_10991_amd as nm
    if family == "norm":
        if not own:
            return _norm_plain(s)
        if not case["train"]:
            return nm.nm_layer_norm(s["x"], s["w"], s["b"], EPS)
        y, mean, rstd = nm.nm_layer_norm(s["x"], s["w"], s["b"], EPS, want_stats=True)
        return (y, *nm.nm_layer_norm_grad(s["g"], s["x"], s["w"], mean, rstd))
    if family == "rotary":
        if own:
            turn = lambda x, sign: nm.nm_rotary(x, s["freqs"], s["positions"], interleaved=case["interleaved"], inverse=sign < 0)     # noqa: E731
        else:
            turn = lambda x, sign: _turn(s, x, sign)                           # noqa: E731
        return (turn(s["x"], 1), turn(s["g"], -1)) if case["train"] else turn(s["x"], 1)
    if not own:
        return _attend_plain(s)
    mask = dict(causal=case["causal"], scale=s["scale"], q_lens=s["q_lens"], k_lens=s["k_lens"])
    if not case["train"]:
        return nm.nm_attention(s["q"], s["k"], s["v"], **mask)
    o, lse = nm.nm_attention(s["q"], s["k"], s["v"], want_lse=True, **mask)
    return (o, *nm.nm_attention_grad(s["g"], s["q"], s["k"], s["v"], o, lse, **mask))


# ---- what a pass needs

def _pairs(case):
    """Pairs of a query and a key that it sees, over the sequences; and the queries and keys that are there."""
    pairs = queries = keys = 0
    for n, m in _lengths(case):
        if case["causal"]:
            first = max(0, n - m)                                              # queries in front of every key see nothing
            pairs += (n - first) * (m - n) + (n * (n + 1) - first * (first + 1)) // 2
        else:
            pairs += n * m
        queries, keys = queries + n, keys + m
    return pairs, queries, keys


def work(case):
    family, e = case["family"], SIZE[case["dtype"]]
    if family == "norm":
        n, C = case["tokens"] * case["width"], case["width"]
        return {"bytes": n * e * (4 if case["train"] else 2) + C * SIZE[case["params"]] * (4 if case["train"] else 2), "flops": n * (20 if case["train"] else 8)}
    if family == "rotary":
        n = case["batch"] * case["length"] * case["heads"] * case["head"]
        passes = 2 if case["train"] else 1
        return {"bytes": 2 * passes * n * e + case["batch"] * case["length"] * 8, "flops": 3 * passes * n}
    pairs, queries, keys = _pairs(case)
    H, K, D = case["heads"], case["kv_heads"], case["head"]
    # q, k, v in and the output out; in training the output's gradient in, and three gradients out
    rows = 2 * H * queries + 2 * K * keys
    return {"bytes": e * D * rows * (2 if case["train"] else 1), "flops": pairs * H * D * (14 if case["train"] else 4)}


# ---- the same in 64 bits

def exact(case, seed):
    s, family = prepare(case, seed), case["family"]
    if family == "norm":
        x, w, b = (s[k].double().requires_grad_(case["train"]) for k in ("x", "w", "b"))
        var, mean = torch.var_mean(x, dim=1, correction=0, keepdim=True)
        y = torch.addcmul(b, (x - mean) * torch.rsqrt(var + EPS), w)
        if not case["train"]:
            return y
        grads = torch.autograd.grad(y, (x, w, b), s["g"].double())
        return (y.detach(), *grads)
    if family == "rotary":
        def turn(x, sign):
            r, out = case["part"], x.double()
            unit = torch.polar(torch.ones((), dtype=torch.float64, device=DEVICE), sign * s["positions"].double().unsqueeze(-1) * s["freqs"]).unsqueeze(2)
            pairs = out[..., :r].unflatten(-1, (r // 2, 2) if case["interleaved"] else (2, r // 2))
            at = -1 if case["interleaved"] else -2
            z = torch.view_as_real(torch.complex(pairs.select(at, 0), pairs.select(at, 1)) * unit)
            out[..., :r] = (z if case["interleaved"] else z.transpose(-1, -2)).flatten(-2)
            return out
        return (turn(s["x"], 1), turn(s["g"], -1)) if case["train"] else turn(s["x"], 1)
    B, H, K = case["batch"], case["heads"], case["kv_heads"]
    G = H // K
    if work(case)["flops"] > 2e13 or B * H > 2048:
        return None
    o = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEVICE)
    grads = [torch.zeros(s[k].shape, dtype=torch.float64, device=DEVICE) for k in "qkv"] if case["train"] else []
    for b, (n, m) in enumerate(_lengths(case)):
        hidden = torch.ones(n, m, dtype=torch.bool, device=DEVICE).triu(m - n + 1) if case["causal"] else None
        for h in range(H):
            at = [(b, slice(n), h), (b, slice(m), h // G), (b, slice(m), h // G)]
            q, k, v = (s[name][w].double() for name, w in zip("qkv", at))
            scores = torch.mm(q, k.t()).mul_(s["scale"])
            if hidden is not None:
                scores.masked_fill_(hidden, float("-inf"))
            p = torch.softmax(scores, -1)
            if case["causal"] and n > m:
                p[:n - m] = 0
            o[at[0]] = torch.mm(p, v)
            if case["train"]:
                g = s["g"][at[0]].double()
                dp = torch.mm(g, v.t())
                ds = p * (dp - (p * dp).sum(1, keepdim=True)) * s["scale"]
                grads[0][at[0]] = torch.mm(ds, k)
                grads[1][at[1]] += torch.mm(ds.t(), q)
                grads[2][at[2]] += torch.mm(p.t(), g)
    return (o, *grads) if case["train"] else o
