"""Performance cases of the operators around the update GEMM: what else a training step, and a served layer, calls.

A case is a dict of plain values.  `listed()` names the ones that are always timed, `draw(rng)` gives further cases of the
same families over their whole range of sizes, `prepare` makes what a program holds before the call, `run` is one pass,
`work` the bytes and operations one pass cannot do without, `exact` the results in 64 bits.  Where `own` is false `run`
computes the operators in elementary torch operations in 32 bits; where it is true it calls the package.

Families
  serve   y = act(x W^T + b) with the weights kept as 8-bit integers and a scale per output channel; x [T x I] is rounded to
          8-bit integers with a scale per token inside the call
  train   the two dense products of a layer in a training step, in 8-bit integers: y = x W^T + b, and dx = g W.  The weights
          move every step, so both of their 8-bit forms (a scale per output, and per input, channel) are made within the pass
  lookup  rows of an embedding table, scaled
  embed   the same and the table's gradient: the rows of the incoming gradient summed by token, a padding token left out
  adamw   one AdamW step over the tensors of a transformer block.  States in binary32, or in 8 bits: e4m3 codes of m and
          of sqrt(v) with a power-of-two scale for every 256 elements, rounded stochastically from counter-based random
          words (key: the seed; counter: the element's quad, the tensor's number, the step)
"""
from __future__ import annotations

import math

import torch

own = False

DEVICE = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"bf16": 2, "f32": 4, "q8": 1}
BETAS, EPS, LR, DECAY = (0.9, 0.999), 1e-8, 1e-3, 0.01
BLOCK = 256                     # elements that share a scale of an 8-bit state


def _i8(name, family, tokens, fin, fout, dtype="bf16", out="bf16", relu=False):
    return {"name": name, "family": family, "tokens": tokens, "in": fin, "out": fout, "dtype": dtype, "out_dtype": out, "relu": relu}


def _embed(name, family, tokens, vocab, width, dtype="bf16", grad="f32", ids="int64"):
    return {"name": name, "family": family, "tokens": tokens, "vocab": vocab, "width": width, "dtype": dtype, "grad": grad, "ids": ids}


def _adamw(name, width, state="f32", param="bf16", grad="f32", master=False):
    return {"name": name, "family": "adamw", "width": width, "state": state, "param": param, "grad": grad, "master": master}


def listed():
    return [
        # one token of a served layer: the latency of a call
        _i8("i8_one_token", "serve", 1, 1024, 4096),
        # a batch of 16 sequences, one token each, through the large decoder MLP layer: the weights are read once
        _i8("i8_decode", "serve", 16, 8192, 28672, relu=True),
        # a prompt batch through the large decoder MLP layer: 32768 tokens, hidden 8192, FFN 28672
        _i8("i8_decoder", "serve", 32768, 8192, 28672),
        # 8 images of 197 positions, odd widths, binary32 tensors
        _i8("i8_train_ragged", "train", 8 * 197, 1001, 1333, dtype="f32", out="f32"),
        # the transformer MLP in training: hidden 1024, FFN 4096, 32 x 512 tokens
        _i8("i8_train", "train", 16384, 1024, 4096),
        # the next tokens of 8 sequences
        _embed("lookup_8", "lookup", 8, 32768, 1024),
        # 32 x 512 tokens of a transformer with hidden 1024
        _embed("embed_train", "embed", 16384, 50001, 1024),
        # a large table: 32768 tokens, hidden 4096, everything in bf16
        _embed("embed_large", "embed", 32768, 120001, 4096, grad="bf16", ids="int32"),
        # a small block, binary32 throughout: launches and host time count
        _adamw("adamw_small", 64, param="f32"),
        # a ViT-Base block, binary32 states and master weights behind bf16 parameters, gradients as the update GEMM writes them
        _adamw("adamw_master", 768, master=True),
        # the same block with 8-bit states, bf16 gradients as the layers return them
        _adamw("adamw_q8", 768, state="q8", grad="bf16"),
        # a large block with 8-bit states
        _adamw("adamw_q8_large", 4096, state="q8"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    family = rng.choice(["serve", "serve", "train", "lookup", "embed", "embed", "adamw", "adamw"])
    if family in ("serve", "train"):
        most = 32768 * 8192 * 28672 // (2 if family == "train" else 1)
        while True:
            T = _log_int(rng, 1 if family == "serve" else 64, 32768)
            if family == "serve" and rng.random() < 0.4:
                T = _log_int(rng, 1, 64)
            I, O = _log_int(rng, 64, 8192), _log_int(rng, 64, 28672)
            if T * I * O <= most:
                break
        dtype = rng.choice(["bf16", "bf16", "f32"])
        c = _i8("", family, T, I, O, dtype=dtype, out=dtype if family == "train" else rng.choice(["bf16", "f32"]), relu=family == "serve" and rng.random() < 0.5)
    elif family in ("lookup", "embed"):
        dtype = rng.choice(["bf16", "bf16", "f32"])
        while True:
            N, V, D = _log_int(rng, 1, 32768), _log_int(rng, 100, 131072), _log_int(rng, 64, 4096)
            if V * D <= 120001 * 4096:
                break
        c = _embed("", family, N, V, D, dtype=dtype, grad=rng.choice(["f32", dtype]), ids=rng.choice(["int32", "int64"]))
    else:
        state = rng.choice(["f32", "q8"])
        param = rng.choice(["bf16", "bf16", "f32"])
        c = _adamw("", _log_int(rng, 24, 3800), state=state, param=param, grad=rng.choice(["f32", param]), master=param == "bf16" and rng.random() < 0.5)
    c.pop("name", None)
    return c


# ---- inputs

def _generator(seed):
    return torch.Generator(device=DEVICE).manual_seed(int(seed) % (1 << 62))


def _activations(gen, T, C, dtype):
    """Normal values under a spread of channel sizes, a few tokens of padding (rows of zeros) where there are many."""
    x = torch.randn(T, C, generator=gen, device=DEVICE)
    x *= torch.randn(C, generator=gen, device=DEVICE).mul_(0.5).exp_()
    if T >= 64:
        x[torch.randint(T, (T // 64,), generator=gen, device=DEVICE)] = 0
    return x.to(dtype)


def _shapes(w):
    """The tensors of a transformer block: two norms, qkv, proj, fc1, fc2."""
    return [(w,), (w,), (3 * w, w), (3 * w,), (w, w), (w,), (w,), (w,), (4 * w, w), (4 * w,), (w, 4 * w), (w,)]


def prepare(case, seed):
    gen, family = _generator(seed), case["family"]
    s = {"case": case}
    if family in ("serve", "train"):
        T, I, O, dtype = case["tokens"], case["in"], case["out"], DTYPES[case["dtype"]]
        s["x"] = _activations(gen, T, I, dtype)
        w = torch.randn(O, I, generator=gen, device=DEVICE) * (I ** -0.5) * torch.rand(O, 1, generator=gen, device=DEVICE).add_(0.5)
        s["bias"] = torch.randn(O, generator=gen, device=DEVICE).to(dtype)
        if family == "serve":
            # kept as 8-bit integers; rows start on 16-byte boundaries
            top = w.abs().amax(1)
            s["ws"] = top / 127
            s["wq"] = torch.zeros(O, -(-I // 16) * 16, dtype=torch.int8, device=DEVICE)[:, :I]
            s["wq"].copy_((w * (127 / top)[:, None]).round_())
        else:
            s["w"] = w.to(dtype)
            size = torch.randn(T, 1, generator=gen, device=DEVICE).exp_()        # gradients: tokens differ in size by far
            s["g"] = (torch.randn(T, O, generator=gen, device=DEVICE) * size * 1e-3).to(dtype)
    elif family in ("lookup", "embed"):
        N, V, D, dtype = case["tokens"], case["vocab"], case["width"], DTYPES[case["dtype"]]
        s["table"] = (torch.randn(V, D, generator=gen, device=DEVICE) * 0.02).to(dtype)
        # the frequency of a word falls with its rank
        u = torch.rand(N, generator=gen, device=DEVICE, dtype=torch.float64)
        ids = (u * math.log(V + 1)).exp_().sub_(1).clamp_(0, V - 1).to(torch.int64)
        s["padding"] = V - 1
        if N >= 64:
            ids[N - N // 16:] = V - 1
        s["ids"] = ids.to(torch.int32 if case["ids"] == "int32" else torch.int64)
        s["scale"] = math.sqrt(D)
        if family == "embed":
            s["g"] = (torch.randn(N, D, generator=gen, device=DEVICE) * 1e-3).to(dtype)
    else:
        state, param = case["state"], DTYPES[case["param"]]
        lists = {k: [] for k in ("p", "master", "g", "m", "v")}
        for shape in _shapes(case["width"]):
            new = lambda: torch.randn(shape, generator=gen, device=DEVICE)       # noqa: E731
            p = new() * 0.02 if len(shape) == 2 else 1 + 0.1 * new()
            size = 1e-3 * new().mul_(1.5).exp_()                                # elements differ in size by far
            r = size * (0.5 + new().abs_())
            m = 0.3 * r * new()
            lists["p"].append(p.to(param))
            lists["master"].append(p if case["master"] else None)
            lists["g"].append((size * new()).to(DTYPES[case["grad"]]))
            if state == "f32":
                lists["m"].append(m)
                lists["v"].append(r.square_())
            else:
                lists["m"].append(_code(m, torch.full((-(-m.numel() // 4), 4), 0x80008000, dtype=torch.int64, device=DEVICE), 0))
                lists["v"].append(_code(r, torch.full((-(-m.numel() // 4), 4), 0x80008000, dtype=torch.int64, device=DEVICE), 16))
        s.update(lists, step=100, seed=int(seed) % (1 << 31))
    return s


# ---- plain forms

def _to_i8(x):
    """(codes, scale): the rows of x in 127 steps of a row's largest magnitude."""
    x = x.float()
    top = x.abs().amax(1, keepdim=True)
    up = torch.where(top > 0, 127 / top, torch.zeros_like(top))
    return (x * up).round_(), top / 127


def _product(q, s, wq, ws, bias, relu, dtype):
    y = (q @ wq.float().t()) * (s * ws.reshape(1, -1))
    if bias is not None:
        y = y + bias.float()
    if relu:
        y = y.clamp_(min=0)
    return y.to(dtype)


def _lookup(s):
    return (s["table"][s["ids"].long()].float() * s["scale"]).to(s["table"].dtype)


def _table_gradient(s):
    case, ids = s["case"], s["ids"].long()
    rows = torch.where((ids == s["padding"])[:, None], torch.zeros((), device=DEVICE), s["g"].float())
    total = torch.zeros(case["vocab"], case["width"], device=DEVICE).index_add_(0, ids, rows)
    return (total * s["scale"]).to(DTYPES[case["grad"]])


_M32 = 0xffffffff


def _random_words(tensors, step, seed):
    """Philox4x32-10 words [quads, 4] of each tensor's quads of elements, as int64."""
    quads = [-(-t.numel() // 4) for t in tensors]
    c0 = torch.cat([torch.arange(q, dtype=torch.int64, device=DEVICE) for q in quads])
    c1 = c0 >> 32
    c0 = c0 & _M32
    c2 = torch.cat([torch.full((q,), k, dtype=torch.int64, device=DEVICE) for k, q in enumerate(quads)])
    c3 = torch.full_like(c0, (1 << 31) + step)
    k0, k1 = seed & _M32, seed >> 32 & _M32
    for _ in range(10):
        p0, p1 = c0 * 0xD2511F53, c2 * 0xCD9E8D57                # 64 bits, wrapped
        c0, c2 = (p1 >> 32 & _M32) ^ c1 ^ k0, (p0 >> 32 & _M32) ^ c3 ^ k1
        c1, c3 = p1 & _M32, p0 & _M32
        k0, k1 = k0 + 0x9E3779B9 & _M32, k1 + 0xBB67AE85 & _M32
    return torch.stack((c0, c1, c2, c3), 1).split(quads)


def _code(u, words, shift):
    """[codes, scales] of an 8-bit state: e4m3 codes of u over a power of two for every BLOCK elements, the smallest that
    holds the block's largest magnitude, rounded to one of the two neighbours by 16 bits of each element's word.  What is
    not negative (shift 16: sqrt(v)) stays above zero where it was."""
    n, blocks = u.numel(), -(-u.numel() // BLOCK)
    flat = torch.zeros(blocks * BLOCK, device=u.device)
    flat[:n] = u.reshape(-1)
    size = flat.abs()
    top = size.view(blocks, BLOCK).amax(1)
    bits = top.view(torch.int32)
    e = (bits >> 23) - 127 - 8 + ((bits & 0x7fffff) > 0x600000)
    e = torch.where(top > 0, e.clamp(-126, 126), torch.zeros_like(e))
    scale, down = (e + 127 << 23).view(torch.float32), (127 - e << 23).view(torch.float32)
    y = (size.view(blocks, BLOCK) * down[:, None]).view(-1)[:n]
    small = y < 2.0 ** -6
    t = torch.where(small, y + 2.0 ** -6, y).view(torch.int32)
    t = t + ((words.reshape(-1)[:n] >> shift & 0xffff) << 4).to(torch.int32)
    code = (t >> 20) - torch.where(small, 968, 960)
    if shift:
        code = torch.where(y > 0, code.clamp(min=1), code)
    code = code | torch.where(flat[:n] < 0, 128, 0)
    return [code.to(torch.uint8).view(torch.float8_e4m3fn).view(u.shape), scale]


def _value(state):
    """The binary32 values of an 8-bit state."""
    codes, scale = state
    return (codes.float().reshape(-1) * scale.repeat_interleave(BLOCK)[:codes.numel()]).view(codes.shape)


def _adamw_step(s):
    case, step = s["case"], s["step"]
    b1, b2 = BETAS
    rate, grow, keep = LR / (1 - b1 ** step), 1 / math.sqrt(1 - b2 ** step), 1 - LR * DECAY
    q8 = case["state"] == "q8"
    words = _random_words(s["p"], step, s["seed"]) if q8 else None
    for k, p in enumerate(s["p"]):
        g, m, v, w = s["g"][k].float(), s["m"][k], s["v"][k], s["master"][k]
        old_m, old_v = (_value(m), _value(v).square_()) if q8 else (m, v)
        new_m = old_m * b1 + g * (1 - b1)
        new_v = old_v * b2 + (g * g) * (1 - b2)
        r = new_v.sqrt()
        new = (w if w is not None else p).float() * keep - (new_m * rate) / (r * grow + EPS)
        p.copy_(new)
        if w is not None:
            w.copy_(new)
        if q8:
            for to, what in ((m, _code(new_m, words[k], 0)), (v, _code(r, words[k], 16))):
                to[0].copy_(what[0])
                to[1].copy_(what[1])
        else:
            m.copy_(new_m)
            v.copy_(new_v)


def run(s):
    case, family = s["case"], s["case"]["family"]
    if own:
        import paper_2203_10991_amd as nm
    if family == "serve":
        if own:
            return nm.nm_linear_i8(s["x"], s["wq"], s["ws"], s["bias"], relu=case["relu"], out_dtype=DTYPES[case["out_dtype"]])
        return _product(*_to_i8(s["x"]), s["wq"], s["ws"], s["bias"], case["relu"], DTYPES[case["out_dtype"]])
    if family == "train":
        if own:
            return nm.nm_linear_i8(s["x"], *nm.nm_quant_i8(s["w"]), s["bias"]), nm.nm_linear_i8(s["g"], *nm.nm_quant_i8_t(s["w"]))
        y = _product(*_to_i8(s["x"]), *_to_i8(s["w"]), s["bias"], False, s["x"].dtype)
        return y, _product(*_to_i8(s["g"]), *_to_i8(s["w"].t()), None, False, s["g"].dtype)
    if family == "lookup":
        return nm.nm_embed(s["table"], s["ids"], s["scale"]) if own else _lookup(s)
    if family == "embed":
        if own:
            return (nm.nm_embed(s["table"], s["ids"], s["scale"]),
                    nm.nm_embed_grad(s["g"], s["ids"], case["vocab"], s["scale"], padding_idx=s["padding"], out_dtype=DTYPES[case["grad"]]))
        return _lookup(s), _table_gradient(s)
    s["step"] += 1
    if own:
        nm.nm_adamw(s["p"], s["g"], s["m"], s["v"], s["step"], lr=LR, betas=BETAS, eps=EPS, weight_decay=DECAY,
                    masters=s["master"] if case["master"] else None, seed=s["seed"])
    else:
        _adamw_step(s)
    return [s["p"], s["m"], s["v"], s["master"]]


# ---- what a pass needs

def work(case):
    family = case["family"]
    if family in ("serve", "train"):
        T, I, O, e = case["tokens"], case["in"], case["out"], SIZE[case["dtype"]]
        if family == "serve":
            return {"bytes": T * I * e + O * I + O * (4 + e) + T * O * SIZE[case["out_dtype"]], "flops": 2 * T * I * O}
        return {"bytes": 2 * e * (T * I + T * O) + e * O * (I + 1), "flops": 4 * T * I * O}
    if family in ("lookup", "embed"):
        N, V, D, e = case["tokens"], case["vocab"], case["width"], SIZE[case["dtype"]]
        b = N * (4 if case["ids"] == "int32" else 8) + 2 * N * D * e
        return {"bytes": b + (N * D * e + V * D * SIZE[case["grad"]] if family == "embed" else 0), "flops": N * D * (2 if family == "embed" else 1)}
    n = sum(math.prod(shape) for shape in _shapes(case["width"]))
    state = SIZE[case["state"]] + (4 / BLOCK if case["state"] == "q8" else 0)
    # parameters, master weights and both states in and out, the gradient in (with master weights the parameters are only written)
    weights = SIZE[case["param"]] + 8 if case["master"] else 2 * SIZE[case["param"]]
    return {"bytes": n * (weights + SIZE[case["grad"]] + 4 * state), "flops": 20 * n}


# ---- the same in 64 bits

def _rows_i8_64(x):
    """Integers and scales of x's rows, from the definition: the nearest of 255 steps of largest/127, ties to even."""
    x = x.double()
    step = x.abs().max(1)[0].div_(127)
    q = torch.nan_to_num(x / step.unsqueeze(1), nan=0.0).round_()
    return q, step


def _linear_64(x, wq, ws, bias, relu):
    q, step = _rows_i8_64(x)
    y = torch.mm(q, wq.double().t().contiguous())
    y.mul_(step.unsqueeze(1)).mul_(ws.double())
    if bias is not None:
        y.add_(bias.double())
    return torch.relu_(y) if relu else y


def _state_64(u, words, shift):
    """An 8-bit state's code values and scales: u over the power of two, down or up to a multiple of the step of its octave."""
    n = u.numel()
    padded = torch.nn.functional.pad(u.reshape(-1), (0, -n % BLOCK)).view(-1, BLOCK)
    top = padded.abs().max(1)[0]
    # the smallest power of two that brings the largest magnitude to 448 or below
    power = torch.where(top > 0, torch.ceil(torch.log2(torch.where(top > 0, top, 1.0) / 448)), 0.0).clamp_(-126, 126)
    y = (padded / torch.exp2(power).unsqueeze(1)).view(-1)[:n]
    octave = torch.frexp(y)[1].clamp_(min=-5) - 4                 # three bits behind the leading one, from 2^-6 on
    step = torch.exp2(octave.double())
    chance = (words.view(-1)[:n] // (1 << shift) % 65536).double() / 65536
    mag = torch.floor(y.abs() / step + chance) * step
    if shift:
        mag = torch.where((y != 0) & (mag == 0), 2.0 ** -9, mag)
    return [(mag * torch.sign(y)).view(u.shape), torch.exp2(power)]


def exact(case, seed):
    s, family = prepare(case, seed), case["family"]
    if family == "serve":
        return _linear_64(s["x"], s["wq"], s["ws"], s["bias"], case["relu"])
    if family == "train":
        return (_linear_64(s["x"], *_rows_i8_64(s["w"]), s["bias"], False),
                _linear_64(s["g"], *_rows_i8_64(s["w"].t()), None, False))
    if family in ("lookup", "embed"):
        ids = s["ids"].long()
        out = torch.index_select(s["table"], 0, ids).double().mul_(s["scale"])
        if family == "lookup":
            return out
        there = (ids != s["padding"]).nonzero().squeeze(1)
        grad = torch.zeros(case["vocab"], case["width"], dtype=torch.float64, device=DEVICE)
        grad.index_put_((ids[there],), s["g"][there].double() * s["scale"], accumulate=True)
        return out, grad
    b1, b2 = BETAS
    t = s["step"] + 1
    words = _random_words(s["p"], t, s["seed"]) if case["state"] == "q8" else None
    out = [[], [], [], []]
    for k, p in enumerate(s["p"]):
        g, m, v, w = s["g"][k].double(), s["m"][k], s["v"][k], s["master"][k]
        if case["state"] == "q8":
            wide = lambda st: st[1].double().repeat_interleave(BLOCK)[:p.numel()].view(p.shape) * st[0].double()      # noqa: E731
            m, v = wide(m), wide(v) ** 2
        m = torch.lerp(m.double(), g, 1 - b1)
        v = torch.lerp(v.double(), g * g, 1 - b2)
        x = p.double() if w is None else w.double()
        x = x - LR * DECAY * x - LR * (m / (1 - b1 ** t)) / ((v / (1 - b2 ** t)).sqrt() + EPS)
        out[0].append(x)
        out[3].append(None if w is None else x)
        if case["state"] == "q8":
            out[1].append(_state_64(m, words[k], 0))
            out[2].append(_state_64(v.sqrt(), words[k], 16))
        else:
            out[1].append(m)
            out[2].append(v)
    return out
