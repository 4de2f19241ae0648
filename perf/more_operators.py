"""The measured operators of a decoder layer: norms, matrix products with their
epilogue, and attention over whole prompts, each forward and backward.

They are what a layer runs beside rotary positions and the paged cache, in the
shapes this package simulates: a decoder layer of 2048 tokens (hidden 4096, 32
query / 8 key-value heads of 128, feed-forward 14336), the design sweep's
largest product (8192 x 8192 x 8192), flash attention of 8 x 4096 tokens with 32
heads, and a decoding batch of 64.  Where `own` is false, run() computes them
from elementary torch operations in 32 bits, rounded once at the end.
"""
from __future__ import annotations

import math
import random

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
BYTES = {"bf16": 2, "f16": 2, "f32": 4}
EPS = 1e-5


def listed():
    return [
        # -- norm ------------------------------------------------------------------
        # a decoding batch between two products: a launch and its latency
        dict(name="norm_decode_64", op="norm", rows=64, dim=4096, type="bf16", center=False, bias=False, backward=False,
             packed=False),
        # an odd width in 32 bits, rows inside wider ones
        dict(name="norm_odd_f32", op="norm", rows=1021, dim=2001, type="f32", center=True, bias=True, backward=False,
             packed=True),
        # a training step of 8 x 4096 tokens, with the gradients of weight and shift
        dict(name="norm_grad_8x4096", op="norm", rows=32768, dim=4096, type="bf16", center=True, bias=True, backward=True,
             packed=False),
        # -- matrix products ---------------------------------------------------------
        # QKV projection of one new token for each of 64 sequences: the weights' bytes
        dict(name="linear_decode_64", op="linear", M=64, N=6144, K=4096, type="bf16", act="none", bias=True, gate=False,
             residual=False, backward=False),
        # down projection of a prompt, onto the residual stream
        dict(name="linear_down_2048", op="linear", M=2048, N=4096, K=14336, type="bf16", act="none", bias=False,
             gate=False, residual=True, backward=False),
        # gradients of the gated feed-forward's first product
        dict(name="linear_gate_grad_2048", op="linear", M=2048, N=14336, K=4096, type="bf16", act="silu", bias=True,
             gate=True, residual=False, backward=True),
        # the design sweep's largest product, with everything an epilogue of an ungated layer has
        dict(name="linear_8192", op="linear", M=8192, N=8192, K=8192, type="f16", act="gelu", bias=True, gate=False,
             residual=True, backward=False),
        # 32-bit values, sizes that no tile and no wide load divides
        dict(name="linear_odd_f32", op="linear", M=1021, N=1000, K=777, type="f32", act="relu", bias=True, gate=False,
             residual=False, backward=False),
        # -- attention over prompts ----------------------------------------------------
        # many short texts seen whole, odd heads
        dict(name="attention_short_24", op="attention", B=24, lo=1, hi=200, Hq=14, Hkv=2, D=96, type="f16", causal=False,
             backward=False, packed=False, lens=11),
        # one prompt, queries, keys and values inside the packed projection
        dict(name="attention_prefill_2048", op="attention", B=1, lo=2048, hi=2048, Hq=32, Hkv=8, D=128, type="bf16",
             causal=True, backward=False, packed=True, lens=1),
        # the simulated flash attention: the largest matrix work
        dict(name="attention_8x4096", op="attention", B=8, lo=4096, hi=4096, Hq=32, Hkv=32, D=128, type="bf16",
             causal=False, backward=False, packed=False, lens=1),
        # a training step on packed texts of different lengths
        dict(name="attention_grad_8", op="attention", B=8, lo=512, hi=8192, Hq=32, Hkv=8, D=128, type="bf16", causal=True,
             backward=True, packed=False, lens=3),
    ]


# ---- drawn cases ----------------------------------------------------------------

def _log(rng, lo, hi):
    """A whole number, uniform over its logarithm."""
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def _width(rng, hi):
    """A width of a layer: mostly of whole 64s, sometimes any number."""
    n = _log(rng, 64, hi)
    return n if rng.random() < 0.3 else max(64, n // 64 * 64)


def _draw_norm(rng):
    center = rng.random() < 0.5
    return dict(rows=_log(rng, 1, 65536), dim=_width(rng, 16384), type=rng.choice(("bf16", "bf16", "f16", "f32")),
                center=center, bias=center and rng.random() < 0.7, backward=rng.random() < 0.5, packed=rng.random() < 0.3)


def _draw_linear(rng):
    act = rng.choice(("none", "none", "relu", "gelu", "silu"))
    return dict(M=_log(rng, 1, 16384), N=_width(rng, 16384), K=_width(rng, 16384),
                type=rng.choice(("bf16", "bf16", "f16", "f32")), act=act, bias=rng.random() < 0.5,
                gate=act == "silu" and rng.random() < 0.6, residual=rng.random() < 0.4, backward=rng.random() < 0.4)


def _draw_attention(rng):
    Hkv, G = rng.choice((1, 2, 3, 4, 8)), rng.choice((1, 2, 4, 5, 7, 8))
    lo = _log(rng, 1, 8192)
    return dict(B=_log(rng, 1, 64), lo=lo, hi=_log(rng, lo, 8192), Hq=Hkv * G, Hkv=Hkv,
                D=rng.choice((64, 80, 96, 128, 128, 256)), type=rng.choice(("bf16", "bf16", "f16", "f32")),
                causal=rng.random() < 0.7, backward=rng.random() < 0.4, packed=rng.random() < 0.4,
                lens=rng.randrange(1 << 20))


_DRAWN = {"norm": _draw_norm, "linear": _draw_linear, "attention": _draw_attention}


def draw(rng):
    largest = {}
    for c in listed():
        w = work(c)
        old = largest.get(c["op"], w)
        largest[c["op"]] = {k: max(old[k], w[k]) for k in w}
    while True:
        op = rng.choice(("norm", "linear", "attention"))
        c = dict(op=op, **_DRAWN[op](rng))
        w = work(c)
        # 32 bits have a sixteenth of the matrix rate
        slow = 16 if c["type"] == "f32" and op != "norm" else 1
        if w["bytes"] <= largest[op]["bytes"] and slow * w["flops"] <= largest[op]["flops"]:
            return c


# ---- inputs ---------------------------------------------------------------------

def _lengths(c):
    """Tokens of each sequence: what a data loader or scheduler knows."""
    rng = random.Random(c["lens"])
    return [_log(rng, c["lo"], c["hi"]) for _ in range(c["B"])]


def prepare(case, seed):
    c = dict(case)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    t = TYPES[c["type"]]
    randn = lambda *shape: torch.randn(shape, generator=gen, device="cuda", dtype=t)  # noqa: E731
    if c["op"] == "norm":
        rows, dim = c["rows"], c["dim"]
        # packed: columns of a projection that holds others behind them
        x = randn(rows, dim + (dim // 4 if c["packed"] else 0))[:, :dim]
        x.mul_(1.5).add_(0.25)
        s = dict(c=c, x=x, weight=randn(dim).mul_(0.1).add_(1.0), bias=randn(dim).mul_(0.1) if c["bias"] else None)
        if c["backward"]:  # what the forward pass kept
            s["mean"] = x.double().mean(1).float() if c["center"] else None
            d = x.double() if s["mean"] is None else x.double() - s["mean"].double()[:, None]
            s.update(dy=randn(rows, dim), rstd=(d.square().mean(1) + EPS).rsqrt().float())
        return s
    if c["op"] == "linear":
        M, N, K = c["M"], c["N"], c["K"]
        s = dict(c=c, x=randn(M, K), weight=randn(N, K).mul_(K ** -0.5), bias=randn(N).mul_(0.5) if c["bias"] else None,
                 gate=randn(M, N) if c["gate"] else None, residual=randn(M, N) if c["residual"] else None)
        if c["backward"]:
            s["dy"] = randn(M, N)
            if c["act"] != "none" or c["gate"]:  # what the forward pass kept
                z = s["x"].float() @ s["weight"].float().T
                s["preact"] = (z if s["bias"] is None else z.add_(s["bias"].float())).to(t)
            else:
                s["preact"] = None
        return s
    lens = _lengths(c)
    T, Hq, Hkv, D = sum(lens), c["Hq"], c["Hkv"], c["D"]
    if c["packed"]:
        q, k, v = randn(T, Hq + 2 * Hkv, D).split((Hq, Hkv, Hkv), 1)
    else:
        q, k, v = randn(T, Hq, D), randn(T, Hkv, D), randn(T, Hkv, D)
    starts = torch.cat((torch.zeros(1, dtype=torch.long), torch.tensor(lens).cumsum(0))).int().cuda()
    s = dict(c=c, q=q, k=k, v=v, starts=starts, lens=lens)
    if c["backward"]:
        o, lse = _attend(c, s)
        s.update(dout=randn(T, Hq, D), out=o.to(t), lse=lse)
    return s


# ---- the operators ----------------------------------------------------------------

def run(state):
    c = state["c"]
    if own:
        return _run_own(c, state)
    return {"norm": _plain_norm, "linear": _plain_linear, "attention": _plain_attention}[c["op"]](c, state)


def _run_own(c, s):
    from paper_2607_11262_amd import ops
    if c["op"] == "norm":
        if not c["backward"]:
            return ops.layer_norm(s["x"], s["weight"], s["bias"], eps=EPS, center=c["center"])
        dx, dw, db = ops.layer_norm_backward(s["dy"], s["x"], s["weight"], s["rstd"], s["mean"], bias=c["bias"])
        return {"dx": dx, "dweight": dw, "dbias": db}
    if c["op"] == "linear":
        act = None if c["act"] == "none" else c["act"]
        if not c["backward"]:
            return ops.linear(s["x"], s["weight"], s["bias"], activation=act, gate=s["gate"], residual=s["residual"])
        dx, dw, db, dg = ops.linear_backward(s["dy"], s["x"], s["weight"], activation=act, preact=s["preact"],
                                             gate=s["gate"], bias=c["bias"])
        return {"dx": dx, "dweight": dw, "dbias": db, "dgate": dg}
    if not c["backward"]:
        return ops.prompt_attention(s["q"], s["k"], s["v"], s["starts"], causal=c["causal"])
    dq, dk, dv = ops.prompt_attention_backward(s["dout"], s["q"], s["k"], s["v"], s["out"], s["lse"], s["starts"],
                                               causal=c["causal"])
    return {"dq": dq, "dk": dk, "dv": dv}


def _plain_norm(c, s):
    x, w = s["x"].float(), s["weight"].float()
    if c["backward"]:
        h = (x if s["mean"] is None else x - s["mean"][:, None]) * s["rstd"][:, None]
        dy = s["dy"].float()
        g = dy * w
        dx = g - h * (g * h).mean(1, keepdim=True)
        if c["center"]:
            dx = dx - g.mean(1, keepdim=True)
        t = s["x"].dtype
        # sums over many rows: 64 bits
        return {"dx": (dx * s["rstd"][:, None]).to(t), "dweight": (dy * h).sum(0, dtype=torch.float64).to(t),
                "dbias": dy.sum(0, dtype=torch.float64).to(t) if c["bias"] else None}
    if c["center"]:
        x = x - x.mean(1, keepdim=True)
    y = x * (x.square().mean(1, keepdim=True) + EPS).rsqrt() * w
    return (y if s["bias"] is None else y + s["bias"].float()).to(s["x"].dtype)


def _activation(act, z):
    if act == "relu":
        return z.clamp(min=0.0)
    if act == "gelu":
        return z * 0.5 * (1.0 + torch.erf(z * 0.5 ** 0.5))
    return z / (1.0 + torch.exp(-z)) if act == "silu" else z


def _slope(act, z):
    if act == "relu":
        return (z > 0).float()
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z * 0.5 ** 0.5)) + z * torch.exp(-0.5 * z * z) * (2.0 * math.pi) ** -0.5
    g = 1.0 / (1.0 + torch.exp(-z))
    return g * (1.0 + z * (1.0 - g))


def _plain_linear(c, s):
    x, w, t = s["x"].float(), s["weight"].float(), s["x"].dtype
    if not c["backward"]:
        y = x @ w.T
        if s["bias"] is not None:
            y = y + s["bias"].float()
        y = _activation(c["act"], y)
        if s["gate"] is not None:
            y = y * s["gate"].float()
        return (y if s["residual"] is None else y + s["residual"].float()).to(t)
    dz, dg = s["dy"].float(), None
    if s["preact"] is not None:
        z = s["preact"].float()
        if s["gate"] is not None:
            dg = (dz * _activation(c["act"], z)).to(t)
            dz = dz * s["gate"].float()
        if c["act"] != "none":
            dz = dz * _slope(c["act"], z)
    return {"dx": (dz @ w).to(t), "dweight": (dz.T @ x).to(t),
            "dbias": dz.sum(0, dtype=torch.float64).to(t) if c["bias"] else None, "dgate": dg}


def _sequences(c, s):
    """Of each sequence its rows and, head by head in 32 bits, queries (scaled),
    keys and values [key-value heads, group or 1, tokens, D]."""
    G, first = c["Hq"] // c["Hkv"], 0
    heads = lambda x: x.float().transpose(0, 1).contiguous()  # noqa: E731
    for n in s["lens"]:
        at = slice(first, first + n)
        first += n
        q = heads(s["q"][at]).mul_(c["D"] ** -0.5).view(c["Hkv"], G * n, c["D"])
        yield n, at, q, heads(s["k"][at]), heads(s["v"][at])


def _scores(c, n, q, k):
    w = (q @ k.transpose(1, 2)).view(c["Hq"], n, n)
    if c["causal"]:
        j = torch.arange(n, device="cuda")
        w.masked_fill_(j > j[:, None], float("-inf"))
    return w


def _attend(c, s):
    """Output and log-sum in 32 bits."""
    out = torch.empty(s["q"].shape, dtype=torch.float32, device="cuda")
    lse = torch.empty(s["q"].shape[:2], dtype=torch.float32, device="cuda")
    for n, at, q, k, v in _sequences(c, s):
        w = _scores(c, n, q, k)
        m = w.amax(-1, keepdim=True)
        w = w.sub_(m).exp_()
        total = w.sum(-1, keepdim=True)
        o = (w.view(c["Hkv"], -1, n) @ v).view(c["Hq"], n, c["D"]) / total
        out[at] = o.transpose(0, 1)
        lse[at] = (m + total.log())[..., 0].T
    return out, lse


def _plain_attention(c, s):
    t = s["q"].dtype
    if not c["backward"]:
        return _attend(c, s)[0].to(t)
    dq, dk, dv = torch.empty_like(s["dout"]), *(s["k"].new_empty(s["k"].shape) for _ in range(2))
    D, Hq, Hkv = c["D"], c["Hq"], c["Hkv"]
    for n, at, q, k, v in _sequences(c, s):
        p = _scores(c, n, q, k).sub_(s["lse"][at].T[..., None]).exp_()
        do = s["dout"][at].float().transpose(0, 1).contiguous()
        delta = (do * s["out"][at].float().transpose(0, 1)).sum(-1, keepdim=True)
        do = do.view(Hkv, -1, D)
        ds = (do @ v.transpose(1, 2)).view(Hq, n, n).sub_(delta).mul_(p).view(Hkv, -1, n)
        dv[at] = (p.view(Hkv, -1, n).transpose(1, 2) @ do).transpose(0, 1).to(t)
        dk[at] = (ds.transpose(1, 2) @ q).transpose(0, 1).to(t)  # q is scaled
        dq[at] = ((ds @ k) * D ** -0.5).view(Hq, n, D).transpose(0, 1).to(t)
    return {"dq": dq, "dk": dk, "dv": dv}


# ---- what a pass cannot do without ------------------------------------------------

def work(case):
    c = case
    e = BYTES[c["type"]]
    if c["op"] == "norm":
        n, dim = c["rows"] * c["dim"], c["dim"]
        if c["backward"]:
            return {"bytes": e * (3 * n + (2 + c["bias"]) * dim) + 4 * c["rows"] * (1 + c["center"]), "flops": 14 * n}
        return {"bytes": e * (2 * n + (1 + c["bias"]) * dim), "flops": 8 * n}
    if c["op"] == "linear":
        M, N, K = c["M"], c["N"], c["K"]
        if c["backward"]:
            kept = c["act"] != "none" or c["gate"]
            return {"bytes": e * (2 * (M * K + N * K) + M * N * (1 + kept + 2 * c["gate"]) + N * c["bias"]),
                    "flops": 4 * M * N * K}
        return {"bytes": e * (M * K + N * K + M * N * (1 + c["gate"] + c["residual"]) + N * c["bias"]),
                "flops": 2 * M * N * K}
    lens = _lengths(c)
    pairs = sum(n * (n + 1) // 2 if c["causal"] else n * n for n in lens)
    T, Hq, Hkv = sum(lens), c["Hq"], c["Hkv"]
    if c["backward"]:
        return {"bytes": 4 * e * T * (Hq + Hkv) * c["D"] + 4 * T * Hq, "flops": 10 * c["D"] * Hq * pairs}
    return {"bytes": 2 * e * T * (Hq + Hkv) * c["D"], "flops": 4 * c["D"] * Hq * pairs}


# ---- from the definitions, in 64 bits ----------------------------------------------

def _leaf(x):
    return None if x is None else x.detach().double().requires_grad_()


def _exact_act(act, z):
    if act == "gelu":  # z times the normal distribution below z
        return z * torch.special.ndtr(z)
    return {"none": lambda a: a, "relu": torch.relu, "silu": lambda a: a * torch.sigmoid(a)}[act](z)


def exact(case, seed):
    s = prepare(case, seed)
    c = s["c"]
    if c["op"] == "norm":
        x, w, b = _leaf(s["x"]), _leaf(s["weight"]), _leaf(s["bias"])
        d = x - x.mean(1, keepdim=True) if c["center"] else x
        y = d / torch.sqrt((d * d).mean(1, keepdim=True) + EPS) * w + (0.0 if b is None else b)
        if not c["backward"]:
            return y.detach()
        y.backward(s["dy"].double())
        return {"dx": x.grad, "dweight": w.grad, "dbias": None if b is None else b.grad}
    if c["op"] == "linear":
        x, w = s["x"].double(), s["weight"].double()
        if not c["backward"]:
            y = torch.mm(x, w.T.contiguous())
            if s["bias"] is not None:
                y += s["bias"].double()
            y = _exact_act(c["act"], y)
            if s["gate"] is not None:
                y = y * s["gate"].double()
            return y if s["residual"] is None else y + s["residual"].double()
        dz, dg = s["dy"].double(), None
        if s["preact"] is not None:
            z, g = _leaf(s["preact"]), _leaf(s["gate"])
            y = _exact_act(c["act"], z)
            (y if g is None else y * g).backward(dz)
            dz, dg = z.grad, None if g is None else g.grad
        return {"dx": torch.mm(dz, w), "dweight": torch.mm(dz.T.contiguous(), x),
                "dbias": dz.sum(0) if c["bias"] else None, "dgate": dg}
    Hq, Hkv, G = c["Hq"], c["Hkv"], c["Hq"] // c["Hkv"]
    results = [torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")]
    if c["backward"]:
        results += [torch.zeros(s["k"].shape, dtype=torch.float64, device="cuda") for _ in range(2)]
    first = 0
    for n in s["lens"]:
        at = slice(first, first + n)
        first += n
        hidden = torch.ones(n, n, dtype=torch.bool, device="cuda").triu(1) if c["causal"] else None
        for h in range(Hq):
            q, k, v = (x.double() for x in (s["q"][at, h], s["k"][at, h // G], s["v"][at, h // G]))
            w = q @ k.T.contiguous() / c["D"] ** 0.5
            if hidden is not None:
                w = w.masked_fill(hidden, -float("inf"))
            w = w.softmax(-1)
            if not c["backward"]:
                results[0][at, h] = w @ v
                continue
            do = s["dout"][at, h].double()
            dw = do @ v.T.contiguous()
            ds = w * (dw - (w * dw).sum(-1, keepdim=True)) / c["D"] ** 0.5
            results[0][at, h] = ds @ k
            results[1][at, h // G] += ds.T.contiguous() @ q
            results[2][at, h // G] += w.T.contiguous() @ do
    return dict(zip(("dq", "dk", "dv"), results)) if c["backward"] else results[0]
