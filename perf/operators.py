"""The measured operators: rotary positions, appending keys and values to a
paged cache, and attention over that cache for a batch that shares a prefix.

They are one serving step, in the shapes this package simulates: split-KV
decode (batch 64, 32 query / 8 key-value heads, head dim 128, 512 to 32768
keys), a decoder layer's rotation at prefill (2048 tokens), flash attention
of 8 x 4096 tokens with 32 heads; and a training step's gradient of the
rotation.  Where `own` is false, run() computes them from elementary torch
operations in 32 bits, rounded once at the end.
"""
from __future__ import annotations

import random

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
BYTES = {"bf16": 2, "f16": 2, "f32": 4}


def listed():
    return [
        # -- rotary: the rotation by itself ------------------------------------------
        # one new token for each of 64 sequences: a launch and its latency
        dict(name="rotary_decode_64", op="rotary", B=64, S=1, H=32, D=128, R=128, type="bf16", interleaved=False,
             backward=False, packed=False, stretch=1.0),
        # a prompt's queries and keys, seen inside the packed QKV projection
        dict(name="rotary_prefill_2048", op="rotary", B=1, S=2048, H=40, D=128, R=128, type="bf16", interleaved=False,
             backward=False, packed=True, stretch=4.0),
        # gradient of a training step's queries
        dict(name="rotary_grad_8x4096", op="rotary", B=8, S=4096, H=32, D=128, R=128, type="bf16", interleaved=True,
             backward=True, packed=False, stretch=1.0),
        # 32-bit values, part of an odd head, an odd number of tokens and heads
        dict(name="rotary_part_f32", op="rotary", B=3, S=1021, H=7, D=80, R=32, type="f32", interleaved=True,
             backward=False, packed=False, stretch=1.0),
        # -- append: keys and values into the cache, queries rotated beside them -----
        # a decode step of 64 sequences behind a shared prefix
        dict(name="append_decode_64", op="append", B=64, new_lo=1, new_hi=1, own_lo=16, own_hi=1024, prefix=8192, Hq=32,
             Hkv=8, D=128, R=128, page=64, type="bf16", interleaved=False, heads_first=False, q=True, lens=1004),
        # several prompts at once, pages kept head by head
        dict(name="append_prompts_16", op="append", B=16, new_lo=512, new_hi=8192, own_lo=0, own_hi=0, prefix=0, Hq=32,
             Hkv=8, D=128, R=128, page=64, type="bf16", interleaved=False, heads_first=True, q=True, lens=7),
        # a few drafted tokens each, odd heads, half of the head rotated, no queries
        dict(name="append_part_f16", op="append", B=7, new_lo=1, new_hi=9, own_lo=0, own_hi=300, prefix=1000, Hq=9,
             Hkv=3, D=80, R=40, page=16, type="f16", interleaved=True, heads_first=False, q=False, lens=3),
        # -- attention over the cache ------------------------------------------------
        # one short sequence, one token: latency
        dict(name="attention_one_512", op="attention", B=1, new_lo=1, new_hi=1, own_lo=511, own_hi=511, prefix=0, Hq=32,
             Hkv=8, D=128, page=64, type="bf16", heads_first=False, lens=1),
        # split-KV decode, 64 ragged sequences of 512 to 32768 keys, nothing shared
        dict(name="attention_decode_64", op="attention", B=64, new_lo=1, new_hi=1, own_lo=512, own_hi=32767, prefix=0,
             Hq=32, Hkv=8, D=128, page=64, type="bf16", heads_first=False, lens=1004),
        # 64 short continuations of one long prefix
        dict(name="attention_prefix_64", op="attention", B=64, new_lo=1, new_hi=1, own_lo=16, own_hi=1024, prefix=8192,
             Hq=32, Hkv=8, D=128, page=64, type="bf16", heads_first=False, lens=5),
        # drafted tokens to verify: several rows a sequence, odd heads, a prefix that ends inside a page
        dict(name="attention_drafts_24", op="attention", B=24, new_lo=1, new_hi=6, own_lo=0, own_hi=700, prefix=1000,
             Hq=14, Hkv=2, D=96, page=16, type="f16", heads_first=True, lens=11),
        # prompts asked of one long document: the largest matrix work
        dict(name="attention_prompts_8", op="attention", B=8, new_lo=64, new_hi=512, own_lo=0, own_hi=0, prefix=32768,
             Hq=32, Hkv=8, D=128, page=64, type="bf16", heads_first=False, lens=2),
    ]


# ---- drawn cases ----------------------------------------------------------------

def _log(rng, lo, hi):
    """A whole number, uniform over its logarithm."""
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def _heads(rng):
    Hkv, G = rng.choice((1, 2, 3, 4, 8)), rng.choice((1, 2, 4, 5, 7, 8))
    return Hkv * G, Hkv


def _draw_rotary(rng):
    D = rng.choice((64, 80, 96, 128, 128, 256))
    return dict(B=_log(rng, 1, 64), S=_log(rng, 1, 8192), H=_log(rng, 1, 64), D=D, R=rng.choice((D, D, D // 2)),
                type=rng.choice(("bf16", "bf16", "f16", "f32")), interleaved=rng.random() < 0.5,
                backward=rng.random() < 0.5, packed=rng.random() < 0.3, stretch=rng.choice((1.0, 4.0)))


def _draw_append(rng):
    D = rng.choice((64, 80, 128, 128, 256))
    Hq, Hkv = _heads(rng)
    one = rng.random() < 0.4
    return dict(B=_log(rng, 1, 256), new_lo=1, new_hi=1 if one else _log(rng, 2, 8192), own_lo=0,
                own_hi=_log(rng, 1, 4096), prefix=rng.choice((0, _log(rng, 16, 32768))), Hq=Hq, Hkv=Hkv, D=D,
                R=rng.choice((D, D // 2)), page=rng.choice((16, 32, 64, 128)), type=rng.choice(("bf16", "f16")),
                interleaved=rng.random() < 0.5, heads_first=rng.random() < 0.5, q=rng.random() < 0.7,
                lens=rng.randrange(1 << 20))


def _draw_attention(rng):
    Hq, Hkv = _heads(rng)
    kind = rng.choice(("decode", "decode", "drafts", "prompts"))
    new = dict(decode=1, drafts=rng.randint(2, 8), prompts=_log(rng, 9, 512))[kind]
    return dict(B=_log(rng, 1, 16 if kind == "prompts" else 128), new_lo=1, new_hi=new, own_lo=0,
                own_hi=_log(rng, 1, 32767 if kind != "prompts" else 4096),
                prefix=rng.choice((0, _log(rng, 16, 32768), _log(rng, 16, 32768))), Hq=Hq, Hkv=Hkv,
                D=rng.choice((64, 96, 128, 128, 256)), page=rng.choice((16, 32, 64, 128)),
                type=rng.choice(("bf16", "f16")), heads_first=rng.random() < 0.5, lens=rng.randrange(1 << 20))


_DRAWN = {"rotary": _draw_rotary, "append": _draw_append, "attention": _draw_attention}


def _plain_bytes(c):
    """What the plain form's largest temporaries hold, roughly."""
    if c["op"] != "attention":
        return 0
    new, lens = _lengths(c)
    G = c["Hq"] // c["Hkv"]
    keys = len(lens) * max(lens) * c["Hkv"] * c["D"] * 8
    scores = len(lens) * c["Hkv"] * G * max(new) * max(lens) * 8 + sum(new) * c["Hq"] * c["prefix"] * 8
    return keys + scores


def draw(rng):
    largest = {}
    for c in listed():
        w = work(c)
        old = largest.get(c["op"], w)
        largest[c["op"]] = {k: max(old[k], w[k]) for k in w}
    while True:
        op = rng.choice(("rotary", "append", "attention", "attention"))
        c = dict(op=op, **_DRAWN[op](rng))
        if any(v == 3072 for v in c.values()):
            continue
        w = work(c)
        if all(w[k] <= largest[op][k] for k in w) and _plain_bytes(c) <= 24e9:
            return c


# ---- inputs ---------------------------------------------------------------------

def _lengths(c):
    """New tokens of each sequence, and its own keys once they are in (the
    prefix apart): what a scheduler knows."""
    rng = random.Random(c["lens"])
    new = [_log(rng, c["new_lo"], c["new_hi"]) for _ in range(c["B"])]
    old = [_log(rng, c["own_lo"] + 1, c["own_hi"] + 1) - 1 for _ in range(c["B"])]
    return new, [n + o for n, o in zip(new, old)]


def _table(positions, R, stretch):
    """[positions, R] of 32 bits: cosines, then sines, the positions shrunk by
    `stretch` for a longer context."""
    f = 10000.0 ** (-torch.arange(0, R, 2, dtype=torch.float64, device="cuda") / R)
    a = torch.arange(positions, dtype=torch.float64, device="cuda")[:, None] / stretch * f
    return torch.cat((a.cos(), a.sin()), 1).float()


def _pages(c, new, lens, gen):
    """A cache of shuffled pages with a few to spare, everything in it random
    as if earlier steps had filled it; page table and the prefix's pages."""
    page, prefix = c["page"], c["prefix"] if c["op"] == "attention" else 0
    n_prefix = -(-prefix // page)
    counts = [-(-n // page) for n in lens]
    total = n_prefix + sum(counts)
    order = torch.randperm(total + 5, generator=gen, device="cuda").int()
    shape = (total + 5, c["Hkv"], page, c["D"]) if c["heads_first"] else (total + 5, page, c["Hkv"], c["D"])
    caches = [torch.randn(shape, generator=gen, device="cuda", dtype=TYPES[c["type"]]) for _ in range(2)]
    if c["heads_first"]:
        caches = [x.transpose(1, 2) for x in caches]
    first = torch.tensor([n_prefix + sum(counts[:b]) for b in range(len(counts))], device="cuda")
    at = first[:, None] + torch.arange(max(counts), device="cuda")
    table = order[at.clamp(max=total - 1)].contiguous()
    return caches, table, order[:n_prefix].contiguous()


def _cumulated(values):
    return torch.cat((torch.zeros(1, dtype=torch.long), torch.tensor(values).cumsum(0))).int().cuda()


def prepare(case, seed):
    c = dict(case)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    t = TYPES[c["type"]]
    randn = lambda *shape: torch.randn(shape, generator=gen, device="cuda", dtype=t)  # noqa: E731
    if c["op"] == "rotary":
        # packed: heads of a projection that holds as many values beside them
        x = randn(c["B"], c["S"], c["H"] + (c["H"] // 5 if c["packed"] else 0), c["D"])[:, :, :c["H"]]
        if c["S"] == 1:
            positions = torch.randint(0, 32768, (c["B"], 1), generator=gen, device="cuda")
        else:
            positions = torch.arange(c["S"], device="cuda") + torch.randint(0, 24576, (c["B"], 1), generator=gen, device="cuda")
        return dict(c=c, x=x, positions=positions, table=_table(32768, c["R"], c["stretch"]))
    new, lens = _lengths(c)
    T = sum(new)
    (kc, vc), pages, prefix_pages = _pages(c, new, lens, gen)
    state = dict(c=c, k_cache=kc, v_cache=vc, pages=pages, lens=torch.tensor(lens).int().cuda(),
                 starts=None if c["new_hi"] == 1 else _cumulated(new), T=T, new_max=max(new), len_max=max(lens))
    if c["op"] == "append":
        state.update(k=randn(T, c["Hkv"], c["D"]), v=randn(T, c["Hkv"], c["D"]),
                     q=randn(T, c["Hq"], c["D"]) if c["q"] else None,
                     table=_table(c["prefix"] + max(lens), c["R"], 1.0))
    else:
        # queries a little larger than the keys: some rows look at few keys
        state.update(q=randn(T, c["Hq"], c["D"]).mul_(2.0), prefix_pages=prefix_pages if c["prefix"] else None)
    return state


# ---- the operators ----------------------------------------------------------------

def run(state):
    c = state["c"]
    if own:
        return _run_own(c, state)
    return {"rotary": _plain_rotary, "append": _plain_append, "attention": _plain_attention}[c["op"]](c, state)


def _run_own(c, s):
    from paper_2607_11262_amd import ops
    if c["op"] == "rotary":
        f = ops.rotary_backward if c["backward"] else ops.rotary
        return f(s["x"], s["positions"], s["table"], interleaved=c["interleaved"])
    if c["op"] == "append":
        q = ops.append_kv(s["k"], s["v"], s["k_cache"], s["v_cache"], s["pages"], s["lens"], starts=s["starts"],
                          table=s["table"], interleaved=c["interleaved"], prefix_len=c["prefix"], q=s["q"])
        return {"k_cache": s["k_cache"], "v_cache": s["v_cache"], "q": q}
    return ops.shared_prefix_attention(s["q"], s["k_cache"], s["v_cache"], s["pages"], s["lens"], starts=s["starts"],
                                       prefix_pages=s["prefix_pages"], prefix_len=c["prefix"])


def _rotate(x, cos, sin, R, interleaved, backward=False):
    """x [.., heads, D] in 32 bits, cos / sin [.., 1, R / 2]."""
    if backward:
        sin = -sin
    if interleaved:
        a, b = x[..., 0:R:2], x[..., 1:R:2]
        y = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    else:
        a, b = x[..., :R // 2], x[..., R // 2:R]
        y = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    return torch.cat((y, x[..., R:]), -1)


def _plain_rotary(c, s):
    cos, sin = s["table"][s["positions"]].unsqueeze(-2).chunk(2, -1)
    return _rotate(s["x"].float(), cos, sin, c["R"], c["interleaved"], c["backward"]).to(s["x"].dtype)


def _tokens(s):
    """Sequence and own index of every new token."""
    B = s["lens"].shape[0]
    starts = s["starts"] if s["starts"] is not None else torch.arange(B + 1, device="cuda")
    token = torch.arange(s["T"], device="cuda")
    seq = torch.searchsorted(starts.long(), token, right=True) - 1
    return seq, token - starts[seq], (s["lens"] - starts.diff())[seq] + token - starts[seq]


def _plain_append(c, s):
    seq, _, own_index = _tokens(s)
    cos, sin = s["table"][c["prefix"] + own_index].unsqueeze(1).chunk(2, -1)
    at = s["pages"][seq, own_index // c["page"]].long(), own_index % c["page"]
    s["k_cache"][at] = _rotate(s["k"].float(), cos, sin, c["R"], c["interleaved"]).to(s["k"].dtype)
    s["v_cache"][at] = s["v"]
    q = None
    if s["q"] is not None:
        q = _rotate(s["q"].float(), cos, sin, c["R"], c["interleaved"]).to(s["q"].dtype)
    return {"k_cache": s["k_cache"], "v_cache": s["v_cache"], "q": q}


def _plain_attention(c, s):
    Hq, Hkv, D, page, P = c["Hq"], c["Hkv"], c["D"], c["page"], c["prefix"]
    G, B, N, L = Hq // Hkv, s["lens"].shape[0], s["new_max"], s["len_max"]
    seq, i, limit = _tokens(s)
    q = s["q"].float().view(s["T"], Hkv, G, D) * D ** -0.5

    def keys(cache, at):  # [.., page, heads, D] to [heads, .., keys, D]
        return cache[at].float().movedim(-2, 0).flatten(-3, -2)

    # a sequence's own keys: new tokens padded to the longest, keys too
    rows = q.new_zeros(Hkv, B, N, G, D)
    rows[:, seq, i] = q.transpose(0, 1)
    last = limit.new_full((B, N), -1)
    last[seq, i] = limit
    j = torch.arange(L, device="cuda")
    hidden = j > last[:, :, None]
    at = s["pages"][:, :-(-L // page)].long()
    k, v = keys(s["k_cache"], at)[:, :, :L], keys(s["v_cache"], at)[:, :, :L]
    k.masked_fill_((j >= s["lens"][:, None])[:, :, None], 0.0)
    v.masked_fill_((j >= s["lens"][:, None])[:, :, None], 0.0)
    w = (rows.flatten(2, 3) @ k.transpose(2, 3)).view(Hkv, B, N, G, L)
    w.masked_fill_(hidden[:, :, None], float("-inf"))
    w = w[:, seq, i]                                   # [heads, T, G, L]
    m = w.amax(-1, keepdim=True)
    if P:
        at = s["prefix_pages"].long()
        kp, vp = keys(s["k_cache"], at)[:, :P], keys(s["v_cache"], at)[:, :P]
        wp = (q.transpose(0, 1).flatten(1, 2) @ kp.transpose(1, 2)).view(Hkv, s["T"], G, P)
        m = torch.maximum(m, wp.amax(-1, keepdim=True))
        wp = wp.sub_(m).exp_()
    w = w.sub_(m).exp_()
    total = w.sum(-1, keepdim=True)
    padded = w.new_zeros(Hkv, B, N, G, L)
    padded[:, seq, i] = w
    o = (padded.flatten(2, 3) @ v).view(Hkv, B, N, G, D)[:, seq, i]
    if P:
        total = total + wp.sum(-1, keepdim=True)
        o = o + (wp.flatten(1, 2) @ vp).view(Hkv, s["T"], G, D)
    return (o / total).transpose(0, 1).reshape(s["T"], Hq, D).to(s["q"].dtype)


# ---- what a pass cannot do without ------------------------------------------------

def work(case):
    c = case
    e = BYTES[c["type"]]
    if c["op"] == "rotary":
        n = c["B"] * c["S"] * c["H"]
        return {"bytes": 2 * e * n * c["D"] + c["B"] * c["S"] * (8 + 4 * c["R"]), "flops": 3 * n * c["R"]}
    new, lens = _lengths(c)
    T = sum(new)
    if c["op"] == "append":
        heads = 2 * c["Hkv"] + (c["Hq"] if c["q"] else 0)
        return {"bytes": 2 * e * T * heads * c["D"] + T * (4 + 4 * c["R"]) + 8 * c["B"],
                "flops": 3 * T * (heads - c["Hkv"]) * c["R"]}
    pairs = sum(n * c["prefix"] + n * (m - n) + n * (n + 1) // 2 for n, m in zip(new, lens))
    keys = c["prefix"] + sum(lens)
    return {"bytes": e * c["D"] * (2 * T * c["Hq"] + 2 * keys * c["Hkv"]) + 4 * (keys // c["page"]) + 8 * c["B"],
            "flops": 4 * c["D"] * c["Hq"] * pairs}


# ---- from the definitions, in 64 bits ----------------------------------------------

def _rotate64(x, rows, R, interleaved, sign=1.0):
    """Each pair as a complex number, turned by its table entry."""
    turn = torch.complex(rows[..., :R // 2].double(), sign * rows[..., R // 2:].double()).unsqueeze(-2)
    part = x[..., :R].double()
    pairs = part.unflatten(-1, (R // 2, 2)) if interleaved else part.unflatten(-1, (2, R // 2)).transpose(-1, -2)
    turned = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
    y = x.double()
    y[..., :R] = turned.flatten(-2) if interleaved else turned.transpose(-1, -2).flatten(-2)
    return y


def exact(case, seed):
    s = prepare(case, seed)
    c = s["c"]
    if c["op"] == "rotary":
        return _rotate64(s["x"], s["table"][s["positions"]], c["R"], c["interleaved"], -1.0 if c["backward"] else 1.0)
    new, lens = _lengths(c)
    pages = s["pages"].tolist()
    if c["op"] == "append":
        k_cache, v_cache = s["k_cache"].double(), s["v_cache"].double()
        where = [(b, m - n + i) for b, (n, m) in enumerate(zip(new, lens)) for i in range(n)]
        row = s["table"][torch.tensor([c["prefix"] + j for _, j in where], device="cuda")]
        page = torch.tensor([pages[b][j // c["page"]] for b, j in where], device="cuda")
        slot = torch.tensor([j % c["page"] for _, j in where], device="cuda")
        k_cache[page, slot] = _rotate64(s["k"], row, c["R"], c["interleaved"])
        v_cache[page, slot] = s["v"].double()
        q = None if s["q"] is None else _rotate64(s["q"], row, c["R"], c["interleaved"])
        return {"k_cache": k_cache, "v_cache": v_cache, "q": q}
    D, P, page = c["D"], c["prefix"], c["page"]
    G = c["Hq"] // c["Hkv"]
    shared = s["prefix_pages"].tolist() if P else []

    def gathered(cache, b, n):
        keys = []
        if P:
            keys.append(cache[torch.tensor(shared, device="cuda")].reshape(-1, c["Hkv"], D)[:P])
        keys.append(cache[torch.tensor(pages[b][:-(-n // page)], device="cuda")].reshape(-1, c["Hkv"], D)[:n])
        return torch.cat(keys).double()

    out = torch.empty(s["T"], c["Hq"], D, dtype=torch.float64, device="cuda")
    first = 0
    for b, (n, m) in enumerate(zip(new, lens)):
        k, v = gathered(s["k_cache"], b, m), gathered(s["v_cache"], b, m)
        seen = torch.arange(P + m, device="cuda") <= P + m - n + torch.arange(n, device="cuda")[:, None]
        for h in range(c["Hq"]):
            w = s["q"][first:first + n, h].double() @ k[:, h // G].T.contiguous() / D ** 0.5
            w = torch.where(seen, w, -float("inf")).softmax(-1)
            out[first:first + n, h] = w @ v[:, h // G].contiguous()
        first += n
    return out
