"""The operators of a decoder layer against their formulas in 64 bits: norms, matrix
products with their epilogue, attention over prompts, forward and backward -- at
the sizes, strides, masks and values where they can go wrong."""
import math

import pytest
import torch

import layer_reference as R
from paper_2607_11262_amd import api, ops

pytestmark = pytest.mark.gpu

BF, HF, F = torch.bfloat16, torch.float16, torch.float32
TYPES = [BF, HF, F]


def gen(seed):
    return torch.Generator().manual_seed(seed)


def randn(g, *shape, dtype=F, scale=1.0, shift=0.0):
    return (torch.randn(shape, generator=g) * scale + shift).to(dtype)


def note(msg):
    print(f"[gpu] {msg}", flush=True)


def close(got, ref, err, dtype, what):
    """got (in dtype) is ref within err and one rounding."""
    assert got.dtype == dtype and got.shape == ref.shape, what
    got, bound = got.detach().cpu().double(), R.rounded(ref, err, dtype)
    bad = ~((got - ref).abs() <= bound) & ~(got == ref) & ~(got.isnan() & ref.isnan())
    if bad.any():
        i = tuple(int(x) for x in bad.nonzero()[0])
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} outside; at {i}: {got[i]} for {ref[i]} +- {bound[i]}")


def d64(*tensors):
    return [None if t is None else t.detach().cpu().double() for t in tensors]


# ---- norm -----------------------------------------------------------------------------

NORM = [(1, 1), (3, 2), (1, 4096), (5, 64), (7, 63), (2, 1000), (9, 1024), (4, 1025), (3, 2048), (6, 8192), (2, 8200),
        (2, 20000), (1, 32768), (2, 33000), (70, 129), (600, 24)]


@pytest.mark.parametrize("center", [True, False])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,dim", NORM)
def test_norm(rows, dim, dtype, center):
    note(f"norm {rows}x{dim} {dtype} {center}")
    g = gen(rows * 7 + dim)
    x, dy = randn(g, rows, dim, dtype=dtype, scale=2.0, shift=0.5), randn(g, rows, dim, dtype=dtype)
    w, b = randn(g, dim, dtype=dtype, scale=0.2, shift=1.0), randn(g, dim, dtype=dtype, scale=0.3)
    mean = torch.empty(rows, device="cuda") if center else None
    rstd = torch.empty(rows, device="cuda")
    for weight, bias in ((w, b), (w, None), (None, b), (None, None)):
        y = ops.layer_norm(x.cuda(), None if weight is None else weight.cuda(), None if bias is None else bias.cuda(), eps=1e-3,
                           center=center, mean=mean, rstd=rstd)
        ref, m, r, err, m_err, r_err = R.norm(*d64(x, weight, bias), 1e-3, center)
        close(y, ref, err, dtype, "y")
        if center:
            close(mean, m, m_err, F, "mean")
        close(rstd, r, r_err, F, "rstd")
        dx, dw, db = ops.layer_norm_backward(dy.cuda(), x.cuda(), None if weight is None else weight.cuda(), rstd, mean,
                                             bias=bias is not None)
        refs = R.norm_gradient(*d64(dy, x, weight, mean, rstd))
        close(dx, refs[0], refs[3], dtype, "dx")
        assert (dw is None) == (weight is None) and (db is None) == (bias is None)
        if dw is not None:
            close(dw, refs[1], refs[4], dtype, "dw")
        if db is not None:
            close(db, refs[2], refs[5], dtype, "db")


@pytest.mark.parametrize("dtype", TYPES)
def test_norm_of_many_rows(dtype):
    g = gen(1)
    x, dy = randn(g, 5003, 72, dtype=dtype), randn(g, 5003, 72, dtype=dtype)
    w = randn(g, 72, dtype=dtype)
    mean, rstd = torch.empty(5003, device="cuda"), torch.empty(5003, device="cuda")
    y = ops.layer_norm(x.cuda(), w.cuda(), mean=mean, rstd=rstd)
    ref = R.norm(*d64(x, w, None), 1e-5, True)
    close(y, ref[0], ref[3], dtype, "y")
    got = ops.layer_norm_backward(dy.cuda(), x.cuda(), w.cuda(), rstd, mean, bias=True)
    again = ops.layer_norm_backward(dy.cuda(), x.cuda(), w.cuda(), rstd, mean, bias=True)
    refs = R.norm_gradient(*d64(dy, x, w, mean, rstd))
    for a, c, r, e, name in zip(got, again, refs, refs[3:], ("dx", "dw", "db")):
        close(a, r, e, dtype, name)
        assert torch.equal(a, c), name


@pytest.mark.parametrize("dtype", TYPES)
def test_norm_layouts(dtype):
    """Strides, alignments, leading dimensions, in place."""
    g = gen(2)
    rows, dim = 6, 136
    x, dy, w, b = (randn(g, *s, dtype=dtype).cuda() for s in ((rows, dim), (rows, dim), (dim,), (dim,)))
    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    y = ops.layer_norm(x, w, b, mean=mean, rstd=rstd)
    grads = ops.layer_norm_backward(dy, x, w, rstd, mean, bias=True)
    for shift in (0, 1, 2, 4, 8):
        def off(t):
            wide = torch.full((*t.shape[:-1], dim + 24), 7.0, device="cuda", dtype=dtype)
            v = wide[..., shift:shift + dim]
            v.copy_(t)
            return v
        xo, do, wo, bo = off(x), off(dy), off(w), off(b)
        out = off(x)
        got = ops.layer_norm(xo, wo, bo, out=out)
        assert got is out
        # another variant takes the sums in another order: the reference decides
        ref = R.norm(*d64(x, w, b), 1e-5, True)
        close(out, ref[0], ref[3], dtype, f"shift {shift}")
        refs = R.norm_gradient(*d64(dy, x, w, mean, rstd))
        for a, r, e in zip(ops.layer_norm_backward(do, xo, wo, rstd, mean, bias=True), refs, refs[3:]):
            close(a, r, e, dtype, f"gradient, shift {shift}")
        rest = out._base.clone()
        rest[..., shift:shift + dim] = 7.0
        assert (rest == 7.0).all()
    assert torch.equal(ops.layer_norm(x.view(2, 3, dim), w, b), y.view(2, 3, dim))
    assert torch.equal(ops.layer_norm(x[0], w, b), y[0])
    d3 = ops.layer_norm_backward(dy.view(3, 2, dim), x.view(3, 2, dim), w, rstd, mean, bias=True)
    assert torch.equal(d3[0], grads[0].view(3, 2, dim)) and torch.equal(d3[1], grads[1])
    one = x[:1].expand(rows, dim)
    assert torch.equal(ops.layer_norm(one, w, b), ops.layer_norm(one.contiguous(), w, b))
    z = x.clone()
    assert ops.layer_norm(z, w, b, out=z) is z and torch.equal(z, y)
    for shape in ((0, dim), (3, 0, dim)):
        assert ops.layer_norm(x.new_empty(shape), w, b).shape == shape
    e = x.new_empty(0, dim)
    dx, dw, db = ops.layer_norm_backward(e, e, w, rstd[:0], mean[:0], bias=True)
    assert dx.shape == (0, dim) and (dw == 0).all() and (db == 0).all()


def test_norm_values():
    """Constant rows, large means, rows that are not finite beside others that are."""
    x = torch.full((2, 512), 3.0, device="cuda")
    assert (ops.layer_norm(x) == 0).all()
    g = gen(5)
    big = randn(g, 3, 4096, scale=1e-3, shift=1000.0)
    ref = R.norm(*d64(big, None, None), 1e-5, True)
    close(ops.layer_norm(big.cuda()), ref[0], ref[3], F, "a mean far from zero")
    x = randn(g, 4, 64).cuda()
    y = ops.layer_norm(x)
    x[1, 3], x[2, 5] = float("inf"), float("nan")
    z = ops.layer_norm(x)
    assert torch.equal(z[[0, 3]], y[[0, 3]]) and z[[1, 2]].isnan().any(1).all()
    assert (ops.layer_norm(torch.zeros(2, 8, device="cuda"), center=False, eps=0.0)).isnan().all()


# ---- products ----------------------------------------------------------------------------

LINEAR = [(1, 1, 1), (1, 64, 64), (3, 5, 7), (2, 130, 33), (16, 256, 512), (17, 200, 96), (33, 7, 1000), (64, 384, 256),
          (100, 128, 2048), (129, 257, 65), (130, 64, 4000), (256, 256, 64), (200, 136, 72), (300, 520, 264)]
ACTS = [None, "relu", "gelu", "gelu_tanh", "silu"]


def linear_case(M, N, K, dtype, seed=0):
    g = gen(M * 31 + N * 7 + K + seed)
    return (randn(g, M, K, dtype=dtype), randn(g, N, K, dtype=dtype, scale=K ** -0.5), randn(g, N, dtype=dtype),
            randn(g, M, N, dtype=dtype), randn(g, M, N, dtype=dtype), randn(g, M, N, dtype=dtype))


def check_linear(M, N, K, dtype, act, with_bias, with_gate, with_residual):
    x, w, b, gate, res, dy = linear_case(M, N, K, dtype)
    b, gate, res = b if with_bias else None, gate if with_gate else None, res if with_residual else None
    cuda = lambda t: None if t is None else t.cuda()  # noqa: E731
    z = torch.empty(M, N, dtype=dtype, device="cuda")
    y = ops.linear(cuda(x), cuda(w), cuda(b), activation=act, gate=cuda(gate), residual=cuda(res), preact=z)
    ref, zr, err, z_err = R.linear(*d64(x, w, b), act, *d64(gate, res))
    close(y, ref, err, dtype, "y")
    close(z, zr, z_err, dtype, "preact")
    got = ops.linear_backward(cuda(dy), cuda(x), cuda(w), activation=act, preact=z, gate=cuda(gate), bias=with_bias)
    refs, errs = R.linear_gradient(*d64(dy, x, w), act, *d64(z, gate), dtype)
    for a, r, e, name, there in zip(got, refs, errs, ("dx", "dw", "db", "dgate"), (True, True, with_bias, with_gate)):
        assert (a is not None) == there
        if there:
            close(a, r, e, dtype, name)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,N,K", LINEAR)
def test_linear(M, N, K, dtype):
    for i, act in enumerate(ACTS):
        note(f"linear {M}x{N}x{K} {dtype} {act}")
        check_linear(M, N, K, dtype, act, i % 2 == 0, act == "silu", i % 3 == 0)


@pytest.mark.parametrize("dtype", TYPES)
def test_linear_epilogues(dtype):
    for act in ACTS:
        for bits in range(8):
            check_linear(20, 48, 40, dtype, act, bool(bits & 1), bool(bits & 2), bool(bits & 4))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,N,K", [(5, 72, 48), (150, 136, 264), (40, 24, 3000)])
def test_linear_layouts(M, N, K, dtype):
    x, w, b, gate, res, dy = (t.cuda() for t in linear_case(M, N, K, dtype))
    z = torch.empty(M, N, dtype=dtype, device="cuda")
    ops.linear(x, w, b, preact=z)
    refs = R.linear(*d64(x, w, b), "silu", *d64(gate, res))
    grads, errs = R.linear_gradient(*d64(dy, x, w), "silu", *d64(z, gate), dtype)
    for shift in (0, 1, 2, 4, 8):
        def off(t):
            wide = torch.full((*t.shape[:-1], t.shape[-1] + 24), float("nan"), device="cuda", dtype=dtype)
            v = wide[..., shift:shift + t.shape[-1]]
            v.copy_(t)
            return v
        out, keep = off(res), off(z)
        got = ops.linear(off(x), off(w), off(b), activation="silu", gate=off(gate), residual=out, out=out, preact=keep)
        assert got is out
        close(out, refs[0], refs[2], dtype, f"shift {shift}")
        for t in (out, keep):
            rest = t._base.clone()
            rest[..., shift:shift + N] = float("nan")
            assert rest.isnan().all()
        got = ops.linear_backward(off(dy), off(x), off(w), activation="silu", preact=off(z), gate=off(gate), bias=True)
        for a, r, e in zip(got, grads, errs):
            close(a, r, e, dtype, f"gradient, shift {shift}")
    y = ops.linear(x, w, b)
    assert torch.equal(ops.linear(x.view(M, 1, K), w, b), y.view(M, 1, N))
    one = x[:1].expand(M, K)
    assert torch.equal(ops.linear(one, w, b), ops.linear(one.contiguous(), w, b))


# Results of many tiles, whose edges and ends of the sum fall inside tiles and stages.
LARGE = [(2048, 2048, 64), (2040, 3000, 104), (4096, 1032, 40), (3500, 1999, 96), (1, 40000, 64), (20000, 8, 32),
         (2056, 3080, 8), (2048, 4096, 200), (70, 136, 9000), (1000, 300, 4104)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,N,K", LARGE)
def test_linear_large(M, N, K, dtype):
    """Against 64-bit products on the card: each tile kernel, each layout of the operands."""
    g = torch.Generator(device="cuda").manual_seed(M + N + K)
    rand = lambda *s: torch.randn(s, generator=g, device="cuda", dtype=dtype)  # noqa: E731
    x, w, b, gate, res, dy = rand(M, K), rand(N, K), rand(N), rand(M, N), rand(M, N), rand(M, N)

    def check(got, a, c, scale=1.0, plus=0.0, err=0.0, what=""):
        """got is a c^T * scale + plus, for a [m, k] and c [n, k] of 64 bits."""
        ref = (a @ c.T.contiguous()) * scale + plus
        size = 2 * (a.shape[1] + 4) * R.E * (a.abs() @ c.abs().T.contiguous()) * abs(scale) + 4 * R.E * ref.abs() + err
        bad = (got.double() - ref).abs() > R.rounded(ref, size, dtype)
        assert not bad.any(), (what, int(bad.sum()), bad.nonzero()[0].tolist())

    xd, wd, gd = x.double(), w.double(), gate.double()
    z = torch.empty(M, N, dtype=dtype, device="cuda")
    y = ops.linear(x, w, b, gate=gate, residual=res, preact=z)
    check(z, xd, wd, plus=b.double(), err=R.E * b.double().abs(), what="preact")
    ref = (xd @ wd.T.contiguous() + b.double()) * gd + res.double()
    size = 2 * (K + 6) * R.E * ((xd.abs() @ wd.abs().T.contiguous() + b.double().abs()) * gd.abs() + res.double().abs())
    assert ((y.double() - ref).abs() <= R.rounded(ref, size, dtype)).all()
    dx, dw, db, _ = ops.linear_backward(dy, x, w, bias=True)
    dyd = dy.double()
    check(dx, dyd, wd.T.contiguous(), what="dx")
    check(dw, dyd.T.contiguous(), xd.T.contiguous(), what="dw")
    assert ((db.double() - dyd.sum(0)).abs() <= R.rounded(dyd.sum(0), (M / 4 + 40) * R.E * dyd.abs().sum(0), dtype)).all()
    # rows behind the operands' ends are not finite and reach nothing
    pad = lambda t: torch.nn.functional.pad(t, (0, 8, 0, 9), value=float("nan"))[:t.shape[0], :t.shape[1]]  # noqa: E731
    assert torch.equal(ops.linear(pad(x), pad(w), b, gate=gate, residual=res), y)
    again = ops.linear_backward(pad(dy), pad(x), pad(w), bias=True)
    assert torch.equal(again[0], dx) and torch.equal(again[1], dw)


def test_linear_of_nothing():
    x, w, b = (t.cuda() for t in (torch.ones(4, 8), torch.ones(6, 8), torch.arange(6.0)))
    assert ops.linear(x[:0], w, b).shape == (0, 6)
    assert ops.linear(x, w[:0], b[:0]).shape == (4, 0)
    assert torch.equal(ops.linear(x[:, :0].contiguous(), w[:, :0].contiguous(), b), b.expand(4, 6))
    dx, dw, db, _ = ops.linear_backward(x.new_empty(0, 6), x[:0], w, bias=True)
    assert dx.shape == (0, 8) and (dw == 0).all() and dw.shape == (6, 8) and (db == 0).all()
    dx, dw, db, _ = ops.linear_backward(x.new_empty(4, 0), x, w[:0], bias=True)
    assert (dx == 0).all() and dx.shape == (4, 8) and dw.shape == (0, 8) and db.shape == (0,)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,N,K", [(150, 140, 72), (3, 40, 600), (256, 256, 256)])
def test_linear_values_not_finite(M, N, K, dtype):
    """An infinity or NaN reaches its own row or column and nothing else; what lies behind
    the operands' ends reaches nothing."""
    g = gen(9)
    x, w = randn(g, M, K, dtype=dtype).cuda(), randn(g, N, K, dtype=dtype).cuda()
    y = ops.linear(x, w)
    pad = torch.full((M + 300, K + 8), float("nan"), device="cuda", dtype=dtype)
    pad[:M, :K] = x
    assert torch.equal(ops.linear(pad[:M, :K], w), y)
    x2, w2 = x.clone(), w.clone()
    x2[1, K - 1], w2[N - 1, 0] = float("inf"), float("nan")
    z = ops.linear(x2, w2)
    hit = torch.zeros(M, N, dtype=torch.bool, device="cuda")
    hit[1], hit[:, N - 1] = True, True
    assert torch.equal(~z.isfinite(), hit) and torch.equal(z[~hit], y[~hit])
    big = torch.tensor([[-1e4, -60.0, -1.0, 0.0, 1.0, 60.0, 1e4, float("nan")]], device="cuda").to(dtype)
    eye = torch.eye(8, device="cuda", dtype=dtype)
    for act in ACTS:
        if dtype == HF and act is None:
            continue
        v = ops.linear(big[:, :7].contiguous(), eye[:7, :7].contiguous(), activation=act).float()[0]
        assert v.isfinite().all(), act
        if act:
            assert v[0] == 0 and v[6] == big[0, 6].float() and v[3] == 0


# ---- attention over prompts ------------------------------------------------------------------

PROMPT = [
    # dtype, Hq, Hkv, D, lengths
    (BF, 1, 1, 64, [1]), (BF, 4, 2, 128, [1, 2, 3, 31, 32, 33]), (HF, 3, 3, 96, [127, 128, 129]), (F, 2, 1, 64, [65, 64, 1]),
    (BF, 5, 1, 80, [200, 0, 7]), (HF, 8, 2, 256, [40, 1, 130]), (F, 2, 2, 256, [70, 33]), (F, 4, 2, 128, [150]),
    (BF, 2, 2, 256, [257]), (HF, 2, 1, 33, [50, 20]), (BF, 2, 1, 8, [300]), (F, 1, 1, 1, [9, 40]), (BF, 8, 8, 128, [384, 90]),
    (HF, 7, 1, 64, [260]), (BF, 16, 2, 128, [1] * 70), (HF, 4, 4, 128, [513]), (BF, 2, 1, 130, [140]), (F, 2, 1, 100, [129, 64]),
]


def prompt_case(Hq, Hkv, D, lens, dtype, seed=0):
    g = gen(Hq * 100 + D + sum(lens) + seed)
    T = sum(lens)
    starts = torch.tensor([0] + lens).cumsum(0).int()
    return (randn(g, T, Hq, D, dtype=dtype, scale=1.5), randn(g, T, Hkv, D, dtype=dtype), randn(g, T, Hkv, D, dtype=dtype), starts,
            randn(g, T, Hq, D, dtype=dtype))


def check_prompt(q, k, v, starts, dout, causal, scale=None, wrap=lambda t: t):
    dtype = q.dtype
    T, Hq, _ = q.shape
    lse = torch.empty(T, Hq, device="cuda")
    st = None if starts is None else starts.cuda()
    qc, kc, vc, dc = (wrap(t.cuda()) for t in (q, k, v, dout))
    o = ops.prompt_attention(qc, kc, vc, st, causal=causal, scale=scale, lse=lse)
    ref, lr, err, l_err = R.prompt(*d64(q, k, v), starts, causal, scale, dtype)
    close(o, ref, err, dtype, "out")
    close(lse, lr, l_err, F, "lse")
    got = ops.prompt_attention_backward(dc, qc, kc, vc, wrap(o), lse, st, causal=causal, scale=scale)
    refs, errs = R.prompt_gradient(*d64(dout, q, k, v, o, lse), starts, causal, scale, dtype)
    for a, r, e, name in zip(got, refs, errs, ("dq", "dk", "dv")):
        close(a, r, e, dtype, name)
    return o, lse, got


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("case", range(len(PROMPT)))
def test_prompt(case, causal):
    dtype, Hq, Hkv, D, lens = PROMPT[case]
    note(f"prompt {PROMPT[case]} {causal}")
    check_prompt(*prompt_case(Hq, Hkv, D, lens, dtype), causal)


@pytest.mark.parametrize("scale", [0.0, -0.3, 2.0])
@pytest.mark.parametrize("dtype", TYPES)
def test_prompt_scales(dtype, scale):
    q, k, v, _, dout = prompt_case(2, 1, 64, [150], dtype)
    check_prompt(q, k, v, None, dout, True, scale)


@pytest.mark.parametrize("dtype,D", [(BF, 128), (HF, 64), (F, 64), (BF, 40), (BF, 256)])
def test_prompt_tokens_outside(dtype, D):
    """Tokens before the first sequence and behind the last: zeros, and no part of others."""
    g = gen(4)
    starts = torch.tensor([37, 90, 90, 221], dtype=torch.int32)
    q, dout = randn(g, 300, 4, D, dtype=dtype), randn(g, 300, 4, D, dtype=dtype)
    k, v = randn(g, 300, 2, D, dtype=dtype), randn(g, 300, 2, D, dtype=dtype)
    for t in (q, k, v, dout):
        t[:37], t[221:] = float("nan"), float("inf")
    lse = torch.empty(300, 4, device="cuda")
    o = ops.prompt_attention(q.cuda(), k.cuda(), v.cuda(), starts.cuda(), lse=lse)
    inside = slice(37, 221)
    alone = (starts - 37).cuda()
    lse2 = torch.empty(184, 4, device="cuda")
    o2 = ops.prompt_attention(*(t[inside].cuda() for t in (q, k, v)), alone, lse=lse2)
    got = ops.prompt_attention_backward(dout.cuda(), q.cuda(), k.cuda(), v.cuda(), o, lse, starts.cuda())
    want = ops.prompt_attention_backward(*(t[inside].cuda() for t in (dout, q, k, v)), o2, lse2, alone)
    for a, b in zip((o, lse, *got), (o2, lse2, *want)):
        assert torch.equal(a[inside], b)
        rest = torch.cat((a[:37], a[221:]))
        assert (rest == (-math.inf if a is lse else 0)).all()


@pytest.mark.parametrize("fill", [float("inf"), float("nan"), -float("inf")])
@pytest.mark.parametrize("dtype,D", [(BF, 128), (HF, 64), (F, 64), (BF, 256), (HF, 72), (BF, 33)])
def test_prompt_later_values_not_finite(dtype, D, fill):
    """What a token must not see reaches neither its result nor its gradient."""
    n, at = 200, 141
    q, k, v, _, dout = (t if t is None else t.cuda() for t in prompt_case(2, 1, D, [n], dtype))
    lse = torch.empty(n, 2, device="cuda")
    o = ops.prompt_attention(q, k, v, lse=lse)
    base = ops.prompt_attention_backward(dout, q, k, v, o, lse)
    for name in ("q", "k", "v", "dout"):
        t = dict(q=q.clone(), k=k.clone(), v=v.clone(), dout=dout.clone())
        t[name][at] = fill
        l2 = torch.empty_like(lse)
        o2 = ops.prompt_attention(t["q"], t["k"], t["v"], lse=l2)
        assert torch.equal(o2[:at], o[:at]) and torch.equal(l2[:at], lse[:at]), name
        if name in ("k", "v"):
            assert not o2[at:].isfinite().all(-1).any(), name
        # scores of one token alone: dq of the tokens before it, dk and dv of the keys behind it
        dq, dk, dv = ops.prompt_attention_backward(t["dout"], t["q"], t["k"], t["v"], o2, l2)
        assert torch.equal(dq[:at], base[0][:at]), name
        if name in ("q", "dout"):
            assert torch.equal(dk[at + 1:], base[1][at + 1:]) and torch.equal(dv[at + 1:], base[2][at + 1:]), name
            assert torch.equal(dq[at + 1:], base[0][at + 1:]), name
            assert dk[:at + 1].isnan().any(-1).all(), name
        if name == "dout":
            assert not dv[:at + 1].isfinite().any(), name


def test_prompt_scores_of_minus_infinity():
    q, k, v, _, _ = prompt_case(1, 1, 64, [40], BF)
    q, k = q.abs() + 0.1, k.clone()
    k[0] = -float("inf")
    lse = torch.empty(40, 1, device="cuda")
    o = ops.prompt_attention(q.cuda(), k.cuda(), v.cuda(), lse=lse)
    assert o[0].isnan().all() and lse[0] == -math.inf and o[1:].isfinite().all()


@pytest.mark.parametrize("dtype,D", [(BF, 128), (HF, 96), (F, 64), (BF, 256), (BF, 64)])
def test_prompt_layouts(dtype, D):
    """Views of a packed projection, heads first, rows that 16 bytes do not divide."""
    q, k, v, starts, dout = prompt_case(4, 2, D, [70, 140], dtype)
    T = q.shape[0]

    def packed(t):
        wide = torch.full((T, t.shape[1] + 3, D), float("nan"), device="cuda", dtype=dtype)
        wide[:, 2:2 + t.shape[1]] = t
        return wide[:, 2:2 + t.shape[1]]

    def heads_first(t):
        return t.transpose(0, 1).contiguous().transpose(0, 1)

    def shifted(by):
        def f(t):
            wide = torch.full((T, t.shape[1], D + 8), float("nan"), device="cuda", dtype=dtype)
            v = wide[..., by:by + D]
            v.copy_(t)
            return v
        return f

    for causal in (True, False):
        for wrap in (packed, heads_first, shifted(1), shifted(2), shifted(8)):
            check_prompt(q, k, v, starts, dout, causal, wrap=wrap)
    # into a given view, the rest as it was
    st = starts.cuda()
    wide = torch.full((T, 9, D + 2), 5.0, device="cuda", dtype=dtype)
    view = wide[:, 3:7, :D]
    assert ops.prompt_attention(q.cuda(), k.cuda(), v.cuda(), st, out=view) is view
    # rows of another alignment may take another kernel: the reference decides
    ref, _, err, _ = R.prompt(*d64(q, k, v), starts, True, None, dtype)
    close(view, ref, err, dtype, "a given view")
    wide[:, 3:7, :D] = 5.0
    assert (wide == 5.0).all()
    one = k[:, :1].cuda().expand(T, 2, D)
    assert torch.equal(ops.prompt_attention(q.cuda(), one, one, st),
                       ops.prompt_attention(q.cuda(), one.contiguous(), one.contiguous(), st))


@pytest.mark.parametrize("B", [1, 62, 63, 64, 65, 200, 4100])
def test_prompt_numbers_of_sequences(B):
    g = gen(B)
    lens = torch.randint(0, 4, (B,), generator=g).tolist()
    lens[-1] = 3
    check_prompt(*prompt_case(2, 1, 64, lens, BF), True)


def test_prompt_long_against_blocks():
    """4500 tokens: rows of the whole against the same rows with 64-bit scores."""
    g = gen(8)
    n, D = 4500, 128
    q, k, v, dout = (randn(g, n, 1, D, dtype=BF) for _ in range(4))
    o, lse, got = ops.prompt_attention(q.cuda(), k.cuda(), v.cuda()), torch.empty(n, 1, device="cuda"), None
    ops.prompt_attention(q.cuda(), k.cuda(), v.cuda(), lse=lse)
    got = ops.prompt_attention_backward(dout.cuda(), q.cuda(), k.cuda(), v.cuda(), o, lse)
    ref, lr, err, l_err = R.prompt(*d64(q, k, v), None, True, None, BF)
    close(o, ref, err, BF, "out")
    close(lse, lr, l_err, F, "lse")
    refs, errs = R.prompt_gradient(*d64(dout, q, k, v, o, lse), None, True, None, BF)
    for a, r, e, name in zip(got, refs, errs, ("dq", "dk", "dv")):
        close(a, r, e, BF, name)
