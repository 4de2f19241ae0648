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


@pytest.mark.parametrize("dtype,D", [(BF, 128), (HF, 64), (F, 64), (BF, 40), (BF, 256), (BF, 33), (F, 130)])
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


# ---- autograd, streams, graphs, refusals ------------------------------------------------------

def directional(f, tensors, dirs, eps=1e-6):
    """Central difference of the 64-bit function f along dirs."""
    up = f(*[t + eps * d for t, d in zip(tensors, dirs)])
    down = f(*[t - eps * d for t, d in zip(tensors, dirs)])
    return (up - down) / (2 * eps)


def check_autograd(op, reference, tensors, seed):
    """Gradients of a weighted sum of op's result against differences of the 64-bit reference:
    the bound is that of 32-bit sums of the terms' size."""
    g = gen(seed)
    leaves = [t.cuda().requires_grad_() for t in tensors]
    y = op(*leaves)
    c = randn(g, *y.shape)
    (y * c.cuda()).sum().backward()
    dirs = [torch.randn(t.shape, generator=g, dtype=torch.float64) for t in tensors]
    got = sum((leaf.grad.cpu().double() * d).sum() for leaf, d in zip(leaves, dirs))
    size = sum((leaf.grad.cpu().double().abs() * d.abs()).sum() for leaf, d in zip(leaves, dirs))
    ref = directional(lambda *a: (reference(*a) * c.double()).sum(), d64(*tensors), dirs)
    # each gradient is off by a few thousand roundings at most (sums of up to 300 products, twice);
    # the difference itself is off by eps^2 and 1e-16 / eps of the sum
    assert abs(got - ref) <= 4096 * R.E * size + 1e-6 * (1 + abs(ref)), (got, ref)


def test_norm_autograd():
    g = gen(1)
    x, w, b = randn(g, 7, 130), randn(g, 130), randn(g, 130)
    check_autograd(lambda x, w, b: ops.layer_norm(x, w, b), lambda x, w, b: R.norm(x, w, b, 1e-5, True)[0], (x, w, b), 2)
    check_autograd(lambda x, w: ops.layer_norm(x.view(7, 10, 13).transpose(0, 1), w, center=False).transpose(0, 1).reshape(7, 130),
                   lambda x, w: R.norm(x.view(70, 13), w, None, 1e-5, False)[0].view(7, 130), (x, w[:13].clone()), 3)
    # only what is asked for
    x1 = x.cuda()
    w1 = w.cuda().requires_grad_()
    ops.layer_norm(x1, w1).sum().backward()
    assert w1.grad is not None and x1.grad is None
    # a gradient that is an expanded view, one that is not contiguous
    x2 = x.cuda().requires_grad_()
    ops.layer_norm(x2, w.cuda()).sum().backward()
    x3 = x.cuda().requires_grad_()
    ops.layer_norm(x3, w.cuda()).t().contiguous().sum().backward()
    assert torch.equal(x2.grad, x3.grad)


@pytest.mark.parametrize("act", ACTS)
def test_linear_autograd(act):
    g = gen(4)
    t = randn(g, 9, 40), randn(g, 24, 40, scale=0.2), randn(g, 24), randn(g, 9, 24), randn(g, 9, 24)
    z = t[0] @ t[1].T + t[2]
    if act == "relu":  # differences do not cross its corner
        t[2].add_(0)
        assert (z.abs() > 1e-4).all()
    check_autograd(lambda x, w, b, gt, r: ops.linear(x, w, b, activation=act, gate=gt, residual=r),
                   lambda x, w, b, gt, r: R.linear(x, w, b, act, gt, r)[0], t, 5)
    check_autograd(lambda x, w: ops.linear(x.view(3, 3, 40), w, activation=act).view(9, 24),
                   lambda x, w: R.linear(x, w, None, act, None, None)[0], t[:2], 6)
    # only what is asked for; the same tensor twice
    w = t[1].cuda().requires_grad_()
    ops.linear(t[0].cuda(), w, activation=act).sum().backward()
    assert w.grad.shape == w.shape
    r = t[3].cuda().requires_grad_()
    y = ops.linear(t[0].cuda(), t[1].cuda(), activation=act, gate=r, residual=r)
    y.sum().backward()
    zd = t[0].double() @ t[1].double().T
    close(r.grad, R.activation(act, zd) + 1, 1e-4 * (1 + zd.abs()), F, "gate and residual")


def test_prompt_autograd():
    g = gen(7)
    starts = torch.tensor([0, 37, 37, 140], dtype=torch.int32)
    q, k, v = randn(g, 140, 4, 32), randn(g, 140, 2, 32), randn(g, 140, 2, 32)
    for causal in (True, False):
        check_autograd(lambda q, k, v: ops.prompt_attention(q, k, v, starts.cuda(), causal=causal),
                       lambda q, k, v: R.prompt(q, k, v, starts, causal, None, F)[0], (q, k, v), 8)
    # one leaf that is queries, keys and values (views of one projection)
    qkv = randn(g, 60, 6, 32)
    check_autograd(lambda x: ops.prompt_attention(*x.split((2, 2, 2), 1)),
                   lambda x: R.prompt(*x.split((2, 2, 2), 1), None, True, None, F)[0], (qkv,), 9)


def test_once_differentiable_and_refused_derivatives():
    from torch.autograd import forward_ad
    x = torch.randn(4, 64, device="cuda", requires_grad=True)
    w = torch.randn(64, 64, device="cuda")
    q = torch.randn(5, 2, 32, device="cuda", requires_grad=True)
    calls = {"norm": lambda t: ops.layer_norm(t), "linear": lambda t: ops.linear(t, w, activation="silu")}
    for name, f in calls.items():
        gx, = torch.autograd.grad(f(x).square().sum(), x, create_graph=True)
        with pytest.raises(RuntimeError):
            gx.sum().backward()
        with forward_ad.dual_level(), torch.no_grad():
            with pytest.raises(ValueError, match="tangent"):
                f(forward_ad.make_dual(x.detach(), torch.ones_like(x)))
    gq, = torch.autograd.grad(ops.prompt_attention(q, q, q).square().sum(), q, create_graph=True)
    with pytest.raises(RuntimeError):
        gq.sum().backward()
    out = torch.empty(4, 64, device="cuda")
    for f in (lambda: ops.layer_norm(x, out=out), lambda: ops.linear(x, w, out=out), lambda: ops.linear(x, w, preact=out),
              lambda: ops.layer_norm(x, rstd=out[:, 0].contiguous()), lambda: ops.prompt_attention(q, q, q, out=torch.empty_like(q))):
        with pytest.raises(ValueError, match="requires a gradient"):
            f()
    for f in (lambda: ops.layer_norm_backward(out, x, None, out[:, 0].contiguous()), lambda: ops.linear_backward(out, x, w),
              lambda: ops.layer_norm(out, out=x), lambda: ops.linear(out, w, out=x)):
        with pytest.raises(ValueError, match="requires a gradient"):
            f()


def test_writes_are_known_to_autograd():
    x = torch.randn(4, 64, device="cuda")
    w = torch.randn(64, 64, device="cuda")
    leaf = torch.randn(4, 64, device="cuda", requires_grad=True)
    q = torch.randn(4, 2, 32, device="cuda")
    lse, rstd = torch.empty(4, 2, device="cuda"), torch.empty(4, device="cuda")
    for t, f in ((x, lambda: ops.layer_norm(x, out=x)), (x, lambda: ops.linear(x, w, out=x, residual=x)),
                 (x, lambda: ops.linear(leaf.detach(), w, preact=x)), (q, lambda: ops.prompt_attention(q.clone(), q.clone(), q.clone(), out=q)),
                 (lse, lambda: ops.prompt_attention(q, q, q, lse=lse)), (rstd, lambda: ops.layer_norm(x, rstd=rstd))):
        before = t._version
        f()
        assert t._version > before
    # an operand changed between forward and backward is noticed
    y = ops.linear(leaf * 1.0, w.clone().requires_grad_())
    wide = (leaf * 2.0)
    y = ops.layer_norm(wide)
    wide.add_(1.0)
    with pytest.raises(RuntimeError, match="modified"):
        y.sum().backward()


def layer_state(dtype=BF, T=300, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    hidden, heads, kv, D, ffn = 256, 4, 2, 64, 512
    rand = lambda *s, scale=1.0: (torch.randn(s, generator=g, device="cuda") * scale).to(dtype)  # noqa: E731
    p = dict(n1=1 + rand(hidden, scale=0.1), wqkv=rand((heads + 2 * kv) * D, hidden, scale=hidden ** -0.5),
             wo=rand(hidden, heads * D, scale=0.06), n2=1 + rand(hidden, scale=0.1), wg=rand(ffn, hidden, scale=hidden ** -0.5),
             wu=rand(ffn, hidden, scale=hidden ** -0.5), wd=rand(hidden, ffn, scale=ffn ** -0.5))
    starts = torch.tensor([0, 1, 130, T], dtype=torch.int32, device="cuda")
    positions = torch.cat([torch.arange(n) for n in (1, 129, T - 130)]).cuda()
    return dict(p=p, x=rand(T, hidden), dy=rand(T, hidden), starts=starts, positions=positions,
                table=ops.rotary_table(T, D), heads=heads, kv=kv, D=D)


def layer(s, x, p):
    """A decoder layer as a user writes it."""
    h = ops.layer_norm(x, p["n1"], center=False)
    q, k, v = ops.linear(h, p["wqkv"]).view(x.shape[0], -1, s["D"]).split((s["heads"], s["kv"], s["kv"]), 1)
    q, k = ops.rotary(q, s["positions"], s["table"]), ops.rotary(k, s["positions"], s["table"])
    x = ops.linear(ops.prompt_attention(q, k, v, s["starts"]).flatten(1), p["wo"], residual=x)
    h = ops.layer_norm(x, p["n2"], center=False)
    return ops.linear(ops.linear(h, p["wg"], activation="silu", gate=ops.linear(h, p["wu"])), p["wd"], residual=x)


def layer64(s, x, p):
    """The same from the formulas in 64 bits, on the CPU."""
    norm = lambda x, w: x / (x.square().mean(1, keepdim=True) + 1e-5).sqrt() * w  # noqa: E731
    rows = s["table"].cpu().double()[s["positions"].cpu()][:, None]

    def turn(t):
        a, b = t.chunk(2, -1)
        c, d = rows.chunk(2, -1)
        return torch.cat((a * c - b * d, b * c + a * d), -1)

    T, G = x.shape[0], s["heads"] // s["kv"]
    q, k, v = (norm(x, p["n1"]) @ p["wqkv"].T).view(T, -1, s["D"]).split((s["heads"], s["kv"], s["kv"]), 1)
    q, k = turn(q), turn(k)
    parts = []
    for a, b in R.spans(T, s["starts"].cpu()):
        w = torch.einsum("ihd,jhd->hij", q[a:b], k[a:b].repeat_interleave(G, 1)) * s["D"] ** -0.5
        w = w.masked_fill(torch.ones(b - a, b - a, dtype=torch.bool).triu(1), -math.inf).softmax(-1)
        parts.append(torch.einsum("hij,jhd->ihd", w, v[a:b].repeat_interleave(G, 1)))
    x = x + torch.cat(parts).flatten(1) @ p["wo"].T
    h = norm(x, p["n2"])
    z = h @ p["wg"].T
    return x + (z * torch.sigmoid(z) * (h @ p["wu"].T)) @ p["wd"].T


@pytest.mark.parametrize("dtype", TYPES)
def test_decoder_layer(dtype):
    """All of them together, forward and backward: the error beside that of the formulas whose
    results of each operator are rounded to the type (about a dozen roundings in a row, each of
    at most u of the values' size, and their sums' worst case is not the root of their number)."""
    s = layer_state(dtype)
    p = {k: v.clone().requires_grad_() for k, v in s["p"].items()}
    x = s["x"].clone().requires_grad_()
    y = layer(s, x, p)
    y.backward(s["dy"])
    p64 = {k: v.detach().cpu().double().requires_grad_() for k, v in s["p"].items()}
    x64 = s["x"].cpu().double().requires_grad_()
    y64 = layer64(s, x64, p64)
    y64.backward(s["dy"].cpu().double())
    for name, a, b in [("y", y, y64), ("x", x.grad, x64.grad)] + [(k, p[k].grad, p64[k].grad) for k in p]:
        a, b = a.detach().cpu().double(), b.detach()
        assert (a - b).norm() <= (24 * R.U[dtype] + 1e-5) * b.norm(), (name, float((a - b).norm() / b.norm()))


def test_decoder_layer_in_a_graph():
    """A training step captured once: replays with other inputs give the eager bits, with eager work
    and synchronizations between them."""
    s = layer_state()
    names = list(s["p"])

    def step(x, dy):
        # leaves of the call's own: no eager graph of them lives while another is captured
        leaf = x.detach().requires_grad_()
        p = {k: v.detach().requires_grad_() for k, v in s["p"].items()}
        y = layer(s, leaf, p)
        return [y.detach(), *torch.autograd.grad(y, [leaf] + [p[k] for k in names], dy)]

    static = s["x"].clone(), s["dy"].clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(*static)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step(*static)
    for seed in range(4):
        g = torch.Generator(device="cuda").manual_seed(seed)
        x, dy = (torch.randn(t.shape, generator=g, device="cuda").to(BF) for t in static)
        static[0].copy_(x)
        static[1].copy_(dy)
        graph.replay()
        eager = step(x, dy)
        torch.cuda.synchronize()
        for a, b in zip(captured, eager):
            assert torch.equal(a, b)


def test_calls_in_two_graphs():
    """Scratch of two captured graphs, replayed in turn and on two streams, is their own."""
    g = torch.Generator(device="cuda").manual_seed(3)
    rand = lambda *t: torch.randn(t, generator=g, device="cuda", dtype=BF)  # noqa: E731
    cases = []
    for M, N, K in ((40, 256, 4096), (24, 384, 8192)):
        x, w, dy, q = rand(M, K), rand(N, K), rand(M, N), rand(M, 4, 64)
        lse = torch.empty(M, 4, device="cuda")

        def calls(x=x, w=w, dy=dy, q=q, lse=lse):
            o = ops.prompt_attention(q, q, q, lse=lse)
            return [ops.linear(x, w), *ops.linear_backward(dy, x, w, bias=True)[:3],
                    *ops.prompt_attention_backward(q, q, q, q, o, lse), *ops.layer_norm_backward(x, x, w[0].contiguous(), lse[:, 0].contiguous())[:2]]

        want = [t.clone() for t in calls()]
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = calls()
        cases.append((graph, got, want, calls))  # calls keeps the inputs that the graph reads
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    for turn in range(6):
        for (graph, got, *_), stream in zip(cases, streams):
            for t in got:
                t.zero_()
            torch.cuda.synchronize()
            with torch.cuda.stream(stream if turn % 2 else torch.cuda.current_stream()):
                graph.replay()
        torch.cuda.synchronize()
        for _, got, want, _ in cases:
            for a, b in zip(got, want):
                assert torch.equal(a, b), turn


def test_layer_on_another_stream():
    """Calls on a side stream, their inputs made on the current one and dropped at once."""
    s = layer_state()
    x, w = s["x"], s["p"]["wqkv"]
    rstd = torch.empty(x.shape[0], device="cuda")
    want_n, want_y = ops.layer_norm(x, rstd=rstd), ops.linear(x, w)
    want_b = ops.linear_backward(want_y, x, w, bias=True)
    want_g = ops.layer_norm_backward(x, x, None, rstd)
    q = want_y.view(-1, 8, 64)
    lse = torch.empty(x.shape[0], 8, device="cuda")
    want_o = ops.prompt_attention(q, q, q, s["starts"], lse=lse)
    want_d = ops.prompt_attention_backward(q, q, q, q, want_o, lse, s["starts"])
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(4):
        copies = [t.clone() for t in (x, w, rstd, want_y, q, want_o, lse, s["starts"])]
        side.wait_stream(torch.cuda.current_stream())
        cx, cw, cr, cy, cq, co, cl, cs = copies
        n, y = ops.layer_norm(cx, stream=side), ops.linear(cx, cw, stream=side)
        b = ops.linear_backward(cy, cx, cw, bias=True, stream=side)
        gr = ops.layer_norm_backward(cx, cx, None, cr, stream=side)
        o = ops.prompt_attention(cq, cq, cq, cs, stream=side)
        d = ops.prompt_attention_backward(cq, cq, cq, cq, co, cl, cs, stream=side)
        del copies, cx, cw, cr, cy, cq, co, cl, cs
        trash = [torch.full((x.numel(),), 7.0, device="cuda", dtype=BF) for _ in range(8)]
        torch.cuda.synchronize()
        del trash
        for a, c in zip((n, y, *b[:3], gr[0], o, *d), (want_n, want_y, *want_b[:3], want_g[0], want_o, *want_d)):
            assert torch.equal(a, c)


@pytest.mark.parametrize("op", ["norm", "linear", "attention"])
def test_what_a_backward_pass_needs_is_of_the_calls_stream(op):
    """What a forward pass on a side stream keeps for its gradient is not in memory that work of the
    current stream still writes."""
    g = torch.Generator(device="cuda").manual_seed(2)
    rows = 1 << 15
    x = torch.randn(rows, 64, generator=g, device="cuda").to(BF).requires_grad_()
    w = torch.randn(64, 64, generator=g, device="cuda").to(BF).requires_grad_()
    kept = dict(norm=[(rows,), (rows,)], linear=[(rows, 32)], attention=[(rows,)])[op]  # float32 of the same bytes
    call = dict(norm=lambda **kw: ops.layer_norm(x, **kw), linear=lambda **kw: ops.linear(x, w, activation="silu", **kw),
                attention=lambda **kw: ops.prompt_attention(x.view(rows, 1, 64), x.view(rows, 1, 64), x.view(rows, 1, 64),
                                                            starts, **kw))[op]
    starts = torch.arange(0, rows + 1, 64, dtype=torch.int32, device="cuda")
    want, = torch.autograd.grad(call().float().square().sum(), x)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    held = [torch.empty(shape, device="cuda") for shape in kept]
    torch.cuda._sleep(50_000_000)  # some 20 ms
    for t in held:
        t.fill_(3.0)
    del held, t  # their memory is free for the current stream, which has yet to write it
    y = call(stream=side)
    side.synchronize()
    torch.cuda.synchronize()
    got, = torch.autograd.grad(y.float().square().sum(), x)
    assert torch.equal(got, want)


def test_copies_are_not_made_on_another_stream():
    x = torch.zeros(4, 3, 16, device="cuda").transpose(0, 1)
    w = torch.zeros(16, 16, device="cuda")
    side = torch.cuda.Stream()
    assert ops.layer_norm(x).shape == x.shape and ops.linear(x, w).shape == x.shape
    rstd = torch.ones(12, device="cuda")
    for f in (lambda: ops.layer_norm(x, stream=side), lambda: ops.linear(x, w, stream=side),
              lambda: ops.linear(x.contiguous(), w, gate=x, stream=side), lambda: ops.linear_backward(x, x, w, stream=side),
              lambda: ops.layer_norm_backward(x, x, None, rstd, stream=side)):
        with pytest.raises(ValueError, match="copied"):
            f()


def test_layer_offsets_past_32_bits():
    """Tensors of more than 2^31 values: their last rows are those of a small call."""
    g = torch.Generator(device="cuda").manual_seed(1)
    rows, dim = 530_000, 4096  # 2.17e9 values
    x = torch.zeros(rows, dim, device="cuda", dtype=BF)
    last = slice(rows - 300, rows)
    x[last] = torch.randn(300, dim, generator=g, device="cuda").to(BF)
    w, v = torch.randn(dim, generator=g, device="cuda").to(BF), torch.randn(64, dim, generator=g, device="cuda").to(BF)
    small = x[last].clone()
    rstd, srstd = torch.empty(rows, device="cuda"), torch.empty(300, device="cuda")
    y = ops.layer_norm(x, w, center=False, rstd=rstd)
    assert torch.equal(y[last], ops.layer_norm(small, w, center=False, rstd=srstd)) and torch.equal(rstd[last], srstd)
    assert not y[:100].any()
    dx, dw, _ = ops.layer_norm_backward(x, x, w, rstd)
    sdx, sdw, _ = ops.layer_norm_backward(small, small, w, srstd)
    assert torch.equal(dx[last], sdx) and not dx[:100].any()
    del y, dx
    z = ops.linear(x, v)
    ref, size = small.double() @ v.double().T.contiguous(), small.double().abs() @ v.double().abs().T.contiguous()
    assert ((z[last].double() - ref).abs() <= R.rounded(ref, 2 * (dim + 4) * R.E * size, BF)).all() and not z[:100].any()
    dz = torch.zeros(rows, 64, device="cuda", dtype=BF)
    dz[last] = torch.randn(300, 64, generator=g, device="cuda").to(BF)
    dx, dv, db, _ = ops.linear_backward(dz, x, v, bias=True)
    d = dz[last].double()
    ref, size = d @ v.double(), d.abs() @ v.double().abs()
    assert ((dx[last].double() - ref).abs() <= R.rounded(ref, 2 * 68 * R.E * size, BF)).all() and not dx[:100].any()
    ref, size = d.T.contiguous() @ small.double(), d.abs().T.contiguous() @ small.double().abs()
    assert ((dv.double() - ref).abs() <= R.rounded(ref, 2 * 304 * R.E * size, BF)).all()
    del x, z, dx, dz
    T, H, D = 135_000, 125, 128  # 2.16e9 values
    q = torch.zeros(T, H, D, device="cuda", dtype=BF)
    k = torch.zeros(T, 1, D, device="cuda", dtype=BF)
    starts = torch.arange(0, T + 1, 100, device="cuda", dtype=torch.int32)
    last = slice(T - 100, T)
    q[last], k[last] = torch.randn(100, H, D, generator=g, device="cuda").to(BF), torch.randn(100, 1, D, generator=g, device="cuda").to(BF)
    lse, slse = torch.empty(T, H, device="cuda"), torch.empty(100, H, device="cuda")
    sq, sk = q[last].clone(), k[last].clone()
    o, so = ops.prompt_attention(q, k, k, starts, lse=lse), ops.prompt_attention(sq, sk, sk, lse=slse)
    assert torch.equal(o[last], so) and torch.equal(lse[last], slse) and not o[:100].any()
    got, want = ops.prompt_attention_backward(q, q, k, k, o, lse, starts), ops.prompt_attention_backward(sq, sq, sk, sk, so, slse)
    assert torch.equal(got[0][last], want[0])
    ref, errs = R.prompt_gradient(*d64(sq, sq, sk, sk, so, slse), None, True, None, BF)
    for a, r, e, name in zip(got[1:], ref[1:], errs[1:], ("dk", "dv")):
        close(a[last], r, e, BF, name)  # the parts of the sum over heads differ with the number of tokens


def test_layer_refusals():
    """Every refused call raises and launches nothing."""
    x, w = torch.zeros(4, 16, device="cuda", dtype=BF), torch.zeros(8, 16, device="cuda", dtype=BF)
    y, v16, v8 = torch.zeros(4, 8, device="cuda", dtype=BF), torch.zeros(16, device="cuda", dtype=BF), torch.zeros(8, device="cuda", dtype=BF)
    f4 = torch.zeros(4, device="cuda")
    q = torch.zeros(4, 2, 16, device="cuda", dtype=BF)
    st, lse = torch.tensor([0, 4], dtype=torch.int32, device="cuda"), torch.zeros(4, 2, device="cuda")
    wide = torch.zeros(4, 32, device="cuda", dtype=BF)
    bad = [
        (ValueError, lambda: ops.layer_norm(x.cpu())), (TypeError, lambda: ops.layer_norm(x.int())), (TypeError, lambda: ops.layer_norm(None)),
        (ValueError, lambda: ops.layer_norm(x, v8)), (TypeError, lambda: ops.layer_norm(x, v16.float())),
        (ValueError, lambda: ops.layer_norm(x, v16, v8)), (ValueError, lambda: ops.layer_norm(wide[:, ::2])),
        (ValueError, lambda: ops.layer_norm(x, out=y)), (ValueError, lambda: ops.layer_norm(x, out=x[:1].expand(4, 16))),
        (ValueError, lambda: ops.layer_norm(x, mean=f4[:3])), (ValueError, lambda: ops.layer_norm(x, rstd=f4.double())),
        (ValueError, lambda: ops.layer_norm(x[:, :0])), (api.GtsError, lambda: ops.layer_norm(x, eps=-1.0)),
        (api.GtsError, lambda: ops.layer_norm(x, eps=math.nan)), (ValueError, lambda: ops.layer_norm(torch.zeros((), device="cuda"))),
        (ValueError, lambda: ops.layer_norm_backward(y, x, v16, f4)), (ValueError, lambda: ops.layer_norm_backward(x, x, v16, None)),
        (ValueError, lambda: ops.layer_norm_backward(x, x, v16, f4[:2])), (TypeError, lambda: ops.layer_norm_backward(x.float(), x, v16, f4)),
        (ValueError, lambda: ops.linear(x, w, activation="tanh")), (ValueError, lambda: ops.linear(x, v16)),
        (ValueError, lambda: ops.linear(y, w)), (TypeError, lambda: ops.linear(x, w.float())), (ValueError, lambda: ops.linear(x, w, v16)),
        (ValueError, lambda: ops.linear(x, w, gate=x)), (ValueError, lambda: ops.linear(x, w, residual=y[:3])),
        (TypeError, lambda: ops.linear(x, w, residual=y.float())), (ValueError, lambda: ops.linear(x, w, out=y[:1].expand(4, 8))),
        (ValueError, lambda: ops.linear(wide[:, ::2], w)), (ValueError, lambda: ops.linear(x, w.cpu())),
        (ValueError, lambda: ops.linear_backward(y, x, w, activation="silu")), (ValueError, lambda: ops.linear_backward(x, x, w)),
        (ValueError, lambda: ops.linear_backward(y, x, w, gate=y)), (ValueError, lambda: ops.linear_backward(y, x, w, activation="silu", preact=x)),
        (ValueError, lambda: ops.prompt_attention(q[0], q, q)), (ValueError, lambda: ops.prompt_attention(q, q[:3], q)),
        (ValueError, lambda: ops.prompt_attention(q, q, q[..., :8])), (api.GtsError, lambda: ops.prompt_attention(q, torch.zeros(4, 3, 16, device="cuda", dtype=BF), torch.zeros(4, 3, 16, device="cuda", dtype=BF))),
        (TypeError, lambda: ops.prompt_attention(q, q.half(), q)), (TypeError, lambda: ops.prompt_attention(q, q, q, st.long())),
        (ValueError, lambda: ops.prompt_attention(q, q, q, st[:1])), (ValueError, lambda: ops.prompt_attention(q, q, q, st.cpu())),
        (ValueError, lambda: ops.prompt_attention(q, q, q, lse=lse.half())), (ValueError, lambda: ops.prompt_attention(q, q, q, out=q[:, :1].expand(4, 2, 16))),
        (api.GtsError, lambda: ops.prompt_attention(q, q, q, scale=math.inf)),
        (ValueError, lambda: ops.prompt_attention_backward(q[:2], q, q, q, q, lse)), (ValueError, lambda: ops.prompt_attention_backward(q, q, q, q, q, f4)),
    ]
    for i, (kind, f) in enumerate(bad):
        with pytest.raises(kind):
            f()
            note(f"refusal {i} missing")
    big = torch.zeros(3, 1, 300, device="cuda", dtype=BF)
    with pytest.raises(api.GtsError):
        ops.prompt_attention(big, big, big)
    torch.cuda.synchronize()


def test_decoder_layer_example():
    import importlib.util
    import os
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    folder = os.path.join(root, "examples")
    sys.path.insert(0, folder)
    try:
        spec = importlib.util.spec_from_file_location("decoder_layer", os.path.join(folder, "decoder_layer.py"))
        example = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(example)
    finally:
        sys.path.remove(folder)
    args = ["--tokens", "128", "--hidden", "256", "--heads", "2", "--kv-heads", "1", "--ffn", "384", "--steps", "3", "--backward"]
    r = example.main(args)
    assert r["measured"] > 0 and r["train"] > 0 and r["simulated"] > 0
    # the captured pass and its gradients are those of the eager calls
    lay = example.Layer(128, 256, 2, 1, 384)
    assert torch.equal(r["out"], lay.step())
    y, grads = lay.train()
    assert torch.equal(y, r["out"]) and len(grads) == len(r["grads"])
    for a, b in zip(grads, r["grads"]):
        assert torch.equal(a, b)
    with pytest.raises(SystemExit):
        example.main(["--hidden", "100"])
