"""The operators of a decoder layer at the edges of what their calls allow."""
import math

import pytest
import torch

import layer_reference as R
from paper_2607_11262_amd import api, ops
from test_gpu_ops_layer import BF, F, HF, TYPES, close, d64, gen, prompt_case, randn

pytestmark = pytest.mark.gpu


# ---- attention over prompts: scales ------------------------------------------------------

def flush_errors(dout, q, k, v, out, starts, causal, scale):
    """What is lost of dq, dk and dv where an exponential is below 2^-126, the smallest number of 32
    bits with all of its bits, and may be 0: 2^-126 of each weight, and of its gradient that times
    |dp - delta|, or 2^-126 where that product is the one below it."""
    G, tiny = q.shape[1] // k.shape[1], 2.0 ** -126
    r = [torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)]
    for a, b in R.spans(q.shape[0], starts):
        for h in range(q.shape[1]):
            x, y = (slice(a, b), h), (slice(a, b), h // G)
            seen = R._scores(q[x], k[y], causal, 1.0) > -math.inf
            size = (dout[x] @ v[y].T - (dout[x] * out[x]).sum(-1, keepdim=True)).abs()
            ds = tiny * (1.0 + size) * seen
            r[0][x] += abs(scale) * (ds @ k[y].abs())
            r[1][y] += abs(scale) * (ds.T @ q[x].abs())
            r[2][y] += tiny * (seen.double().T @ dout[x].abs())
    return r


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("scale", [0.0, -0.0, -0.3, -1e-30, 2.0])
@pytest.mark.parametrize("dtype,D", [(BF, 64), (BF, 128), (BF, 256), (HF, 96), (HF, 256), (F, 64), (F, 256), (BF, 33)])
def test_prompt_scales_of_any_sign(dtype, D, scale, causal):
    """Lengths that no tile divides: what is hidden behind a sequence's end stays so."""
    for lens in ([1], [33], [150], [64, 70], [31, 0, 97]):
        q, k, v, starts, dout = prompt_case(2, 1, D, lens, dtype)
        st, lse = starts.cuda(), torch.empty(q.shape[:2], device="cuda")
        qc, kc, vc, dc = (t.cuda() for t in (q, k, v, dout))
        o = ops.prompt_attention(qc, kc, vc, st, causal=causal, scale=scale, lse=lse)
        ref, lr, err, l_err = R.prompt(*d64(q, k, v), starts, causal, scale, dtype)
        close(o, ref, err, dtype, "out")
        close(lse, lr, l_err, F, "lse")
        got = ops.prompt_attention_backward(dc, qc, kc, vc, o, lse, st, causal=causal, scale=scale)
        refs, errs = R.prompt_gradient(*d64(dout, q, k, v, o, lse), starts, causal, scale, dtype)
        flushed = flush_errors(*d64(dout, q, k, v, o), starts, causal, scale)
        for a, r, e, f, name in zip(got, refs, errs, flushed, ("dq", "dk", "dv")):
            close(a, r, e + f, dtype, name)


# ---- norm: gradients in place ------------------------------------------------------------

def norm_gradient_into(dy, x, weight, rstd, mean, dx):
    """gts_layer_norm_backward with a dx of the caller's: (dweight, dbias)."""
    rows, dim = x.shape
    dw, db = torch.empty_like(weight), torch.empty_like(weight)
    scratch = torch.empty(ops._scratch_of("gts_layer_norm_backward_scratch", rows, dim), device="cuda", dtype=torch.uint8)
    ops._call("gts_layer_norm_backward", ops._pack_norm_grad(
        dy.data_ptr(), x.data_ptr(), weight.data_ptr(), ops._ptr(mean), rstd.data_ptr(), dx.data_ptr(), dw.data_ptr(), db.data_ptr(),
        dy.stride(0), x.stride(0), dx.stride(0), rows, dim, ops._TYPES[x.dtype], 0 if mean is None else ops.CENTER,
        scratch.data_ptr(), scratch.numel()), torch.cuda.current_stream().cuda_stream)
    return dw, db


@pytest.mark.parametrize("center", [True, False])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,dim", [(50, 3), (300, 136), (300, 137), (9, 2048), (9, 2045), (40, 8200), (40, 8201),
                                      (70, 20000), (5, 16385)])
def test_norm_gradient_in_place(rows, dim, dtype, center):
    g = gen(rows + dim)
    x, dy, w = (t.cuda() for t in (randn(g, rows, dim, dtype=dtype, shift=0.5), randn(g, rows, dim, dtype=dtype), randn(g, dim, dtype=dtype)))
    mean, rstd = torch.empty(rows, device="cuda") if center else None, torch.empty(rows, device="cuda")
    ops.layer_norm(x, w, center=center, mean=mean, rstd=rstd)
    want = ops.layer_norm_backward(dy, x, w, rstd, mean, bias=True)
    refs = R.norm_gradient(*d64(dy, x, w, mean, rstd))
    for a, r, e, name in zip(want, refs, refs[3:], ("dx", "dw", "db")):
        close(a, r, e, dtype, name)
    for which in ("dy", "x", "neither"):
        dy1, x1 = dy.clone(), x.clone()
        dx = dict(dy=dy1, x=x1, neither=torch.empty_like(x))[which]
        got = (dx, *norm_gradient_into(dy1, x1, w, rstd, mean, dx))
        for a, b, name in zip(got, want, ("dx", "dw", "db")):
            assert torch.equal(a, b), (which, name)


# ---- norm: many rows -----------------------------------------------------------------------

@pytest.mark.parametrize("dtype,dim", [(BF, 3), (HF, 7), (F, 2)])
def test_norm_of_more_rows_than_a_row_of_the_grid(dtype, dim):
    """More workgroups of 1024 threads than 2^32 threads hold."""
    rows = (1 << 22) + 5
    g = torch.Generator(device="cuda").manual_seed(dim)
    x, dy = (torch.randn(rows, dim, generator=g, device="cuda").to(dtype) for _ in range(2))
    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    y = ops.layer_norm(x, eps=0.1, mean=mean, rstd=rstd)
    few = torch.cat((torch.arange(40), torch.arange(rows // 2 - 20, rows // 2 + 20), torch.arange(rows - 40, rows))).cuda()
    ref = R.norm(*d64(x[few], None, None), 0.1, True)
    close(y[few], ref[0], ref[3], dtype, "y")
    # every row: what a call of the same rows in parts gives
    part = 1 << 20
    for i in range(0, rows, part):
        assert torch.equal(y[i:i + part], ops.layer_norm(x[i:i + part], eps=0.1))
    dx, _, db = ops.layer_norm_backward(dy, x, None, rstd, mean, bias=True)
    refs = R.norm_gradient(*d64(dy[few], x[few], None, mean[few], rstd[few]))
    close(dx[few], refs[0], refs[3], dtype, "dx")
    for i in range(0, rows, part):
        at = slice(i, i + part)
        assert torch.equal(dx[at], ops.layer_norm_backward(dy[at], x[at], None, rstd[at], mean[at])[0])
    total = dy.double().sum(0)
    # 512 strips of rows, each a sum of its own, then their sum
    assert ((db.double() - total).abs() <= R.rounded(total, (rows / 512 + 600) * R.E * dy.double().abs().sum(0), dtype)).all()


# ---- products: tall and narrow ---------------------------------------------------------------

@pytest.mark.parametrize("dtype", [BF, F])
def test_product_of_more_rows_than_small_tiles_take(dtype):
    """Results that 2^23 tiles of 128 rows hold, and tiles of 64 rows do not."""
    rows = 64 * (1 << 23) + 77
    x = (torch.arange(rows, device="cuda", dtype=torch.int32) % 251).to(dtype).view(rows, 1)
    y = ops.linear(x, torch.tensor([[2.0]], device="cuda", dtype=dtype))
    assert torch.equal(y, x * 2)


# ---- batches of nothing ------------------------------------------------------------------------

@pytest.mark.parametrize("shape", [(0, 16), (3, 0, 16), (0, 5, 16), (2, 0, 3, 16)])
@pytest.mark.parametrize("params", [False, True])
def test_batches_of_nothing_have_gradients(shape, params):
    """A batch without a token is a training step like any other: zeros for the parameters."""
    leaf = lambda *s: torch.ones(s, device="cuda").requires_grad_()  # noqa: E731
    x, gate, res = leaf(*shape), leaf(*shape[:-1], 8), leaf(*shape[:-1], 8)
    w, b, weight, bias = leaf(16), leaf(16), leaf(8, 16), leaf(8)
    if not params:
        w, b, weight, bias = (t.detach() for t in (w, b, weight, bias))
    h = ops.layer_norm(x, w, b)
    y = ops.linear(h, weight, bias, activation="silu", gate=gate, residual=res)
    assert h.shape == shape and y.shape == (*shape[:-1], 8) and h.requires_grad and y.requires_grad
    y.sum().backward()
    for t in (x, gate, res):
        assert t.grad is not None and t.grad.shape == t.shape
    for t in (w, b, weight, bias) if params else ():
        assert t.grad is not None and (t.grad == 0).all()


def test_sums_of_nothing_have_gradients():
    """Rows of no values: the product is its bias, the operands' gradients are empty."""
    x, w = torch.ones(2, 3, 0, device="cuda").requires_grad_(), torch.ones(4, 0, device="cuda").requires_grad_()
    b = torch.arange(4.0, device="cuda").requires_grad_()
    y = ops.linear(x, w, b)
    assert torch.equal(y, b.detach().expand(2, 3, 4))
    y.sum().backward()
    assert x.grad.shape == x.shape and w.grad.shape == w.shape and (b.grad == 6).all()


def test_prompts_of_nothing_have_gradients():
    q, k, v = (torch.ones(0, h, 32, device="cuda").requires_grad_() for h in (4, 2, 2))
    for starts in (None, torch.zeros(4, dtype=torch.int32, device="cuda")):
        o = ops.prompt_attention(q, k, v, starts)
        assert o.shape == q.shape and o.requires_grad
        o.sum().backward()
        assert all(t.grad.shape == t.shape for t in (q, k, v))


# ---- float16: gradients that are small or large ------------------------------------------------

def half_gradient(dout, q, k, v, out, lse, causal, scale):
    """dq, dk, dv of one sequence in 64 bits, and their errors before the last rounding, of a
    gradient that keeps weights and their gradients as float16 of the size that suits them.  A weight
    is rounded by 2^-11 of itself or, lifted by 2^10, half of the smallest number, 2^-25, below 2^-14.
    A weight's gradient is rounded by 2^-11 of itself or, scaled so that the largest of its row (for dq) or
    of its key (for dk) is 2^8 at least, 2^-25: 2^-33 of that largest.  Otherwise as in 32 bits."""
    exact = R.prompt_gradient(dout, q, k, v, out, lse, None, causal, scale, F)
    refs, errs = exact
    G, u = q.shape[1] // k.shape[1], R.U[HF]
    for h in range(q.shape[1]):
        x, y = (slice(None), h), (slice(None), h // G)
        s = R._scores(q[x], k[y], causal, scale)
        seen = s > -math.inf
        p = torch.exp(s - lse[x][:, None])
        ds = p * (dout[x] @ v[y].T - (dout[x] * out[x]).sum(-1, keepdim=True))
        size = ds.abs()
        errs[0][x] += abs(scale) * ((u * size + 2.0 ** -33 * size.amax(1, keepdim=True) * seen) @ k[y].abs())
        errs[1][y] += abs(scale) * ((u * size + 2.0 ** -33 * size.amax(0, keepdim=True) * seen).T @ q[x].abs())
        errs[2][y] += (u * p + 2.0 ** -35 * seen).T @ dout[x].abs()
    return refs, errs


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("D,Hq,Hkv", [(64, 2, 1), (128, 4, 2), (256, 2, 2), (33, 2, 1), (200, 1, 1)])
@pytest.mark.parametrize("powers", [(-14, 0, 0), (-14, -6, 0), (-14, 6, 0), (10, -6, 4), (10, 6, 4), (8, 0, 6), (-12, -8, 8)])
def test_prompt_gradient_of_any_size_in_float16(powers, D, Hq, Hkv, causal):
    """dout times 2^powers[0], keys times 2^powers[1] and queries divided by it, values times
    2^powers[2]: scores stay, their gradients leave the range of float16 where the results do not."""
    q, k, v, _, dout = prompt_case(Hq, Hkv, D, [150], F)
    scale = D ** -0.5
    q, k = (q * 2.0 ** -powers[1]).half(), (k * 2.0 ** powers[1]).half()
    v, dout = (v * 2.0 ** powers[2]).half(), (dout * 2.0 ** powers[0]).half()
    qc, kc, vc, dc = (t.cuda() for t in (q, k, v, dout))
    lse = torch.empty(150, Hq, device="cuda")
    o = ops.prompt_attention(qc, kc, vc, causal=causal, lse=lse)
    assert o.isfinite().all()
    got = ops.prompt_attention_backward(dc, qc, kc, vc, o, lse, causal=causal)
    refs, errs = half_gradient(*d64(dout, q, k, v, o, lse), causal, scale)
    for a, r, e, name in zip(got, refs, errs, ("dq", "dk", "dv")):
        # a result whose bound reaches past the largest number may be infinite
        reaches = r.abs() + R.rounded(r, e, HF) >= torch.finfo(HF).max
        a = a.cpu()
        assert (a.isfinite() | reaches & (a.sign() == r.sign())).all(), name
        compared = a.isfinite()
        close(torch.where(compared, a, 0), torch.where(compared, r, 0.0), e, HF, name)


@pytest.mark.parametrize("D", [64, 33])
def test_prompt_gradient_of_equal_weights_of_many_keys(D):
    """Weights 1 / n of which float16 as it stands has few bits, and would round all to the same side."""
    n = 332_222 if D == 64 else 166_932  # 2^24 / n is near 50.5 and 100.5
    g = torch.Generator(device="cuda").manual_seed(1)
    rand = lambda: torch.randn(n, 1, D, generator=g, device="cuda").half()  # noqa: E731
    q, k, v, dout = torch.zeros(n, 1, D, device="cuda", dtype=HF), rand(), rand(), (rand() + 1).half()
    lse = torch.empty(n, 1, device="cuda")
    o = ops.prompt_attention(q, k, v, causal=False, lse=lse)
    dq, dk, dv = ops.prompt_attention_backward(dout, q, k, v, o, lse, causal=False)
    do, vd, kd = dout[:, 0].double(), v[:, 0].double(), k[:, 0].double()
    p = torch.exp(-lse[0, 0].double())  # the same for all
    # weights of one rounding; sums in 32 bits, 16 terms a matrix instruction, whose order within is not known
    steps = 2 * (n / 16 + 100) * R.E
    ref = (do.sum(0) * p).expand(n, D)
    err = (R.U[HF] + steps) * do.abs().sum(0) * p
    close(dv[:, 0], ref.cpu(), err.cpu().expand(n, D), HF, "dv")
    assert not dk.any()
    few = slice(1000, 1040)  # dq of some rows
    ds = p * (do[few] @ vd.T.contiguous() - (do[few] * o[few, 0].double()).sum(1, keepdim=True))
    ref = D ** -0.5 * (ds @ kd)
    sizes = (ds.abs() @ kd.abs()) * D ** -0.5
    off = p * 2 * (D + 4) * R.E * (do[few].abs() @ vd.abs().T.contiguous() + (do[few] * o[few, 0].double()).abs().sum(1, keepdim=True))
    err = (R.U[HF] + steps) * sizes + (off + 2.0 ** -33 * ds.abs().amax(1, keepdim=True)) @ kd.abs() * D ** -0.5
    close(dq[few, 0], ref.cpu(), err.cpu(), HF, "dq")


# ---- refusals ------------------------------------------------------------------------------------

def test_numbers_that_no_field_takes_are_refused():
    x, q = torch.zeros(4, 16, device="cuda"), torch.zeros(4, 2, 0, device="cuda")
    lse = torch.zeros(4, 2, device="cuda")
    for eps in (1e300, -1e300, math.inf):
        with pytest.raises(api.GtsError):
            ops.layer_norm(x, eps=eps)
    for eps in ("small", None):
        with pytest.raises(TypeError):
            ops.layer_norm(x, eps=eps)
    for f in (lambda: ops.prompt_attention(q, q, q), lambda: ops.prompt_attention_backward(q, q, q, q, q, lse)):
        with pytest.raises(api.GtsError, match="head dim 0"):
            f()


# ---- norm: widths at the limits of the kernels -----------------------------------------------------

@pytest.mark.parametrize("center", [True, False])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("limit", [4, 8, 128, 256, 512, 1024, 2048, 4096, 8192, 16384])
def test_norm_widths_about_the_limits(limit, dtype, center):
    for dim in (limit - 1, limit, limit + 1):
        g = gen(dim)
        x, dy, w, b = (randn(g, *s, dtype=dtype) for s in ((5, dim), (5, dim), (dim,), (dim,)))
        mean, rstd = torch.empty(5, device="cuda") if center else None, torch.empty(5, device="cuda")
        y = ops.layer_norm(x.cuda(), w.cuda(), b.cuda(), eps=1e-3, center=center, mean=mean, rstd=rstd)
        ref = R.norm(*d64(x, w, b), 1e-3, center)
        close(y, ref[0], ref[3], dtype, f"y of {dim}")
        got = ops.layer_norm_backward(dy.cuda(), x.cuda(), w.cuda(), rstd, mean, bias=True)
        refs = R.norm_gradient(*d64(dy, x, w, mean, rstd))
        for a, r, e, name in zip(got, refs, refs[3:], ("dx", "dw", "db")):
            close(a, r, e, dtype, f"{name} of {dim}")


# ---- products: in place ------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,N,K", [(5, 72, 48), (5, 71, 48), (150, 136, 264), (150, 135, 264), (40, 24, 3000), (700, 512, 64)])
def test_products_in_place(M, N, K, dtype):
    """out over gate or residual, and in the C call of the gradient dz over dy: the bits of a result apart."""
    g = gen(M + N + K)
    x, w, gate, res, dy, z = (randn(g, *s, dtype=dtype).cuda() for s in ((M, K), (N, K), (M, N), (M, N), (M, N), (M, N)))
    want = ops.linear(x, w, activation="gelu", gate=gate, residual=res)
    for which in ("gate", "residual"):
        t = dict(gate=gate.clone(), residual=res.clone())
        out = t[which]
        assert ops.linear(x, w, activation="gelu", out=out, **t) is out and torch.equal(out, want), which
    scratch = torch.empty(ops._scratch_of("gts_linear_backward_scratch", M, N), device="cuda", dtype=torch.uint8)
    results = []
    for dz in (torch.empty_like(dy), dy):
        dgate, dbias = torch.empty_like(dy), torch.empty(N, device="cuda", dtype=dtype)
        ops._call("gts_linear_backward", ops._pack_linear_grad(
            dy.data_ptr(), z.data_ptr(), gate.data_ptr(), dz.data_ptr(), dgate.data_ptr(), dbias.data_ptr(), N, N, N, N, N, M, N,
            ops._TYPES[dtype], ops.ACTIVATIONS["gelu"], scratch.data_ptr(), scratch.numel()), torch.cuda.current_stream().cuda_stream)
        results.append((dz, dgate, dbias))
    for a, b, name in zip(*results, ("dz", "dgate", "dbias")):
        assert torch.equal(a, b), name


# ---- streams -------------------------------------------------------------------------------------------

def test_a_call_on_another_stream_behind_late_inputs():
    """Inputs whose work on the current stream is late, a wait behind them, a call on a side stream, the
    inputs dropped at once: the caller's order holds."""
    g = torch.Generator(device="cuda").manual_seed(4)
    x = torch.randn(300, 256, generator=g, device="cuda").to(BF)
    w = torch.randn(512, 256, generator=g, device="cuda").to(BF)
    q = torch.randn(300, 4, 64, generator=g, device="cuda").to(BF)
    lse = torch.empty(300, 4, device="cuda")
    o = ops.prompt_attention(q, q, q, lse=lse)
    want = [ops.layer_norm(x), ops.linear(x, w), o, *ops.prompt_attention_backward(q, q, q, q, o, lse)]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(5):
        torch.cuda._sleep(200_000)
        cx, cw, cq, co, cl = (t.clone() for t in (x, w, q, o, lse))
        side.wait_stream(torch.cuda.current_stream())
        got = [ops.layer_norm(cx, stream=side), ops.linear(cx, cw, stream=side), ops.prompt_attention(cq, cq, cq, stream=side),
               *ops.prompt_attention_backward(cq, cq, cq, cq, co, cl, stream=side)]
        del cx, cw, cq, co, cl
        trash = [torch.full((n,), 9.0, device="cuda") for n in (300 * 128, 512 * 128, 300 * 128, 1200)]
        torch.cuda.synchronize()
        del trash
        for a, b in zip(got, want):
            assert torch.equal(a, b)
