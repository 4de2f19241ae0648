"""The operators of a decoder layer in 64 bits on the CPU, from their formulas, and how
far a kernel's result may be from them.

u is the unit roundoff of the result's type and e that of 32 bits.  A sum of n
products in 32 bits is off by at most n e times the sum of their absolute values
(twice that where the matrix instructions' own order is not known); a value computed in 32
bits and rounded once adds u times itself.  What is rounded to the tensors' type
before a product (softmax weights, their gradients, dz) adds u times each term, and in
float16 half of its smallest number."""
import math

import torch

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
TINY = {torch.bfloat16: 2.0 ** -126, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -126}
E = 2.0 ** -24


def rounded(ref, err, dtype):
    """Bound of a result that is off by err in 32 bits and then rounded."""
    return 1.01 * err + 1.01 * U[dtype] * ref.abs() + 1.01 * TINY[dtype]


# ---- norm ---------------------------------------------------------------------------

def _sum_steps(n):
    """Roundings behind one another in a sum over a row: those of a thread (32, or every
    1024th value of a long row), of a wave and of the waves."""
    return max(32, n // 1024 + 1) + 6 + 16 + 2


def norm(x, weight, bias, eps, center):
    """(y, mean, rstd, bound of y, of mean, of rstd) of 64-bit x [rows, dim]."""
    k = _sum_steps(x.shape[1])
    mean = x.mean(1, keepdim=True) if center else torch.zeros(x.shape[0], 1, dtype=x.dtype)
    d = x - mean
    rstd = (d.square().mean(1, keepdim=True) + eps).rsqrt()
    off = (k + 2) * E * x.abs().mean(1, keepdim=True) if center else torch.zeros_like(mean)
    # a wrong mean adds off^2 to the variance, each difference is rounded
    var = 2 * k * E + 6 * E + (off * rstd).square() + 2 * E * (x.abs() * rstd).square().mean(1, keepdim=True).sqrt()
    h = d * rstd
    h_err = (off + E * d.abs()) * rstd + h.abs() * (var + 4 * E)
    w = torch.ones(x.shape[1], dtype=x.dtype) if weight is None else weight
    b = torch.zeros(x.shape[1], dtype=x.dtype) if bias is None else bias
    y = h * w + b
    err = h_err * w.abs() + 2 * E * ((h * w).abs() + b.abs())
    return y, mean[:, 0], rstd[:, 0], err, off[:, 0] + 1e-30, rstd[:, 0] * (var[:, 0] + 4 * E)


def norm_gradient(dy, x, weight, mean, rstd):
    """(dx, dw, db, their errors in 32 bits), center where mean is given."""
    rows, n = x.shape
    k = _sum_steps(n) + 8
    w = torch.ones(n, dtype=x.dtype) if weight is None else weight
    r = rstd[:, None]
    h = (x if mean is None else x - mean[:, None]) * r
    g = dy * w
    mg, mgh = g.mean(1, keepdim=True), (g * h).mean(1, keepdim=True)
    dx = r * (g - h * mgh - (mg if mean is not None else 0.0))
    size = g.abs() + g.abs().mean(1, keepdim=True) + h.abs() * (g * h).abs().mean(1, keepdim=True)
    steps = rows / 512 + 600 + 16  # rows of a workgroup, then the parts
    return (dx, (dy * h).sum(0), dy.sum(0), 2 * k * E * r * size, steps * E * (dy * h).abs().sum(0),
            steps * E * dy.abs().sum(0))


# ---- products --------------------------------------------------------------------------

def activation(name, z):
    if name == "relu":
        return z.clamp(min=0.0)
    if name == "gelu":
        return 0.5 * z * torch.erfc(-z / math.sqrt(2.0))
    if name == "gelu_tanh":
        return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z ** 3)))
    return z * torch.sigmoid(z) if name == "silu" else z


def slope(name, z):
    z = z.clone().requires_grad_()
    with torch.enable_grad():  # of a formula above, in 64 bits
        g, = torch.autograd.grad(activation(name, z).sum(), z)
    return g


def _shape_error(name, z):
    """Of an activation or its slope computed in 32 bits, absolute and relative to 1 + |z|:
    the arguments of exp and erfc are rounded, so their values are off by e times the
    argument (z^2, or for the tanh form its cubic, which stops at 30)."""
    if name in (None, "relu"):
        return torch.zeros_like(z)
    arg = z.square().clamp(max=200.0) + 16.0  # beyond, the function is 0 or z in 32 bits
    return 4 * E * arg * (1.0 + z.abs())


def linear(x, w, bias, act, gate, residual):
    """(out, z, error of out and of z in 32 bits)."""
    z, size = x @ w.T, x.abs() @ w.abs().T
    z_err = 2 * (x.shape[1] + 4) * E * size
    if bias is not None:
        z = z + bias
        z_err = z_err + E * (size + bias.abs())
    y = activation(act, z)
    err = 1.2 * z_err + (_shape_error(act, z) * torch.exp(-z.clamp(max=0.0).square() / 4) if act else 0.0)
    if gate is not None:
        y, err = y * gate, err * gate.abs() + 2 * E * (y * gate).abs()
    if residual is not None:
        y = y + residual
    return y, z, err + 2 * E * y.abs() + (E * residual.abs() if residual is not None else 0.0), z_err


def linear_gradient(dy, x, w, act, z, gate, dtype):
    """dx, dw, db, dgate and their errors in 32 bits."""
    dz, dz_err, dg, dg_err = dy, torch.zeros_like(dy), None, None
    if gate is not None:
        dg = dy * activation(act, z)
        dg_err = dy.abs() * _shape_error(act, z) + 2 * E * dg.abs()
        dz = dz * gate
    if act:
        dz_err = dz.abs() * _shape_error(act, z)
        dz = dz * slope(act, z)
    dz_err = dz_err + 3 * E * dz.abs()
    db, db_err = dz.sum(0), dz_err.sum(0) + (dz.shape[0] / 4 + 40) * E * dz.abs().sum(0)
    if act or gate is not None:  # rounded for the products
        dz_err = dz_err + U[dtype] * dz.abs() + TINY[dtype]
    M, N = dz.shape
    dx_err = dz_err @ w.abs() + 2 * (N + 4) * E * (dz.abs() @ w.abs())
    dw_err = dz_err.T @ x.abs() + 2 * (M + 4) * E * (dz.abs().T @ x.abs())
    return (dz @ w, dz.T @ x, db, dg), (dx_err, dw_err, db_err, dg_err)


# ---- attention over prompts ---------------------------------------------------------------

def spans(T, starts):
    return [(0, T)] if starts is None else [(int(a), int(b)) for a, b in zip(starts[:-1], starts[1:]) if b > a]


def _scores(q, k, causal, scale):
    s = q @ k.T * scale
    if causal:
        s = s.masked_fill(torch.ones(s.shape, dtype=torch.bool).triu(1), -math.inf)
    return s


def _score_error(q, k, scale):
    D = q.shape[1]
    return 2 * (D + 4) * E * (q.abs() @ k.abs().T) * abs(scale)


def prompt(q, k, v, starts, causal, scale, dtype):
    """(out, lse, error of out before its rounding, of lse)."""
    T, Hq, D = q.shape
    G = Hq // k.shape[1]
    scale = D ** -0.5 if scale is None else scale
    out, err = torch.zeros(T, Hq, D, dtype=torch.float64), torch.zeros(T, Hq, D, dtype=torch.float64)
    lse = torch.full((T, Hq), -math.inf, dtype=torch.float64)
    lse_err = torch.zeros(T, Hq, dtype=torch.float64)
    for a, b in spans(T, starts):
        for h in range(Hq):
            qh, kh, vh = q[a:b, h], k[a:b, h // G], v[a:b, h // G]
            s = _scores(qh, kh, causal, scale)
            d = (_score_error(qh, kh, scale) + 6 * E * s.abs().where(s.isfinite(), torch.zeros_like(s))).amax(-1, keepdim=True)
            w = s.softmax(-1)
            out[a:b, h], lse[a:b, h] = w @ vh, s.logsumexp(-1)
            n = b - a
            rel = U[dtype] * (dtype != torch.float32) + 2 * d + (2 * n + 64) * E
            err[a:b, h] = rel * (w @ vh.abs()) + (TINY[dtype] * vh.abs().sum(0) if dtype == torch.float16 else 0.0)
            lse_err[a:b, h] = d[:, 0] + (n + 64) * E + 4 * E * lse[a:b, h].abs()
    return out, lse, err, lse_err


def prompt_gradient(dout, q, k, v, out, lse, starts, causal, scale, dtype):
    """dq, dk, dv and their errors in 32 bits, from the given out and lse."""
    T, Hq, D = q.shape
    G = Hq // k.shape[1]
    scale = D ** -0.5 if scale is None else scale
    r = [torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)]
    f = [torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)]
    u = U[dtype] if dtype != torch.float32 else 0.0
    tiny = TINY[dtype] if dtype == torch.float16 else 0.0
    for a, b in spans(T, starts):
        n = b - a
        for h in range(Hq):
            x = slice(a, b), h
            y = slice(a, b), h // G
            s = _scores(q[x], k[y], causal, scale)
            seen = s > -math.inf
            p = torch.exp(s - lse[x][:, None])
            p_err = p * 1.1 * (_score_error(q[x], k[y], scale) + 4 * E * (s.where(seen, torch.zeros_like(s)).abs()
                                                                      + lse[x].abs()[:, None]) + 4 * E)
            dp = dout[x] @ v[y].T
            delta = (dout[x] * out[x]).sum(-1, keepdim=True)
            dp_err = (2 * (D + 4) * E * (dout[x].abs() @ v[y].abs().T)
                      + (D + 4) * E * (dout[x] * out[x]).abs().sum(-1, keepdim=True) + E * (dp - delta).abs())
            ds = p * (dp - delta)
            ds_err = p_err * (dp - delta).abs() + p * dp_err + 2 * E * ds.abs() + (u * ds.abs() + tiny * seen)
            p_err = p_err + u * p + tiny * seen
            steps = 2 * (n * G + 8) * E
            r[0][x] += scale * (ds @ k[y])
            f[0][x] += abs(scale) * (ds_err @ k[y].abs() + steps * (ds.abs() @ k[y].abs()))
            r[1][y] += scale * (ds.T @ q[x])
            f[1][y] += abs(scale) * (ds_err.T @ q[x].abs() + steps * (ds.abs().T @ q[x].abs()))
            r[2][y] += p.T @ dout[x]
            f[2][y] += p_err.T @ dout[x].abs() + steps * (p.T @ dout[x].abs())
    return r, f
