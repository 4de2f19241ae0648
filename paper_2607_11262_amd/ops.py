"""Operators of the steps whose tile graphs this package simulates, as
hand-written kernels on the card (C ABI: include/gts_ops.h).

The serving step: rotary positions, appending keys and values to a paged cache, and
attention over that cache for a batch whose sequences share a prefix.

    from paper_2607_11262_amd import ops
    table = ops.rotary_table(65536, 128)                   # once
    q = ops.append_kv(k, v, k_cache, v_cache, pages, lens, table=table, q=q,
                      prefix_len=P)                        # a decode step: one
    o = ops.shared_prefix_attention(q, k_cache, v_cache, pages, lens,
                                    prefix_pages=shared, prefix_len=P)

    y = ops.rotary(x, positions, table)                    # a training step
    dx = ops.rotary_backward(dy, positions, table)         # (autograd calls it too)

The rest of a decoder layer, at prefill and in training: norms, matrix products
with their epilogue, attention over whole prompts.

    h = ops.layer_norm(x, w_norm, center=False)
    q, k, v = ops.linear(h, w_qkv).view(T, -1, D).split((Hq, Hkv, Hkv), 1)
    o = ops.prompt_attention(ops.rotary(q, positions, table), ops.rotary(k, positions, table), v, starts)
    x = ops.linear(o.flatten(1), w_o, residual=x)
    h = ops.layer_norm(x, w_norm2, center=False)
    x = ops.linear(ops.linear(h, w_gate, activation="silu", gate=ops.linear(h, w_up)), w_down, residual=x)
    x.backward(dx)                                         # or the *_backward calls

Shapes.  q [T, Hq, D], k and v [T, Hkv, D]: the new tokens of all sequences one
behind the other, sequence b's at starts[b] .. starts[b + 1] (starts=None: the
same number each; for prompts one sequence).  Caches [pages, page, Hkv, D] in any
memory order whose last dimension is contiguous (pages kept head by head are a
transposed view), page a power of two.  page_table [B, max_pages] int32; lens [B] int32 counts a
sequence's own keys with its new ones, the shared prefix apart.  Types: bfloat16,
float16, float32.

Errors are ValueError / TypeError for shapes, types and devices, and
api.GtsError for what the library refuses.  Work is enqueued on `stream`
(default: the current one) and not waited for; outputs and scratch are
allocated on it, and tensors handed to another stream than the current one are
kept from reuse until it has run (record_stream).  The caller orders the
streams.  Every call may be captured into a graph (a backward pass too, where no
eager autograd graph of the same leaves lives meanwhile: that is torch's rule).  For
autograd the caller's tensors that a call writes (out, q_out, lse, scratch, preact,
mean, rstd, the caches) are modified in place.
"""
from __future__ import annotations

import ctypes
import functools
import math
import operator
import struct

import torch
from torch.autograd import forward_ad

from . import api

F32, BF16, F16 = 0, 1, 2
INTERLEAVED, BACKWARD, ZERO_REST = 1, 2, 4
_TYPES = {torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16}

A_COLUMNS, B_COLUMNS, CENTER, CAUSAL = 1, 2, 1, 1
ACTIVATIONS = {None: 0, "relu": 1, "gelu": 2, "gelu_tanh": 3, "silu": 4}

EXPORTS = ("gts_rotary_table", "gts_rotary", "gts_append_kv", "gts_shared_prefix_attention",
           "gts_shared_prefix_attention_scratch", "gts_layer_norm", "gts_layer_norm_backward",
           "gts_layer_norm_backward_scratch", "gts_matmul", "gts_matmul_scratch", "gts_linear_backward",
           "gts_linear_backward_scratch", "gts_prompt_attention", "gts_prompt_attention_backward",
           "gts_prompt_attention_backward_scratch")

_u32, _i64, _vp, _f32 = ctypes.c_uint32, ctypes.c_int64, ctypes.c_void_p, ctypes.c_float


class _RotaryArgs(ctypes.Structure):
    _fields_ = [("x", _vp), ("out", _vp), ("positions", _vp), ("table", _vp), ("x_stride", _i64 * 3),
                ("out_stride", _i64 * 3), ("pos_stride", _i64 * 2), ("table_stride", _i64), ("batch", _u32),
                ("tokens", _u32), ("heads", _u32), ("dim", _u32), ("rot_dim", _u32), ("n_positions", _u32),
                ("dtype", _u32), ("pos_bytes", _u32), ("flags", _u32), ("reserved", _u32)]


class _Cache(ctypes.Structure):
    _fields_ = [("k", _vp), ("v", _vp), ("k_stride", _i64 * 3), ("v_stride", _i64 * 3), ("n_pages", _u32),
                ("page", _u32), ("heads", _u32), ("dim", _u32), ("dtype", _u32), ("reserved", _u32)]


class _Batch(ctypes.Structure):
    _fields_ = [("starts", _vp), ("lens", _vp), ("page_table", _vp), ("table_stride", _i64), ("batch", _u32),
                ("tokens", _u32), ("max_pages", _u32), ("prefix_len", _u32)]


class _AppendArgs(ctypes.Structure):
    _fields_ = [("cache", _Cache), ("batch", _Batch), ("k", _vp), ("v", _vp), ("q", _vp), ("q_out", _vp),
                ("k_stride", _i64 * 2), ("v_stride", _i64 * 2), ("q_stride", _i64 * 2), ("q_out_stride", _i64 * 2),
                ("table", _vp), ("table_stride", _i64), ("q_heads", _u32), ("rot_dim", _u32), ("n_positions", _u32),
                ("flags", _u32)]


class _AttentionArgs(ctypes.Structure):
    _fields_ = [("cache", _Cache), ("batch", _Batch), ("q", _vp), ("out", _vp), ("lse", _vp), ("q_stride", _i64 * 2),
                ("out_stride", _i64 * 2), ("prefix_pages", _vp), ("n_prefix_pages", _u32), ("q_heads", _u32),
                ("scale", _f32), ("reserved", _u32), ("scratch", _vp), ("scratch_bytes", ctypes.c_uint64)]


class _NormArgs(ctypes.Structure):
    _fields_ = [("x", _vp), ("out", _vp), ("weight", _vp), ("bias", _vp), ("mean", _vp), ("rstd", _vp), ("x_stride", _i64),
                ("out_stride", _i64), ("rows", _u32), ("dim", _u32), ("eps", _f32), ("dtype", _u32), ("flags", _u32),
                ("reserved", _u32)]


class _NormGradArgs(ctypes.Structure):
    _fields_ = [("dy", _vp), ("x", _vp), ("weight", _vp), ("mean", _vp), ("rstd", _vp), ("dx", _vp), ("dweight", _vp),
                ("dbias", _vp), ("dy_stride", _i64), ("x_stride", _i64), ("dx_stride", _i64), ("rows", _u32),
                ("dim", _u32), ("dtype", _u32), ("flags", _u32), ("scratch", _vp), ("scratch_bytes", ctypes.c_uint64)]


class _MatmulArgs(ctypes.Structure):
    _fields_ = [("a", _vp), ("b", _vp), ("out", _vp), ("preact", _vp), ("bias", _vp), ("gate", _vp), ("residual", _vp),
                ("a_stride", _i64), ("b_stride", _i64), ("out_stride", _i64), ("preact_stride", _i64),
                ("gate_stride", _i64), ("residual_stride", _i64), ("m", _u32), ("n", _u32), ("k", _u32), ("dtype", _u32),
                ("activation", _u32), ("flags", _u32), ("scratch", _vp), ("scratch_bytes", ctypes.c_uint64)]


class _LinearGradArgs(ctypes.Structure):
    _fields_ = [("dy", _vp), ("preact", _vp), ("gate", _vp), ("dz", _vp), ("dgate", _vp), ("dbias", _vp),
                ("dy_stride", _i64), ("preact_stride", _i64), ("gate_stride", _i64), ("dz_stride", _i64),
                ("dgate_stride", _i64), ("m", _u32), ("n", _u32), ("dtype", _u32), ("activation", _u32), ("scratch", _vp),
                ("scratch_bytes", ctypes.c_uint64)]


class _PromptArgs(ctypes.Structure):
    _fields_ = [("q", _vp), ("k", _vp), ("v", _vp), ("out", _vp), ("lse", _vp), ("starts", _vp), ("q_stride", _i64 * 2),
                ("k_stride", _i64 * 2), ("v_stride", _i64 * 2), ("out_stride", _i64 * 2), ("batch", _u32),
                ("tokens", _u32), ("q_heads", _u32), ("kv_heads", _u32), ("dim", _u32), ("dtype", _u32), ("scale", _f32),
                ("flags", _u32)]


class _PromptGradArgs(ctypes.Structure):
    _fields_ = [("dout", _vp), ("q", _vp), ("k", _vp), ("v", _vp), ("out", _vp), ("lse", _vp), ("starts", _vp),
                ("dq", _vp), ("dk", _vp), ("dv", _vp)] + [
        (x + "_stride", _i64 * 2) for x in ("dout", "q", "k", "v", "out", "dq", "dk", "dv")] + [
        ("batch", _u32), ("tokens", _u32), ("q_heads", _u32), ("kv_heads", _u32), ("dim", _u32), ("dtype", _u32),
        ("scale", _f32), ("flags", _u32), ("scratch", _vp), ("scratch_bytes", ctypes.c_uint64)]


# The structures' values in one call each, as the C side lays them out: a call of
# a small batch is bound by the host.
_pack_rotary = struct.Struct("=4Q3q3q2qq10I").pack
_pack_cache_batch = "2Q3q3q6I3Qq4I"
_pack_append = struct.Struct("=" + _pack_cache_batch + "4Q2q2q2q2qQq4I").pack
_pack_attention = struct.Struct("=" + _pack_cache_batch + "3Q2q2qQ2IfIQQ").pack

_pack_norm = struct.Struct("=6Q2q2If3I").pack
_pack_norm_grad = struct.Struct("=8Q3q4IQQ").pack
_pack_matmul = struct.Struct("=7Q6q6IQQ").pack
_pack_linear_grad = struct.Struct("=6Q5q4IQQ").pack
_pack_prompt = struct.Struct("=6Q8q6IfI").pack
_pack_prompt_grad = struct.Struct("=10Q16q6IfIQQ").pack

_bound, _calls = None, {}  # the library the calls are bound to


def lib():
    """The loaded libgts.so with the operators' argument types (raises if it
    has not been built)."""
    global _bound
    L = api.lib()
    if _bound is not L:
        for name in EXPORTS:
            getattr(L, name).restype = ctypes.c_int
        L.gts_rotary_table.argtypes = [_vp, _u32, _u32, _vp, ctypes.c_double, _vp]
        for name in ("gts_rotary", "gts_append_kv", "gts_shared_prefix_attention", "gts_layer_norm",
                     "gts_layer_norm_backward", "gts_matmul", "gts_linear_backward", "gts_prompt_attention",
                     "gts_prompt_attention_backward"):
            getattr(L, name).argtypes = [_vp, _vp]
            _calls[name] = getattr(L, name)
        for name, sizes in (("gts_shared_prefix_attention_scratch", 5), ("gts_layer_norm_backward_scratch", 2),
                            ("gts_matmul_scratch", 3), ("gts_linear_backward_scratch", 2),
                            ("gts_prompt_attention_backward_scratch", 5)):
            getattr(L, name).argtypes = [_u32] * sizes + [ctypes.POINTER(ctypes.c_uint64)]
        _scratch_bytes.cache_clear()
        _scratch_of.cache_clear()
        _bound = L
    return L


# ---- checks and streams -----------------------------------------------------------

def _refuse(ok, why):
    if not ok:
        raise ValueError(why)


def _data(t, name, dims, like=None):
    """t is a tensor on the GPU with `dims` dimensions and a contiguous last
    one, of the type and on the device of `like`; returns its strides."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} is a tensor: got {type(t).__name__}")
    if t.dim() != dims:
        raise ValueError(f"{name} has {t.dim()} dimensions, not {dims}")
    if not t.is_cuda:
        raise ValueError(f"{name} is not on the GPU")
    strides = t.stride()
    if strides[-1] != 1 and t.shape[-1] > 1 and t.numel():
        raise ValueError(f"{name}: the last dimension is not contiguous")
    if like is None:
        if t.dtype not in _TYPES:
            raise TypeError(f"{name} is {t.dtype}: bfloat16, float16 or float32")
    elif t.dtype != like.dtype:
        raise TypeError(f"{name} is {t.dtype}, not {like.dtype}")
    elif t.get_device() != like.get_device():
        raise ValueError(f"{name} is on {t.device}, not {like.device}")
    return strides


def _index(t, name, dims, like, types=(torch.int32,)):
    """t is a tensor of whole numbers beside `like`; returns its strides."""
    if not isinstance(t, torch.Tensor) or t.dtype not in types:
        raise TypeError(f"{name} is a tensor of {' or '.join(str(x) for x in types)}")
    if t.dim() != dims:
        raise ValueError(f"{name} has {t.dim()} dimensions, not {dims}")
    if t.device != like.device:
        raise ValueError(f"{name} is on {t.device}, not {like.device}")
    return t.stride()


def _table(table, like, D):
    """Positions, rotated values and row stride of a rotary table."""
    if not isinstance(table, torch.Tensor) or table.dtype != torch.float32:
        raise TypeError("table is a float32 tensor (rotary_table)")
    if table.dim() != 2 or table.device != like.device:
        raise ValueError(f"table is [positions, rotated values] on {like.device}")
    (n, rot), (row, one) = table.shape, table.stride()
    if one != 1 and rot > 1:
        raise ValueError("table: its rows are not contiguous")
    if not 0 < rot <= D:
        raise ValueError(f"table turns {rot} values of a head of {D}")
    return n, rot, row


class _On:
    """The stream of a call, current while outputs are allocated and the work
    is enqueued, with the device of the tensors current."""

    def __init__(self, stream, like, tensors):
        _refuse(stream is None or stream.device == like.device, f"stream is not on {like.device}")
        self.like, self.stream, self.tensors = like, stream, tensors
        self.guard = torch.cuda.device(like.device) if stream is None else torch.cuda.stream(stream)

    def __enter__(self):
        if self.stream is not None and self.stream != torch.cuda.current_stream(self.like.device):
            for t in self.tensors:
                if t is not None:
                    t.record_stream(self.stream)
        self.guard.__enter__()
        return torch.cuda.current_stream(self.like.device).cuda_stream

    def __exit__(self, *exc):
        self.guard.__exit__(*exc)


class _Here:
    """The same for a call on the current stream of the current device."""

    def __init__(self, device):
        self.device = device

    def __enter__(self):
        return torch._C._cuda_getCurrentRawStream(self.device)

    def __exit__(self, *exc):
        pass


def _on(stream, like, *tensors):
    device = like.get_device()
    if stream is None and device == torch._C._cuda_getDevice():
        return _Here(device)
    return _On(stream, like, tensors)


def _call(name, args, stream):
    if _bound is None or _bound is not api._lib:
        lib()
    rc = _calls[name](args, stream)
    if rc != api.GTS_OK:
        raise api.GtsError(rc, name, api.lib().gts_last_error().decode())


def _ptr(t):
    return 0 if t is None else t.data_ptr()


def _no_gradient(what, *tensors):
    """Refuses a tensor that wants a derivative which the operator does not have
    and would drop without a word: by reverse mode, or a tangent."""
    if torch.is_grad_enabled():
        for t in tensors:
            if t is not None and t.requires_grad:
                raise ValueError(f"{what} requires a gradient, which it does not get here: use torch.no_grad()")
    _no_tangent(what, *tensors)


def _no_tangent(what, *tensors):
    if forward_ad._current_level >= 0:  # inside forward_ad.dual_level()
        for t in tensors:
            if t is not None and forward_ad.unpack_dual(t).tangent is not None:
                raise ValueError(f"{what} has a tangent: the operators have no forward-mode derivative")


def _wrote(*tensors):
    """Tells autograd of the caller's tensors that a call has written, so that
    the backward of an operation that saved one of them earlier raises."""
    tensors = [t for t in tensors if t is not None]
    if tensors:
        torch.autograd.graph.increment_version(tensors)


def _scale(scale, D):
    """scale as its field takes it; by default that of heads of D (heads of 0 are refused by the library)."""
    return max(D, 1) ** -0.5 if scale is None else _f32(scale).value


def _disjoint(strides, shape, name):
    """An output whose elements overlap (an expanded view) would be written
    from several places."""
    if 0 in strides and any(s == 0 and n > 1 for s, n in zip(strides, shape)):
        raise ValueError(f"{name} is an expanded view")


# ---- rotary ---------------------------------------------------------------------

def rotary_frequencies(dim, *, base=10000.0, scaling=None):
    """Radians a position of the dim / 2 pairs, as floats, and the factor on
    cosines and sines.  `scaling` stretches them to longer contexts:

    None                       base ** (-2 i / dim)
    {"kind": "linear", "factor": f}
        every frequency divided by f (positions interpolated)
    {"kind": "ntk", "factor": f}
        base times f ** (dim / (dim - 2)): the slowest pair stretched by f,
        the fastest left alone
    {"kind": "ramp", "factor": f, "original": n, "fast": 32, "slow": 1}
        pairs that turn more than `fast` times in the original n positions
        are left alone, those that turn less than `slow` times are divided by
        f, a linear ramp over the pair's number between; cosines and sines
        times 0.1 ln f + 1 (the YaRN method of Peng et al., 2023)."""
    _refuse(dim >= 2 and dim % 2 == 0, f"rotated part of {dim} values: even and at least 2")
    _refuse(base > 1, f"base {base}: more than 1")
    half, factor, mscale = dim // 2, 1.0, 1.0
    kind = None if scaling is None else scaling.get("kind")
    if scaling is not None:
        _refuse(kind in ("linear", "ntk", "ramp"), f"unknown scaling {kind!r}")
        known = {"kind", "factor"} | ({"original", "fast", "slow"} if kind == "ramp" else set())
        _refuse(set(scaling) <= known, f"scaling {kind!r} takes {sorted(known)}")
        factor = float(scaling.get("factor", 1.0))
        _refuse(math.isfinite(factor) and factor >= 1, f"scaling factor {factor}: at least 1")
    if kind == "ntk" and dim > 2:
        base = base * factor ** (dim / (dim - 2))
    f = [base ** (-2.0 * i / dim) for i in range(half)]
    if kind == "linear":
        f = [x / factor for x in f]
    if kind == "ramp":
        _refuse("original" in scaling and scaling["original"] >= 1, "scaling 'ramp' takes the original length")
        n, fast, slow = float(scaling["original"]), float(scaling.get("fast", 32)), float(scaling.get("slow", 1))
        _refuse(fast > slow > 0, "scaling 'ramp': fast > slow > 0")
        # the (fractional) number of the pair that turns `turns` times in n positions
        pair = lambda turns: dim * math.log(n / (turns * 2 * math.pi)) / (2 * math.log(base))  # noqa: E731
        lo, hi = max(math.floor(pair(fast)), 0), min(math.ceil(pair(slow)), dim - 1)  # hi may lie behind the last pair
        keep = [1.0 - min(max((i - lo) / max(hi - lo, 1e-3), 0.0), 1.0) for i in range(half)]
        f = [x * k + x / factor * (1.0 - k) for x, k in zip(f, keep)]
        mscale = 0.1 * math.log(factor) + 1.0
    return f, mscale


def rotary_table(n_positions, dim, *, base=10000.0, scaling=None, device="cuda", stream=None):
    """[n_positions, dim] float32: row p holds the cosines of position p's
    dim / 2 angles, then the sines (computed in 64 bits, rounded once).
    `dim` is the rotated part of the head."""
    f, mscale = rotary_frequencies(dim, base=base, scaling=scaling)
    _refuse(n_positions > 0, f"table of {n_positions} positions")
    like = torch.empty(0, device=device)
    _refuse(like.is_cuda, "the table lives on the GPU")
    with _on(stream, like) as s:
        table = torch.empty((n_positions, dim), dtype=torch.float32, device=like.device)
        rc = lib().gts_rotary_table(table.data_ptr(), n_positions, dim, (ctypes.c_double * len(f))(*f), mscale, s)
    if rc != api.GTS_OK:
        raise api.GtsError(rc, "gts_rotary_table", api.lib().gts_last_error().decode())
    return table


def _rotary(x, positions, table, flags, out, stream):
    dims = x.dim() if isinstance(x, torch.Tensor) else 0
    if dims != 3 and dims != 4:
        raise ValueError("x is a tensor [tokens, heads, dim] or [batch, tokens, heads, dim]")
    xs = _data(x, "x", dims)
    shape = x.shape
    B, S, H, D = (1, *shape) if dims == 3 else shape
    n_pos, rot, row = _table(table, x, D)
    pdims = positions.dim() if isinstance(positions, torch.Tensor) else 0
    ps = _index(positions, "positions", pdims, x, (torch.int64, torch.int32))
    if not (pdims == 1 and positions.shape[0] == S or pdims == 2 and dims == 4 and positions.shape == (B, S)):
        raise ValueError(f"positions {tuple(positions.shape)} for {B} x {S} tokens: [tokens] or [batch, tokens]")
    if out is not None:
        _disjoint(_data(out, "out", dims, x), out.shape, "out")
        _refuse(out.shape == shape, f"out is {tuple(out.shape)}, not {tuple(shape)}")
    with _on(stream, x, x, positions, table, out) as s:
        y = x.new_empty(shape) if out is None else out
        ys = y.stride()
        if dims == 3:
            xs, ys = (0, *xs), (0, *ys)
        _call("gts_rotary", _pack_rotary(
            x.data_ptr(), y.data_ptr(), positions.data_ptr(), table.data_ptr(), xs[0], xs[1], xs[2], ys[0], ys[1], ys[2],
            0 if pdims == 1 else ps[0], ps[-1], row, B, S, H, D, rot, n_pos, _TYPES[x.dtype],
            8 if positions.dtype == torch.int64 else 4, flags, 0), s)
    _wrote(out)
    return y


class _Rotary(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, positions, table, flags, stream):
        ctx.save_for_backward(positions, table)
        ctx.flags = flags
        return _rotary(x, positions, table, flags, None, stream)

    @staticmethod
    def backward(ctx, dy):
        positions, table = ctx.saved_tensors
        if dy.stride(-1) != 1:
            dy = dy.contiguous()
        # a linear map: its gradient has one of its own, the map again
        return _Rotary.apply(dy, positions, table, ctx.flags ^ BACKWARD, None), None, None, None, None


def _turn(x, positions, table, flags, out, stream):
    if isinstance(table, torch.Tensor):
        _no_gradient("table", table)
    if isinstance(x, torch.Tensor):
        _no_tangent("x", x)
        if x.requires_grad and torch.is_grad_enabled():
            _refuse(out is None, "out: x requires a gradient")
            return _Rotary.apply(x, positions, table, flags, stream)
    if isinstance(out, torch.Tensor):
        _no_gradient("out", out)
    return _rotary(x, positions, table, flags, out, stream)


def rotary(x, positions, table, *, interleaved=False, out=None, stream=None):
    """x [tokens, heads, D] or [batch, tokens, heads, D] with the leading
    table.shape[1] values of every head turned by the table's row of the
    token's position (int32 or int64 [tokens] or [batch, tokens]); the values
    behind them copied.  Pairs are (i, i + R / 2), or (2 i, 2 i + 1) when
    interleaved.  out=x rotates in place (any other overlap of the two mixes
    rotated values with others).  Differentiable in x by reverse mode, to any
    order (out is then refused); a table that requires a gradient, an out that
    does and tangents of forward mode are refused, torch.func's transforms raise.
    A position outside the table gives NaN."""
    return _turn(x, positions, table, INTERLEAVED if interleaved else 0, out, stream)


def rotary_backward(dy, positions, table, *, interleaved=False, out=None, stream=None):
    """The gradient of rotary's x from that of its result: the transposed
    rotation (scaled as the table is)."""
    return _turn(dy, positions, table, (INTERLEAVED if interleaved else 0) | BACKWARD, out, stream)


# ---- paged cache ------------------------------------------------------------------

def _cache_batch(k_cache, v_cache, T, page_table, lens, starts, prefix_len, like, written):
    """The packed values of gts_kv_cache and gts_kv_batch; the cache's heads and
    dim, and the number of sequences."""
    ks, vs = _data(k_cache, "k_cache", 4, like), _data(v_cache, "v_cache", 4, like)
    shape = k_cache.shape
    if v_cache.shape != shape:
        raise ValueError(f"k_cache {tuple(shape)} and v_cache {tuple(v_cache.shape)} differ in shape")
    if written:
        _disjoint(ks, shape, "k_cache")
        _disjoint(vs, shape, "v_cache")
    pages, page, heads, dim = shape
    ps = _index(page_table, "page_table", 2, like)
    ls = _index(lens, "lens", 1, like)
    B, max_pages = lens.shape[0], page_table.shape[1]
    if page_table.shape[0] != B or (ps[1] != 1 and max_pages > 1):
        raise ValueError(f"page_table is [{B}, pages], its rows contiguous: got {tuple(page_table.shape)}")
    if ls[0] != 1 and B > 1:
        raise ValueError("lens is not contiguous")
    if starts is not None:
        ss = _index(starts, "starts", 1, like)
        if starts.shape[0] != B + 1 or ss[0] != 1:
            raise ValueError(f"starts is [{B + 1}] and contiguous")
    prefix_len = operator.index(prefix_len)
    if not 0 <= prefix_len < 1 << 31:
        raise ValueError(f"prefix of {prefix_len} keys")
    return (k_cache.data_ptr(), v_cache.data_ptr(), ks[0], ks[1], ks[2], vs[0], vs[1], vs[2], pages, page, heads, dim,
            _TYPES[like.dtype], 0, _ptr(starts), lens.data_ptr(), page_table.data_ptr(), ps[0], B, T, max_pages,
            prefix_len), heads, dim, B


def append_kv(k, v, k_cache, v_cache, page_table, lens, *, starts=None, table=None, interleaved=False, prefix_len=0,
              q=None, q_out=None, stream=None):
    """Writes the new tokens' keys and values into their slots of the cache.
    With a table the keys are rotated on the way, and q (if given) into q_out
    (default: a new tensor), which is returned.  New token i of the n of
    sequence b becomes its own key lens[b] - n + i, in page
    page_table[b, key // page], at position prefix_len + key.  A page number
    outside the cache writes nothing.  A token outside every sequence, or with
    a negative key, writes nothing either; its rows of a new q_out are zeros, of
    a given one as they were.  Two tokens must not share a slot.  Has no
    gradient."""
    ks, vs = _data(k, "k", 3), _data(v, "v", 3, k)
    T, Hkv, D = k.shape
    if v.shape != k.shape:
        raise ValueError(f"k {tuple(k.shape)} and v {tuple(v.shape)} differ in shape")
    packed, heads, dim, _ = _cache_batch(k_cache, v_cache, T, page_table, lens, starts, prefix_len, k, True)
    if heads != Hkv or dim != D:
        raise ValueError(f"caches of {heads} heads of {dim} for keys of {Hkv} heads of {D}")
    n_pos, rot, row = (0, 0, 0) if table is None else _table(table, k, D)
    Hq, qs, os, flags = 0, (0, 0), (0, 0), INTERLEAVED if interleaved else 0
    if q is not None:
        qs = _data(q, "q", 3, k)
        Hq = q.shape[1]
        if q.shape[0] != T or q.shape[2] != D:
            raise ValueError(f"q is {tuple(q.shape)}: [{T}, heads, {D}]")
    if q_out is not None:
        _refuse(q is not None, "q_out without q")
        _disjoint(_data(q_out, "q_out", 3, k), q_out.shape, "q_out")
        _refuse(q_out.shape == q.shape, f"q_out is {tuple(q_out.shape)}, not {tuple(q.shape)}")
    _no_gradient("a tensor of the append", k, v, q, k_cache, v_cache, table, q_out)
    with _on(stream, k, k, v, k_cache, v_cache, page_table, lens, starts, table, q, q_out) as s:
        if q is not None:
            if q_out is None:
                q_out = q.new_empty(q.shape)
                flags |= ZERO_REST
            os = q_out.stride()
        _call("gts_append_kv", _pack_append(
            *packed, k.data_ptr(), v.data_ptr(), _ptr(q), _ptr(q_out), ks[0], ks[1], vs[0], vs[1], qs[0], qs[1], os[0], os[1],
            _ptr(table), row, Hq, rot, n_pos, flags), s)
    _wrote(k_cache, v_cache, q_out)
    return q_out


@functools.lru_cache(maxsize=256)
def _scratch_bytes(B, T, Hq, Hkv, D):
    n = ctypes.c_uint64(0)
    rc = lib().gts_shared_prefix_attention_scratch(B, T, Hq, Hkv, D, ctypes.byref(n))
    if rc != api.GTS_OK:
        raise api.GtsError(rc, "gts_shared_prefix_attention_scratch", api.lib().gts_last_error().decode())
    return int(n.value)


def attention_scratch_bytes(sequences, tokens, q_heads, kv_heads, dim):
    """Bytes of scratch shared_prefix_attention needs for a batch of these
    sizes, whatever its lengths."""
    return _scratch_bytes(sequences, tokens, q_heads, kv_heads, dim)


def shared_prefix_attention(q, k_cache, v_cache, page_table, lens, *, starts=None, prefix_pages=None, prefix_len=0,
                            scale=None, out=None, lse=None, scratch=None, stream=None):
    """Attention of the new tokens' q [T, Hq, D] over the cache: every token
    sees the prefix_len keys in prefix_pages (int32 [n]) and its sequence's own
    keys up to its own (lens counts them with the new ones).  Query head h reads key-value head h // (Hq / Hkv).
    scale defaults to D ** -0.5.  Without a prefix this is attention over a
    paged cache, one token a sequence or many.  A token without a key gives
    zeros and a log-sum of -inf; one whose keys all score -inf is 0 / 0, NaN.

    16-bit caches with rows aligned to 16 bytes have softmax weights rounded to
    their type for the product with the values, and read the prefix once for the
    whole batch; 32 bits, odd head dims and unaligned rows take a kernel that
    reads each key for every query head.

    out [T, Hq, D] and lse (float32 [T, Hq], natural logarithm) receive the
    results if given; scratch (uint8, attention_scratch_bytes) is allocated if
    not.  Returns out.  Has no gradient."""
    qs = _data(q, "q", 3)
    T, Hq, D = q.shape
    packed, heads, dim, B = _cache_batch(k_cache, v_cache, T, page_table, lens, starts, prefix_len, q, False)
    if dim != D:
        raise ValueError(f"caches of head dim {dim} for queries of {D}")
    n_prefix = 0
    if prefix_pages is not None:
        pps = _index(prefix_pages, "prefix_pages", 1, q)
        n_prefix = prefix_pages.shape[0]
        _refuse(pps[0] == 1 or n_prefix <= 1, "prefix_pages is not contiguous")
    if out is not None:
        _disjoint(_data(out, "out", 3, q), out.shape, "out")
        _refuse(out.shape == q.shape, f"out is {tuple(out.shape)}, not {tuple(q.shape)}")
    if lse is not None:
        _refuse(isinstance(lse, torch.Tensor) and lse.dtype == torch.float32 and lse.shape == (T, Hq)
                and lse.is_contiguous() and lse.device == q.device, f"lse is a contiguous float32 [{T}, {Hq}]")
    if scratch is not None:
        _refuse(isinstance(scratch, torch.Tensor) and scratch.dtype == torch.uint8 and scratch.is_contiguous()
                and scratch.device == q.device, "scratch is a contiguous uint8 tensor")
        _refuse(scratch.data_ptr() % 16 == 0, "scratch is not aligned to 16 bytes")
    _no_gradient("a tensor of the attention", q, k_cache, v_cache, out, lse)
    need = _scratch_bytes(B, T, Hq, heads, D)
    written = out, lse, scratch
    with _on(stream, q, q, k_cache, v_cache, page_table, lens, starts, prefix_pages, out, lse, scratch) as s:
        if out is None:
            out = q.new_empty(q.shape)
        if scratch is None:
            scratch = q.new_empty(need, dtype=torch.uint8)
        os = out.stride()
        _call("gts_shared_prefix_attention", _pack_attention(
            *packed, q.data_ptr(), out.data_ptr(), _ptr(lse), qs[0], qs[1], os[0], os[1], _ptr(prefix_pages), n_prefix, Hq,
            _scale(scale, D), 0, scratch.data_ptr(), scratch.numel()), s)
    _wrote(*written)
    return out


# ---- norms --------------------------------------------------------------------------

@functools.lru_cache(maxsize=1024)
def _scratch_of(name, *sizes):
    n = ctypes.c_uint64(0)
    rc = getattr(lib(), name)(*sizes, ctypes.byref(n))
    if rc != api.GTS_OK:
        raise api.GtsError(rc, name, api.lib().gts_last_error().decode())
    return int(n.value)


def _scratch(like, name, *sizes):
    """Scratch of a call, allocated on its stream: (tensor or None, bytes)."""
    n = _scratch_of(name, *sizes)
    return (like.new_empty(n, dtype=torch.uint8) if n else None), n


def _vector(t, name, n, like):
    """t is None or a contiguous [n] of the type and on the device of `like`."""
    if t is not None:
        s = _data(t, name, 1, like)
        if t.shape[0] != n or (n > 1 and s[0] != 1):
            raise ValueError(f"{name} is a contiguous [{n}]: got {tuple(t.shape)}")


def _matrix(t, name, shape, like, written=False):
    """t is None or a matrix of that shape; returns its row stride."""
    if t is None:
        return 0
    s = _data(t, name, 2, like)
    if t.shape != shape:
        raise ValueError(f"{name} is {tuple(t.shape)}, not {tuple(shape)}")
    if written:
        _disjoint(s, shape, name)
    return s[0]


def _stats(t, name, rows, like):
    if t is not None and not (isinstance(t, torch.Tensor) and t.dtype == torch.float32 and t.shape == (rows,)
                              and t.is_contiguous() and t.get_device() == like.get_device()):
        raise ValueError(f"{name} is a contiguous float32 [{rows}] beside x")


def _flat(x, name="x", stream=None):
    """x [..., dim] as rows [n, dim]: a view where its layout has one, else a copy on the
    current stream, which a call on another one does not wait for and so refuses."""
    if not isinstance(x, torch.Tensor):
        raise TypeError(f"{name} is a tensor: got {type(x).__name__}")
    if x.dim() == 2:
        return x
    if x.dim() < 1:
        raise ValueError(f"{name} has no dimensions")
    flat = x.reshape(math.prod(x.shape[:-1]), x.shape[-1])  # sizes that an empty x leaves open with -1
    if stream is not None and flat.data_ptr() != x.data_ptr():
        raise ValueError(f"{name}: its rows are not evenly apart, so that it would be copied on another stream")
    return flat


def _norm(x, weight, bias, eps, center, out, mean, rstd, stream):
    xs = _data(x, "x", 2)
    rows, dim = x.shape
    _refuse(dim > 0, "x has rows of no values")
    _vector(weight, "weight", dim, x)
    _vector(bias, "bias", dim, x)
    os = _matrix(out, "out", x.shape, x, True)
    _stats(mean, "mean", rows, x)
    _stats(rstd, "rstd", rows, x)
    with _on(stream, x, x, weight, bias, out, mean, rstd) as s:
        y = x.new_empty((rows, dim)) if out is None else out
        _call("gts_layer_norm", _pack_norm(
            x.data_ptr(), y.data_ptr(), _ptr(weight), _ptr(bias), _ptr(mean), _ptr(rstd), xs[0],
            dim if out is None else os, rows, dim, _f32(eps).value, _TYPES[x.dtype], CENTER if center else 0, 0), s)
    _wrote(out, mean, rstd)
    return y


def _keep(stream, like, *tensors):
    """Tensors that a call on `stream` allocates there, and its backward pass reads on the current one."""
    if stream is not None:
        current = torch.cuda.current_stream(like.device)
        for t in tensors:
            if t is not None:
                t.record_stream(current)


class _Norm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, eps, center, stream):
        _data(x, "x", 2)
        with _on(stream, x):
            mean = x.new_empty(x.shape[0], dtype=torch.float32) if center else None
            rstd = x.new_empty(x.shape[0], dtype=torch.float32)
        y = _norm(x, weight, bias, eps, center, None, mean, rstd, stream)
        _keep(stream, x, mean, rstd)
        ctx.save_for_backward(x, weight, mean, rstd)
        ctx.bias = bias is not None
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        x, weight, mean, rstd = ctx.saved_tensors
        need = ctx.needs_input_grad
        dx, dw, db = _norm_backward(_rows(dy), x, weight, rstd, mean, need[0], weight is not None and need[1],
                                    ctx.bias and need[2], None)
        return dx, dw, db, None, None, None


def _rows(t):
    return t if t.stride(-1) == 1 or t.shape[-1] <= 1 else t.contiguous()


def layer_norm(x, weight=None, bias=None, *, eps=1e-5, center=True, out=None, mean=None, rstd=None, stream=None):
    """Rows of x [..., dim] with their mean taken off and divided by the root of
    their mean square plus eps, times weight [dim], plus bias [dim]; without `center`
    the mean stays (RMS norm).  out=x writes over x (another overlap of the two mixes rows).  mean and rstd (float32, one
    a row) receive what layer_norm_backward takes.  Differentiable once in x, weight and
    bias by reverse mode (out, mean and rstd are then refused)."""
    _no_tangent_of("a tensor of the norm", x, weight, bias)
    shape = x.shape if isinstance(x, torch.Tensor) else None
    flat = _flat(x, "x", stream)
    if _wants_gradient(x, weight, bias):
        _refuse(out is None and mean is None and rstd is None, "out, mean and rstd are refused: an input requires a gradient")
        y = _Norm.apply(flat, weight, bias, eps, center, stream)
    else:
        _no_gradient("out of the norm", out, mean, rstd)
        if out is not None:
            _refuse(isinstance(out, torch.Tensor) and out.shape == shape, f"out is a tensor {tuple(shape)}")
            flat_out = _flat(out, "out")
            _refuse(flat_out.data_ptr() == out.data_ptr(), "out: its rows are not evenly apart")
            _norm(flat, weight, bias, eps, center, flat_out, mean, rstd, stream)
            return out
        y = _norm(flat, weight, bias, eps, center, None, mean, rstd, stream)
    return y if y.shape == shape else y.view(shape)


def _norm_backward(dy, x, weight, rstd, mean, want_dx, want_dw, want_db, stream):
    xs = _data(x, "x", 2)
    rows, dim = x.shape
    _refuse(dim > 0, "x has rows of no values")
    dys = _matrix(dy, "dy", x.shape, x)
    _vector(weight, "weight", dim, x)
    _stats(mean, "mean", rows, x)
    _stats(rstd, "rstd", rows, x)
    with _on(stream, x, x, dy, weight, mean, rstd) as s:
        dx = x.new_empty((rows, dim)) if want_dx else None
        dw = x.new_empty(dim) if want_dw else None
        db = x.new_empty(dim) if want_db else None
        scratch, n = _scratch(x, "gts_layer_norm_backward_scratch", rows, dim) if want_dw or want_db else (None, 0)
        _call("gts_layer_norm_backward", _pack_norm_grad(
            dy.data_ptr(), x.data_ptr(), _ptr(weight), _ptr(mean), rstd.data_ptr(), _ptr(dx), _ptr(dw), _ptr(db), dys, xs[0],
            dim, rows, dim, _TYPES[x.dtype], 0 if mean is None else CENTER, _ptr(scratch), n), s)
    return dx, dw, db


def layer_norm_backward(dy, x, weight, rstd, mean=None, *, bias=False, stream=None):
    """(dx, dweight, dbias) of layer_norm from the gradient of its result, x and the
    statistics that the forward pass left; mean=None is the norm without `center`.
    dweight is None without a weight, dbias unless `bias` asks for it."""
    _no_gradient("a tensor of the norm's gradient", dy, x, weight, rstd, mean)
    _refuse(isinstance(rstd, torch.Tensor), "rstd is a float32 tensor, one value a row")
    flat = _flat(x, "x", stream)
    _refuse(isinstance(dy, torch.Tensor) and dy.shape == x.shape, "dy has the shape of x")
    dx, dw, db = _norm_backward(_flat(dy, "dy", stream), flat, weight, rstd, mean, True, weight is not None, bias, stream)
    return dx.view(x.shape), dw, db


# ---- products -------------------------------------------------------------------------

def _activation(name):
    if name not in ACTIVATIONS:
        raise ValueError(f"activation {name!r}: one of {list(ACTIVATIONS)}")
    return ACTIVATIONS[name]


def _matmul(a, b, out, preact, bias, gate, residual, strides, m, n, k, act, flags, s):
    """One product on stream s; strides of a, b, out, preact, gate, residual."""
    scratch, size = _scratch(out, "gts_matmul_scratch", m, n, k)
    _call("gts_matmul", _pack_matmul(
        a.data_ptr(), b.data_ptr(), out.data_ptr(), _ptr(preact), _ptr(bias), _ptr(gate), _ptr(residual), *strides, m, n, k,
        _TYPES[out.dtype], act, flags, _ptr(scratch), size), s)


def _linear(x, weight, bias, act, gate, residual, out, preact, stream):
    xs = _data(x, "x", 2)
    ws = _data(weight, "weight", 2, x)
    (M, K), N = x.shape, weight.shape[0]
    if weight.shape[1] != K:
        raise ValueError(f"weight is {tuple(weight.shape)} for x of {K} columns: [columns of the result, {K}]")
    _vector(bias, "bias", N, x)
    gs, rs = _matrix(gate, "gate", (M, N), x), _matrix(residual, "residual", (M, N), x)
    os, ps = _matrix(out, "out", (M, N), x, True), _matrix(preact, "preact", (M, N), x, True)
    with _on(stream, x, x, weight, bias, gate, residual, out, preact) as s:
        y = x.new_empty((M, N)) if out is None else out
        _matmul(x, weight, y, preact, bias, gate, residual, (xs[0], ws[0], N if out is None else os, ps, gs, rs), M, N, K, act,
                0, s)
    _wrote(out, preact)
    return y


class _Linear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, act, gate, residual, stream):
        preact = None
        if (act or gate is not None) and any(t is not None and t.requires_grad for t in (x, weight, bias, gate)):
            _data(x, "x", 2)
            with _on(stream, x):
                preact = x.new_empty((x.shape[0], weight.shape[0]))
        y = _linear(x, weight, bias, act, gate, residual, None, preact, stream)
        _keep(stream, x, preact)
        ctx.save_for_backward(x, weight, preact, gate)
        ctx.act, ctx.bias, ctx.residual = act, bias is not None, residual is not None
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        x, weight, preact, gate = ctx.saved_tensors
        need = ctx.needs_input_grad
        dres = dy if ctx.residual and need[5] else None
        if not (need[0] or need[1] or need[2] or need[4]):
            return None, None, None, None, None, dres, None
        dx, dw, db, dg = _linear_backward(_rows(dy), x, weight, ctx.act, preact, gate, need[0], need[1], ctx.bias and need[2],
                                          gate is not None and need[4], None)
        return dx, dw, db, None, dg, dres, None


def _wants_gradient(*tensors):
    return torch.is_grad_enabled() and any(isinstance(t, torch.Tensor) and t.requires_grad for t in tensors)


def _no_tangent_of(what, *tensors):
    _no_tangent(what, *(t for t in tensors if isinstance(t, torch.Tensor)))


def linear(x, weight, bias=None, *, activation=None, gate=None, residual=None, out=None, preact=None, stream=None):
    """act(x weight^T + bias) * gate + residual, in one pass: x [..., K], weight
    [N, K], bias [N]; gate and residual have the result's shape [..., N].  `activation` is
    None, "relu", "gelu" (by the normal distribution), "gelu_tanh" or "silu"; with gate
    the result is that of a gated layer.  All of it is computed in 32 bits and rounded
    once.  out may be gate or residual, and shares no memory with x, weight or bias; preact (of
    the result's shape and type) receives x weight^T + bias for linear_backward, and shares none with any.  Differentiable once in x, weight,
    bias, gate and residual by reverse mode (out and preact are then refused)."""
    act = _activation(activation)
    _no_tangent_of("a tensor of the product", x, weight, bias, gate, residual)
    flat = _flat(x, "x", stream)
    _refuse(isinstance(weight, torch.Tensor) and weight.dim() == 2, "weight is a matrix [N, K]")
    shape = (*x.shape[:-1], weight.shape[0])
    for t, name in ((gate, "gate"), (residual, "residual"), (out, "out"), (preact, "preact")):
        if t is not None:
            _refuse(isinstance(t, torch.Tensor) and t.shape == shape, f"{name} is a tensor {shape}")
    g, r = (None if t is None else _flat(t, "gate or residual", stream) for t in (gate, residual))
    if _wants_gradient(x, weight, bias, gate, residual):
        _refuse(out is None and preact is None, "out and preact are refused: an input requires a gradient")
        y = _Linear.apply(flat, weight, bias, act, g, r, stream)
    else:
        _no_gradient("out of the product", out, preact)
        o, z = (None if t is None else _flat(t) for t in (out, preact))
        for t, f, name in ((out, o, "out"), (preact, z, "preact")):
            _refuse(t is None or f.data_ptr() == t.data_ptr(), f"{name}: its rows are not evenly apart")
        y = _linear(flat, weight, bias, act, g, r, o, z, stream)
        if out is not None:
            return out
    return y if y.shape == shape else y.view(shape)


def _linear_backward(dy, x, weight, act, preact, gate, want_dx, want_dw, want_db, want_dg, stream):
    xs, ws = _data(x, "x", 2), _data(weight, "weight", 2, x)
    (M, K), N = x.shape, weight.shape[0]
    if weight.shape[1] != K:
        raise ValueError(f"weight is {tuple(weight.shape)} for x of {K} columns")
    dys = _matrix(dy, "dy", (M, N), x)
    ps, gs = _matrix(preact, "preact", (M, N), x), _matrix(gate, "gate", (M, N), x)
    if preact is None and (act or gate is not None):
        raise ValueError("preact is missing: linear left it for an activation or a gate")
    with _on(stream, x, x, weight, dy, preact, gate) as s:
        dz, zs = dy, dys
        db = x.new_empty(N) if want_db else None
        dg = x.new_empty((M, N)) if want_dg else None
        own = (act or gate is not None) and (want_dx or want_dw)
        if own:
            dz, zs = x.new_empty((M, N)), N
        if own or want_db or want_dg:
            scratch, n = _scratch(x, "gts_linear_backward_scratch", M, N) if want_db else (None, 0)
            _call("gts_linear_backward", _pack_linear_grad(
                dy.data_ptr(), _ptr(preact), _ptr(gate), dz.data_ptr() if own else 0, _ptr(dg), _ptr(db), dys, ps, gs, zs, N,
                M, N, _TYPES[x.dtype], act, _ptr(scratch), n), s)
        dx = dw = None
        if want_dx:
            dx = x.new_empty((M, K))
            _matmul(dz, weight, dx, None, None, None, None, (zs, ws[0], K, 0, 0, 0), M, K, N, 0, B_COLUMNS, s)
        if want_dw:
            dw = x.new_empty((N, K))
            _matmul(dz, x, dw, None, None, None, None, (zs, xs[0], K, 0, 0, 0), N, K, M, 0, A_COLUMNS | B_COLUMNS, s)
    return dx, dw, db, dg


def linear_backward(dy, x, weight, *, activation=None, preact=None, gate=None, bias=False, stream=None):
    """(dx, dweight, dbias, dgate) of linear from the gradient of its result, its
    operands and, with an activation or a gate, the preact that it left.  dbias is None
    unless `bias` asks for it, dgate without a gate.  The gradient of residual is dy.
    What is multiplied (dy times the gate and the activation's slope) is in dy's type."""
    act = _activation(activation)
    _no_gradient("a tensor of the product's gradient", dy, x, weight, preact, gate)
    flat = _flat(x, "x", stream)
    _refuse(isinstance(weight, torch.Tensor) and weight.dim() == 2, "weight is a matrix [N, K]")
    shape = (*x.shape[:-1], weight.shape[0])
    for t, name in ((dy, "dy"), (preact, "preact"), (gate, "gate")):
        if t is not None or name == "dy":
            _refuse(isinstance(t, torch.Tensor) and t.shape == shape, f"{name} is a tensor {shape}")
    z, g = (None if t is None else _flat(t, "preact or gate", stream) for t in (preact, gate))
    dx, dw, db, dg = _linear_backward(_flat(dy, "dy", stream), flat, weight, act, z, g, True, True, bias, gate is not None, stream)
    return dx.view(x.shape), dw, db, None if dg is None else dg.view(shape)


# ---- attention over prompts ---------------------------------------------------------------

def _prompt_shapes(q, k, v, starts):
    qs, ks, vs = _data(q, "q", 3), _data(k, "k", 3, q), _data(v, "v", 3, q)
    T, Hq, D = q.shape
    if k.shape != v.shape or k.shape[0] != T or k.shape[2] != D:
        raise ValueError(f"q {tuple(q.shape)}, k {tuple(k.shape)}, v {tuple(v.shape)}: [{T}, heads, {D}], k and v alike")
    B = 1
    if starts is not None:
        ss = _index(starts, "starts", 1, q)
        B = starts.shape[0] - 1
        if B < 1 or ss[0] != 1:
            raise ValueError("starts is [sequences + 1] and contiguous")
    return qs, ks, vs, B, T, Hq, k.shape[1], D


def _lse_like(lse, T, Hq, q):
    _refuse(isinstance(lse, torch.Tensor) and lse.dtype == torch.float32 and lse.shape == (T, Hq) and lse.is_contiguous()
            and lse.device == q.device, f"lse is a contiguous float32 [{T}, {Hq}]")


def _prompt(q, k, v, starts, causal, scale, out, lse, stream):
    qs, ks, vs, B, T, Hq, Hkv, D = _prompt_shapes(q, k, v, starts)
    if out is not None:
        _disjoint(_data(out, "out", 3, q), out.shape, "out")
        _refuse(out.shape == q.shape, f"out is {tuple(out.shape)}, not {tuple(q.shape)}")
    if lse is not None:
        _lse_like(lse, T, Hq, q)
    with _on(stream, q, q, k, v, starts, out, lse) as s:
        o = q.new_empty(q.shape) if out is None else out
        os = o.stride()
        _call("gts_prompt_attention", _pack_prompt(
            q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), _ptr(lse), _ptr(starts), qs[0], qs[1], ks[0], ks[1], vs[0],
            vs[1], os[0], os[1], B, T, Hq, Hkv, D, _TYPES[q.dtype], _scale(scale, D), CAUSAL if causal else 0), s)
    _wrote(out, lse)
    return o


class _Prompt(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, starts, causal, scale, stream):
        _data(q, "q", 3)
        with _on(stream, q):
            lse = q.new_empty(q.shape[:2], dtype=torch.float32)
        o = _prompt(q, k, v, starts, causal, scale, None, lse, stream)
        _keep(stream, q, o, lse)
        ctx.save_for_backward(q, k, v, o, lse, starts)
        ctx.causal, ctx.scale = causal, scale
        return o

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dout):
        q, k, v, o, lse, starts = ctx.saved_tensors
        dq, dk, dv = _prompt_backward(_rows(dout), q, k, v, o, lse, starts, ctx.causal, ctx.scale, None)
        return dq, dk, dv, None, None, None, None


def prompt_attention(q, k, v, starts=None, *, causal=True, scale=None, out=None, lse=None, stream=None):
    """Attention over whole prompts: q [T, Hq, D], k and v [T, Hkv, D], the tokens of
    sequence b at starts[b] .. starts[b + 1] (int32 [B + 1], ascending; None: one
    sequence).  A token sees the keys of its sequence, with `causal` those up to its own.
    Query head h reads key-value head h // (Hq / Hkv); scale defaults to D ** -0.5.  A token
    outside every sequence gives zeros and a log-sum of -inf.  out (which shares no memory
    with the inputs) and lse (float32 [T, Hq], natural logarithm) receive the results if given.  Softmax weights are rounded
    to the tensors' type for the product with the values.  Differentiable once in q, k and
    v by reverse mode (out and lse are then refused)."""
    _no_tangent_of("a tensor of the attention", q, k, v)
    if _wants_gradient(q, k, v):
        _refuse(out is None and lse is None, "out and lse are refused: an input requires a gradient")
        return _Prompt.apply(q, k, v, starts, causal, scale, stream)
    _no_gradient("out of the attention", out, lse)
    return _prompt(q, k, v, starts, causal, scale, out, lse, stream)


def _prompt_backward(dout, q, k, v, out, lse, starts, causal, scale, stream):
    qs, ks, vs, B, T, Hq, Hkv, D = _prompt_shapes(q, k, v, starts)
    ds, os = _data(dout, "dout", 3, q), _data(out, "out", 3, q)
    _refuse(dout.shape == q.shape and out.shape == q.shape, f"dout and out are {tuple(q.shape)}")
    _lse_like(lse, T, Hq, q)
    with _on(stream, q, dout, q, k, v, out, lse, starts) as s:
        dq, dk, dv = q.new_empty(q.shape), k.new_empty(k.shape), v.new_empty(v.shape)
        scratch, n = _scratch(q, "gts_prompt_attention_backward_scratch", B, T, Hq, Hkv, D)
        _call("gts_prompt_attention_backward", _pack_prompt_grad(
            dout.data_ptr(), q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), lse.data_ptr(), _ptr(starts),
            dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), ds[0], ds[1], qs[0], qs[1], ks[0], ks[1], vs[0], vs[1], os[0], os[1],
            Hq * D, D, Hkv * D, D, Hkv * D, D, B, T, Hq, Hkv, D, _TYPES[q.dtype], _scale(scale, D), CAUSAL if causal else 0,
            _ptr(scratch), n), s)
    return dq, dk, dv


def prompt_attention_backward(dout, q, k, v, out, lse, starts=None, *, causal=True, scale=None, stream=None):
    """(dq, dk, dv) of prompt_attention from the gradient of its result, its inputs,
    its result and the log-sums that it left; causal and scale as in the forward call.
    Weights and their gradients are rounded to the tensors' type for the products (in
    float16 scaled by powers of two, so that no size of dout or v loses them), and
    summed over a key-value head's query heads in 32 bits.  Tokens outside every
    sequence get zeros.  The same bits on every run."""
    _no_gradient("a tensor of the attention's gradient", dout, q, k, v, out, lse)
    return _prompt_backward(dout, q, k, v, out, lse, starts, causal, scale, stream)
