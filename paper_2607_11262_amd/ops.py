"""Operators of the serving step whose tile graphs this package simulates, as
hand-written kernels on the card (C ABI: include/gts_ops.h): rotary positions,
appending keys and values to a paged cache, and attention over that cache for a
batch whose sequences share a prefix.

    from paper_2607_11262_amd import ops
    table = ops.rotary_table(65536, 128)                   # once
    q = ops.append_kv(k, v, k_cache, v_cache, pages, lens, table=table, q=q,
                      prefix_len=P)                        # a decode step: one
    o = ops.shared_prefix_attention(q, k_cache, v_cache, pages, lens,
                                    prefix_pages=shared, prefix_len=P)

    y = ops.rotary(x, positions, table)                    # a training step
    dx = ops.rotary_backward(dy, positions, table)         # (autograd calls it too)

Shapes.  q [T, Hq, D], k and v [T, Hkv, D]: the new tokens of all sequences one
behind the other, sequence b's at starts[b] .. starts[b + 1] (starts=None: the
same number each).  Caches [pages, page, Hkv, D] in any memory order whose last
dimension is contiguous (pages kept head by head are a transposed view), page a
power of two.  page_table [B, max_pages] int32; lens [B] int32 counts a
sequence's own keys with its new ones, the shared prefix apart.  Types: bfloat16,
float16, float32.

Errors are ValueError / TypeError for shapes, types and devices, and
api.GtsError for what the library refuses.  Work is enqueued on `stream`
(default: the current one) and not waited for; outputs and scratch are
allocated on it, and tensors handed to another stream than the current one are
kept from reuse until it has run (record_stream).  The caller orders the
streams.  Every call may be captured into a graph.  For autograd the caller's
tensors that a call writes (out, q_out, lse, scratch, the caches) are modified in
place.
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

EXPORTS = ("gts_rotary_table", "gts_rotary", "gts_append_kv", "gts_shared_prefix_attention",
           "gts_shared_prefix_attention_scratch")

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


# The structures' values in one call each, as the C side lays them out: a call of
# a small batch is bound by the host.
_pack_rotary = struct.Struct("=4Q3q3q2qq10I").pack
_pack_cache_batch = "2Q3q3q6I3Qq4I"
_pack_append = struct.Struct("=" + _pack_cache_batch + "4Q2q2q2q2qQq4I").pack
_pack_attention = struct.Struct("=" + _pack_cache_batch + "3Q2q2qQ2IfIQQ").pack

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
        for name in ("gts_rotary", "gts_append_kv", "gts_shared_prefix_attention"):
            getattr(L, name).argtypes = [_vp, _vp]
            _calls[name] = getattr(L, name)
        L.gts_shared_prefix_attention_scratch.argtypes = [_u32] * 5 + [ctypes.POINTER(ctypes.c_uint64)]
        _scratch_bytes.cache_clear()
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
    if strides[-1] != 1 and t.shape[-1] > 1:
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
            D ** -0.5 if scale is None else _f32(scale).value, 0, scratch.data_ptr(), scratch.numel()), s)
    _wrote(*written)
    return out
