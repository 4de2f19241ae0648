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
streams.  Every call may be captured into a graph.
"""
from __future__ import annotations

import ctypes
import functools
import math

import torch

from . import api

F32, BF16, F16 = 0, 1, 2
INTERLEAVED, BACKWARD = 1, 2
MAX_ATTENTION_DIM = 256  # GTS_OPS_MAX_ATTN
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


_bound = None


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
        L.gts_shared_prefix_attention_scratch.argtypes = [_u32] * 5 + [ctypes.POINTER(ctypes.c_uint64)]
        _bound = L
    return L


# ---- checks and streams -----------------------------------------------------------

def _refuse(ok, why):
    if not ok:
        raise ValueError(why)


def _data(t, name, dims, like=None):
    """t is a tensor on the GPU with `dims` dimensions and a contiguous last
    one, of the type and on the device of `like`."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} is a tensor: got {type(t).__name__}")
    _refuse(t.dim() == dims, f"{name} has {t.dim()} dimensions, not {dims}")
    _refuse(t.is_cuda, f"{name} is not on the GPU")
    _refuse(t.stride(-1) == 1 or t.shape[-1] <= 1, f"{name}: the last dimension is not contiguous")
    if like is None:
        if t.dtype not in _TYPES:
            raise TypeError(f"{name} is {t.dtype}: bfloat16, float16 or float32")
    else:
        if t.dtype != like.dtype:
            raise TypeError(f"{name} is {t.dtype}, not {like.dtype}")
        _refuse(t.device == like.device, f"{name} is on {t.device}, not {like.device}")


def _index(t, name, dims, like, types=(torch.int32,)):
    if not isinstance(t, torch.Tensor) or t.dtype not in types:
        raise TypeError(f"{name} is a tensor of {' or '.join(str(x) for x in types)}")
    _refuse(t.dim() == dims, f"{name} has {t.dim()} dimensions, not {dims}")
    _refuse(t.device == like.device, f"{name} is on {t.device}, not {like.device}")


def _table(table, like, D):
    if not isinstance(table, torch.Tensor) or table.dtype != torch.float32:
        raise TypeError("table is a float32 tensor (rotary_table)")
    _refuse(table.dim() == 2 and table.device == like.device and (table.stride(1) == 1 or table.shape[1] <= 1),
            f"table is [positions, rotated values] on {like.device}, its rows contiguous")
    _refuse(0 < table.shape[1] <= D, f"table turns {table.shape[1]} values of a head of {D}")


class _On:
    """The stream of a call, current while outputs are allocated and the work
    is enqueued, with the device of the tensors current."""

    def __init__(self, stream, like, tensors):
        self.guard = None
        device = like.device
        if stream is None:
            self.stream = torch.cuda.current_stream(device)
            if device.index != torch.cuda.current_device():
                self.guard = torch.cuda.device(device)
        else:
            _refuse(stream.device == device, f"stream is on {stream.device}, the tensors on {device}")
            self.stream = stream
            self.guard = torch.cuda.stream(stream)  # also makes its device current
            if stream != torch.cuda.current_stream(device):
                for t in tensors:
                    if t is not None:
                        t.record_stream(stream)

    def __enter__(self):
        if self.guard is not None:
            self.guard.__enter__()
        return self.stream.cuda_stream

    def __exit__(self, *exc):
        if self.guard is not None:
            self.guard.__exit__(*exc)


def _call(name, args, stream):
    rc = getattr(lib(), name)(ctypes.byref(args), stream)
    if rc != api.GTS_OK:
        raise api.GtsError(rc, name, api.lib().gts_last_error().decode())


def _ptr(t):
    return None if t is None else t.data_ptr()


def _disjoint(t, name):
    """An output whose elements overlap (an expanded view) would be written
    from several places."""
    _refuse(all(s != 0 or n <= 1 for s, n in zip(t.stride(), t.shape)), f"{name} is an expanded view")


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
        lo, hi = max(math.floor(pair(fast)), 0), min(math.ceil(pair(slow)), half - 1)
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
    with _On(stream, like, ()) as s:
        table = torch.empty((n_positions, dim), dtype=torch.float32, device=like.device)
        rc = lib().gts_rotary_table(table.data_ptr(), n_positions, dim, (ctypes.c_double * len(f))(*f), mscale, s)
    if rc != api.GTS_OK:
        raise api.GtsError(rc, "gts_rotary_table", api.lib().gts_last_error().decode())
    return table


def _rotary(x, positions, table, flags, out, stream):
    _refuse(isinstance(x, torch.Tensor) and x.dim() in (3, 4), "x is [tokens, heads, dim] or [batch, tokens, heads, dim]")
    _data(x, "x", x.dim())
    B, S, H, D = (1, *x.shape) if x.dim() == 3 else x.shape
    _table(table, x, D)
    _index(positions, "positions", positions.dim() if isinstance(positions, torch.Tensor) else 0, x,
           (torch.int64, torch.int32))
    shared = positions.dim() == 1
    _refuse(positions.shape == ((S,) if shared else (B, S)) and (shared or x.dim() == 4),
            f"positions {tuple(positions.shape)} for {B} x {S} tokens: [tokens] or [batch, tokens]")
    if out is not None:
        _data(out, "out", x.dim(), x)
        _refuse(out.shape == x.shape, f"out is {tuple(out.shape)}, not {tuple(x.shape)}")
        _disjoint(out, "out")
    with _On(stream, x, (x, positions, table, out)) as s:
        if out is None:
            out = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        xs, os, ps = x.stride(), out.stride(), positions.stride()
        if x.dim() == 3:
            xs, os = (0, *xs), (0, *os)
        args = _RotaryArgs(x.data_ptr(), out.data_ptr(), positions.data_ptr(), table.data_ptr(), xs[:3], os[:3],
                           (0, ps[0]) if shared else ps, table.stride(0), B, S, H, D, table.shape[1], table.shape[0],
                           _TYPES[x.dtype], positions.element_size(), flags, 0)
        _call("gts_rotary", args, s)
    return out


class _Rotary(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, positions, table, interleaved, stream):
        ctx.save_for_backward(positions, table)
        ctx.interleaved, ctx.stream = interleaved, stream
        return _rotary(x, positions, table, INTERLEAVED if interleaved else 0, None, stream)

    @staticmethod
    def backward(ctx, dy):
        positions, table = ctx.saved_tensors
        if dy.stride(-1) != 1:
            dy = dy.contiguous()
        dx = _rotary(dy, positions, table, (INTERLEAVED if ctx.interleaved else 0) | BACKWARD, None, None)
        return dx, None, None, None, None


def rotary(x, positions, table, *, interleaved=False, out=None, stream=None):
    """x [tokens, heads, D] or [batch, tokens, heads, D] with the leading
    table.shape[1] values of every head turned by the table's row of the
    token's position (int32 or int64 [tokens] or [batch, tokens]); the values
    behind them copied.  Pairs are (i, i + R / 2), or (2 i, 2 i + 1) when
    interleaved.  out=x rotates in place.  Differentiable in x (without out).
    A position outside the table gives NaN."""
    if out is None and torch.is_grad_enabled() and isinstance(x, torch.Tensor) and x.requires_grad:
        return _Rotary.apply(x, positions, table, interleaved, stream)
    return _rotary(x, positions, table, INTERLEAVED if interleaved else 0, out, stream)


def rotary_backward(dy, positions, table, *, interleaved=False, out=None, stream=None):
    """The gradient of rotary's x from that of its result: the transposed
    rotation (scaled as the table is)."""
    return _rotary(dy, positions, table, (INTERLEAVED if interleaved else 0) | BACKWARD, out, stream)


# ---- paged cache ------------------------------------------------------------------

def _cache(k_cache, v_cache, like):
    _data(k_cache, "k_cache", 4, like)
    _data(v_cache, "v_cache", 4, like)
    _refuse(k_cache.shape == v_cache.shape,
            f"k_cache {tuple(k_cache.shape)} and v_cache {tuple(v_cache.shape)} differ in shape")
    pages, page, heads, dim = k_cache.shape
    return _Cache(k_cache.data_ptr(), v_cache.data_ptr(), k_cache.stride()[:3], v_cache.stride()[:3], pages, page,
                  heads, dim, _TYPES[k_cache.dtype], 0)


def _batch(T, page_table, lens, starts, prefix_len, like):
    _index(page_table, "page_table", 2, like)
    _index(lens, "lens", 1, like)
    B = lens.shape[0]
    _refuse(page_table.shape[0] == B and (page_table.stride(1) == 1 or page_table.shape[1] <= 1),
            f"page_table is [{B}, pages], its rows contiguous: got {tuple(page_table.shape)}")
    _refuse(lens.stride(0) == 1 or B <= 1, "lens is not contiguous")
    if starts is not None:
        _index(starts, "starts", 1, like)
        _refuse(starts.shape[0] == B + 1 and starts.stride(0) == 1, f"starts is [{B + 1}] and contiguous")
    _refuse(0 <= prefix_len < 1 << 31, f"prefix of {prefix_len} keys")
    return _Batch(_ptr(starts), lens.data_ptr(), page_table.data_ptr(), page_table.stride(0), B, T,
                  page_table.shape[1], prefix_len)


def append_kv(k, v, k_cache, v_cache, page_table, lens, *, starts=None, table=None, interleaved=False, prefix_len=0,
              q=None, q_out=None, stream=None):
    """Writes the new tokens' keys and values into their slots of the cache.
    With a table the keys are rotated on the way, and q (if given) into q_out
    (default: a new tensor), which is returned.  New token i of the n of
    sequence b becomes its own key lens[b] - n + i, in page
    page_table[b, key // page], at position prefix_len + key.  A page number
    outside the cache writes nothing.  Two tokens must not share a slot."""
    _data(k, "k", 3)
    _data(v, "v", 3, k)
    T, Hkv, D = k.shape
    _refuse(v.shape == k.shape, f"k {tuple(k.shape)} and v {tuple(v.shape)} differ in shape")
    cache = _cache(k_cache, v_cache, k)
    _refuse(k_cache.shape[2:] == k.shape[1:],
            f"caches of {tuple(k_cache.shape[2:])} (heads, dim) for keys of {tuple(k.shape[1:])}")
    _disjoint(k_cache, "k_cache")
    _disjoint(v_cache, "v_cache")
    batch = _batch(T, page_table, lens, starts, prefix_len, k)
    if table is not None:
        _table(table, k, D)
    if q is not None:
        _data(q, "q", 3, k)
        _refuse(q.shape[0] == T and q.shape[2] == D, f"q is {tuple(q.shape)}: [{T}, heads, {D}]")
    if q_out is not None:
        _refuse(q is not None, "q_out without q")
        _data(q_out, "q_out", 3, k)
        _refuse(q_out.shape == q.shape, f"q_out is {tuple(q_out.shape)}, not {tuple(q.shape)}")
        _disjoint(q_out, "q_out")
    with _On(stream, k, (k, v, k_cache, v_cache, page_table, lens, starts, table, q, q_out)) as s:
        if q is not None and q_out is None:
            q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        args = _AppendArgs(cache, batch, k.data_ptr(), v.data_ptr(), _ptr(q), _ptr(q_out), k.stride()[:2],
                           v.stride()[:2], (0, 0) if q is None else q.stride()[:2],
                           (0, 0) if q is None else q_out.stride()[:2], _ptr(table),
                           0 if table is None else table.stride(0), 0 if q is None else q.shape[1],
                           0 if table is None else table.shape[1], 0 if table is None else table.shape[0],
                           INTERLEAVED if interleaved else 0)
        _call("gts_append_kv", args, s)
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
    sees the prefix_len keys in prefix_pages (int32 [n], read once for the
    whole batch) and its sequence's own keys up to its own (lens counts them
    with the new ones).  Query head h reads key-value head h // (Hq / Hkv).
    scale defaults to D ** -0.5.  Without a prefix this is attention over a
    paged cache, one token a sequence or many.  A token without a key gives
    zeros and a log-sum of -inf.

    out [T, Hq, D] and lse (float32 [T, Hq], natural logarithm) receive the
    results if given; scratch (uint8, attention_scratch_bytes) is allocated if
    not.  Returns out."""
    _data(q, "q", 3)
    T, Hq, D = q.shape
    cache = _cache(k_cache, v_cache, q)
    Hkv = k_cache.shape[2]
    _refuse(k_cache.shape[3] == D, f"caches of head dim {k_cache.shape[3]} for queries of {D}")
    batch = _batch(T, page_table, lens, starts, prefix_len, q)
    n_prefix = 0
    if prefix_pages is not None:
        _index(prefix_pages, "prefix_pages", 1, q)
        _refuse(prefix_pages.stride(0) == 1 or prefix_pages.shape[0] <= 1, "prefix_pages is not contiguous")
        n_prefix = prefix_pages.shape[0]
    if out is not None:
        _data(out, "out", 3, q)
        _refuse(out.shape == q.shape, f"out is {tuple(out.shape)}, not {tuple(q.shape)}")
        _disjoint(out, "out")
    if lse is not None:
        _refuse(isinstance(lse, torch.Tensor) and lse.dtype == torch.float32 and lse.shape == (T, Hq)
                and lse.is_contiguous() and lse.device == q.device, f"lse is a contiguous float32 [{T}, {Hq}]")
    if scratch is not None:
        _refuse(isinstance(scratch, torch.Tensor) and scratch.dtype == torch.uint8 and scratch.is_contiguous()
                and scratch.device == q.device, "scratch is a contiguous uint8 tensor")
        _refuse(scratch.data_ptr() % 16 == 0, "scratch is not aligned to 16 bytes")
    need = _scratch_bytes(batch.batch, T, Hq, Hkv, D)
    with _On(stream, q, (q, k_cache, v_cache, page_table, lens, starts, prefix_pages, out, lse, scratch)) as s:
        if out is None:
            out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        if scratch is None and need:
            scratch = torch.empty(need, dtype=torch.uint8, device=q.device)
        args = _AttentionArgs(cache, batch, q.data_ptr(), out.data_ptr(), _ptr(lse), q.stride()[:2], out.stride()[:2],
                              _ptr(prefix_pages), n_prefix, Hq, D ** -0.5 if scale is None else scale, 0, _ptr(scratch),
                              0 if scratch is None else scratch.numel())
        _call("gts_shared_prefix_attention", args, s)
    return out
