"""The operators' C ABI without a GPU: every entry point the header declares is
exported and bound, the structures have the header's layout, and arguments are
refused with the documented codes before anything is launched."""
import ctypes
import math
import os
import re
import subprocess

import pytest

from paper_2607_11262_amd import api, ops

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ARG, RANGE, SCRATCH = -1, -4, -6
FAKE = 4096  # never followed: every call here is refused first


def header():
    return open(os.path.join(ROOT, "include", "gts_ops.h")).read()


def test_exports_match_header():
    names = set(re.findall(r"^\s*int\s+(gts_\w+)\s*\(", header(), re.M))
    assert names == set(ops.EXPORTS)
    for n in names:
        assert hasattr(ops.lib(), n), n


def test_structures_match_header(tmp_path):
    """Sizes and offsets as a C compiler sees them."""
    pairs = {"gts_rotary_args": ops._RotaryArgs, "gts_kv_cache": ops._Cache, "gts_kv_batch": ops._Batch,
             "gts_append_args": ops._AppendArgs, "gts_attention_args": ops._AttentionArgs}
    lines = []
    for name, s in pairs.items():
        lines.append(f'printf("%zu\\n", sizeof({name}));')
        lines += [f'printf("%zu\\n", offsetof({name}, {f[0]}));' for f in s._fields_]
    src = tmp_path / "layout.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "gts_ops.h"\nint main(void) {\n' + "\n".join(lines)
                   + "\nreturn 0;\n}\n")
    subprocess.check_call(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(tmp_path / "layout")])
    got = [int(x) for x in subprocess.check_output([str(tmp_path / "layout")]).split()]
    want = []
    for s in pairs.values():
        want.append(ctypes.sizeof(s))
        want += [getattr(s, f[0]).offset for f in s._fields_]
    assert got == want


def test_packed_values_match_structures():
    """The calls pack the structures' values themselves: the same bytes as the
    ctypes structures, whose layout is the header's."""
    import struct

    def same(packer, cls, fields):
        flat = []
        for v in fields.values():
            flat += list(v) if isinstance(v, tuple) else [v]
        n = 0

        def fill(c):
            out = {}
            for f in c._fields_:
                if issubclass(f[1], ctypes.Structure):
                    out[f[0]] = f[1](**fill(f[1]))
                else:
                    out[f[0]] = fields[(c.__name__, f[0])]
            return out

        assert packer(*flat) == bytes(cls(**fill(cls))), cls.__name__
        assert struct.calcsize("=Q") == 8 and n == 0

    def values(*classes):
        """Distinct values, in the order of the members."""
        out, k = {}, 1
        for c in classes:
            for name, kind in c._fields_:
                if issubclass(kind, ctypes.Structure):
                    continue
                if issubclass(kind, ctypes.Array):
                    out[(c.__name__, name)] = tuple(range(k, k + kind._length_))
                    k += kind._length_
                else:
                    out[(c.__name__, name)] = 0.5 if kind is ctypes.c_float else k
                    k += 1
        return out

    same(ops._pack_rotary, ops._RotaryArgs, values(ops._RotaryArgs))
    same(ops._pack_append, ops._AppendArgs, values(ops._Cache, ops._Batch, ops._AppendArgs))
    same(ops._pack_attention, ops._AttentionArgs, values(ops._Cache, ops._Batch, ops._AttentionArgs))


def rotary_args(**kw):
    d = dict(x=FAKE, out=FAKE, positions=FAKE, table=FAKE, x_stride=(0, 64, 16), out_stride=(0, 64, 16), pos_stride=(0, 1),
             table_stride=16, batch=1, tokens=2, heads=4, dim=16, rot_dim=16, n_positions=8, dtype=ops.BF16, pos_bytes=8,
             flags=0, reserved=0)
    return ops._RotaryArgs(**{**d, **kw})


def cache(**kw):
    d = dict(k=FAKE, v=FAKE, k_stride=(128, 32, 16), v_stride=(128, 32, 16), n_pages=3, page=4, heads=2, dim=16,
             dtype=ops.BF16, reserved=0)
    return ops._Cache(**{**d, **kw})


def batch(**kw):
    d = dict(starts=FAKE, lens=FAKE, page_table=FAKE, table_stride=1, batch=2, tokens=2, max_pages=1, prefix_len=0)
    return ops._Batch(**{**d, **kw})


def append_args(c=None, b=None, **kw):
    d = dict(cache=c or cache(), batch=b or batch(), k=FAKE, v=FAKE, q=None, q_out=None, table=FAKE, table_stride=16,
             q_heads=0, rot_dim=16, n_positions=8, flags=0)
    return ops._AppendArgs(**{**d, **kw})


def attention_args(c=None, b=None, **kw):
    d = dict(cache=c or cache(), batch=b or batch(), q=FAKE, out=FAKE, lse=None, q_stride=(64, 16), out_stride=(64, 16),
             prefix_pages=None, n_prefix_pages=0, q_heads=4, scale=0.25, reserved=0, scratch=FAKE, scratch_bytes=1 << 40)
    return ops._AttentionArgs(**{**d, **kw})


def refused(name, args, code, word=""):
    rc = getattr(ops.lib(), name)(None if args is None else ctypes.byref(args), None)
    assert rc == code, (name, rc, api.lib().gts_last_error())
    assert word in api.lib().gts_last_error().decode()


def test_rotary_refusals():
    refused("gts_rotary", None, ARG)
    for code, kw in ((ARG, dict(dtype=3)), (RANGE, dict(dim=0)), (RANGE, dict(dim=15)), (RANGE, dict(dim=514)),
                     (RANGE, dict(rot_dim=0)), (RANGE, dict(rot_dim=3)), (RANGE, dict(rot_dim=18)),
                     (RANGE, dict(n_positions=0)), (ARG, dict(flags=4)), (ARG, dict(reserved=1)), (ARG, dict(pos_bytes=2)),
                     (RANGE, dict(heads=65536)), (RANGE, dict(batch=65536, tokens=65536)), (ARG, dict(x=None)),
                     (ARG, dict(out=None)), (ARG, dict(positions=None)), (ARG, dict(table=None))):
        refused("gts_rotary", rotary_args(**kw), code)
    for kw in (dict(batch=0), dict(tokens=0), dict(heads=0, x=None)):  # nothing to do
        refused("gts_rotary", rotary_args(**kw), 0)
    L, f = ops.lib(), (ctypes.c_double * 8)(*[1.0] * 8)
    assert L.gts_rotary_table(None, 8, 16, f, 1.0, None) == ARG
    assert L.gts_rotary_table(FAKE, 8, 16, None, 1.0, None) == ARG
    assert L.gts_rotary_table(FAKE, 0, 16, f, 1.0, None) == RANGE
    assert L.gts_rotary_table(FAKE, 8, 15, f, 1.0, None) == RANGE
    assert L.gts_rotary_table(FAKE, 8, 1024, f, 1.0, None) == RANGE
    assert L.gts_rotary_table(FAKE, 8, 16, f, math.inf, None) == ARG
    f[3] = math.nan
    assert L.gts_rotary_table(FAKE, 8, 16, f, 1.0, None) == ARG and b"freq[3]" in L.gts_last_error()


@pytest.mark.parametrize("name,make", [("gts_append_kv", append_args), ("gts_shared_prefix_attention", attention_args)])
def test_cache_and_batch_refusals(name, make):
    refused(name, None, ARG)
    for code, kw in ((ARG, dict(dtype=7)), (ARG, dict(reserved=1)), (RANGE, dict(heads=0)), (RANGE, dict(page=0)),
                     (RANGE, dict(page=6)), (RANGE, dict(page=1 << 17)), (RANGE, dict(n_pages=1 << 31)), (ARG, dict(k=None)),
                     (ARG, dict(v=None)), (RANGE, dict(dim=0)), (RANGE, dict(dim=1024))):
        refused(name, make(c=cache(**kw)), code)
    for code, kw in ((RANGE, dict(batch=0)), (RANGE, dict(batch=1 << 31)), (RANGE, dict(tokens=1 << 31)), (ARG, dict(lens=None)),
                     (ARG, dict(page_table=None)), (ARG, dict(starts=None, tokens=3)), (RANGE, dict(prefix_len=1 << 31))):
        refused(name, make(b=batch(**kw)), code)
    refused(name, make(b=batch(tokens=0)), 0)


def test_append_refusals():
    for code, kw in ((ARG, dict(flags=2)), (RANGE, dict(rot_dim=18)), (RANGE, dict(rot_dim=0)), (RANGE, dict(n_positions=0)),
                     (ARG, dict(k=None)), (ARG, dict(v=None)), (RANGE, dict(q=FAKE, q_out=FAKE)),
                     (ARG, dict(q=FAKE, q_heads=4))):
        refused("gts_append_kv", append_args(**kw), code)


def test_attention_refusals():
    for code, kw in ((RANGE, dict(q_heads=0)), (RANGE, dict(q_heads=3)), (RANGE, dict(q_heads=65538)), (ARG, dict(reserved=1)),
                     (ARG, dict(scale=math.nan)), (ARG, dict(scale=math.inf)), (ARG, dict(q=None)), (ARG, dict(out=None))):
        refused("gts_shared_prefix_attention", attention_args(**kw), code)
    name = "gts_shared_prefix_attention"
    refused(name, attention_args(b=batch(prefix_len=9)), ARG, "prefix_pages")
    refused(name, attention_args(b=batch(prefix_len=9), prefix_pages=FAKE, n_prefix_pages=2), RANGE, "2 prefix pages")
    refused(name, attention_args(b=batch(tokens=1 << 30)), RANGE)
    n = ctypes.c_uint64()
    L = ops.lib()
    assert L.gts_shared_prefix_attention_scratch(2, 2, 4, 2, 16, None) == ARG
    for sizes in ((0, 2, 4, 2, 16), (2, 2, 4, 3, 16), (2, 2, 4, 0, 16), (2, 2, 0, 2, 16), (2, 2, 4, 2, 0), (2, 2, 4, 2, 300)):
        assert L.gts_shared_prefix_attention_scratch(*sizes, ctypes.byref(n)) == RANGE, sizes
    assert L.gts_shared_prefix_attention_scratch(2, 2, 4, 2, 128, ctypes.byref(n)) == 0
    if n.value:
        a = attention_args(c=cache(dim=128), scratch_bytes=n.value - 1)
        refused(name, a, SCRATCH, str(n.value))
        refused(name, attention_args(c=cache(dim=128), scratch=None), SCRATCH)


def test_frequencies():
    f, m = ops.rotary_frequencies(8)
    assert f == [10000.0 ** (-i / 4) for i in range(4)] and m == 1.0
    g, _ = ops.rotary_frequencies(8, scaling={"kind": "linear", "factor": 4})
    assert g == [x / 4 for x in f]
    g, _ = ops.rotary_frequencies(8, scaling={"kind": "ntk", "factor": 16})
    assert g[0] == 1.0 and math.isclose(g[3], f[3] / 16) and f[1] / 16 < g[1] < f[1]
    f, _ = ops.rotary_frequencies(128)
    g, m = ops.rotary_frequencies(128, scaling={"kind": "ramp", "factor": 8, "original": 4096})
    assert math.isclose(m, 0.1 * math.log(8) + 1)
    turns = [4096 * x / (2 * math.pi) for x in f]
    for x, y, t in zip(f, g, turns):
        assert x / 8 * (1 - 1e-12) <= y <= x
        if t > 34:
            assert y == x
        if t < 0.9:
            assert math.isclose(y, x / 8)
    assert sorted(g, reverse=True) == g


@pytest.mark.parametrize("dim,original,factor", [(128, 4096, 8), (128, 32768, 4), (128, 65536, 4), (128, 131072, 4),
                                                 (64, 131072, 4), (16, 1 << 20, 2)])
def test_ramp_frequencies(dim, original, factor):
    """Every pair of the ramp, its end behind the last pair where that still
    turns more than once in the original positions."""
    base = 10000.0
    f, _ = ops.rotary_frequencies(dim)
    g, _ = ops.rotary_frequencies(dim, scaling={"kind": "ramp", "factor": factor, "original": original})
    # the number of the pair whose angle turns n times: original base^(-2 i / dim) = 2 pi n
    number = lambda n: dim / 2 * math.log(original / (2 * math.pi * n), base)  # noqa: E731
    lo, hi = max(math.floor(number(32)), 0), math.ceil(number(1))
    assert hi < dim
    for i, (x, y) in enumerate(zip(f, g)):
        t = min(max((i - lo) / (hi - lo), 0.0), 1.0)
        assert math.isclose(y, x * (1 - t) + x / factor * t, rel_tol=1e-12), i
        if original * x / (2 * math.pi) > 1.001 and i < hi:
            assert y > x / factor * (1 + 1e-9), i  # turns more than once: not divided in full


def test_append_flags():
    defined = dict(re.findall(r"#define\s+GTS_(\w+)\s+(\d+)u", header()))
    assert (ops.INTERLEAVED, ops.BACKWARD, ops.ZERO_REST) == tuple(
        int(defined[x]) for x in ("ROTARY_INTERLEAVED", "ROTARY_BACKWARD", "APPEND_ZERO_REST"))
    for flags in (0, 1, 4, 5):
        refused("gts_append_kv", append_args(b=batch(tokens=0), flags=flags), 0)  # nothing to do
        refused("gts_append_kv", append_args(flags=flags, q=FAKE, q_heads=4), ARG, "q_out")
    for flags in (2, 8, 6, 1 << 31):
        refused("gts_append_kv", append_args(flags=flags), ARG, "flag bits")
