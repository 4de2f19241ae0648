"""The C ABI of a decoder layer's operators without a GPU: the structures have the
header's layout, calls pack the same bytes, and arguments are refused with the documented
codes before anything is launched."""
import ctypes
import math
import os
import re
import struct
import subprocess

import pytest

from paper_2607_11262_amd import api, ops

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ARG, RANGE, SCRATCH = -1, -4, -6
FAKE = 4096  # never followed: every call here is refused first, or has nothing to do

STRUCTS = {"gts_norm_args": (ops._NormArgs, ops._pack_norm), "gts_norm_grad_args": (ops._NormGradArgs, ops._pack_norm_grad),
           "gts_matmul_args": (ops._MatmulArgs, ops._pack_matmul),
           "gts_linear_grad_args": (ops._LinearGradArgs, ops._pack_linear_grad),
           "gts_prompt_args": (ops._PromptArgs, ops._pack_prompt),
           "gts_prompt_grad_args": (ops._PromptGradArgs, ops._pack_prompt_grad)}


def test_structures_match_header(tmp_path):
    lines = []
    for name, (s, _) in STRUCTS.items():
        lines.append(f'printf("%zu\\n", sizeof({name}));')
        lines += [f'printf("%zu\\n", offsetof({name}, {f[0]}));' for f in s._fields_]
    src = tmp_path / "layout.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "gts_ops.h"\nint main(void) {\n' + "\n".join(lines)
                   + "\nreturn 0;\n}\n")
    subprocess.check_call(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(tmp_path / "layout")])
    got = [int(x) for x in subprocess.check_output([str(tmp_path / "layout")]).split()]
    want = []
    for s, _ in STRUCTS.values():
        want.append(ctypes.sizeof(s))
        want += [getattr(s, f[0]).offset for f in s._fields_]
    assert got == want


@pytest.mark.parametrize("name", STRUCTS)
def test_packed_values_match_structures(name):
    cls, pack = STRUCTS[name]
    values, flat, k = {}, [], 1
    for f, kind in cls._fields_:
        if issubclass(kind, ctypes.Array):
            values[f] = tuple(range(k, k + kind._length_))
            flat += values[f]
            k += kind._length_
        else:
            values[f] = 0.5 if kind is ctypes.c_float else k
            flat.append(values[f])
            k += 1
    assert pack(*flat) == bytes(cls(**values))


def test_constants_match_header():
    text = open(os.path.join(ROOT, "include", "gts_ops.h")).read()
    defined = {k: int(v) for k, v in re.findall(r"#define\s+GTS_(\w+)\s+(\d+)u", text)}
    assert (ops.A_COLUMNS, ops.B_COLUMNS, ops.CENTER, ops.CAUSAL) == tuple(
        defined[x] for x in ("MATMUL_A_COLUMNS", "MATMUL_B_COLUMNS", "NORM_CENTER", "PROMPT_CAUSAL"))
    for name, value in ops.ACTIVATIONS.items():
        assert defined["ACT_" + (name or "none").upper()] == value


def refused(name, args, code, word=""):
    rc = getattr(ops.lib(), name)(None if args is None else ctypes.byref(args), None)
    assert rc == code, (name, rc, api.lib().gts_last_error())
    assert word in api.lib().gts_last_error().decode()


def scratch_of(name, *sizes):
    n = ctypes.c_uint64()
    rc = getattr(ops.lib(), name)(*sizes, ctypes.byref(n))
    return rc if rc else n.value


def make(cls, **base):
    return lambda **kw: cls(**{**base, **kw})


norm = make(ops._NormArgs, x=FAKE, out=FAKE, x_stride=8, out_stride=8, rows=2, dim=8, eps=1e-5, dtype=ops.BF16)
norm_grad = make(ops._NormGradArgs, dy=FAKE, x=FAKE, mean=FAKE, rstd=FAKE, dx=FAKE, dweight=FAKE, dy_stride=8, x_stride=8,
                 dx_stride=8, rows=2, dim=8, dtype=ops.BF16, flags=1, scratch=FAKE, scratch_bytes=1 << 40)
matmul = make(ops._MatmulArgs, a=FAKE, b=FAKE, out=FAKE, a_stride=8, b_stride=8, out_stride=8, m=4, n=8, k=8, dtype=ops.BF16,
              scratch=FAKE, scratch_bytes=1 << 40)
linear_grad = make(ops._LinearGradArgs, dy=FAKE, preact=FAKE, gate=FAKE, dz=FAKE, dgate=FAKE, dbias=FAKE, dy_stride=8, m=4, n=8,
                   dtype=ops.BF16, activation=4, scratch=FAKE, scratch_bytes=1 << 40)
SIZES = dict(batch=1, tokens=4, q_heads=4, kv_heads=2, dim=16, dtype=ops.BF16, scale=0.25, flags=1)
prompt = make(ops._PromptArgs, q=FAKE, k=FAKE, v=FAKE, out=FAKE, starts=FAKE, **SIZES)
prompt_grad = make(ops._PromptGradArgs, dout=FAKE, q=FAKE, k=FAKE, v=FAKE, out=FAKE, lse=FAKE, starts=FAKE, dq=FAKE, dk=FAKE,
                   dv=FAKE, scratch=FAKE, scratch_bytes=1 << 40, **SIZES)


def test_norm_refusals():
    name = "gts_layer_norm"
    refused(name, None, ARG)
    for code, kw in ((ARG, dict(dtype=3)), (RANGE, dict(dim=0)), (RANGE, dict(dim=(1 << 24) + 1)), (RANGE, dict(rows=1 << 31)),
                     (ARG, dict(flags=2)), (ARG, dict(reserved=1)), (ARG, dict(eps=-1.0)), (ARG, dict(eps=math.inf)),
                     (ARG, dict(eps=math.nan)), (ARG, dict(x=None)), (ARG, dict(out=None))):
        refused(name, norm(**kw), code)
    refused(name, norm(rows=0, x=None, out=None), 0)
    name = "gts_layer_norm_backward"
    refused(name, None, ARG)
    for code, kw in ((ARG, dict(dtype=3)), (RANGE, dict(dim=0)), (ARG, dict(flags=2)), (ARG, dict(x=None)), (ARG, dict(dy=None)),
                     (ARG, dict(rstd=None)), (ARG, dict(mean=None)), (ARG, dict(scratch=FAKE + 4))):
        refused(name, norm_grad(**kw), code)
    refused(name, norm_grad(dx=None, dweight=None), 0)
    refused(name, norm_grad(rows=0, dweight=None), 0)
    need = scratch_of("gts_layer_norm_backward_scratch", 2, 8)
    if need:
        refused(name, norm_grad(scratch_bytes=need - 1), SCRATCH, str(need))
        refused(name, norm_grad(scratch=None), SCRATCH)
    assert ops.lib().gts_layer_norm_backward_scratch(2, 8, None) == ARG
    assert scratch_of("gts_layer_norm_backward_scratch", 2, 0) == RANGE


def test_product_refusals():
    name = "gts_matmul"
    refused(name, None, ARG)
    for code, kw in ((ARG, dict(dtype=3)), (ARG, dict(activation=5)), (ARG, dict(flags=4)), (RANGE, dict(n=(1 << 24) + 1)),
                     (RANGE, dict(m=1 << 31)), (RANGE, dict(k=1 << 31)), (RANGE, dict(m=(1 << 31) - 1, n=1 << 24)),
                     (ARG, dict(a=None)), (ARG, dict(b=None)), (ARG, dict(out=None))):
        refused(name, matmul(**kw), code)
    refused(name, matmul(m=0, a=None, out=None), 0)
    refused(name, matmul(n=0, a=None, out=None), 0)
    need = scratch_of("gts_matmul_scratch", 8, 8, 1 << 20)
    if need:
        refused(name, matmul(m=8, k=1 << 20, scratch_bytes=need - 1), SCRATCH, str(need))
        refused(name, matmul(m=8, k=1 << 20, scratch=None), SCRATCH)
    assert ops.lib().gts_matmul_scratch(2, 8, 4, None) == ARG
    assert scratch_of("gts_matmul_scratch", 1 << 31, 8, 4) == RANGE
    name = "gts_linear_backward"
    refused(name, None, ARG)
    for code, kw in ((ARG, dict(dtype=3)), (ARG, dict(activation=9)), (RANGE, dict(n=(1 << 24) + 1)), (ARG, dict(dy=None)),
                     (ARG, dict(preact=None)), (ARG, dict(preact=None, activation=0)), (SCRATCH, dict(scratch=None))):
        if code == SCRATCH and not scratch_of("gts_linear_backward_scratch", 4, 8):
            continue
        refused(name, linear_grad(**kw), code)
    for kw in (dict(n=0), dict(m=0, dbias=None), dict(dz=None, dgate=None, dbias=None)):
        refused(name, linear_grad(**kw), 0)
    for sizes in ((0, 0), (0, 8), (8, 0)):
        assert scratch_of("gts_linear_backward_scratch", *sizes) >= 0


@pytest.mark.parametrize("name,args", [("gts_prompt_attention", prompt), ("gts_prompt_attention_backward", prompt_grad)])
def test_prompt_refusals(name, args):
    refused(name, None, ARG)
    for code, kw in ((ARG, dict(dtype=3)), (RANGE, dict(dim=0)), (RANGE, dict(dim=257)), (RANGE, dict(q_heads=0)),
                     (RANGE, dict(kv_heads=0)), (RANGE, dict(q_heads=3)), (RANGE, dict(q_heads=65538)), (RANGE, dict(batch=0)),
                     (RANGE, dict(tokens=1 << 31)), (RANGE, dict(batch=1 << 31)), (ARG, dict(flags=2)),
                     (ARG, dict(scale=math.nan)), (ARG, dict(scale=math.inf)), (ARG, dict(starts=None, batch=2)),
                     (ARG, dict(q=None)), (ARG, dict(k=None)), (ARG, dict(v=None)), (ARG, dict(out=None))):
        refused(name, args(**kw), code)
    refused(name, args(tokens=0, q=None), 0)
    if name.endswith("backward"):
        for kw in (dict(dout=None), dict(lse=None), dict(dq=None), dict(dk=None), dict(dv=None)):
            refused(name, args(**kw), ARG)
        need = scratch_of("gts_prompt_attention_backward_scratch", 1, 4, 4, 2, 16)
        if need:
            refused(name, args(scratch_bytes=need - 1), SCRATCH, str(need))
            refused(name, args(scratch=None), SCRATCH)
        assert ops.lib().gts_prompt_attention_backward_scratch(1, 4, 4, 2, 16, None) == ARG
        assert scratch_of("gts_prompt_attention_backward_scratch", 1, 4, 4, 3, 16) == RANGE


def test_host_tensors_are_refused_with_a_gradient_too():
    torch = pytest.importorskip("torch")
    x = torch.zeros(4, 16, requires_grad=True)
    q = x.view(4, 1, 16)
    for f in (lambda: ops.layer_norm(x), lambda: ops.linear(x, x, activation="relu"), lambda: ops.prompt_attention(q, q, q)):
        with pytest.raises(ValueError, match="not on the GPU"):
            f()


def test_offsets_of_packing_are_native():
    assert struct.calcsize("=Q") == 8 and struct.calcsize("=I") == 4
