"""The serving-step operators against their formulas in 64 bits: rotary
positions with their gradient, the paged append, and attention over the cache
with and without a shared prefix -- at the sizes, strides, masks and values where
they can go wrong."""
import pytest
import torch

import ops_reference as R
from paper_2607_11262_amd import api, ops

pytestmark = pytest.mark.gpu

BF, HF, F = torch.bfloat16, torch.float16, torch.float32


def randn(gen, *shape, dtype=F, scale=1.0):
    return (torch.randn(shape, generator=gen) * scale).to(dtype)


def gen(seed):
    return torch.Generator().manual_seed(seed)


def note(msg):
    print(f"[gpu] {msg}", flush=True)


def close(got, ref, bound, what):
    got = got.detach().cpu().double()
    bad = ~((got - ref).abs() <= bound) & ~((got == ref))
    if bad.any():
        i = tuple(int(x) for x in bad.nonzero()[0])
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} outside; at {i}: {got[i]} for {ref[i]} +- {bound[i]}")


# ---- rotary -----------------------------------------------------------------------

def test_table():
    for dim, scaling in ((2, None), (6, {"kind": "linear", "factor": 4}), (64, {"kind": "ntk", "factor": 8}),
                         (128, {"kind": "ramp", "factor": 16, "original": 4096}), (512, None)):
        note(f"table {dim} {scaling}")
        f, m = ops.rotary_frequencies(dim, scaling=scaling)
        t = ops.rotary_table(301, dim, scaling=scaling).cpu().double()
        angle = torch.arange(301, dtype=torch.float64)[:, None] * torch.tensor(f, dtype=torch.float64)
        ref = torch.cat((angle.cos(), angle.sin()), 1) * m
        assert ((t - ref).abs() <= 1.001 * R.E * ref.abs() + 1e-12).all()
    # far positions keep their angle: it is never rounded to 32 bits
    t = ops.rotary_table(1_000_003, 16).cpu().double()
    f, _ = ops.rotary_frequencies(16)
    angle = 1_000_002 * torch.tensor(f, dtype=torch.float64)
    assert ((t[-1] - torch.cat((angle.cos(), angle.sin()))).abs() < 1e-7).all()


ROTARY = [
    # type, B, S, H, D, R, interleaved
    (BF, 2, 5, 3, 128, 128, False), (BF, 2, 5, 3, 128, 128, True), (HF, 1, 1, 1, 2, 2, False),
    (HF, 3, 7, 5, 80, 40, False), (HF, 3, 7, 5, 80, 40, True), (F, 2, 3, 7, 80, 32, True), (F, 1, 33, 2, 96, 96, False),
    (BF, 1, 9, 2, 10, 6, False), (F, 2, 2, 3, 14, 10, True), (BF, 4, 1, 32, 128, 64, False), (HF, 1, 3, 2, 512, 512, True),
    (BF, 1, 129, 40, 64, 64, False), (F, 1, 2, 1, 512, 2, False),
]


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("dtype,B,S,H,D,rot,inter", ROTARY)
def test_rotary(dtype, B, S, H, D, rot, inter, backward):
    note(f"rotary {dtype} {B}x{S}x{H}x{D} rot {rot} interleaved {inter} backward {backward}")
    g = gen(B * 1000 + S * 10 + H + D)
    x = randn(g, B, S, H, D, dtype=dtype)
    pos = torch.randint(0, 5000, (B, S), generator=g)
    table = ops.rotary_table(5000, rot, scaling={"kind": "linear", "factor": 3})
    ref, size = R.rotate(x.double(), table.cpu().double()[pos], inter, backward)
    f = ops.rotary_backward if backward else ops.rotary
    y = f(x.cuda(), pos.cuda(), table, interleaved=inter)
    close(y, ref, R.rotation_bound(ref, size, dtype), "y")
    if rot < D:
        assert torch.equal(y[..., rot:].cpu(), x[..., rot:])
    # 32-bit positions, one row for every batch entry
    y1 = f(x.cuda(), pos[0].int().cuda(), table, interleaved=inter)
    ref, size = R.rotate(x.double(), table.cpu().double()[pos[:1]], inter, backward)
    close(y1, ref, R.rotation_bound(ref, size, dtype), "shared positions")


@pytest.mark.parametrize("inter", [False, True])
def test_rotary_layouts(inter):
    """Strides, alignments and orders other than a fresh tensor's."""
    g = gen(3)
    B, S, H, D = 2, 6, 4, 64
    table = ops.rotary_table(64, D)
    pos = torch.randint(0, 64, (B, S), generator=g).cuda()
    dense = randn(g, B, S, H, D, dtype=BF).cuda()
    ref = ops.rotary(dense, pos, table, interleaved=inter)
    heads_first = dense.transpose(1, 2).contiguous().transpose(1, 2)
    assert torch.equal(ops.rotary(heads_first, pos, table, interleaved=inter), ref)
    packed = torch.randn(B, S, H + 3, D, device="cuda").to(BF)
    packed[:, :, 1:H + 1] = dense
    before = packed.clone()
    view = packed[:, :, 1:H + 1]
    assert torch.equal(ops.rotary(view, pos, table, interleaved=inter), ref)
    # each alignment down to one element
    for shift in (1, 2, 4):
        wide = torch.zeros(B, S, H, D + 8, device="cuda", dtype=BF)
        off = wide[..., shift:shift + D]
        off.copy_(dense)
        assert torch.equal(ops.rotary(off, pos, table, interleaved=inter), ref), shift
    # a table and positions that are views
    t2 = torch.zeros(64, D + 1, device="cuda")[:, 1:]
    t2.copy_(table)
    p2 = torch.zeros(B, S, 2, device="cuda", dtype=torch.int64)[..., 1]
    p2.copy_(pos)
    assert torch.equal(ops.rotary(dense, p2, t2, interleaved=inter), ref)
    # in place, inside the packed tensor: nothing else changes
    out = ops.rotary(view, pos, table, interleaved=inter, out=view)
    assert out is view and torch.equal(view, ref)
    before[:, :, 1:H + 1] = ref
    assert torch.equal(packed, before)
    # an expanded input
    one = dense[:1].expand(B, S, H, D)
    assert torch.equal(ops.rotary(one, pos, table, interleaved=inter),
                       ops.rotary(one.contiguous(), pos, table, interleaved=inter))
    # [tokens, heads, D]
    flat = ops.rotary(dense.flatten(0, 1), pos.flatten(), table, interleaved=inter)
    assert torch.equal(flat, ref.flatten(0, 1))


def test_rotary_edges():
    table = ops.rotary_table(10, 8)
    x = torch.ones(4, 1, 12, device="cuda", dtype=BF)
    y = ops.rotary(x, torch.tensor([-1, 0, 9, 10], device="cuda"), table)
    assert y[[0, 3], :, :8].isnan().all() and not y[[1, 2]].isnan().any() and (y[..., 8:] == 1).all()
    assert torch.equal(y[1], x[1])  # position 0
    for shape in ((0, 3, 12), (3, 0, 12)):
        assert ops.rotary(x.new_zeros(shape), torch.zeros(shape[0], device="cuda", dtype=torch.int32), table).shape == shape
    # infinities and NaN stay in their own pairs
    x = torch.zeros(1, 2, 8, device="cuda")
    x[0, 0, 1], x[0, 1, 6] = float("inf"), float("nan")
    y = ops.rotary(x, torch.tensor([3], device="cuda"), table)
    hit = torch.zeros(1, 2, 8, dtype=torch.bool)
    hit[0, 0, [1, 5]] = hit[0, 1, [2, 6]] = True
    assert torch.equal(~y.isfinite().cpu(), hit)


@pytest.mark.parametrize("inter", [False, True])
def test_rotary_gradient(inter):
    """Against the formula's transposed rotation and against differences of the
    64-bit formula, through autograd, with broadcast inputs and gradients."""
    g = gen(8)
    B, S, H, D, rot = 3, 4, 5, 24, 16
    table = ops.rotary_table(100, rot, scaling={"kind": "ramp", "factor": 4, "original": 32})
    pos = torch.randint(0, 100, (B, S), generator=g)
    x, dy = randn(g, B, S, H, D), randn(g, B, S, H, D)
    leaf = x.cuda().requires_grad_()
    y = ops.rotary(leaf, pos.cuda(), table, interleaved=inter)
    (dx,) = torch.autograd.grad(y, leaf, dy.cuda())
    rows = table.cpu().double()[pos]
    ref, size = R.rotate(dy.double(), rows, inter, True)
    close(dx, ref, R.rotation_bound(ref, size, F), "dx")
    assert torch.equal(dx, ops.rotary_backward(dy.cuda(), pos.cuda(), table, interleaved=inter))
    # differences: the map is linear, so a step of 1 has no error of its own
    base, _ = R.rotate(x.double(), rows, inter)
    for _ in range(12):
        at = tuple(int(torch.randint(0, n, (1,), generator=g)) for n in x.shape)
        step = x.double().clone()
        step[at] += 1.0
        slope = ((R.rotate(step, rows, inter)[0] - base) * dy.double()).sum()
        assert abs(float(dx[at]) - float(slope)) <= 1e-6 * max(1.0, float(dy.abs().max()) * 2)
    # the same gradient everywhere (an expanded tensor of ones), one input for
    # all batch entries
    leaf = x[:1].cuda().requires_grad_()
    ops.rotary(leaf.expand(B, S, H, D), pos.cuda(), table, interleaved=inter).sum().backward()
    ref, size = R.rotate(torch.ones(B, S, H, D, dtype=torch.float64), rows, inter, True)
    close(leaf.grad, ref.sum(0, keepdim=True), 4 * R.rotation_bound(ref, size, F).sum(0, keepdim=True) + 1e-6, "broadcast")
    with torch.no_grad():
        assert not ops.rotary(leaf, pos[:1].cuda(), table).requires_grad


def test_gradient_of_the_gradient():
    """d/d(dy) of the gradient is the rotation; out has no gradient."""
    g = gen(18)
    table = ops.rotary_table(50, 12)
    pos = torch.arange(4, device="cuda")
    x, dy, z = (randn(g, 4, 3, 16).cuda() for _ in range(3))
    leaf, dleaf = x.clone().requires_grad_(), dy.clone().requires_grad_()
    (dx,) = torch.autograd.grad(ops.rotary(leaf, pos, table, interleaved=True), leaf, dleaf, create_graph=True)
    (ddy,) = torch.autograd.grad(dx, dleaf, z)
    assert torch.equal(ddy, ops.rotary(z, pos, table, interleaved=True))
    (dx,) = torch.autograd.grad(ops.rotary_backward(dleaf, pos, table), dleaf, z)
    assert torch.equal(dx, ops.rotary(z, pos, table))
    for f in (ops.rotary, ops.rotary_backward):
        with pytest.raises(ValueError, match="gradient"):
            f(leaf, pos, table, out=torch.empty_like(x))
        with torch.no_grad():
            assert torch.equal(f(leaf, pos, table, out=torch.empty_like(x)), f(x, pos, table))


def test_serving_operators_refuse_gradients():
    g = gen(19)
    kc, vc = (x.cuda() for x in cache(g, 2, 16, 2, 64, BF))
    q, k, v = (randn(g, 1, h, 64, dtype=BF).cuda() for h in (4, 2, 2))
    pages, lens = torch.tensor([[1]], device="cuda", dtype=torch.int32), torch.tensor([3], device="cuda", dtype=torch.int32)
    before = kc.clone(), vc.clone()
    for at in range(3):
        x = [t.clone().requires_grad_(i == at) for i, t in enumerate((q, k, v))]
        with pytest.raises(ValueError, match="gradient"):
            ops.append_kv(x[1], x[2], kc, vc, pages, lens, q=x[0])
    with pytest.raises(ValueError, match="gradient"):
        ops.shared_prefix_attention(q.clone().requires_grad_(), kc, vc, pages, lens)
    assert torch.equal(kc, before[0]) and torch.equal(vc, before[1])
    with torch.no_grad():
        out = ops.shared_prefix_attention(q.clone().requires_grad_(), kc, vc, pages, lens)
    assert torch.equal(out, ops.shared_prefix_attention(q, kc, vc, pages, lens))


# ---- append -----------------------------------------------------------------------

def cache(g, n_pages, page, H, D, dtype, heads_first=False, fill=None):
    shape = (n_pages, H, page, D) if heads_first else (n_pages, page, H, D)
    pair = [randn(g, *shape, dtype=dtype) if fill is None else torch.full(shape, fill, dtype=dtype) for _ in range(2)]
    return [x.transpose(1, 2) if heads_first else x for x in pair]


def on_gpu(t):
    """A copy with the same strides."""
    out = torch.empty_strided(t.shape, t.stride(), dtype=t.dtype, device="cuda")
    return out.copy_(t)


APPEND = [
    # type, Hq, Hkv, D, rot, page, counts, lens, prefix, interleaved, heads_first
    (BF, 32, 8, 128, 128, 64, None, [1, 64, 65, 200], 0, False, False),
    (BF, 4, 4, 64, 32, 16, [0, 3, 1, 20, 0], [5, 3, 17, 40, 0], 1000, True, True),
    (HF, 9, 3, 80, 40, 16, [2, 2, 5], [2, 33, 5], 77, True, False),
    (F, 2, 1, 10, 6, 1, [1, 4], [1, 9], 3, False, False),
    (HF, 6, 2, 256, 256, 256, [300], [300], 0, False, True),
    (BF, 1, 1, 2, 2, 8, [1] * 70, list(range(1, 71)), 5, False, False),
    # fewer own keys than new tokens: the first ones have no place
    (BF, 2, 2, 16, 16, 4, [5, 2], [3, 0], 9, False, False),
]


@pytest.mark.parametrize("dtype,Hq,Hkv,D,rot,page,counts,lens,prefix,inter,heads_first", APPEND)
def test_append(dtype, Hq, Hkv, D, rot, page, counts, lens, prefix, inter, heads_first):
    note(f"append {dtype} {Hq}/{Hkv}x{D} rot {rot} page {page} counts {counts and counts[:6]} lens {lens[:6]}")
    g = gen(D + len(lens))
    B = len(lens)
    n = [1] * B if counts is None else counts
    T = sum(n)
    max_pages = max(-(-m // page) for m in lens) + 1
    n_pages = B * max_pages + 3
    kc, vc = cache(g, n_pages, page, Hkv, D, dtype, heads_first)
    table_pages = torch.randperm(n_pages, generator=g)[:B * max_pages].view(B, max_pages).int()
    k, v, q = (randn(g, T, h, D, dtype=dtype) for h in (Hkv, Hkv, Hq))
    starts = None if counts is None else torch.tensor([0] + counts).cumsum(0).int()
    tab = ops.rotary_table(prefix + max(lens) + 1, rot)
    kg, vg = on_gpu(kc), on_gpu(vc)
    qo = torch.full((T, Hq, D), 7.0, dtype=dtype, device="cuda")
    got = ops.append_kv(k.cuda(), v.cuda(), kg, vg, table_pages.cuda(), torch.tensor(lens).int().cuda(),
                        starts=None if starts is None else starts.cuda(), table=tab, interleaved=inter, prefix_len=prefix,
                        q=q.cuda(), q_out=qo)
    assert got is qo
    rk, rv, rq = kc.double().clone(), vc.clone(), torch.full((T, Hq, D), 7.0, dtype=torch.float64)
    bk, bq = torch.zeros_like(rk), torch.zeros_like(rq)
    for b, (first, cnt) in enumerate(R.own_counts(B, T, starts)):
        for i in range(cnt):
            j = lens[b] - cnt + i
            if j < 0:
                continue
            row = tab.cpu().double()[prefix + j]
            p, s = int(table_pages[b, j // page]), j % page
            y, size = R.rotate(k[first + i].double(), row, inter)
            rk[p, s], bk[p, s] = y, R.rotation_bound(y, size, dtype)
            rv[p, s] = v[first + i]
            y, size = R.rotate(q[first + i].double(), row, inter)
            rq[first + i], bq[first + i] = y, R.rotation_bound(y, size, dtype)
    close(kg, rk, bk, "k_cache")
    assert torch.equal(vg.cpu(), rv)
    close(qo, rq, bq, "q")


def test_large_calls_agree_with_small_ones():
    """From 2^19 units (rotary) and 64 MB (append) on a thread takes two units:
    the same bits as calls of a part each, tokens that end inside a workgroup."""
    g = torch.Generator(device="cuda").manual_seed(6)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda", dtype=BF)  # noqa: E731
    x, tab = rnd(70001, 1, 128), ops.rotary_table(70001, 96)
    pos = torch.randperm(70001, generator=g, device="cuda")
    for inter in (False, True):
        big = ops.rotary(x, pos, tab, interleaved=inter)
        parts = [ops.rotary(x[i:i + 30000], pos[i:i + 30000], tab, interleaved=inter) for i in range(0, 70001, 30000)]
        note(f"large rotary, interleaved {inter}")
        assert torch.equal(big, torch.cat(parts))
    T, H, D, page = 17003, 5, 128, 64
    k, v, q = rnd(T, H, D), rnd(T, H, D), rnd(T, 9, D)
    counts = [5000, 1, 12002]
    starts = torch.tensor([0] + counts).cumsum(0).int().cuda()
    lens = torch.tensor(counts).int().cuda()
    pages = torch.randperm(3 * 190, generator=g, device="cuda").int().view(3, 190)
    caches = [[torch.zeros(3 * 190, page, H, D, device="cuda", dtype=BF) for _ in range(2)] for _ in range(2)]
    a = ops.append_kv(k, v, *caches[0], pages, lens, starts=starts, table=tab, q=q)
    out = []
    for b in range(3):
        i, j = int(starts[b]), int(starts[b + 1])
        for m in range(i, j, 4000):
            n = min(m + 4000, j)
            out.append(ops.append_kv(k[m:n], v[m:n], *caches[1], pages[b:b + 1],
                                     torch.tensor([n - i], device="cuda", dtype=torch.int32), table=tab, q=q[m:n]))
    note("large append")
    assert torch.equal(a, torch.cat(out))
    assert torch.equal(caches[0][0], caches[1][0]) and torch.equal(caches[0][1], caches[1][1])


def test_append_without_rotation_and_bad_pages():
    g = gen(1)
    kc, vc = (x.cuda() for x in cache(g, 4, 4, 2, 8, BF))
    k0, v0 = kc.clone(), vc.clone()
    k, v = randn(g, 4, 2, 8, dtype=BF).cuda(), randn(g, 4, 2, 8, dtype=BF).cuda()
    # page numbers outside the cache, and a key past the table: written nowhere
    pages = torch.tensor([[2], [-1], [4], [0]], device="cuda", dtype=torch.int32)
    lens = torch.tensor([3, 1, 1, 5], device="cuda", dtype=torch.int32)
    assert ops.append_kv(k, v, kc, vc, pages, lens) is None
    k0[2, 2], v0[2, 2] = k[0], v[0]
    assert torch.equal(kc, k0) and torch.equal(vc, v0)
    # a position past the rotary table: NaN, visibly
    tab = ops.rotary_table(2, 8)
    q = randn(g, 1, 4, 8, dtype=BF).cuda()
    r = ops.append_kv(k[:1], v[:1], kc, vc, pages[:1], lens[:1], table=tab, q=q)
    assert r.isnan().all() and kc[2, 2].isnan().all() and torch.equal(vc[2, 2], v[0])
    # tokens of no sequence, and no tokens at all
    starts = torch.tensor([0, 1, 1], device="cuda", dtype=torch.int32)
    kc.copy_(k0)
    ops.append_kv(k, v, kc, vc, pages[:2], lens[:2], starts=starts)
    k0[2, 2] = k[0]
    assert torch.equal(kc, k0)
    ops.append_kv(k[:0], v[:0], kc, vc, pages[:2], lens[:2], starts=starts)
    # queries in place
    q2 = q.clone()
    tab = ops.rotary_table(16, 4)
    assert ops.append_kv(k[:1], v[:1], kc, vc, pages[:1], lens[:1], table=tab, q=q2, q_out=q2) is q2
    assert torch.equal(q2, ops.rotary(q, lens[:1] - 1, tab))


# ---- attention --------------------------------------------------------------------

def attention_case(dtype, Hq, Hkv, D, page, counts, lens, prefix, heads_first=False, seed=0, fill=float("nan"), scale=None,
                   size=1.0, spare_tokens=0, drop_pages=()):
    """A batch over a cache whose unused slots hold `fill`, kernels against
    the formula."""
    g = gen(seed + D + len(lens))
    B = len(lens)
    n = [1] * B if counts is None else counts
    T = sum(n) + spare_tokens
    own_pages = [max(-(-m // page), 0) for m in lens]
    max_pages = max(own_pages + [1])
    n_prefix = -(-prefix // page)
    n_pages = n_prefix + sum(own_pages) + 2
    kc, vc = cache(g, n_pages, page, Hkv, D, dtype, heads_first, fill)
    order = torch.randperm(n_pages, generator=g).tolist()
    shared = order[:n_prefix]
    table = torch.full((B, max_pages), -7, dtype=torch.int32)
    at = n_prefix
    for b, c in enumerate(own_pages):
        table[b, :c] = torch.tensor(order[at:at + c], dtype=torch.int32)
        at += c
    for where, m in [(shared, prefix)] + [(table[b].tolist(), lens[b]) for b in range(B)]:
        for j in range(m):
            kc[where[j // page], j % page] = randn(g, Hkv, D, dtype=dtype, scale=size)
            vc[where[j // page], j % page] = randn(g, Hkv, D, dtype=dtype)
    for b, i in drop_pages:
        table[b, i] = -1
    q = randn(g, T, Hq, D, dtype=dtype, scale=size)
    starts = None if counts is None else torch.tensor([0] + counts).cumsum(0).int()
    lens_t = torch.tensor(lens).int()
    shared_t = torch.tensor(shared).int() if n_prefix else None
    ref = R.attention(q, kc, vc, table, lens_t, starts, shared_t, prefix, scale)
    lse = torch.full((T, Hq), 3.0, device="cuda")
    out = ops.shared_prefix_attention(q.cuda(), on_gpu(kc), on_gpu(vc), table.cuda(), lens_t.cuda(),
                                      starts=None if starts is None else starts.cuda(),
                                      prefix_pages=None if shared_t is None else shared_t.cuda(), prefix_len=prefix,
                                      scale=scale, lse=lse, out=torch.full_like(q.cuda(), 5.0))
    close(out, ref[0], ref[2], "out")
    close(lse, ref[1], ref[3], "lse")
    return out


ATTENTION = {
    "one key": (BF, 4, 2, 128, 64, None, [1], 0),
    "one key of a prefix": (BF, 4, 2, 128, 64, None, [0], 1),
    "decode": (BF, 32, 8, 128, 64, None, [1, 63, 64, 65, 127, 128, 129, 300], 0),
    "decode, prefix": (BF, 8, 2, 128, 64, None, [5, 0, 200, 64], 333),
    "decode, prefix of whole tiles": (BF, 4, 1, 128, 128, None, [128, 256], 256),
    "decode float16": (HF, 14, 2, 96, 16, None, [7, 99, 200], 70),
    "drafts": (BF, 14, 2, 96, 16, [1, 6, 3, 0, 5], [1, 6, 150, 9, 131], 100),
    "drafts, heads first": (HF, 8, 8, 64, 32, [4, 4, 4], [4, 40, 133], 65),
    "prompts": (BF, 4, 2, 64, 64, [70, 1, 130], [70, 1, 130], 200),
    "prompts without a prefix": (HF, 5, 1, 128, 16, [33, 129], [40, 260], 0),
    "chunk of a prompt": (BF, 2, 1, 128, 64, [150], [400], 0),
    "many heads": (BF, 64, 1, 64, 16, None, [33, 90], 40),
    "large head": (BF, 8, 2, 256, 32, [3, 1], [70, 200], 130),
    "24 rows of a large head": (BF, 8, 1, 256, 32, [3, 1], [70, 200], 130),
    "prompts of a large head": (HF, 4, 1, 256, 16, [40, 33], [60, 40], 70),
    "32 rows": (BF, 8, 1, 128, 16, [4, 3], [90, 75], 300),
    "64 rows": (HF, 16, 2, 128, 16, [3, 2, 4], [90, 75, 64], 100),
    "small head": (HF, 3, 3, 8, 8, [2, 1], [9, 30], 20),
    "head of 16": (BF, 6, 2, 16, 4, None, [3, 50, 5], 33),
    "odd head": (BF, 6, 2, 33, 4, None, [3, 50], 33),
    "32 bits": (F, 6, 3, 64, 16, [1, 4], [40, 70], 50),
    # the prefix dealt out: in pieces (8 workgroups a head, 3 segments), and whole
    # (2 workgroups a head, 3 segments), a piece of each left for the line
    "prefix in pieces": (BF, 64, 64, 64, 64, [150, 1, 149], [150, 20, 160], 1601),
    "prefix dealt out whole": (HF, 1024, 256, 8, 16, [50, 46], [50, 60], 100),
    "page of one": (BF, 2, 1, 64, 1, None, [70, 3], 9),
    "many sequences": (BF, 2, 1, 64, 16, None, [1 + (i * 37) % 90 for i in range(300)], 20),
    "empty rows": (BF, 4, 2, 64, 16, [3, 1, 2, 0], [1, 0, 0, 50], 0),
    "empty own part behind a prefix": (HF, 4, 2, 128, 16, [3, 1], [1, 0], 17),
    "nothing anywhere": (BF, 4, 2, 128, 16, None, [0, 0], 0),
}


@pytest.mark.parametrize("name", ATTENTION)
def test_attention(name):
    note(f"attention: {name}")
    attention_case(*ATTENTION[name], heads_first="heads first" in name)


FOUR_ROWS = [(HF, 64, 1100), (BF, 128, 2600), (HF, 256, 1300), (BF, 24, 700)]


@pytest.mark.parametrize("dtype,D,prefix", FOUR_ROWS)
def test_attention_of_4096_rows(dtype, D, prefix):
    """The join by four rows a wave: every width of head, more partial results of a
    row than lanes, rows without a key."""
    note(f"4096 rows of {D}, prefix {prefix}")
    attention_case(dtype, 64, 1, D, 16, None, [(i * 13) % 70 for i in range(64)], prefix)
    attention_case(dtype, 64, 16, D, 16, [30, 0, 4, 30], [20, 0, 9, 45], 0, seed=1)


@pytest.mark.parametrize("B", [1, 62, 63, 64, 65])
def test_attention_numbers_of_sequences(B):
    """Up to 63 sequences' bounds are looked up in one load; some are empty, and
    the last tokens are no one's."""
    counts = [(i * 7 + 1) % 4 for i in range(B)]
    note(f"{B} sequences")
    attention_case(BF, 4, 2, 64, 16, counts, [c + (i * 5) % 40 for i, c in enumerate(counts)], 20, spare_tokens=2)


def test_attention_masked_values():
    """What is masked never reaches a result, whatever it holds."""
    for fill in (float("inf"), float("-inf"), float("nan"), torch.finfo(BF).min):
        note(f"masked slots hold {fill}")
        attention_case(BF, 8, 2, 128, 16, [2, 1, 3], [5, 37, 140], 33, fill=fill)


def test_attention_later_tokens_hold_nothing_finite():
    """Keys and values behind a token's own are masked for it even when
    another row of the same tile sees them."""
    g = gen(4)
    for dtype in (BF, HF, F):
        kc, vc = (x.cuda() for x in cache(g, 4, 16, 1, 64, dtype))
        q = randn(g, 6, 4, 64, dtype=dtype).cuda()
        pages = torch.tensor([[1, 3]], device="cuda", dtype=torch.int32)
        lens = torch.tensor([20], device="cuda", dtype=torch.int32)
        starts = torch.tensor([0, 6], device="cuda", dtype=torch.int32)
        ref = ops.shared_prefix_attention(q, kc, vc, pages, lens, starts=starts)
        for bad in (float("nan"), float("inf"), float("-inf")):
            k1, v1 = kc.clone(), vc.clone()
            k1[3, 1], v1[3, 1] = bad, bad  # own key 17: token 3's
            out = ops.shared_prefix_attention(q, k1, v1, pages, lens, starts=starts)
            note(f"token 3's key and value hold {bad} {dtype}")
            assert torch.equal(out[:3], ref[:3]) and out[3:].isnan().all()
            k1 = kc.clone()
            out = ops.shared_prefix_attention(q, k1, v1, pages, lens, starts=starts)
            assert torch.equal(out[:3], ref[:3]) and not out[3:].isfinite().any()


def test_attention_values():
    """Scores that differ by hundreds, one sharp key, scales of either sign."""
    attention_case(BF, 4, 2, 128, 16, [2, 1], [90, 300], 150, size=8.0)
    attention_case(HF, 4, 2, 64, 16, None, [90, 300], 150, size=8.0, scale=0.5)
    attention_case(BF, 4, 2, 64, 16, None, [90, 130], 150, scale=-0.2)
    attention_case(BF, 4, 2, 64, 16, None, [90, 130], 150, scale=0.0)


def test_attention_missing_pages_and_spare_tokens():
    attention_case(BF, 4, 2, 128, 16, [2, 1], [90, 300], 40, drop_pages=((0, 0), (1, 3), (1, 10), (1, 18)), seed=5)
    attention_case(BF, 4, 2, 128, 16, None, [16], 0, drop_pages=((0, 0),))  # its only page
    # tokens of no sequence get zeros
    attention_case(HF, 4, 2, 64, 16, [2, 3], [90, 30], 40, spare_tokens=5)


@pytest.mark.parametrize("dtype,D", [(BF, 64), (F, 64), (HF, 33)])
def test_lengths_past_the_pages(dtype, D):
    """Keys that lens counts but no page can hold do not exist, however many."""
    g = gen(14)
    kc, vc = (x.cuda() for x in cache(g, 4, 16, 2, D, dtype))
    q = randn(g, 3, 4, D, dtype=dtype).cuda()
    pages = torch.tensor([[1, 3], [2, 0]], device="cuda", dtype=torch.int32)
    starts = torch.tensor([0, 2, 3], device="cuda", dtype=torch.int32)
    lens = torch.tensor([34, 32], device="cuda", dtype=torch.int32)  # all see 32 keys
    ref = ops.shared_prefix_attention(q, kc, vc, pages, lens, starts=starts)
    far = torch.tensor([2 ** 31 - 1, 1 << 30], device="cuda", dtype=torch.int32)
    note(f"{far.tolist()} keys in two pages of 16 {dtype} {D}")
    assert torch.equal(ops.shared_prefix_attention(q, kc, vc, pages, far, starts=starts), ref)


def test_attention_one_long_prompt():
    """2100 tokens of one sequence (33 segments of 128 rows for the first of
    two heads' groups): the places of segments far down the line."""
    attention_case(BF, 2, 1, 16, 64, [2100, 1], [2100, 5], 70)


def test_attention_long_against_rows_of_parts():
    """70001 own keys behind 40003 shared ones: the join of many parts; checked
    on the GPU in 64 bits."""
    g = torch.Generator(device="cuda").manual_seed(2)
    D, H, page, P, L = 128, 2, 64, 40003, 70001
    n = -(-P // page) + -(-L // page)
    kc, vc = (torch.randn(n, page, H, D, generator=g, device="cuda", dtype=BF) for _ in range(2))
    order = torch.randperm(n, generator=g, device="cuda").int()
    shared, own = order[:-(-P // page)], order[-(-P // page):][None].contiguous()
    q = torch.randn(2, 4, D, generator=g, device="cuda", dtype=BF) * 3
    starts = torch.tensor([0, 2], device="cuda", dtype=torch.int32)
    lens = torch.tensor([L], device="cuda", dtype=torch.int32)
    out = ops.shared_prefix_attention(q, kc, vc, own, lens, starts=starts, prefix_pages=shared, prefix_len=P)
    k = torch.cat((kc[shared.long()].flatten(0, 1)[:P], kc[own[0].long()].flatten(0, 1)[:L])).double()
    v = torch.cat((vc[shared.long()].flatten(0, 1)[:P], vc[own[0].long()].flatten(0, 1)[:L])).double()
    for i in range(2):
        for h in range(4):
            keys = P + L - 1 + i
            s = k[:keys, h // 2] @ q[i, h].double() * D ** -0.5
            w = s.softmax(0)
            ref, spread = w @ v[:keys, h // 2], w @ v[:keys, h // 2].abs()
            d = (D + 6) * R.E * (k[:keys, h // 2].abs() @ q[i, h].double().abs() * D ** -0.5).max()
            assert ((out[i, h].double() - ref).abs() <= (2.01 * R.U[BF] + 2 * d + keys / 8 * R.E) * spread).all()


def test_offsets_past_32_bits():
    """Pages whose elements lie past 2^32 bytes and 2^31 elements: append and
    attention agree with a small cache."""
    g = gen(9)
    page, H, D = 16, 2, 64
    far = (1 << 31) // 2 + 1024  # elements between pages: page 3 starts past 2^31
    buf = [torch.zeros(3 * far + page * H * D, dtype=BF, device="cuda") for _ in range(2)]
    kc, vc = (b.as_strided((4, page, H, D), (far, H * D, D, 1)) for b in buf)
    ks, vs = (torch.zeros(4, page, H, D, dtype=BF, device="cuda") for _ in range(2))
    pages = torch.tensor([[3, 0, 2, 1]], device="cuda", dtype=torch.int32)
    lens = torch.tensor([60], device="cuda", dtype=torch.int32)
    starts = torch.tensor([0, 60], device="cuda", dtype=torch.int32)
    k, v, q = (randn(g, 60, h, D, dtype=BF).cuda() for h in (H, H, 4))
    tab = ops.rotary_table(60, D)
    outs = []
    for a, b in ((kc, vc), (ks, vs)):
        qr = ops.append_kv(k, v, a, b, pages, lens, starts=starts, table=tab, q=q)
        outs.append(ops.shared_prefix_attention(qr, a, b, pages, lens, starts=starts))
    assert torch.equal(kc, ks) and torch.equal(vc, vs) and torch.equal(outs[0], outs[1])
    assert outs[0].isfinite().all() and (outs[0] != 0).any()


def step(state):
    q = ops.append_kv(state["k"], state["v"], state["kc"], state["vc"], state["pages"], state["lens"], table=state["tab"],
                      prefix_len=state["P"], q=state["q"])
    return ops.shared_prefix_attention(q, state["kc"], state["vc"], state["pages"], state["lens"],
                                       prefix_pages=state["shared"], prefix_len=state["P"])


def decode_state(B=6, P=200, seed=1):
    g = torch.Generator(device="cuda").manual_seed(seed)
    page, H, D, Hq = 16, 2, 128, 8
    n_prefix, per = -(-P // page), 8
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda", dtype=BF)  # noqa: E731
    return dict(P=P, kc=rnd(n_prefix + B * per, page, H, D), vc=rnd(n_prefix + B * per, page, H, D), k=rnd(B, H, D),
                v=rnd(B, H, D), q=rnd(B, Hq, D), tab=ops.rotary_table(400, D),
                shared=torch.arange(n_prefix, device="cuda", dtype=torch.int32),
                pages=(n_prefix + torch.arange(B * per, device="cuda", dtype=torch.int32)).view(B, per),
                lens=torch.arange(1, B + 1, device="cuda", dtype=torch.int32) * 15)


def test_decode_steps_in_a_graph():
    """The step captured once and replayed while the lengths grow, with eager
    work between the replays, against the eager step."""
    s = decode_state()
    step(s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(s)
    for i in range(4):
        s["lens"] += 1
        for x in ("q", "k", "v"):
            s[x].copy_(torch.randn_like(s[x]))
        graph.replay()
        torch.cuda.synchronize()
        kept = got.clone()
        eager = step(s)
        torch.cuda.synchronize()
        note(f"replay {i}")
        assert torch.equal(kept, eager)


def test_another_stream():
    """A step enqueued on a side stream, its inputs made and dropped on the
    current one; calls of two states interleaved on two streams."""
    a, b = decode_state(seed=1), decode_state(seed=2, P=0, B=9)
    ra, rb = step(a), step(b)
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    outs = []
    for _ in range(5):
        for s, st in ((a, s1), (b, s2)):
            st.wait_stream(torch.cuda.current_stream())
            q = ops.append_kv(s["k"].clone(), s["v"].clone(), s["kc"], s["vc"], s["pages"], s["lens"], table=s["tab"],
                              prefix_len=s["P"], q=s["q"].clone(), stream=st)
            with torch.cuda.stream(st):
                outs.append(ops.shared_prefix_attention(q, s["kc"], s["vc"], s["pages"], s["lens"],
                                                        prefix_pages=s["shared"], prefix_len=s["P"]))
    torch.cuda.synchronize()
    for i, o in enumerate(outs):
        assert torch.equal(o, rb if i % 2 else ra)


def test_repeated_calls_agree():
    """No atomics, no state between calls: the same bits each time, on a
    scratch that holds another call's."""
    s, t = decode_state(B=5, P=350), decode_state(B=3, P=30, seed=7)
    need = ops.attention_scratch_bytes(5, 5, 8, 2, 128)
    scratch = torch.full((need + 16,), 255, dtype=torch.uint8, device="cuda")
    first = None
    for _ in range(3):
        out = ops.shared_prefix_attention(s["q"], s["kc"], s["vc"], s["pages"], s["lens"], prefix_pages=s["shared"],
                                          prefix_len=s["P"], scratch=scratch)
        ops.shared_prefix_attention(t["q"], t["kc"], t["vc"], t["pages"], t["lens"], prefix_pages=t["shared"],
                                    prefix_len=t["P"], scratch=scratch)
        first = out if first is None else first
        assert torch.equal(out, first)


# ---- refusals ---------------------------------------------------------------------

def test_refusals():
    """Every refused call raises and launches nothing."""
    x = torch.zeros(2, 3, 4, 16, device="cuda", dtype=BF)
    pos = torch.zeros(3, device="cuda", dtype=torch.int64)
    tab = ops.rotary_table(8, 16)
    bad = [
        (ValueError, lambda: ops.rotary(x.cpu(), pos, tab)),
        (ValueError, lambda: ops.rotary(x[..., ::2], pos, tab)),
        (ValueError, lambda: ops.rotary(x[0, 0], pos, tab)),
        (TypeError, lambda: ops.rotary(x.double(), pos, tab)),
        (TypeError, lambda: ops.rotary(x, pos.float(), tab)),
        (ValueError, lambda: ops.rotary(x, pos[:2], tab)),
        (ValueError, lambda: ops.rotary(x, pos, ops.rotary_table(8, 32))),
        (TypeError, lambda: ops.rotary(x, pos, tab.half())),
        (TypeError, lambda: ops.rotary(x, pos, tab, out=x.half())),
        (ValueError, lambda: ops.rotary(x, pos, tab, out=x[:1].expand_as(x))),
        (api.GtsError, lambda: ops.rotary(x[..., :15], pos, tab[:, :14])),   # odd head
        (api.GtsError, lambda: ops.rotary(x, pos, tab[:, :15])),             # odd part
        (ValueError, lambda: ops.rotary_table(8, 7)),
        (ValueError, lambda: ops.rotary_table(0, 8)),
        (api.GtsError, lambda: ops.rotary_table(8, 514)),
        (ValueError, lambda: ops.rotary_table(8, 8, scaling={"kind": "other"})),
        (ValueError, lambda: ops.rotary_table(8, 8, scaling={"kind": "linear", "factor": 0.5})),
        (ValueError, lambda: ops.rotary_table(8, 8, scaling={"kind": "ramp", "factor": 2})),
        (ValueError, lambda: ops.rotary_table(8, 8, scaling={"kind": "ntk", "factor": 2, "original": 8})),
    ]
    kc, vc = (torch.zeros(3, 4, 2, 16, device="cuda", dtype=BF) for _ in range(2))
    k, q = torch.zeros(2, 2, 16, device="cuda", dtype=BF), torch.zeros(2, 4, 16, device="cuda", dtype=BF)
    pages, lens = torch.zeros(2, 1, device="cuda", dtype=torch.int32), torch.ones(2, device="cuda", dtype=torch.int32)
    starts = torch.tensor([0, 1, 2], device="cuda", dtype=torch.int32)
    odd = torch.zeros(3, 5, 2, 16, device="cuda", dtype=BF)
    for f in (lambda q, kc, vc, p, n, **kw: ops.append_kv(k, k, kc, vc, p, n, **{**kw, **({} if q is None else {"q": q})}),
              ops.shared_prefix_attention):
        bad += [
            (TypeError, lambda f=f: f(q, kc.half(), vc, pages, lens)),
            (ValueError, lambda f=f: f(q, kc, vc[:2], pages, lens)),
            (ValueError, lambda f=f: f(q, kc[..., :8], vc[..., :8], pages, lens)),
            (TypeError, lambda f=f: f(q, kc, vc, pages.long(), lens)),
            (TypeError, lambda f=f: f(q, kc, vc, pages, lens.long())),
            (ValueError, lambda f=f: f(q, kc, vc, pages[:1], lens)),
            (ValueError, lambda f=f: f(q, kc, vc, pages.cpu(), lens)),
            (ValueError, lambda f=f: f(q, kc, vc, pages, lens, starts=starts[:2])),
            (ValueError, lambda f=f: f(q, kc, vc, pages, lens, prefix_len=-1)),
            (api.GtsError, lambda f=f: f(q, odd, odd, pages, lens)),                       # pages of 5
            (api.GtsError, lambda f=f: f(q, kc, vc, pages.expand(2, 1)[:0], lens[:0])),    # no sequence
        ]
    bad += [
        (api.GtsError, lambda: ops.append_kv(k, k, kc, vc, torch.cat([pages, pages[:1]]), torch.cat([lens, lens[:1]]))),
        (ValueError, lambda: ops.append_kv(k, k[:1], kc, vc, pages, lens)),
        (ValueError, lambda: ops.append_kv(k, k, kc, vc, pages, lens, q_out=q)),
        (ValueError, lambda: ops.append_kv(k, k, kc[:1].expand_as(kc), vc, pages, lens)),
        (api.GtsError, lambda: ops.shared_prefix_attention(q[:, :3], kc, vc, pages, lens)),  # 3 heads over 2
        (api.GtsError, lambda: ops.shared_prefix_attention(q, kc, vc, pages, lens, prefix_len=1)),
        (api.GtsError, lambda: ops.shared_prefix_attention(q, kc, vc, pages, lens, prefix_pages=lens, prefix_len=9)),
        (api.GtsError, lambda: ops.shared_prefix_attention(q, kc, vc, pages, lens, scale=float("nan"))),
        (ValueError, lambda: ops.shared_prefix_attention(q, kc, vc, pages, lens, lse=torch.zeros(2, 3, device="cuda"))),
        (ValueError, lambda: ops.shared_prefix_attention(q, kc, vc, pages, lens, out=q[:1])),
    ]
    for i, (kind, f) in enumerate(bad):
        with pytest.raises(kind):
            f()
            note(f"refusal {i} was not refused")
    torch.cuda.synchronize()
    assert (kc == 0).all()


def test_decode_step_example():
    """The example's step against the formula, with and without a prefix, and
    its two times."""
    import os
    import sys
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import decode_step
    for prefix in (0, 70):
        d = decode_step.Decode([90, 130, 201], prefix, q_heads=8, kv_heads=2)
        us, out = decode_step.measure(d, 3)
        note(f"example, prefix {prefix}: {us:.1f} us a step")
        ref = d.step()
        torch.cuda.synchronize()
        assert torch.equal(out, ref) and us > 0
        rows = d.table.cpu().double()[prefix + d.lens.cpu().long() - 1]
        q, _ = R.rotate(d.q.cpu().double(), rows)
        q16 = ops.rotary(d.q, (prefix + d.lens - 1), d.table).cpu()
        assert ((q16.double() - q).abs() <= 2 ** -8 * q.abs() + 1e-6).all()
        want = R.attention(q16, d.k_cache.cpu(), d.v_cache.cpu(), d.pages.cpu(), d.lens.cpu(), None,
                           None if not prefix else d.prefix_pages.cpu(), prefix)
        close(out, want[0], want[2], "out")
    r = decode_step.main(["--batch", "3", "--kv-max", "1024", "--prefix", "128", "--steps", "2"])
    assert r["simulated"] > 0 and r["out"].isfinite().all()


def test_append_returns_zeros_for_tokens_without_a_place():
    """Queries of tokens outside every sequence, or with fewer own keys than new
    tokens, in a result that the call allocates: zeros, whatever the memory
    held, and so the same attention behind a prefix each time."""
    g = gen(23)
    D, page, P, counts, lens, spare = 64, 16, 20, [5, 0, 3], [2, 0, 9], 4
    kc, vc = (x.cuda() for x in cache(g, 6, page, 2, D, BF))
    T = sum(counts) + spare
    k, v, q = (randn(g, T, h, D, dtype=BF).cuda() for h in (2, 2, 4))
    pages = torch.tensor([[0], [1], [2]], device="cuda", dtype=torch.int32)
    shared = torch.tensor([3, 4], device="cuda", dtype=torch.int32)
    starts = torch.tensor([0, 5, 5, 8], device="cuda", dtype=torch.int32)
    lens_t = torch.tensor(lens, device="cuda", dtype=torch.int32)
    placed = torch.tensor([False] * 3 + [True] * 5 + [False] * spare, device="cuda")
    tab = ops.rotary_table(64, D)
    for inter in (False, True):
        for table in (tab, None):
            given = torch.full_like(q, 7.0)
            ops.append_kv(k, v, kc, vc, pages, lens_t, starts=starts, table=table, interleaved=inter, prefix_len=P, q=q,
                          q_out=given)
            outs = []
            for fill in (float("nan"), 3.0):
                for _ in range(4):  # blocks of the size of q, to be taken again
                    torch.full_like(q, fill)
                got = ops.append_kv(k, v, kc, vc, pages, lens_t, starts=starts, table=table, interleaved=inter,
                                    prefix_len=P, q=q)
                assert (got[~placed] == 0).all() and torch.equal(got[placed], given[placed])
                outs.append(ops.shared_prefix_attention(got, kc, vc, pages, lens_t, starts=starts, prefix_pages=shared,
                                                        prefix_len=P))
            assert torch.equal(outs[0], outs[1]) and outs[0].isfinite().all()
            assert (given[~placed] == 7).all()  # what the caller hands in keeps its rows


@pytest.mark.parametrize("dtype,D,group,counts", [
    (BF, 64, 4, None), (HF, 128, 4, None), (BF, 256, 8, None), (BF, 128, 8, [3, 4, 2, 3]), (BF, 128, 4, [13, 12, 9, 10]),
    (HF, 256, 4, [13, 12, 9, 10]), (BF, 64, 4, [40, 33, 35, 37]), (HF, 128, 4, [40, 33, 35, 37]), (F, 64, 4, [3, 4, 2, 3]),
    (HF, 33, 4, None)])
@pytest.mark.parametrize("prefix", [0, 33, 150])
def test_attention_scores_of_minus_infinity(dtype, D, group, counts, prefix):
    """Keys whose score is -inf weigh nothing beside others; a row that has no
    other keys is 0 / 0, unlike a row without a key, which is zeros."""
    note(f"-inf scores {dtype} {D} group {group} counts {counts} prefix {prefix}")
    g = gen(31)
    page, H = 16, 2
    lens = [70, 50, 150, 0]
    n = [1] * 4 if counts is None else counts
    T = sum(n)
    n_prefix, n_pages = -(-prefix // page), 40
    kc, vc = cache(g, n_pages, page, H, D, dtype)
    q = randn(g, T, group * H, D, dtype=dtype).abs() + 0.1
    order = torch.randperm(n_pages, generator=g).int()
    shared = order[:n_prefix]
    table = torch.full((4, 10), -1, dtype=torch.int32)
    at = n_prefix
    for b, m in enumerate(lens):
        c = -(-m // page)
        table[b, :c] = order[at:at + c]
        at += c
    starts = None if counts is None else torch.tensor([0] + counts).cumsum(0).int()
    # sequence 0: every key; 1: its first two pages (rows of its first tokens may see
    # no other); 2: a page in the middle; the prefix: all of it
    finite = table.clone()
    finite[0], finite[1, :2], finite[2, 4] = -1, -1, -1
    for b in range(4):
        for x in table[b][(finite[b] < 0) & (table[b] >= 0)].tolist():
            kc[x, :, :, 1] = -float("inf")
    for x in shared.tolist():
        kc[x, :, :, 0] = -float("inf")
    lens_t = torch.tensor(lens).int()
    # the same without those keys; the rows that have keys
    want = R.attention(q, kc, vc, finite, lens_t, starts, None, 0)
    ones = torch.zeros_like(kc), torch.ones_like(vc)
    has = R.attention(q, *ones, table, lens_t, starts, shared if prefix else None, prefix)[1] > -float("inf")
    lse = torch.full((T, group * H), 3.0, device="cuda")
    out = ops.shared_prefix_attention(q.cuda(), kc.cuda(), vc.cuda(), table.cuda(), lens_t.cuda(),
                                      starts=None if starts is None else starts.cuda(),
                                      prefix_pages=shared.cuda() if prefix else None, prefix_len=prefix, lse=lse)
    none = want[1] == -float("inf")
    assert (none & has).any() and (~none).any() and (has.all() if prefix else not has.all())
    close(lse, want[1], want[3], "lse")
    got = out.cpu()
    assert got[none & has].isnan().all() and (got[none & ~has] == 0).all()
    close(out[~none.cuda()], want[0][~none], want[2][~none], "out")


def test_tangents_are_refused():
    """Forward-mode derivatives, which no operator has, are refused and not
    dropped."""
    import torch.autograd.forward_ad as fw
    g = gen(41)
    table, pos = ops.rotary_table(50, 64), torch.arange(2, device="cuda")
    kc, vc = (x.cuda() for x in cache(g, 2, 16, 2, 64, F))
    q, k, v = (randn(g, 2, h, 64).cuda() for h in (4, 2, 2))
    pages, lens = torch.tensor([[1]], device="cuda", dtype=torch.int32), torch.tensor([3], device="cuda", dtype=torch.int32)
    before = kc.clone(), vc.clone()
    calls = [lambda t: ops.rotary(t(q), pos, table), lambda t: ops.rotary(q, pos, t(table)),
             lambda t: ops.rotary_backward(t(q), pos, table), lambda t: ops.rotary(q, pos, table, out=t(q.clone())),
             lambda t: ops.append_kv(t(k), v, kc, vc, pages, lens), lambda t: ops.append_kv(k, t(v), kc, vc, pages, lens),
             lambda t: ops.append_kv(k, v, t(kc), vc, pages, lens), lambda t: ops.append_kv(k, v, kc, vc, pages, lens, q=t(q)),
             lambda t: ops.append_kv(k, v, kc, vc, pages, lens, table=t(table)),
             lambda t: ops.shared_prefix_attention(t(q), kc, vc, pages, lens),
             lambda t: ops.shared_prefix_attention(q, kc, t(vc), pages, lens),
             lambda t: ops.shared_prefix_attention(q, kc, vc, pages, lens, out=t(q.clone()))]
    with fw.dual_level():
        for i, f in enumerate(calls):
            with pytest.raises(ValueError, match="tangent"):
                f(lambda x: fw.make_dual(x, torch.ones_like(x)))
                note(f"tangent {i} was not refused")
    assert torch.equal(kc, before[0]) and torch.equal(vc, before[1])
    with fw.dual_level():  # a level alone is no reason
        assert torch.equal(ops.rotary(q, pos, table), ops.rotary(q.clone(), pos, table))


def test_gradients_that_would_be_lost_are_refused():
    """A table has no gradient, and neither has what an operator writes to."""
    g = gen(42)
    table, pos = ops.rotary_table(50, 64), torch.arange(2, device="cuda")
    kc, vc = (x.cuda() for x in cache(g, 2, 16, 2, 64, F))
    q, k, v = (randn(g, 2, h, 64).cuda() for h in (4, 2, 2))
    pages, lens = torch.tensor([[1]], device="cuda", dtype=torch.int32), torch.tensor([3], device="cuda", dtype=torch.int32)
    leaf = lambda x: x.clone().requires_grad_()  # noqa: E731
    calls = [lambda: ops.rotary(q, pos, leaf(table)), lambda: ops.rotary(leaf(q), pos, leaf(table)),
             lambda: ops.rotary_backward(q, pos, leaf(table)), lambda: ops.rotary(q, pos, table, out=leaf(q)),
             lambda: ops.append_kv(k, v, kc, vc, pages, lens, table=leaf(table)),
             lambda: ops.append_kv(k, v, kc, vc, pages, lens, q=q, q_out=leaf(q)),
             lambda: ops.shared_prefix_attention(q, kc, vc, pages, lens, out=leaf(q)),
             lambda: ops.shared_prefix_attention(q, kc, vc, pages, lens, lse=leaf(q[..., 0].contiguous()))]
    for i, f in enumerate(calls):
        with pytest.raises(ValueError, match="gradient"):
            f()
            note(f"gradient {i} was not refused")
        with torch.no_grad():
            f()


def test_writes_are_known_to_autograd():
    """A tensor that an earlier operation saved and one of the operators has
    since written to is an error in that operation's backward, as with torch's
    own in-place operations."""
    g = gen(43)
    table, pos = ops.rotary_table(50, 64), torch.arange(2, device="cuda")
    q, k, v = (randn(g, 2, h, 64).cuda() for h in (4, 2, 2))
    pages, lens = torch.tensor([[1]], device="cuda", dtype=torch.int32), torch.tensor([3], device="cuda", dtype=torch.int32)
    kc, vc = (x.cuda() for x in cache(g, 2, 16, 2, 64, F))
    lse, q_out, out = torch.zeros(2, 4, device="cuda"), torch.zeros_like(q), torch.zeros_like(q)
    scratch = torch.zeros(ops.attention_scratch_bytes(1, 2, 4, 2, 64), device="cuda", dtype=torch.uint8)
    writes = [(lambda: ops.rotary(q, pos, table, out=q), (q,)),
              (lambda: ops.rotary_backward(q, pos, table, out=out), (out,)),
              (lambda: ops.append_kv(k, v, kc, vc, pages, lens, q=q, q_out=q_out), (kc, vc, q_out)),
              (lambda: ops.shared_prefix_attention(q, kc, vc, pages, lens, out=out, lse=lse), (out, lse)),
              (lambda: ops.shared_prefix_attention(q, kc, vc, pages, lens, scratch=scratch), (scratch,))]
    for i, (write, written) in enumerate(writes):
        note(f"write {i}")
        others = [x for x in (q, k, v, kc, vc, lse, q_out, out, table, scratch) if not any(x is y for y in written)]
        versions = [x._version for x in others]
        for x in written:
            w = torch.ones((), device="cuda", requires_grad=True)
            y = w * x.float() if x.dtype == torch.uint8 else w * x
            before = x._version
            write()
            assert x._version > before
            if x.dtype != torch.uint8:
                with pytest.raises(RuntimeError, match="inplace"):
                    y.sum().backward()
        assert [x._version for x in others] == versions
    with torch.inference_mode():
        c = torch.zeros_like(kc), torch.zeros_like(vc)
        ops.append_kv(k, v, *c, pages, lens)
        assert ops.rotary(q, pos, table, out=q) is q


def test_scales_and_prefix_lengths_of_no_call():
    """Refused with the documented errors, whatever their kind."""
    kc, vc = (torch.zeros(3, 4, 2, 16, device="cuda", dtype=BF) for _ in range(2))
    k, q = torch.zeros(2, 2, 16, device="cuda", dtype=BF), torch.zeros(2, 4, 16, device="cuda", dtype=BF)
    pages, lens = torch.zeros(2, 1, device="cuda", dtype=torch.int32), torch.ones(2, device="cuda", dtype=torch.int32)
    attend_ = lambda **kw: ops.shared_prefix_attention(q, kc, vc, pages, lens, **kw)  # noqa: E731
    for kind, f in ((api.GtsError, lambda: attend_(scale=1e39)), (api.GtsError, lambda: attend_(scale=-float("inf"))),
                    (TypeError, lambda: attend_(scale="1")), (TypeError, lambda: attend_(prefix_len=0.5)),
                    (ValueError, lambda: attend_(prefix_len=1 << 31)), (ValueError, lambda: attend_(prefix_len=-1 << 40)),
                    (TypeError, lambda: ops.append_kv(k, k, kc, vc, pages, lens, prefix_len=1.5))):
        with pytest.raises(kind):
            f()
    torch.cuda.synchronize()
    assert torch.equal(attend_(scale=1), attend_(scale=1.0))


# ---- launches of 2^32 threads and more -----------------------------------------------

@pytest.mark.parametrize("dtype,Hq,Hkv,D", [(F, 64, 8, 2), (HF, 24, 8, 8)])
def test_attention_of_more_rows_than_a_grid_is_wide(dtype, Hq, Hkv, D):
    """2^26 rows and a few of 64 threads each: the row kernel, and the join by one
    row a wave.  All see one key, so that the result is its value."""
    T = (1 << 26) // Hq + 3
    note(f"{T} x {Hq} rows {dtype}")
    g = torch.Generator(device="cuda").manual_seed(71)
    kc, vc = (torch.randn(2, 4, Hkv, D, generator=g, device="cuda").to(dtype) for _ in range(2))
    q = torch.randn(T, Hq, D, generator=g, device="cuda", dtype=dtype)
    pages = torch.full((1, 1), -1, device="cuda", dtype=torch.int32)
    lens, shared = torch.zeros(1, device="cuda", dtype=torch.int32), torch.ones(1, device="cuda", dtype=torch.int32)
    lse = torch.full((T, Hq), 7.0, device="cuda")
    out = ops.shared_prefix_attention(q, kc, vc, pages, lens, prefix_pages=shared, prefix_len=1, lse=lse)
    v, k = (c[1, 0].repeat_interleave(Hq // Hkv, 0) for c in (vc, kc))
    assert (out == v).all()
    for t in range(0, T, 1 << 18):
        s = (q[t:t + (1 << 18)].float() * k.float()).sum(-1) * D ** -0.5
        size = (q[t:t + (1 << 18)].float() * k.float()).abs().sum(-1)
        assert ((lse[t:t + (1 << 18)] - s).abs() <= (D + 10) * R.E * size + 4 * R.E).all()


def test_rotary_of_more_units_than_a_grid_is_wide():
    """2^33 units and a few (34 GB of heads of 2), two a thread: every token as in a
    small call."""
    n, H, times = 4096, 8192, 257
    g = torch.Generator(device="cuda").manual_seed(72)
    x = torch.randn(1, H, 2, generator=g, device="cuda", dtype=BF)
    tab = ops.rotary_table(n, 2)
    pos = torch.randperm(n, generator=g, device="cuda")
    ref = ops.rotary(x.expand(n, H, 2), pos, tab)
    note(f"{n * times} tokens of {H} heads of 2")
    out = torch.empty(times, n, H, 2, device="cuda", dtype=BF)
    ops.rotary(x.expand(n * times, H, 2), pos.repeat(times), tab, out=out.flatten(0, 1))
    for i in range(times):
        assert torch.equal(out[i], ref), i


# ---- segments of many rows: the tiles' masks -------------------------------------------

# New tokens of a sequence and query heads of a group: 48 rows (two of the four waves
# take rows of their own), 80 and 160 (all four, the second in two segments).
MANY_ROWS = [(12, 4), (20, 4), (20, 8)]


@pytest.mark.parametrize("fill", [float("inf"), float("-inf"), float("nan"), torch.finfo(BF).min])
@pytest.mark.parametrize("dtype,D", [(BF, 64), (HF, 128), (BF, 256), (BF, 96)])
def test_masked_values_of_many_rows(dtype, D, fill):
    note(f"masked slots hold {fill}, many rows {dtype} {D}")
    fill = fill if dtype == BF or fill != torch.finfo(BF).min else torch.finfo(HF).min
    attention_case(dtype, 8, 2, D, 16, [12, 20, 40], [25, 37, 140], 33, fill=fill)
    attention_case(dtype, 4, 1, D, 64, [12, 20, 9], [12, 90, 4], 0, fill=fill)


@pytest.mark.parametrize("dtype,D", [(BF, 64), (HF, 128), (BF, 256), (BF, 96)])
def test_missing_pages_of_many_rows(dtype, D):
    note(f"missing pages, many rows {dtype} {D}")
    drop = ((0, 0), (0, 4), (1, 2), (1, 3), (2, 0))
    attention_case(dtype, 8, 2, D, 16, [12, 40, 20], [90, 300, 16], 40, drop_pages=drop, seed=5)
    attention_case(dtype, 8, 2, D, 8, [12, 40, 20], [90, 300, 16], 0, drop_pages=drop, seed=6)
    attention_case(dtype, 8, 2, D, 64, [12, 40, 20], [90, 300, 20], 0, drop_pages=((0, 1), (1, 0), (1, 4)), seed=7)


@pytest.mark.parametrize("rows", [(1, 4), (3, 8)] + MANY_ROWS)
@pytest.mark.parametrize("dtype,D", [(BF, 64), (HF, 128), (BF, 256), (F, 64)])
def test_missing_pages_of_the_prefix(dtype, D, rows):
    """Pages of the prefix outside the cache: the same as a prefix without their
    keys."""
    n, G = rows
    g, page, H, P = gen(51), 16, 2, 300
    note(f"prefix without pages 0, 7 and 18 {dtype} {D} rows {rows}")
    kc, vc = (x.cuda() for x in cache(g, 24, page, H, D, dtype))
    q = randn(g, 2 * n, G * H, D, dtype=dtype)
    order = torch.randperm(24, generator=g)[:19].int()
    shared = order.clone()
    shared[[0, 7, 18]] = torch.tensor([-1, 24, 1 << 30], dtype=torch.int32)
    own = torch.tensor([[23, 22], [21, 20]], dtype=torch.int32)
    lens = torch.tensor([0, 20]).int()
    want = R.attention(q, kc.cpu(), vc.cpu(), own, lens, None, shared, P)
    lse = torch.zeros(2 * n, G * H, device="cuda")
    out = ops.shared_prefix_attention(q.cuda(), kc, vc, own.cuda(), lens.cuda(), prefix_pages=shared.cuda(), prefix_len=P,
                                      lse=lse)
    close(out, want[0], want[2], "out")
    close(lse, want[1], want[3], "lse")


@pytest.mark.parametrize("at", [0, 37, 70, 75, 79])
@pytest.mark.parametrize("n,G", [(2, 4), (5, 5)] + MANY_ROWS)
@pytest.mark.parametrize("dtype,D", [(BF, 64), (HF, 128), (BF, 256), (BF, 96), (F, 64)])
def test_values_not_finite_behind_some_rows(dtype, D, n, G, at):
    """One value of one key is not finite: it is in that dim of the rows that see
    the key, and nowhere else."""
    g, H, L = gen(52), 2, 80
    note(f"a value of key {at} of {L}, {n} tokens x {G} heads {dtype} {D}")
    kc, vc = cache(g, 6, 16, H, D, dtype)
    q = randn(g, n, G * H, D, dtype=dtype)
    pages, lens = torch.tensor([[4, 1, 5, 0, 2]], dtype=torch.int32), torch.tensor([L]).int()
    want = R.attention(q, kc, vc, pages, lens, None)
    seen = torch.arange(L - n, L) >= at
    for bad, d in ((float("inf"), 3), (float("-inf"), D - 1), (float("nan"), 8)):
        v1 = vc.clone()
        v1[pages[0, at // 16], at % 16, 1, d] = bad  # key-value head 1
        lse = torch.zeros(n, G * H, device="cuda")
        out = ops.shared_prefix_attention(q.cuda(), kc.cuda(), v1.cuda(), pages.cuda(), lens.cuda(), lse=lse)
        close(lse, want[1], want[3], "lse")
        out = out.cpu()
        hit = out[seen][:, G:, d]
        assert (hit.isnan() if bad != bad else hit == bad).all(), f"{bad} in dim {d}"
        out[:, G:, d][seen] = 0
        ref = want[0].clone()
        ref[:, G:, d][seen] = 0
        close(out, ref, want[2], f"without {bad} in dim {d}")


@pytest.mark.parametrize("n,G", MANY_ROWS)
@pytest.mark.parametrize("dtype,D", [(BF, 64), (HF, 128), (BF, 256)])
def test_keys_not_finite_behind_some_rows(dtype, D, n, G):
    g, H, L, at = gen(53), 2, 80, 72
    note(f"key {at} of {L} holds nothing finite, {n} tokens x {G} heads {dtype} {D}")
    kc, vc = cache(g, 6, 16, H, D, dtype)
    q = randn(g, n, G * H, D, dtype=dtype)
    pages, lens = torch.tensor([[4, 1, 5, 0, 2]], dtype=torch.int32), torch.tensor([L]).int()
    want = R.attention(q, kc, vc, pages, lens, None)
    first = at - (L - n)  # the first token that sees it
    for bad in (float("inf"), float("-inf"), float("nan")):
        k1, v1 = kc.clone(), vc.clone()
        k1[pages[0, at // 16], at % 16] = bad
        v1[pages[0, at // 16], at % 16] = bad
        out = ops.shared_prefix_attention(q.cuda(), k1.cuda(), v1.cuda(), pages.cuda(), lens.cuda())
        assert out[first:].isnan().all()
        close(out[:first], want[0][:first], want[2][:first], f"before {bad}")


@pytest.mark.parametrize("dtype,D", [(BF, 64), (HF, 128), (BF, 256)])
def test_lengths_past_the_pages_of_many_rows(dtype, D):
    g = gen(54)
    kc, vc = (x.cuda() for x in cache(g, 8, 16, 2, D, dtype))
    q = randn(g, 60, 8, D, dtype=dtype).cuda()
    pages = torch.tensor([[1, 3, 5, 7], [2, 0, 4, 6]], device="cuda", dtype=torch.int32)
    starts = torch.tensor([0, 40, 60], device="cuda", dtype=torch.int32)
    lens = torch.tensor([64 + 40, 64 + 20], device="cuda", dtype=torch.int32)  # all see 64 keys
    ref = ops.shared_prefix_attention(q, kc, vc, pages, lens, starts=starts)
    far = torch.tensor([2 ** 31 - 1, 1 << 30], device="cuda", dtype=torch.int32)
    note(f"{far.tolist()} keys in four pages of 16, many rows {dtype} {D}")
    assert torch.equal(ops.shared_prefix_attention(q, kc, vc, pages, far, starts=starts), ref)
    want = R.attention(q.cpu(), kc.cpu(), vc.cpu(), pages.cpu(), lens.cpu(), starts.cpu())
    close(ref, want[0], want[2], "out")


@pytest.mark.parametrize("dtype,D,n,G", [(BF, 64, 5, 2), (HF, 128, 30, 4), (F, 64, 4, 2)])
def test_the_same_number_of_tokens_each(dtype, D, n, G):
    """starts=None with several tokens a sequence: the same bits as with starts."""
    g, H, B = gen(55), 2, 3
    kc, vc = (x.cuda() for x in cache(g, 16, 16, H, D, dtype))
    k, v, q = (randn(g, B * n, h, D, dtype=dtype).cuda() for h in (H, H, G * H))
    pages = torch.randperm(16, generator=g)[:15].view(3, 5).int().cuda()
    lens = torch.tensor([n, n + 40, 77], device="cuda", dtype=torch.int32)
    starts = torch.arange(B + 1, device="cuda", dtype=torch.int32) * n
    tab = ops.rotary_table(80, D)
    got = []
    for s in (None, starts):
        k1, v1 = kc.clone(), vc.clone()
        q1 = ops.append_kv(k, v, k1, v1, pages, lens, starts=s, table=tab, q=q)
        got.append((k1, v1, q1, ops.shared_prefix_attention(q1, k1, v1, pages, lens, starts=s)))
    note(f"{B} x {n} tokens {dtype} {D}")
    assert all(torch.equal(a, b) for a, b in zip(*got)) and not torch.equal(got[0][0], kc)
    want = R.attention(got[0][2].cpu(), got[0][0].cpu(), got[0][1].cpu(), pages.cpu(), lens.cpu())
    close(got[0][3], want[0], want[2], "out")


# ---- layouts of the paged operators ------------------------------------------------------

def shifted(t, by):
    """The same values, `by` elements behind a 16-byte boundary, rows `by` further apart."""
    wide = torch.zeros(*t.shape[:-1], t.shape[-1] + 8, dtype=t.dtype, device="cuda")
    off = wide[..., by:by + t.shape[-1]]
    off.copy_(t)
    return off


def odd_rows(t):
    """The same values in rows an odd number of elements apart."""
    off = torch.zeros(*t.shape[:-1], t.shape[-1] + 1, dtype=t.dtype, device="cuda")[..., :t.shape[-1]]
    return off.copy_(t)


def paged(g, dtype, D, H, G, page=16, prefix=40, counts=(5, 1, 14), lens=(9, 70, 33)):
    """Inputs of both operators on the GPU: a packed projection's q, k and v."""
    T, B = sum(counts), len(counts)
    n = -(-max(lens) // page)
    n_prefix = -(-prefix // page)
    order = torch.randperm(B * n + n_prefix, generator=g).int()
    packed = randn(g, T, (G + 2) * H, D, dtype=dtype).cuda()
    q, k, v = packed[:, :G * H], packed[:, G * H:(G + 1) * H], packed[:, (G + 1) * H:]
    kc, vc = (x.cuda() for x in cache(g, B * n + n_prefix, page, H, D, dtype))
    return dict(q=q, k=k, v=v, kc=kc, vc=vc, pages=order[n_prefix:].view(B, n).cuda(), shared=order[:n_prefix].cuda(),
                P=prefix, lens=torch.tensor(lens).int().cuda(),
                starts=torch.tensor([0, *counts]).cumsum(0).int().cuda(), tab=ops.rotary_table(200, D // 2 * 2))


def attend(s, **kw):
    s = {**s, **kw}
    return ops.shared_prefix_attention(s["q"], s["kc"], s["vc"], s["pages"], s["lens"], starts=s["starts"],
                                       prefix_pages=s["shared"], prefix_len=s["P"], out=s.get("out"), lse=s.get("lse"))


def append(s, inter=False, **kw):
    s = {**s, **kw}
    return ops.append_kv(s["k"], s["v"], s["kc"], s["vc"], s["pages"], s["lens"], starts=s["starts"], table=s["tab"],
                         interleaved=inter, prefix_len=s["P"], q=s["q"], q_out=s.get("q_out"))


@pytest.mark.parametrize("dtype,D,inter", [(BF, 64, False), (HF, 128, True), (BF, 40, False), (F, 64, False), (F, 64, True),
                                           (F, 512, False)])
def test_append_layouts(dtype, D, inter):
    """Every layout of k, v, q, the result and the caches gives the bits of
    contiguous ones, whose values are those of the formula."""
    g = gen(61)
    s = paged(g, dtype, D, 2, 3)
    dense = {x: s[x].contiguous() for x in "qkv"}
    kc, vc = s["kc"].clone(), s["vc"].clone()
    ref = append(s, inter, **dense, kc=kc, vc=vc)
    rows = s["tab"].cpu().double()
    at = [(b, j) for b, (n, m) in enumerate(zip((5, 1, 14), (9, 70, 33))) for j in range(m - n, m)]
    row = rows[[s["P"] + j for _, j in at]]
    slots = torch.stack([s["pages"].cpu()[b, j // 16] for b, j in at]).long(), torch.tensor([j % 16 for _, j in at])
    for got, x in ((ref, "q"), (kc.cpu()[slots], "k")):
        y, size = R.rotate(s[x].cpu().double(), row, inter)
        close(got, y, R.rotation_bound(y, size, dtype), x)
    assert torch.equal(vc.cpu()[slots], s["v"].cpu())

    def same(what, **kw):
        note(f"append {dtype} {D} interleaved {inter}: {what}")
        k1, v1 = kw.pop("kc", s["kc"].clone()), kw.pop("vc", s["vc"].clone())
        got = append(s, inter, kc=k1, vc=v1, **kw)
        assert torch.equal(got, ref) and torch.equal(k1, kc) and torch.equal(v1, vc), what

    same("views of a packed projection")
    heads_first = lambda x: x.transpose(1, 2).contiguous().transpose(1, 2)  # noqa: E731
    same("keys head by head", kc=heads_first(s["kc"]))
    same("values head by head", vc=heads_first(s["vc"]))
    for by in (1, 2, 4):
        for x in "qkv":
            same(f"{x} shifted by {by}", **{x: shifted(s[x], by)})
        same(f"result shifted by {by}", q_out=shifted(torch.zeros_like(dense["q"]), by))
        same(f"keys' cache shifted by {by}", kc=shifted(s["kc"], by))
        same(f"values' cache shifted by {by}", vc=shifted(s["vc"], by))
    for x in "qkv":
        same(f"{x} in odd rows", **{x: odd_rows(s[x])})
    same("result in odd rows", q_out=odd_rows(torch.zeros_like(dense["q"])))
    same("caches in odd rows", kc=odd_rows(s["kc"]), vc=odd_rows(s["vc"]))
    # into the packed projection itself: nothing else in it changes
    whole = torch.cat((s["q"], s["k"], s["v"]), 1)
    G = s["q"].shape[1]
    same("in place", q=whole[:, :G], q_out=whole[:, :G], k=whole[:, G:G + 2], v=whole[:, G + 2:])
    assert torch.equal(whole[:, :G], ref) and torch.equal(whole[:, G:], torch.cat((s["k"], s["v"]), 1))


@pytest.mark.parametrize("dtype,D,G", [(BF, 64, 3), (HF, 128, 4), (BF, 256, 4), (HF, 80, 4), (F, 64, 2), (HF, 33, 2)])
def test_attention_layouts(dtype, D, G):
    g = gen(62)
    s = paged(g, dtype, D, 2, G)
    dense = s["q"].contiguous()
    want = R.attention(dense.cpu(), s["kc"].cpu(), s["vc"].cpu(), s["pages"].cpu(), s["lens"].cpu(), s["starts"].cpu(),
                       s["shared"].cpu(), s["P"])
    ref = attend(s, q=dense)
    close(ref, want[0], want[2], "out")
    bits = ref.clone()

    def check(what, same, **kw):
        """`same`: the kernel that contiguous tensors take, so its bits."""
        note(f"attention {dtype} {D}: {what}")
        lse = torch.zeros(dense.shape[:2], device="cuda")
        got = attend(s, lse=lse, **kw)
        close(got, want[0], want[2], what)
        close(lse, want[1], want[3], what)
        if same:
            assert torch.equal(got, bits), what

    check("queries of a packed projection", D % 8 == 0)
    heads_first = lambda x: x.transpose(1, 2).contiguous().transpose(1, 2)  # noqa: E731
    check("keys head by head", True, kc=heads_first(s["kc"]))
    check("values head by head", True, vc=heads_first(s["vc"]))
    check("a result inside a packed tensor", True, out=torch.zeros_like(torch.cat((s["q"], s["k"]), 1))[:, :dense.shape[1]])
    check("a result two elements off", True, out=shifted(torch.zeros_like(dense), 2))
    # rows that cannot be loaded 16 bytes at a time, or stored four
    for by in (1, 2, 4):
        check(f"queries shifted by {by}", False, q=shifted(s["q"], by))
        check(f"keys shifted by {by}", False, kc=shifted(s["kc"], by))
        check(f"values shifted by {by}", False, vc=shifted(s["vc"], by))
    check("a result one element off", False, out=shifted(torch.zeros_like(dense), 1))
    check("a result in odd rows", False, out=odd_rows(torch.zeros_like(dense)))
    check("queries in odd rows", False, q=odd_rows(s["q"]))
    check("caches in odd rows", False, kc=odd_rows(s["kc"]), vc=odd_rows(s["vc"]))
    check("caches in rows of 8 more", False, kc=shifted(s["kc"], 0), vc=shifted(s["vc"], 0))
    buf = torch.zeros(dense.numel() + 8, dtype=dtype, device="cuda")
    check("the result's neighbours", True, out=buf[4:4 + dense.numel()].view(dense.shape))
    assert (buf[:4] == 0).all() and (buf[4 + dense.numel():] == 0).all()


@pytest.mark.parametrize("counts,lens", [((1, 1, 1), (9, 70, 33)), ((30, 1, 14), (40, 70, 33))])
def test_slots_far_apart(counts, lens):
    """Slots of a page 2^26 elements and more apart, so that 16 rows pass 2 GiB:
    the general way of loading, with pages of 16."""
    g = gen(63)
    s = paged(g, BF, 64, 2, 4, counts=counts, lens=lens)
    ref = attend(s)
    n, page, H, D = s["kc"].shape
    slot = (1 << 26) + 8
    buf = torch.empty((page - 1) * slot + n * H * D, dtype=BF, device="cuda")
    far = buf.as_strided((n, page, H, D), (H * D, slot, D, 1))
    for x in ("kc", "vc"):
        far.copy_(s[x])
        note(f"{x} with slots {slot} elements apart, {counts} tokens")
        assert torch.equal(attend(s, **{x: far}), ref)
    far.zero_()
    kc, vc = s["kc"].clone(), s["vc"].clone()
    zero = torch.zeros_like(kc)
    append(s, kc=far, vc=vc)
    append(s, kc=zero, vc=s["vc"].clone())
    assert torch.equal(far, zero) and torch.equal(kc, s["kc"])


def test_function_transforms_raise():
    """torch.func's transforms hand over tensors without memory: an error, not a
    lost derivative."""
    g = gen(44)
    table, pos = ops.rotary_table(50, 64), torch.arange(2, device="cuda")
    q = randn(g, 2, 4, 64).cuda()
    turn = lambda x: ops.rotary(x, pos, table)  # noqa: E731
    for f in (lambda: torch.func.grad(lambda x: turn(x).sum())(q), lambda: torch.func.jvp(turn, (q,), (q,)),
              lambda: torch.func.vmap(turn)(q[None]), lambda: torch.func.jvp(lambda t: ops.rotary(q, pos, t), (table,), (table,))):
        with pytest.raises((RuntimeError, ValueError)):
            f()
