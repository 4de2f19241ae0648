"""The operators in 64 bits on the CPU, from their formulas, and how far a
kernel's result may be from them.

u is the unit roundoff of the result's type (2^-8, 2^-11, 2^-24) and e that
of 32 bits.  A rotated value is two products and a sum in 32 bits (at most 3 e
of |a c| + |b s|), rounded once.  An attention score is a sum of D products
(D + 2 roundings of 32 bits); an error d of a score changes its weight by a
factor of at most exp(d) and the sum of weights too; a weight may be rounded to
the values' type before it is multiplied (u, and in float16, whose numbers end
at 2^-24, half of that), the sum of n products and the join of the parts add
their roundings in 32 bits, and the result is rounded once."""
import torch

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
E = 2.0 ** -24


def rotate(x, rows, interleaved=False, backward=False):
    """x [.., heads, D], rows [.., R] of the table, both on the CPU in 64 bits;
    the result and sum of the absolute products."""
    R = rows.shape[-1]
    c, s = rows[..., None, :R // 2], rows[..., None, R // 2:]
    if backward:
        s = -s
    ia = torch.arange(0, R, 2) if interleaved else torch.arange(R // 2)
    ib = ia + (1 if interleaved else R // 2)
    a, b = x[..., ia], x[..., ib]
    y, size = x.clone(), torch.zeros_like(x)
    y[..., ia], size[..., ia] = a * c - b * s, (a * c).abs() + (b * s).abs()
    y[..., ib], size[..., ib] = b * c + a * s, (b * c).abs() + (a * s).abs()
    return y, size


def rotation_bound(ref, size, dtype):
    tiny = 2.0 ** -24 if dtype == torch.float16 else 2.0 ** -126
    return U[dtype] * 1.001 * ref.abs() + 3.01 * E * size + tiny


def own_counts(B, T, starts):
    """(first token, number of new tokens) of each sequence."""
    s = [b * (T // B) for b in range(B + 1)] if starts is None else starts.tolist()
    return [(s[b], s[b + 1] - s[b]) for b in range(B)]


def pages_of(row, n, n_pages, page):
    """(page, slot) of keys 0 .. n - 1, None where no page holds them."""
    row = row.tolist()
    return [(row[j // page], j % page) if j // page < len(row) and 0 <= row[j // page] < n_pages else None
            for j in range(n)]


def attention(q, k_cache, v_cache, page_table, lens, starts=None, prefix_pages=None, prefix_len=0, scale=None):
    """(out, lse, bound of out, bound of lse), all tensors on the CPU."""
    T, Hq, D = q.shape
    n_pages, page, Hkv, _ = k_cache.shape
    G, dtype = Hq // Hkv, q.dtype
    scale = D ** -0.5 if scale is None else scale
    out, bound = torch.zeros(T, Hq, D, dtype=torch.float64), torch.full((T, Hq, D), 1e-30, dtype=torch.float64)
    lse = torch.full((T, Hq), -float("inf"), dtype=torch.float64)
    lse_bound = torch.zeros(T, Hq, dtype=torch.float64)
    shared = [] if prefix_pages is None else pages_of(prefix_pages, prefix_len, n_pages, page)
    for b, (first, n) in enumerate(own_counts(len(lens), T, starts)):
        if n <= 0:
            continue
        m = int(lens[b])
        where = shared + pages_of(page_table[b], max(m, 0), n_pages, page)
        there = [j for j, x in enumerate(where) if x is not None]
        if not there:
            continue
        pg = torch.tensor([where[j][0] for j in there])
        sl = torch.tensor([where[j][1] for j in there])
        k, v = k_cache[pg, sl].double(), v_cache[pg, sl].double()  # [keys, Hkv, D]
        at = torch.tensor(there)
        for i in range(n):
            limit = len(shared) + m - n + i if m - n + i >= 0 else len(shared) - 1
            seen = at <= limit
            if not seen.any():
                continue
            for h in range(Hkv):
                qr = q[first + i, h * G:(h + 1) * G].double()
                ks, vs = k[seen, h], v[seen, h]
                s = qr @ ks.T * scale
                d = (D + 6) * E * (qr.abs() @ ks.abs().T * abs(scale)).amax(-1, keepdim=True) + 4 * E * s.abs().amax(-1, keepdim=True)
                w = s.softmax(-1)
                rows = slice(h * G, (h + 1) * G)
                out[first + i, rows] = w @ vs
                lse[first + i, rows] = s.logsumexp(-1)
                spread = w @ vs.abs()
                keys = int(seen.sum())
                rel = 2.01 * U[dtype] + 2 * d + (keys / 16 + 64) * 2 * E
                tiny = 2.0 ** -25 * vs.abs().sum(0) if dtype == torch.float16 else 0.0
                bound[first + i, rows] = rel * spread + tiny + (2.0 ** -25 if dtype == torch.float16 else 1e-30)
                lse_bound[first + i, rows] = d[:, 0] + (keys / 16 + 64) * 2 * E + 4 * E * lse[first + i, rows].abs()
    return out, lse, bound, lse_bound
