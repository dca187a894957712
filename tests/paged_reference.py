"""Plain evaluation in 64 bits of the operators on a paged cache, and how far fp32 kernels may be from it."""
import torch

E4M3_MAX = 448.0
U = 2.0 ** -24  # half a step of fp32, relative


def fill_pool(n_pages, heads, tokens, dim, cache, gen, scale_exp=(-3, 3)):
    """Random pages as a cache holds them -> (pages, scales or None); scales are powers of two."""
    x = torch.randn((n_pages, heads, tokens, dim), generator=gen)
    if cache == "bf16":
        return x.to(torch.bfloat16), None
    s = torch.exp2(torch.randint(scale_exp[0], scale_exp[1] + 1, (n_pages, heads), generator=gen).float())
    return (x * 40.0).to(torch.float8_e4m3fn), s


def dequantised(pages, scale):
    x = pages.float().double()
    return x if scale is None else x * scale.double()[:, :, None, None]


def rows_of(pages, scale, table_row, h, tokens):
    """K or V rows [tokens][D] of one head, and which of them have a page."""
    P, n_pages = pages.shape[2], pages.shape[0]
    n = -(-tokens // P)
    ids = table_row[:n].long()
    ok = (ids >= 0) & (ids < n_pages)
    x = dequantised(pages[ids.clamp(0, n_pages - 1), h:h + 1], None if scale is None else scale[ids.clamp(0, n_pages - 1), h:h + 1])
    return x[:, 0].reshape(-1, pages.shape[3])[:tokens], ok.repeat_interleave(P)[:tokens]


def attend(q, k, v, seen, scale, out, two_terms):
    """q [m][D], k, v [t][D] double, seen [m][t] -> (result [m][D], tolerance [m][D]).

    Tolerance, first order.  A logit is off by the fp32 accumulation of D exact products (D U sum|q k|), the factors it is multiplied
    with (three roundings) and exp2 (2 ulp); a relative error d of all weights moves the result by at most 2 d sum p |v|.  The
    weights enter the product with the values as bf16 terms (2^-18 of a weight left out with two, 2^-8 with one), the scale of the
    values is one more rounding, and at most a quarter of the tokens are added up in sequence (32 at a time in four waves, each
    time as up to 32 roundings), some more in folding.  Then the output's own rounding."""
    m, D = q.shape
    res = torch.zeros((m, v.shape[1]), dtype=torch.float64)
    tol = torch.zeros_like(res)
    w = (q @ k.T) * scale
    size = (q.abs() @ k.abs().T) * scale
    for i in range(m):
        j = seen[i]
        if not j.any():
            continue
        x = w[i, j]
        p = torch.softmax(x, 0)
        res[i] = p @ v[j]
        d = (D + 8) * U * float(size[i, j].max()) + 8 * U * float(x.abs().max()) + 8 * U
        spread = p @ v[j].abs()
        rel = 2 * d + (2.0 ** -18 if two_terms else 2.0 ** -8) + (int(j.sum()) / 4 + 64) * U
        tol[i] = spread * rel + (2.0 ** -8 if out == "bf16" else U) * res[i].abs() + 1e-30
    return res, tol


def attention(q, pages, table, lengths, offsets, scale, out, listed=None):
    """All sequences; pages = (k, v, ks, vs).  Rows outside the offsets are NaN in the result."""
    k_pages, v_pages, ks, vs = pages
    n, Hq, D = q.shape
    Hkv, P = k_pages.shape[1], k_pages.shape[2]
    G = Hq // Hkv
    res = torch.full((n, Hq, D), float("nan"), dtype=torch.float64)
    tol = torch.zeros_like(res)
    for b in range(lengths.shape[0]):
        lo, hi = (int(offsets[b]), int(offsets[b + 1])) if offsets is not None else (b, b + 1)
        t = min(max(int(lengths[b]), 0), table.shape[1] * P)
        m = hi - lo
        for h in range(Hkv):
            k, ok = rows_of(k_pages, ks, table[b], h, t)
            v, _ = rows_of(v_pages, vs, table[b], h, t)
            seen = ok[None, :] & (torch.arange(t)[None, :] <= (t - m + torch.arange(m))[:, None])
            if listed is not None:
                i = listed[b, h].long()
                i = i[(i >= 0) & (i < t)]
                k, v, seen = k[i], v[i], ok[i][None, :]
            for g in range(h * G, h * G + G):
                r, e = attend(q[lo:hi, g].double(), k, v, seen, scale, out, out == "f32")
                res[lo:hi, g], tol[lo:hi, g] = r, e
    return res, tol


def rotated(x, pos, table, style):
    """x [n][heads][D] double by rows `pos` of the table."""
    r = table.shape[1]
    c, s = table[pos].double()[:, None, :].chunk(2, -1)
    y = x.clone()
    a, b = (slice(0, r // 2), slice(r // 2, r)) if style == "halves" else (slice(0, r, 2), slice(1, r, 2))
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., b] * c + x[..., a] * s
    return y


def power_scale(amax):
    """Smallest power of two s with amax <= 448 s, not below 2^-100."""
    s = 2.0 ** -100
    while amax > E4M3_MAX * s:
        s *= 2.0
    return s


def append(x, pages, scale, table, lengths, offsets):
    """Values [n][heads][D] in 64 bits join their pages -> (values of the pool, scales, tolerance, which rows were written or kept).

    Tolerance of a new value: half a step of e4m3 (2^-4 of it, or half the subnormal step 2^-10 s), of a bf16 value 2^-8; plus three
    fp32 roundings of the rotation, relative to the larger of a pair (bounded by the row's largest value).  An old value in a page
    whose scale grew moves by half the new scale's subnormal step at most."""
    heads, P, D = pages.shape[1], pages.shape[2], pages.shape[3]
    val = dequantised(pages, scale)
    new_scale = None if scale is None else scale.double().clone()
    tol = torch.zeros_like(val)
    cap = table.shape[1] * P
    for b in range(lengths.shape[0]):
        lo, hi = (int(offsets[b]), int(offsets[b + 1])) if offsets is not None else (b, b + 1)
        at = int(lengths[b]) - (hi - lo)
        touched = {}
        for i in range(lo, hi):
            p = at + i - lo
            if 0 <= p < cap:
                touched.setdefault(p // P, []).append((p % P, i))
        for e, rows in touched.items():
            page = int(table[b, e])
            if not 0 <= page < pages.shape[0]:
                continue
            slots, toks = [r[0] for r in rows], [r[1] for r in rows]
            for h in range(heads):
                y = x[toks, h]
                t = 3 * U * y.abs().amax(-1, keepdim=True).expand_as(y)
                if scale is None:
                    t = t + 2.0 ** -8 * y.abs()
                else:
                    s = power_scale(float(y.abs().max()))
                    if slots[0] > 0:
                        old = float(scale[page, h])
                        if s > old:
                            tol[page, h, : slots[0]] = 2.0 ** -10 * s
                        s = max(s, old)
                    new_scale[page, h] = s
                    t = t + torch.maximum(2.0 ** -4 * y.abs(), torch.full_like(y, 2.0 ** -10 * s))
                val[page, h, slots] = y
                tol[page, h, slots] = t
    return val, new_scale, tol
