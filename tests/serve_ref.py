"""The serving operators in 64 bits on the CPU, from their definitions, a row at
a time; and the rounding bounds that their GPU results are held to."""
import math

import numpy as np

HALF_ULP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}      # largest relative error of one rounding


def frequencies(rot, scaling="none", base=10000.0, factor=1.0, orig_len=0, low=0.0, high=0.0):
    """(radians per position of each pair, factor on cosine and sine)."""
    half = rot // 2
    if scaling == "base":
        base = base * factor ** (rot / (rot - 2))
    f = [base ** (-2.0 * i / rot) for i in range(half)]
    if scaling == "linear":
        return np.array(f) / factor, 1.0
    if scaling == "yarn":
        pair = lambda turns: rot * math.log(orig_len / (2 * math.pi * turns)) / (2 * math.log(base))
        lo = min(max(math.floor(pair(high)), 0), half - 1)
        hi = max(min(math.ceil(pair(low)), half - 1), 0)
        w = [min(max((i - lo) / max(hi - lo, 0.001), 0.0), 1.0) for i in range(half)]
        return np.array([(1 - x) * y + x * y / factor for x, y in zip(w, f)]), 1.0 + 0.1 * math.log(factor)
    if scaling == "wavelength":
        s = [min(max((orig_len * y / (2 * math.pi) - low) / (high - low), 0.0), 1.0) for y in f]
        return np.array([x * y + (1 - x) * y / factor for x, y in zip(s, f)]), 1.0
    return np.array(f), 1.0


def rope(x, heads, hd, rot, positions, layout="half", back=False, mscale=0.0, **scaling):
    """Rows [T][heads * hd] (float64) turned by their positions."""
    f, m = frequencies(rot, **scaling)
    m = mscale or m
    y = np.array(x, dtype=np.float64).reshape(len(x), heads, hd)
    angle = np.asarray(positions, dtype=np.float64)[:, None] * f
    c, s = m * np.cos(angle)[:, None], m * np.sin(angle)[:, None] * (-1.0 if back else 1.0)
    i, j = (slice(0, rot // 2), slice(rot // 2, rot)) if layout == "half" else (slice(0, rot, 2), slice(1, rot, 2))
    a, b = y[..., i].copy(), y[..., j].copy()
    y[..., i], y[..., j] = a * c - b * s, b * c + a * s
    return y.reshape(len(x), heads * hd)


def rope_bound(x, heads, hd, rot, y, dtype, layout="half", m=1.0):
    """Largest error of each element of y: its rounding, and the fp32 cosine, sine
    and products of its pair.  bf16: cosine and sine to 2^-17 (the hardware's; the
    angle's fraction of a turn is good to 2^-26); fp32: 2^-23.3 from the fraction,
    2^-23 from the functions, 2^-24 each from the scale and the products: 2^-21."""
    a = np.abs(np.array(x, dtype=np.float64).reshape(len(x), heads, hd))
    pair = np.zeros_like(a)
    i, j = (slice(0, rot // 2), slice(rot // 2, rot)) if layout == "half" else (slice(0, rot, 2), slice(1, rot, 2))
    pair[..., i] = pair[..., j] = a[..., i] + a[..., j]
    return HALF_ULP[dtype] * np.abs(y) + (2.0 ** -17 if dtype == "bf16" else 2.0 ** -21) * abs(m) * pair.reshape(y.shape)


def page_map(kv_len, n_new, free_pages, free_at, table, page, T, pos0):
    """The tables of a step, request by request and token by token."""
    table = np.array(table)
    start, slots, positions, at = [0], [-1] * T, [0] * T, free_at
    width = table.shape[1] if table.ndim == 2 else 0
    row = 0
    for r, (kv, n) in enumerate(zip(kv_len, n_new)):
        kv = max(int(kv), 0)
        n = min(max(int(n), 0), kv)
        have = min(-(-(kv - n) // page), width)
        for j in range(have, min(-(-kv // page), width)):
            table[r, j] = free_pages[at] if 0 <= at < len(free_pages) else -1
            at += 1
        for i in range(kv - n, kv):
            if row < T:
                p = int(table[r, i // page]) if i // page < width else -1
                slots[row] = p * page + i % page if p >= 0 else -1
                positions[row] = pos0 + i
            row += 1
        start.append(row)
    return table, start, slots, positions, at


def attention(q, K, V, hq, prefix_table, prefix_len, table, kv_len, start, page, scale=None):
    """(out [T][hq * hd], lse [hq][T], weight) in 64 bits; rows of no request are NaN.
    weight is sum p |v|: what a relative error of each probability can do to out.
    K, V [n_pages][heads][page][hd]; pages outside the cache hold no keys."""
    n_pages, hk, _, hd = K.shape
    T, g = len(q), hq // hk
    scale = 1.0 / math.sqrt(hd) if scale is None else scale
    q = np.array(q, dtype=np.float64).reshape(T, hq, hd)
    out, weight, lse = np.full((T, hq, hd), np.nan), np.full((T, hq, hd), np.nan), np.full((hq, T), np.nan)

    def rows(tab, n):
        """(page, offset) of the tokens 0 .. n - 1 that lie in the cache."""
        at = [(int(tab[j // page]), j % page, j) for j in range(n)]
        return [x for x in at if 0 <= x[0] < n_pages]

    shared = rows(prefix_table, prefix_len)
    for r in range(len(start) - 1):
        n = start[r + 1] - start[r]
        own = rows(table[r], kv_len[r]) if len(kv_len) else []
        for i in range(n):
            last = (kv_len[r] if len(kv_len) else 0) - n + i
            seen = shared + [x for x in own if x[2] <= last]
            t = start[r] + i
            if not seen:
                out[t], weight[t], lse[:, t] = 0.0, 0.0, -np.inf
                continue
            p, o = np.array([x[0] for x in seen]), np.array([x[1] for x in seen])
            for h in range(hk):
                Kh, Vh = K[p, h, o].astype(np.float64), V[p, h, o].astype(np.float64)
                x = slice(h * g, (h + 1) * g)
                with np.errstate(invalid="ignore", over="ignore"):
                    s = q[t, x] @ Kh.T * scale
                    m = s.max(-1, keepdims=True)
                    e = np.exp(s - m)
                    l = e.sum(-1, keepdims=True)
                    out[t, x], weight[t, x] = e / l @ Vh, e / l @ np.abs(Vh)
                    lse[x, t] = (m + np.log(l))[:, 0]
    return out.reshape(T, hq * hd), lse, weight.reshape(T, hq * hd)


def attention_bound(out, weight, keys):
    """Largest error of out: each probability rounded to bf16 (2^-8 of weight), the
    result rounded (2^-8 of out, and of the first error), and the fp32 parts: scores
    of at most 2^7 products whose magnitudes sum to under 2^6 here are good to 2^-11
    (2^7 2^-24 2^6) and so are the probabilities, the sums over `keys` to keys 2^-24."""
    small = 2.0 ** -11 + 2.0 ** -22 + keys * 2.0 ** -24
    return (2.0 ** -8 * 1.01 + 2.0 * small) * weight + 2.0 ** -8 * np.abs(out) + 1e-30


def lse_bound(lse, keys):
    """fp32 log-sum-exp: scores to 2^-11 (see attention_bound), the sum over `keys`
    to keys 2^-24, the logarithm and its rounding to 2^-22 of the result."""
    return 2.0 ** -11 + keys * 2.0 ** -24 + 2.0 ** -22 * np.abs(lse)
