"""Head norms, drafted trees and rules on logits in 64 bits on the CPU, from their
definitions, a row at a time; and the rounding bounds that GPU results are held to."""
import math

import numpy as np

import serve_ref as R

HALF_ULP = R.HALF_ULP
# cosine and sine of a bf16 row, and of an fp32 one with the products (serve_ref.rope_bound)
TRIG = {"bf16": 2.0 ** -17, "f32": 2.0 ** -21}


def heads(x, hd):
    x = np.array(x, dtype=np.float64)
    return x.reshape(len(x), x.shape[1] // hd, hd)


def normed(x, g, hd, eps):
    """(n = x r, z = n g, r) of each head."""
    x = heads(x, hd)
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    return x * r, x * r * (1.0 if g is None else np.asarray(g, np.float64)), r


def pair_sums(a, rot, layout):
    """|a| of an element and of the one that it turns with; 0 where nothing turns."""
    a, p = np.abs(a), np.zeros_like(a)
    i, j = (slice(0, rot // 2), slice(rot // 2, rot)) if layout == "half" else (slice(0, rot, 2), slice(1, rot, 2))
    p[..., i] = p[..., j] = a[..., i] + a[..., j]
    return p


def norm_rope(x, g, hd, rot, pos, dtype, layout="half", eps=1e-6, mscale=0.0, **scaling):
    """(rows, the largest error of each element).  The sum of hd squares in fp32 is good
    to hd 2^-24, r to half of that and its own instruction's 2^-23; two products, 2^-24
    each: (hd / 2 + 6) 2^-24 in all; then the turn (serve_ref.rope_bound)."""
    _, z, _ = normed(x, g, hd, eps)
    flat = z.reshape(len(z), z.shape[1] * hd)
    y = R.rope(flat, z.shape[1], hd, rot, pos, layout, False, mscale, **scaling)
    m = mscale or R.frequencies(max(rot, 4), **scaling)[1]
    rel = (hd / 2 + 6) * 2.0 ** -24
    turn = pair_sums(z, rot, layout)
    err = HALF_ULP[dtype] * np.abs(y).reshape(z.shape) + (TRIG[dtype] + rel) * abs(m) * turn + 1.01 * rel * np.abs(z)
    return y, err.reshape(y.shape) + 1e-30


def norm_rope_bwd(dy, x, g, hd, rot, pos, dtype, layout="half", eps=1e-6, mscale=0.0, **scaling):
    """((dx, its largest error), (dg, its largest error)).  As for the forward; the mean is a
    sum of hd products (hd 2^-24 of their magnitudes), dg one of all rows and heads."""
    n, _, r = normed(x, g, hd, eps)
    m = mscale or R.frequencies(max(rot, 4), **scaling)[1]
    dz = R.rope(dy, n.shape[1], hd, rot, pos, layout, True, mscale, **scaling).reshape(n.shape)
    gain = 1.0 if g is None else np.asarray(g, np.float64)
    w = dz * gain
    mean = (w * n).mean(-1, keepdims=True)
    dx = r * (w - n * mean)
    dz_err = TRIG[dtype] * abs(m) * pair_sums(heads(dy, hd), rot, layout)
    w_err = dz_err * np.abs(gain)
    size = np.abs(w) + np.abs(n) * (np.abs(w) * np.abs(n)).mean(-1, keepdims=True)
    err = r * (w_err + np.abs(n) * (w_err * np.abs(n)).mean(-1, keepdims=True)) + r * size * (2 * hd + 16) * 2.0 ** -24
    err = 1.01 * err + HALF_ULP[dtype] * np.abs(dx) + 1e-30
    terms = n.shape[0] * n.shape[1]
    dg = (dz * n).sum((0, 1))
    dg_err = 1.01 * ((dz_err * np.abs(n)).sum((0, 1)) + np.abs(dz * n).sum((0, 1)) * (terms + hd / 2 + 8) * 2.0 ** -24) + 1e-30
    return (dx.reshape(len(n), -1), err.reshape(len(n), -1)), (dg, dg_err)


def tree_map(parent, kv_len, start, T, max_new, pos0):
    """(masks as whole numbers, positions), node by node."""
    masks, positions = [0] * T, [0] * T
    for r, kv in enumerate(kv_len):
        n = start[r + 1] - start[r]
        for i in range(min(n, max_new)):
            t = start[r] + i
            if t >= T:
                break
            p = int(parent[t])
            masks[t] = 1 << i | (masks[start[r] + p] if 0 <= p < i else 0)
            positions[t] = min(max(pos0 + int(kv) - n + bin(masks[t]).count("1") - 1, 0), 2 ** 31 - 1)
    return masks, positions


def words(masks, max_new):
    """Whole numbers as rows of int64 words."""
    w = -(-max_new // 64)
    return np.array([[m >> 64 * i & 2 ** 64 - 1 for i in range(w)] for m in masks], dtype=np.uint64).reshape(-1, w).view(np.int64)


def random_tree(rng, n, roots=1):
    """Parents: the first `roots` nodes have none, the others an earlier one."""
    return [-1 if i < roots else int(rng.integers(0, i)) for i in range(n)]


def attention(q, K, V, hq, prefix_table, prefix_len, table, kv_len, start, page, masks, scale=None, max_kv=None):
    """serve_ref.attention whose rows see of their request's new tokens those in their mask."""
    n_pages, hk, _, hd = K.shape
    T, g = len(q), hq // hk
    scale = 1.0 / math.sqrt(hd) if scale is None else scale
    q = np.array(q, dtype=np.float64).reshape(T, hq, hd)
    out, weight, lse = np.full((T, hq, hd), np.nan), np.full((T, hq, hd), np.nan), np.full((hq, T), np.nan)

    def rows(tab, n):
        at = [(int(tab[j // page]), j % page, j) for j in range(n)]
        return [x for x in at if 0 <= x[0] < n_pages]

    shared = rows(prefix_table, prefix_len)
    for r in range(len(start) - 1):
        n = start[r + 1] - start[r]
        kv = max(int(kv_len[r]), 0) if len(kv_len) else 0
        own = rows(table[r], kv if max_kv is None else min(kv, max_kv))
        for i in range(n):
            t = start[r] + i
            if t >= T:
                break
            seen = shared + [x for x in own if x[2] < kv - n or masks[t] >> (x[2] - (kv - n)) & 1]
            if not seen:
                out[t], weight[t], lse[:, t] = 0.0, 0.0, -np.inf
                continue
            p, o = np.array([x[0] for x in seen]), np.array([x[1] for x in seen])
            for h in range(hk):
                Kh, Vh = K[p, h, o].astype(np.float64), V[p, h, o].astype(np.float64)
                x = slice(h * g, (h + 1) * g)
                s = q[t, x] @ Kh.T * scale
                m = s.max(-1, keepdims=True)
                e = np.exp(s - m)
                l = e.sum(-1, keepdims=True)
                out[t, x], weight[t, x] = e / l @ Vh, e / l @ np.abs(Vh)
                lse[x, t] = (m + np.log(l))[:, 0]
    return out.reshape(T, hq * hd), lse, weight.reshape(T, hq * hd)


def logits(l, start, V, history=None, prompt_len=None, hist_len=None, draft=None, masks=None, repetition=None, presence=None,
           frequency=None, bias_start=None, bias_token=None, bias=None, allowed=None, allowed_row=None, dtype="f32"):
    """(rows, the largest error of each element, which elements a rule touches).  Rows of no
    request are NaN.  At most five fp32 roundings, each of half a step of what is
    there, and the result's."""
    T = len(l)
    y, err, touched = np.full((T, V), np.nan), np.zeros((T, V)), np.zeros((T, V), bool)
    for r in range(len(start) - 1):
        end = 0 if hist_len is None or history is None else min(max(int(hist_len[r]), 0), history.shape[1])
        past = 0 if prompt_len is None else min(max(int(prompt_len[r]), 0), end)
        for t in range(max(start[r], 0), min(start[r + 1], T)):
            x = np.array(l[t], dtype=np.float64)
            prompt, count = np.zeros(V, bool), np.zeros(V)
            for j in range(end):
                v = int(history[r, j])
                if 0 <= v < V:
                    if j < past:
                        prompt[v] = True
                    else:
                        count[v] += 1
            if draft is not None:
                for j in range(min(start[r + 1], T) - start[r]):
                    v = int(draft[start[r] + j])
                    if masks[t] >> j & 1 and 0 <= v < V:
                        count[v] += 1
            rep = 1.0 if repetition is None else float(repetition[r])
            f = 0.0 if frequency is None else float(frequency[r])
            p = 0.0 if presence is None else float(presence[r])
            seen = prompt | (count > 0)
            if repetition is None and presence is None and frequency is None:
                seen[:] = False
                count[:] = 0
            with np.errstate(invalid="ignore"):
                x = np.where(seen, np.where(x > 0, x / rep, x * rep), x)
                size = np.abs(x) + abs(f) * count + abs(p)
                x = np.where(count > 0, x - f * count - p, x)
                touched[t] |= seen
                if bias_start is not None:
                    lo = min(max(int(bias_start[r]), 0), len(bias))
                    hi = min(max(int(bias_start[r + 1]), lo), len(bias))
                    last = {int(bias_token[j]): float(bias[j]) for j in range(lo, hi)}
                    for v, b in last.items():
                        if 0 <= v < V:
                            x[v] += b
                            size[v] += abs(b)
                            touched[t, v] = True
                e = 5 * 2.0 ** -24 * size + HALF_ULP[dtype] * np.abs(x) + 1e-30
            if allowed is not None:
                s = t if allowed_row is None else int(allowed_row[t])
                if 0 <= s < len(allowed):
                    bits = np.unpackbits(np.asarray(allowed[s], dtype="<u4").view(np.uint8), bitorder="little")[:V]
                    hidden = bits == 0
                    x[hidden], e[hidden], touched[t, hidden] = -np.inf, 0.0, True
            y[t], err[t] = x, e
    return y, err, touched
