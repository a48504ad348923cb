"""Head norms, drafted trees and rules on logits on the GPU against their definitions in 64
bits (tests/verify_ref.py), element by element within the bounds derived there: odd
and smallest sizes, layouts, far positions, strides and alignments, masks that leave
nothing, infinities and NaN in masked places, batches cut at their rows, bounds above
and below the lengths; gradients against the formula's and against differences;
streams, graphs, workspace contents; and a run of them together as a program uses
them."""
import math

import numpy as np
import pytest
import torch

import serve_ref as R
import verify_ref as W
from paper_2502_10940_amd import cola
from test_gpu_serve import ATTN, DEV, DT, KERNELS, ROPE, SCALINGS, Batch, f64, i32, pitched, rand

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _device():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    cola.lib()
    yield


def gain(seed, hd, dtype):
    return (1.0 + 0.3 * rand(seed, (hd,), "f32")).to(DT[dtype])


def workspace(d, fill=0xFF):
    return torch.full((cola.norm_rope_workspace_bytes(d),), fill, dtype=torch.uint8, device=DEV)


# ---------------------------------------------------------------------------
# norms
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("layout", ("half", "interleaved"))
@pytest.mark.parametrize("dtype", ("bf16", "f32"))
@pytest.mark.parametrize("case", range(len(ROPE)), ids=["%dx%d+%dx%d-%d" % c for c in ROPE])
def test_norm_rope(case, dtype, layout):
    """Both directions, gains given and not."""
    T, hq, hk, hd, rot = ROPE[case]
    name = sorted(SCALINGS)[case % len(SCALINGS)]
    if name == "base" and rot <= 2:
        name = "linear"
    sc = dict(SCALINGS[name], base=500000.0 if case % 2 else 10000.0)
    rng = np.random.default_rng(200 + case)
    pos = rng.integers(0, 1 << 20, T)
    pos[0] = (2 ** 31 - 1) if case % 2 else -5
    m = 1.25 if case % 3 == 0 else 0.0
    eps = 1e-6 if case % 2 else 0.37
    d = cola.rope_desc(T, hq, hk, hd, rot, dtype, layout, name, mscale=m, **sc)
    kw = dict(layout=layout, eps=eps, mscale=m, scaling=name, **sc)
    x = {n: rand(case + i, (T, max(h, 1) * hd), dtype) for i, (n, h) in enumerate((("q", hq), ("k", hk)))}
    dy = {n: rand(case + 70 + i, (T, max(h, 1) * hd), dtype) for i, (n, h) in enumerate((("q", hq), ("k", hk)))}
    g = {"q": gain(case, hd, dtype), "k": gain(case + 9, hd, dtype)}
    if case % 4 == 3:
        g["k" if case % 8 == 3 else "q"] = None
    there = {"q": hq > 0, "k": hk > 0}
    pick = lambda t, n: t if there[n] else None
    out = {n: torch.full_like(x[n], math.nan) for n in "qk"}
    cola.norm_rope_fwd(d, pick(x["q"], "q"), pick(x["k"], "k"), g["q"], g["k"], i32(pos), pick(out["q"], "q"), pick(out["k"], "k"), eps=eps)
    dx = {n: torch.full_like(x[n], math.nan) for n in "qk"}
    dg = {n: torch.full((hd,), math.nan, device=DEV) for n in "qk"}
    cola.norm_rope_bwd(d, pick(dy["q"], "q"), pick(dy["k"], "k"), pick(x["q"], "q"), pick(x["k"], "k"), g["q"], g["k"], i32(pos),
                       pick(dx["q"], "q"), pick(dx["k"], "k"), pick(dg["q"], "q"), pick(dg["k"], "k"), workspace(d), eps=eps)
    torch.cuda.synchronize()
    for n in "qk":
        if not there[n]:
            assert torch.isnan(out[n]).all() and torch.isnan(dx[n]).all() and torch.isnan(dg[n]).all()
            continue
        gn = None if g[n] is None else f64(g[n])
        ref, bound = W.norm_rope(f64(x[n]), gn, hd, rot, pos, dtype, **kw)
        err = np.abs(f64(out[n]) - ref)
        assert (err <= bound).all(), (n, (err / bound).max())
        (rx, bx), (rg, bg) = W.norm_rope_bwd(f64(dy[n]), f64(x[n]), gn, hd, rot, pos, dtype, **kw)
        err = np.abs(f64(dx[n]) - rx)
        assert (err <= bx).all(), (n, (err / bx).max())
        err = np.abs(f64(dg[n]) - rg)
        assert (err <= bg).all(), (n, (err / bg).max())


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
def test_norm_rope_of_zeros_at_the_least_eps(dtype):
    """2^-126, the smallest eps there is: a head of zeros gives zeros, and gradients of
    dz 2^63 (exact; the hardware's 1 / sqrt is off by an ulp of 2^-23, the result is
    rounded)."""
    T, h, hd = 5, 3, 64
    d = cola.rope_desc(T, h, 0, hd, 0, dtype=dtype)                      # nothing turns
    q, dy = torch.zeros(T, h * hd, dtype=DT[dtype], device=DEV), rand(1, (T, h * hd), dtype)
    out, dx = torch.full_like(q, math.nan), torch.full_like(q, math.nan)
    dg = torch.full((hd,), math.nan, device=DEV)
    cola.norm_rope_fwd(d, q, None, None, None, None, out, None, eps=2.0 ** -126)
    cola.norm_rope_bwd(d, dy, None, q, None, None, None, None, dx, None, dg, None, workspace(d), eps=2.0 ** -126)
    torch.cuda.synchronize()
    assert (out == 0).all() and (dg == 0).all()
    want = f64(dy) * 2.0 ** 63
    tol = 2.0 ** -22 + torch.finfo(DT[dtype]).eps / 2
    assert (np.abs(f64(dx) - want) <= tol * np.abs(want)).all()


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
@pytest.mark.parametrize("layout", ("half", "interleaved"))
def test_norm_rope_pitches_alignment_and_in_place(dtype, layout):
    """Slices of one buffer at an odd pitch and start: the bits of tight rows, nothing else
    touched; in place too, in both directions."""
    T, hq, hk, hd, seq = 37, 4, 2, 64, 10
    q, k, dq, dk = (rand(i, (T, h * hd), dtype) for i, h in enumerate((hq, hk, hq, hk)))
    gq, gk = gain(5, hd + 3, dtype)[3:].clone(), gain(6, hd + 3, dtype)[3:]      # the second 3 elements off
    want = [torch.empty_like(q), torch.empty_like(k)]
    d = cola.rope_desc(T, hq, hk, hd, dtype=dtype, layout=layout, seq_len=seq)
    cola.norm_rope_fwd(d, q, k, gq, gk, None, *want)
    back = [torch.empty_like(q), torch.empty_like(k)]
    dg = [torch.empty(hd, device=DEV) for _ in range(2)]
    cola.norm_rope_bwd(d, dq, dk, q, k, gq, gk, None, *back, *dg, workspace(d))
    for ldi, ldk, off in ((hq * hd + hk * hd, hq * hd + hk * hd, 8), (hq * hd + 3, hk * hd + 1, 1), (hq * hd + 37, hk * hd, 5)):
        (pq, bq), (pk, bk) = pitched(q, ldi, off), pitched(k, ldk, off)
        oq, ob = pitched(torch.zeros_like(q), hq * hd + 5, 3)
        ok, okb = pitched(torch.zeros_like(k), hk * hd + 7, 1)
        d = cola.rope_desc(T, hq, hk, hd, dtype=dtype, layout=layout, seq_len=seq, ldq=ldi, ldk=ldk, ldqo=hq * hd + 5, ldko=hk * hd + 7)
        cola.norm_rope_fwd(d, pq, pk, gq, gk, None, oq, ok)
        assert torch.equal(oq, want[0]) and torch.equal(ok, want[1])
        for b, n in ((ob, q), (okb, k)):
            assert torch.isnan(b).sum() == b.numel() - n.numel()         # the padding stayed
        # the gradients' rows at the outputs' pitches, results over the inputs
        oq.copy_(dq), ok.copy_(dk)
        got = [torch.empty(hd, device=DEV) for _ in range(2)]
        cola.norm_rope_bwd(d, oq, ok, pq, pk, gq, gk, None, pq, pk, *got, workspace(d))
        assert torch.equal(pq, back[0]) and torch.equal(pk, back[1])
        assert all(torch.equal(a, b) for a, b in zip(got, dg))
        for b, n in ((bq, q), (bk, k)):
            assert torch.isnan(b).sum() == b.numel() - n.numel()
        pq.copy_(q), pk.copy_(k)
        d = cola.rope_desc(T, hq, hk, hd, dtype=dtype, layout=layout, seq_len=seq, ldq=ldi, ldk=ldk, ldqo=ldi, ldko=ldk)
        cola.norm_rope_fwd(d, pq, pk, gq, gk, None, pq, pk)
        assert torch.equal(pq, want[0]) and torch.equal(pk, want[1])
    # over the gradients' rows
    d = cola.rope_desc(T, hq, hk, hd, dtype=dtype, layout=layout, seq_len=seq)
    a, b = dq.clone(), dk.clone()
    cola.norm_rope_bwd(d, a, b, q, k, gq, gk, None, a, b, None, None, workspace(d))
    assert torch.equal(a, back[0]) and torch.equal(b, back[1])


@pytest.mark.parametrize("layout", ("half", "interleaved"))
def test_norm_gradient_against_differences(layout):
    """<dx, e> + <dg, f> against a central difference of <y, c> along (e, f) on the GPU, in
    fp32: what the same difference of the 64-bit forward is off, and the roundings of
    the two forwards (2^-20 of a pair's magnitudes in each element) over the step."""
    T, h, hd, rot = 6, 2, 32, 24
    x, e, c = (rand(s, (T, h * hd), "f32") for s in (1, 2, 3))
    g, f = gain(4, hd, "f32"), rand(5, (hd,), "f32")
    pos = [0, 1, 5, 100, 70000, 3]
    d = cola.rope_desc(T, h, 0, hd, rot, "f32", layout)
    s = 2.0 ** -5
    y = []
    for k in (s, -s):
        out = torch.empty_like(x)
        cola.norm_rope_fwd(d, x + k * e, None, g + k * f, None, i32(pos), out, None)
        y.append((f64(out) * f64(c)).sum())
    dx, dg = torch.empty_like(x), torch.empty(hd, device=DEV)
    cola.norm_rope_bwd(d, c, None, x, None, g, None, i32(pos), dx, None, dg, None, workspace(d))
    grad = (f64(dx) * f64(e)).sum() + (f64(dg) * f64(f)).sum()
    ref = lambda k: (W.norm_rope(f64(x + k * e), f64(g + k * f), hd, rot, pos, "f32", layout)[0] * f64(c)).sum()
    (rx, bx), (rg, bg) = W.norm_rope_bwd(f64(c), f64(x), f64(g), hd, rot, pos, "f32", layout)
    exact = (rx * f64(e)).sum() + (rg * f64(f)).sum()
    cut = abs((ref(s) - ref(-s)) / (2 * s) - exact)
    _, yb = W.norm_rope(f64(x), f64(g), hd, rot, pos, "f32", layout)
    rounding = 2 * 1.2 * (yb * np.abs(f64(c))).sum() / (2 * s)
    own = (bx * np.abs(f64(e))).sum() + (bg * np.abs(f64(f))).sum()
    assert abs((y[0] - y[1]) / (2 * s) - grad) <= cut + rounding + own


def test_norm_rope_of_no_rows_and_no_gains():
    d = cola.rope_desc(0, 2, 2, 64)
    dg = [torch.full((64,), 7.0, device=DEV) for _ in range(2)]
    x = torch.zeros((0, 128), dtype=torch.bfloat16, device=DEV)
    cola.norm_rope_bwd(d, x, x, x, x, None, None, None, x, x, *dg, None)
    assert all((t == 0).all() for t in dg)
    cola.norm_rope_fwd(d, x, x, None, None, None, x, x)


@pytest.mark.parametrize("value", (0.0, math.inf, math.nan, 3.0e38))
def test_norm_rope_rows_do_not_reach_each_other(value):
    """A head of zeros gives zeros and finite gradients; one of anything else leaves the rows
    and heads beside it as they are."""
    T, h, hd = 21, 4, 64
    q, dy, g = rand(1, (T, h * hd), "bf16"), rand(2, (T, h * hd), "bf16"), gain(3, hd, "bf16")
    d = cola.rope_desc(T, h, 0, hd)

    def both(q):
        out, dx = torch.empty_like(q), torch.empty_like(q)
        dg = torch.empty(hd, device=DEV)
        cola.norm_rope_fwd(d, q, None, g, None, None, out, None)
        cola.norm_rope_bwd(d, dy, None, q, None, g, None, None, dx, None, dg, None, workspace(d))
        return out, dx, dg

    a = both(q)
    z = q.clone()
    z[5, hd:2 * hd] = value
    b = both(z)
    keep = torch.ones_like(q, dtype=torch.bool)
    keep[5, hd:2 * hd] = False
    for u, v in zip(a[:2], b[:2]):
        assert torch.equal(u[keep], v[keep])
    if value == 0.0:
        assert (b[0][5, hd:2 * hd] == 0).all() and all(torch.isfinite(t.float()).all() for t in b)


@pytest.mark.parametrize("dtype, layout", [("bf16", "half"), ("bf16", "interleaved"), ("f32", "half")])
def test_large_norm_results_are_the_small_ones(dtype, layout):
    """Sizes whose results go past the caches: every row has the bits that a small call
    gives it, and dg is within its bound."""
    T, hq, hk, hd = 9001, 24, 8, 128
    q, k, dq, dk = (rand(i, (T, h * hd), dtype) for i, h in enumerate((hq, hk, hq, hk)))
    gq, gk = gain(5, hd, dtype), gain(6, hd, dtype)
    pos = torch.randint(0, 1 << 20, (T,), device=DEV, dtype=torch.int32)
    o = [torch.empty_like(q), torch.empty_like(k)]
    dx = [torch.empty_like(q), torch.empty_like(k)]
    dg = [torch.empty(hd, device=DEV) for _ in range(2)]
    d = cola.rope_desc(T, hq, hk, hd, dtype=dtype, layout=layout)
    cola.norm_rope_fwd(d, q, k, gq, gk, pos, *o)
    cola.norm_rope_bwd(d, dq, dk, q, k, gq, gk, pos, *dx, *dg, workspace(d))
    for lo, n in ((0, 3), (4000, 17), (T - 5, 5)):
        part = [t[lo:lo + n].clone() for t in (q, k, dq, dk, pos)]
        s = [torch.empty_like(part[0]), torch.empty_like(part[1])]
        sd = cola.rope_desc(n, hq, hk, hd, dtype=dtype, layout=layout)
        cola.norm_rope_fwd(sd, part[0], part[1], gq, gk, part[4], *s)
        assert all(torch.equal(a[lo:lo + n], b) for a, b in zip(o, s))
        cola.norm_rope_bwd(sd, part[2], part[3], part[0], part[1], gq, gk, part[4], *s, None, None, workspace(sd))
        assert all(torch.equal(a[lo:lo + n], b) for a, b in zip(dx, s))
    p = pos.cpu().numpy()
    for y, x, g, got in ((dq, q, gq, dg[0]), (dk, k, gk, dg[1])):
        _, (ref, bound) = W.norm_rope_bwd(f64(y), f64(x), f64(g), hd, hd, p, dtype, layout)
        # 2^18 terms at random signs: far inside the bound, which takes the worst order
        assert (np.abs(f64(got) - ref) <= bound).all() and np.abs(f64(got) - ref).max() < 2.0 ** -12 * np.abs(ref).max()


# rows of many heads, an odd number of them; single rows; one element a head
@pytest.mark.parametrize("T, hq, hk, hd, rot", [(1, 4099, 3, 64, 64), (3, 1025, 1026, 8, 8), (2, 70001, 5, 1, 0), (5, 129, 700, 80, 40), (1, 1, 9001, 3, 2)])
def test_norm_rope_of_many_heads(T, hq, hk, hd, rot):
    q, k, dq, dk = (rand(i, (T, h * hd), "bf16") for i, h in enumerate((hq, hk, hq, hk)))
    gq, gk = gain(5, hd, "bf16"), gain(6, hd, "bf16")
    pos = np.random.default_rng(T).integers(0, 5000, T)
    d = cola.rope_desc(T, hq, hk, hd, rot)
    o, dx, dg = [torch.empty_like(q), torch.empty_like(k)], [torch.empty_like(q), torch.empty_like(k)], [torch.empty(hd, device=DEV) for _ in range(2)]
    cola.norm_rope_fwd(d, q, k, gq, gk, i32(pos), *o)
    cola.norm_rope_bwd(d, dq, dk, q, k, gq, gk, i32(pos), *dx, *dg, workspace(d))
    for x, dy, g, y, u, v in ((q, dq, gq, o[0], dx[0], dg[0]), (k, dk, gk, o[1], dx[1], dg[1])):
        ref, bound = W.norm_rope(f64(x), f64(g), hd, rot, pos, "bf16")
        assert (np.abs(f64(y) - ref) <= bound).all()
        (rx, bx), (rg, bg) = W.norm_rope_bwd(f64(dy), f64(x), f64(g), hd, rot, pos, "bf16")
        assert (np.abs(f64(u) - rx) <= bx).all() and (np.abs(f64(v) - rg) <= bg).all()


def test_norm_rope_past_4_gib():
    """Rows at a pitch that puts the last ones past 2^32 bytes: the bits of tight rows, both ways."""
    T, h, hd, ld = 1100, 2, 64, (1 << 21) + 8
    x, dy, g = rand(1, (T, h * hd), "bf16"), rand(2, (T, h * hd), "bf16"), gain(3, hd, "bf16")
    d, far = cola.rope_desc(T, h, 0, hd), cola.rope_desc(T, h, 0, hd, ldq=ld)
    want, dx, dg = torch.empty_like(x), torch.empty_like(x), torch.empty(hd, device=DEV)
    cola.norm_rope_fwd(d, x, None, g, None, None, want, None)
    cola.norm_rope_bwd(d, dy, None, x, None, g, None, None, dx, None, dg, None, workspace(d))
    big, _ = pitched(x, ld, fill=0.0)
    out, dg2 = torch.empty_like(x), torch.empty(hd, device=DEV)
    cola.norm_rope_fwd(far, big, None, g, None, None, out, None)
    assert torch.equal(out, want)
    cola.norm_rope_bwd(far, dy, None, big, None, g, None, None, big, None, dg2, None, workspace(far))
    assert torch.equal(big, dx) and torch.equal(dg2, dg)


def test_norm_gradients_do_not_depend_on_the_workspace_s_contents_or_the_run():
    T, hq, hk, hd = 700, 5, 3, 96
    q, k, dq, dk = (rand(i, (T, h * hd), "bf16") for i, h in enumerate((hq, hk, hq, hk)))
    gq, gk = gain(5, hd, "bf16"), gain(6, hd, "bf16")
    d = cola.rope_desc(T, hq, hk, hd, 48)
    got = []
    for fill in (0, 0xFF, 0x7F, 0):
        o = [torch.empty_like(q), torch.empty_like(k), torch.empty(hd, device=DEV), torch.empty(hd, device=DEV)]
        cola.norm_rope_bwd(d, dq, dk, q, k, gq, gk, None, *o, workspace(d, fill))
        got.append(o)
    assert all(torch.equal(a, b) for o in got[1:] for a, b in zip(got[0], o))


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
@pytest.mark.parametrize("case", [(1, 1, 1, 64, 64, 16), (19, 8, 2, 128, 128, 32), (33, 5, 5, 80, 40, 16), (7, 0, 3, 33, 0, 64),
                                  (300, 16, 4, 64, 64, 128)], ids=str)
def test_norm_append(case, dtype):
    """As norm_rope_fwd's rows, in their slots; rows without a slot, and slots without a row, are left."""
    T, hq, hk, hd, rot, page = case
    pages = -(-T // page) + 2
    q, k, v = (rand(i, (T, max(h, 1) * hd), dtype) for i, h in enumerate((hq, hk, hk)))
    gq, gk = gain(4, hd, dtype), gain(5, hd, dtype)
    rng = np.random.default_rng(T)
    slots = rng.permutation(pages * page)[:T]
    bad = rng.random(T) < 0.2
    slots[bad] = rng.choice([-1, pages * page, 2 ** 31 - 1, -2 ** 31], bad.sum())
    pos = rng.integers(0, 1 << 17, T)
    K, V = (rand(9 + i, (pages, hk, page, hd), dtype) for i in range(2))
    K0, V0 = K.clone(), V.clone()
    qo = torch.full_like(q, math.nan)
    d = cola.rope_desc(T, hq, hk, hd, rot, dtype)
    c = cola.cache_desc(pages, page, hk, hd, dtype)
    cola.norm_append(d, c, q if hq else None, k, v, gq, gk, i32(pos), i32(slots), qo if hq else None, K, V)
    want = [torch.empty_like(q), torch.empty_like(k)]
    cola.norm_rope_fwd(d, q if hq else None, k, gq, gk, i32(pos), want[0] if hq else None, want[1])
    if hq:
        assert torch.equal(qo, want[0])
    for t in range(T):
        if not bad[t]:
            K0[slots[t] // page, :, slots[t] % page] = want[1][t].view(hk, hd)
            V0[slots[t] // page, :, slots[t] % page] = v[t].view(hk, hd)
    assert torch.equal(K, K0) and torch.equal(V, V0)


# ---------------------------------------------------------------------------
# trees
# ---------------------------------------------------------------------------

def run_tree_map(parent, kv, start, T, max_new, pos0):
    w = -(-max_new // 64)
    mask = torch.full((T, w), -7, dtype=torch.int64, device=DEV)
    pos = torch.full((T,), -7, dtype=torch.int32, device=DEV)
    n = T if start is None else len(start) - 1
    cola.tree_map(cola.tree_map_desc(n, T, max_new, pos0), i32(parent), i32(kv), None if start is None else i32(start), mask, pos)
    torch.cuda.synchronize()
    m, p = W.tree_map(parent, kv, list(range(T + 1)) if start is None else start, T, max_new, pos0)
    assert np.array_equal(mask.cpu().numpy(), W.words(m, max_new)) and pos.cpu().tolist() == p


@pytest.mark.parametrize("max_new", (1, 2, 63, 64, 65, 128, 129, 200, 256))
@pytest.mark.parametrize("n_req", (1, 5, 300))
def test_tree_map(n_req, max_new):
    rng = np.random.default_rng(n_req + max_new)
    new = rng.integers(0, max_new + 1, n_req)
    new[0] = max_new
    start = np.concatenate([[3], 3 + np.cumsum(new)])
    T = int(start[-1]) + 5
    parent = rng.integers(-3, 300, T)                                 # rows of no request hold anything
    for r, n in enumerate(new):
        parent[start[r]:start[r] + n] = list(range(-1, n - 1)) if r == 1 else W.random_tree(rng, n, 1 + r % 2)
    run_tree_map(parent, rng.integers(0, 5000, n_req) + new, start, T, max_new, 77)


def test_tree_map_edges():
    rng = np.random.default_rng(0)
    # parents that are none: the node itself, a later one, anything
    run_tree_map([0, 5, 1, -9, 2 ** 31 - 1, -2 ** 31, 4], [7], [0, 7], 7, 7, 0)
    # more nodes than max_new, and than rows; a chain; kv_len below the nodes; positions at the ends of their range
    chain = list(range(-1, 99))
    run_tree_map(chain, [100], [0, 100], 100, 70, 0)
    run_tree_map(chain[:40], [100], [0, 100], 40, 100, 3)
    run_tree_map(chain, [3], [0, 100], 100, 100, 0)
    run_tree_map(chain, [2 ** 31 - 1], [0, 100], 100, 128, 2 ** 31 - 1)
    # a row each; nothing at all
    run_tree_map(rng.integers(-2, 3, 9), rng.integers(1, 9, 9), None, 9, 4, 5)
    run_tree_map([1, 2, 3], [], [0], 3, 64, 0)
    run_tree_map([1, 2, 3], [5, 5], [3, 3, 3], 3, 200, 0)


class TreeBatch(Batch):
    """A batch whose new tokens see each other by masks: whole numbers, a bit for each."""

    def __init__(self, *a, masks="trees", **kw):
        super().__init__(*a, **kw)
        rng = np.random.default_rng(a[0] + 1000)
        self.masks = [0] * self.T
        for r, n in enumerate(self.new):
            parent = W.random_tree(rng, n, 1 + r % 3)
            for i in range(n):
                t = self.start[r] + i
                up = self.masks[self.start[r] + parent[i]] if parent[i] >= 0 else 0
                self.masks[t] = {"trees": up | 1 << i, "chains": (2 << i) - 1,
                                 "any": int(rng.integers(0, 2 ** 62)) * 2 ** 200 // 3 ** int(rng.integers(0, 90)) % 2 ** n if (i + r) % 4 else 0}[masks]
                if masks == "any":                                    # bits that have no token
                    self.masks[t] |= 2 ** (64 * (-(-self.max_new // 64))) - 2 ** min(n, 64 * (-(-self.max_new // 64)))

    def run(self, ws_fill=0xFF, lse=True, start=True, stream=None):
        d, c = self.desc()
        q = self.q if not self.ldq else pitched(self.q, self.ldq, 8)[0]
        out = torch.full((self.T, self.ldo or self.hq * self.hd), 7.0, dtype=torch.bfloat16, device=DEV)
        ls = torch.full((self.hq, self.T), 7.0, device=DEV) if lse else None
        n = cola.tree_attn_workspace_bytes(d, c)
        ws = torch.full((n,), ws_fill, dtype=torch.uint8, device=DEV) if n else None
        cola.tree_attn(d, c, q, self.K, self.V, i32(self.ptab) if self.L else None, i32(self.tab) if self.max_kv else None,
                       i32(self.kv) if self.max_kv else None, i32(self.start) if start else None,
                       torch.from_numpy(W.words(self.masks[:self.T], self.max_new)).to(DEV), out, ls, ws, stream=stream)
        torch.cuda.synchronize()
        return out, ls

    def reference(self):
        return W.attention(f64(self.q), f64(self.K), f64(self.V), self.hq, self.ptab, self.L, self.tab, self.kv, self.start, self.page,
                           self.masks, self.scale or None)


TREES = {k: v for k, v in KERNELS.items() if max(v[0]) <= 256}


@pytest.mark.parametrize("masks", ("trees", "any"))
@pytest.mark.parametrize("hd", (64, 128))
@pytest.mark.parametrize("name", sorted(TREES))
def test_tree_attention_kernels(name, hd, masks):
    new, kv, L, hq, hk = TREES[name]
    print("trees", name, hd, masks, flush=True)
    TreeBatch(len(name) + hd, new, kv, L, hq, hk, hd, 16 if hd == 64 else 64, pad=2, masks=masks).check()


@pytest.mark.parametrize("name", sorted(k for k in ATTN if max(ATTN[k]["new"]) <= 256))
def test_tree_attention(name):
    print("trees", name, ATTN[name], flush=True)
    TreeBatch(len(name), **ATTN[name]).check()


# trees that begin and end everywhere in a block of 32 and a stage of 64 keys
@pytest.mark.parametrize("hd, hq", [(64, 1), (128, 2), (64, 4), (128, 8)])
@pytest.mark.parametrize("n", (1, 2, 7, 16, 31, 32, 33, 63, 64, 65, 100, 129, 255, 256))
def test_tree_attention_of_every_size_and_place(n, hd, hq):
    old = [0, 1, 31, 32, 63, 64, 65, 97]
    TreeBatch(n, [n] * len(old), [n + o for o in old], 0, hq, 1, hd, 16, masks="any" if n % 2 else "trees").check()


@pytest.mark.parametrize("name", ("along-one", "along-two", "along-wide", "one-one", "two-two", "wide-wide", "wide-two", "parts-own"))
def test_a_chain_sees_what_causal_rows_see(name):
    """Within the bounds of both; up to 32 rows of a head the kernels are the same, and so are the bits."""
    new, kv, L, hq, hk = TREES[name]
    b = TreeBatch(3, new, kv, L, hq, hk, 64, 16, masks="chains")
    out, lse = b.check()
    want, wl = Batch.run(b)
    if max(new) * hq // hk <= 32:
        assert torch.equal(out, want) and torch.equal(lse, wl)


# Few requests with long caches: parts cut by the lengths, under bounds near and far; the
# largest number of requests that are counted, and one more; and kinds that no other case has
CUT = {"near": ([40, 100, 7], [5000, 300, 7000], 0, 2, 1, None), "far": ([40, 100, 7], [5000, 300, 7000], 0, 2, 1, 60000),
       "empty": ([129, 0, 35], [3000, 40, 35], 0, 1, 1, 9000), "prefix": ([70, 33], [2500, 6000], 1300, 2, 2, None), "one": ([200], [9000], 0, 4, 2, None),
       "mixed": ([34, 256, 1, 90], [34, 4000, 5000, 90], 0, 1, 1, None), "256": ([5] * 255 + [36], [5 + 3 * i for i in range(255)] + [1500], 0, 1, 1, 4000),
       "257": ([5] * 256 + [36], [5 + i for i in range(256)] + [1500], 0, 1, 1, 4000), "wide": ([100, 80], [5000, 3000], 0, 1, 1, None),
       "wide-prefix": ([100, 80], [900, 300], 1300, 1, 1, None), "tiles-prefix": ([200, 180], [500, 700], 1300, 1, 1, None),
       "along-four": ([40, 60, 9], [70, 60, 30], 90, 1, 1, None), "along-tiles": ([200, 150], [220, 150], 90, 1, 1, None), "four-prefix": ([40, 9], [900, 300], 1300, 1, 1, None),
       "tiles-many": ([130] * 40, [130 + 20 * i for i in range(40)], 0, 8, 8, None),
       "wide-direct": ([70, 80], [200, 90], 0, 1, 1, None), "tiles-direct": ([150, 80], [200, 90], 0, 1, 1, None)}


@pytest.mark.parametrize("hd", (64, 128))
@pytest.mark.parametrize("name", sorted(CUT))
def test_tree_attention_cut_by_the_lengths(name, hd):
    new, kv, L, hq, hk, max_kv = CUT[name]
    print("trees", name, hd, flush=True)
    TreeBatch(40 + hd, new, kv, L, hq, hk, hd, 64, masks="any", max_kv=max_kv, pad=3).check()


@pytest.mark.parametrize("hd", (64, 128))
def test_far_bounds_cut_trees_where_near_ones_do(hd):
    """A max_kv far above the lengths (a program's context length): the parts end where the lengths say, as under a bound
    that is the longest length, as long as the workspace has room for them."""
    cut = []
    for max_kv in (7000, 1 << 20):
        b = TreeBatch(60 + hd, [40, 100, 7], [5000, 300, 7000], 0, 2, 1, hd, 64, max_kv=max_kv)
        b.check()
        d, c = b.desc()
        ws = torch.zeros(cola.tree_attn_workspace_bytes(d, c), dtype=torch.uint8, device=DEV)
        out, lse = torch.empty_like(b.q), torch.empty((b.hq, b.T), device=DEV)
        cola.tree_attn(d, c, b.q, b.K, b.V, None, i32(b.tab), i32(b.kv), i32(b.start), torch.from_numpy(W.words(b.masks, b.max_new)).to(DEV), out, lse, ws)
        cut.append((int(ws[-64:-60].view(torch.int32)[0]), out, lse))
    assert cut[0][0] == cut[1][0] == 256
    assert torch.equal(cut[0][1], cut[1][1]) and torch.equal(cut[0][2], cut[1][2])


def test_tree_attention_without_starts_pitches_and_scale():
    b = TreeBatch(1, [1] * 9, [4, 0, 17, 60, 33, 1, 16, 100, 12], 40, 4, 2, 64, 16, pad=3, ldq=4 * 64 + 24, ldo=4 * 64 + 8, scale=0.3)
    a, la = b.check()
    c, lc = b.check(start=False)
    assert torch.equal(a, c) and torch.equal(la, lc)
    d, _ = b.run(lse=False)
    assert torch.equal(a, d)


def test_tree_attention_bounds_above_the_lengths():
    kw = dict(new=[1, 3, 2], kv=[20, 65, 2], L=50, hq=4, hk=2, hd=64, page=16)
    for extra in (dict(max_kv=3000), dict(max_new=200), dict(max_kv=1000, max_new=256)):
        TreeBatch(7, **kw, **extra).check()


@pytest.mark.parametrize("max_kv", (3, 20, 40, 57))
def test_tree_attention_of_keys_past_max_kv(max_kv):
    """Tokens past max_kv are not seen, the tree's own among them."""
    b = TreeBatch(3, [20, 9], [60, 30], 0, 2, 2, 64, 16, masks="any")
    ref, rl, w = W.attention(f64(b.q), f64(b.K), f64(b.V), 2, [], 0, b.tab, b.kv, b.start, 16, b.masks, max_kv=max_kv)
    b.max_kv = max_kv
    b.tab = np.ascontiguousarray(b.tab[:, :-(-max_kv // 16)])
    out, lse = b.run()
    assert (np.abs(f64(out) - ref) <= R.attention_bound(ref, w, 60)).all()
    fin = np.isfinite(rl)
    assert (np.isneginf(f64(lse)) == ~fin).all() and (np.abs(f64(lse) - np.where(fin, rl, 0))[fin] <= R.lse_bound(rl[fin], 60)).all()


def test_tree_attention_rows_past_max_new_are_left():
    b = TreeBatch(4, [20, 9], [60, 30], 30, 2, 2, 64, 16)
    ref, _, w = b.reference()
    b.max_new = 12
    out, _ = b.run()
    keep = list(range(12)) + list(range(20, 29))
    assert (out[12:20] == 7).all()
    assert (np.abs(f64(out) - ref) <= R.attention_bound(ref, w, 90))[keep].all()


@pytest.mark.parametrize("hd", (64, 128))
@pytest.mark.parametrize("name, new, kv, L, rows", [("one", [2, 5], [9, 40], 0, 4), ("two", [5, 20], [9, 40], 1300, 12), ("wide", [30, 90], [60, 300], 0, 75),
                                                    ("past", [4, 9, 2], [4, 20, 2], 20, 4)])
def test_trees_of_a_batch_cut_at_its_rows(name, new, kv, L, rows, hd):
    """Nodes that have no row are still counted, and are in the cache for the rows that name them."""
    b = TreeBatch(30 + hd, new, kv, L, 2, 2, hd, 16, masks="any")
    ref, rl, w = b.reference()
    b.T, b.q = rows, b.q[:rows].contiguous()
    out, lse = b.run()
    keys = L + max(kv)
    assert (np.abs(f64(out) - ref[:rows]) <= R.attention_bound(ref, w, keys)[:rows]).all()
    fin = np.isfinite(rl[:, :rows])
    assert (np.abs(f64(lse) - np.where(fin, rl[:, :rows], 0))[fin] <= R.lse_bound(rl[:, :rows][fin], keys)).all()


@pytest.mark.parametrize("value", (math.inf, -math.inf, math.nan))
@pytest.mark.parametrize("new, hq", [([3, 5], 1), ([20, 9], 1), ([70, 30], 2)])
@pytest.mark.parametrize("hd", (64, 128))
def test_nodes_that_a_row_does_not_see_do_not_reach_it(new, hq, hd, value):
    """K and V of one node not finite: rows whose masks leave it out keep their bits."""
    b = TreeBatch(11, new, [n + 37 for n in new], 20, hq, 1, hd, 16)
    want, wl = b.run()
    for r, j in ((0, 1), (1, 0), (1, new[1] - 1), (0, new[0] // 2)):
        token = 37 + j
        page, at = int(b.tab[r, token // 16]), token % 16
        for c in (b.K, b.V):
            keep = c[page, :, at].clone()
            c[page, :, at] = value
            out, lse = b.run()
            hidden = [t for t in range(b.T) if not (b.start[r] <= t < b.start[r + 1] and b.masks[t] >> j & 1)]
            assert torch.equal(out[hidden], want[hidden]) and torch.equal(lse[:, hidden], wl[:, hidden])
            seen = [t for t in range(b.T) if t not in hidden]
            if c is b.V and not math.isnan(value):
                assert (out[seen] == value).all()
            elif math.isnan(value):
                assert torch.isnan(out[seen]).all()
            c[page, :, at] = keep


@pytest.mark.parametrize("bad", (-1, 10 ** 6, 2 ** 31 - 1, -2 ** 31))
@pytest.mark.parametrize("new, hq", [([3, 5], 1), ([20, 9], 1), ([70, 30], 2)])
def test_trees_over_missing_pages(new, hq, bad):
    b = TreeBatch(12, new, [n + 100 for n in new], 40, hq, 1, 64, 16, masks="any")
    b.tab[0, 1], b.tab[1, 100 // 16], b.tab[0, -(-b.kv[0] // 16) - 1] = bad, bad, bad
    b.check()


def test_tree_attention_past_4_gib():
    """Pages of a cache of more than 2^32 bytes, at its far end."""
    page, hk, hd = 128, 8, 128
    pages = (1 << 32) // (page * hk * hd * 2) + 40
    for new, kv in (([4], [300]), ([24], [300]), ([60], [300])):
        b = TreeBatch(13, new, kv, 0, hk, hk, hd, page)
        K, V = (torch.zeros((pages, hk, page, hd), dtype=torch.bfloat16, device=DEV) for _ in range(2))
        far = [pages - 1 - i for i in range(b.K.shape[0])]
        for big, small in ((K, b.K), (V, b.V)):
            big[far] = small
        want, wl = b.run()
        b.tab = np.where(b.tab >= 0, pages - 1 - b.tab, b.tab)
        b.K, b.V = K, V
        out, lse = b.run()
        assert torch.equal(out, want) and torch.equal(lse, wl)
        del K, V
        b.K = b.V = None


def test_tree_attention_does_not_depend_on_the_workspace_s_contents_or_the_run():
    b = TreeBatch(9, [3, 1, 20], [50, 600, 20], 700, 8, 2, 128, 16, pad=5)
    a = b.run(ws_fill=0)
    for fill in (0xFF, 0x7F, 0):
        c = b.run(ws_fill=fill)
        assert torch.equal(a[0], c[0]) and torch.equal(a[1], c[1])


# ---------------------------------------------------------------------------
# logits
# ---------------------------------------------------------------------------

class Rows:
    """Logits of a step and the rules on them, each left out where its name is in `without`."""

    def __init__(self, seed, rows, V, dtype, max_hist=60, n_bias=9, max_new=None, pad=0, lead=0, ldl=0, ldo=0, lda=0, without=(), states=5):
        rng = np.random.default_rng(seed)
        n = len(rows)
        self.start = [lead]
        for x in rows:
            self.start.append(self.start[-1] + x)
        self.T, self.V, self.dtype = self.start[-1] + pad, V, dtype
        self.max_new = max(list(rows) + [1]) if max_new is None else max_new
        self.l = rand(seed, (self.T, V), dtype, 3.0)
        token = lambda *s: np.where(rng.random(s) < 0.1, rng.choice([-1, V, 2 ** 31 - 1, -2 ** 31], s), rng.integers(0, min(V, 40), s) ** 2 % V)
        self.u = dict(history=token(n, max_hist), prompt_len=rng.integers(-2, max_hist + 3, n), hist_len=rng.integers(-2, max_hist + 3, n),
                      draft=token(self.T), repetition=np.float32(rng.choice([0.7, 1.0, 1.3], n)), presence=np.float32(rng.choice([0, 0.5, -0.25], n)),
                      frequency=np.float32(rng.choice([0, 0.4, 1.5], n)), bias_token=token(n * n_bias), bias=np.float32(rng.standard_normal(n * n_bias) * 4),
                      bias_start=np.concatenate([[-1 if seed % 2 else 0], np.sort(rng.integers(0, n * n_bias + 3, n))]),
                      allowed=rng.integers(0, 2 ** 32, (states, lda or -(-V // 32)), dtype=np.uint32), allowed_row=rng.integers(-1, states + 1, self.T))
        self.masks = [0] * self.T
        for r, k in enumerate(rows):
            parent = W.random_tree(rng, k)
            for i in range(k):
                t = self.start[r] + i
                self.masks[t] = (1 << i | (self.masks[self.start[r] + parent[i]] if parent[i] >= 0 else 0)) & (2 ** (64 * -(-self.max_new // 64)) - 1)
        for k in without:
            self.u.pop(k)
        if "bias_start" in without:
            self.u.pop("bias", None), self.u.pop("bias_token", None)
        self.ldl, self.ldo, self.lda, self.max_hist, self.n = ldl, ldo, lda, max_hist, n

    def tensors(self):
        u = {k: torch.from_numpy(v.view(np.int32).copy()).to(DEV) if k == "allowed" else torch.from_numpy(v).to(DEV) if v.dtype == np.float32 else i32(v)
             for k, v in self.u.items()}
        if "draft" in u:
            u["mask"] = torch.from_numpy(W.words(self.masks, self.max_new)).to(DEV)
        return u

    def desc(self, ldl=None, ldo=None):
        u = self.u
        return cola.logits_desc(self.T, self.V, self.n, self.max_hist, self.max_new, self.dtype, len(u.get("bias", ())), len(u.get("allowed", ())),
                                self.ldl if ldl is None else ldl, self.ldo if ldo is None else ldo, self.lda)

    def run(self, start=True, in_place=False, stream=None):
        l = pitched(self.l, self.ldl, 1)[0] if self.ldl else self.l.clone()
        out, buf = pitched(torch.full_like(self.l, 7.0), self.ldo, 3, fill=7.0) if self.ldo else (torch.full_like(self.l, 7.0), None)
        d = self.desc()
        if in_place:
            out, buf, d = l, None, self.desc(self.ldl, self.ldl)
        cola.logits_adjust(d, cola.logits_rules(**self.tensors()), l, i32(self.start) if start else None, out, stream=stream)
        torch.cuda.synchronize()
        if buf is not None:
            assert (buf == 7).sum() >= buf.numel() - out.numel(), "the padding is left"
        return out

    def check(self, **kw):
        out = self.run(**kw)
        kwargs = dict(self.u)
        if "draft" in kwargs:
            kwargs["masks"] = self.masks
        ref, bound, touched = W.logits(f64(self.l), self.start, self.V, dtype=self.dtype, **kwargs)
        got, lo, hi = f64(out), self.start[0], self.start[-1]
        left = self.l if kw.get("in_place") else torch.full_like(self.l, 7.0)
        for x in (slice(0, lo), slice(hi, self.T)):
            assert torch.equal(out[x], left[x]), "rows of no request are left"
        got, ref, bound, touched = got[lo:hi], ref[lo:hi], bound[lo:hi], touched[lo:hi]
        assert (np.isneginf(got) == np.isneginf(ref)).all()
        fin = np.isfinite(ref)
        err = np.abs(got - np.where(fin, ref, 0))
        assert (err[fin] <= bound[fin]).all(), (err[fin] / bound[fin]).max()
        same = torch.from_numpy(~touched).to(DEV)
        assert torch.equal(out[lo:hi][same], self.l[lo:hi][same]), "what no rule touches keeps its bits"
        return out


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
@pytest.mark.parametrize("V", (1, 7, 31, 32, 33, 1000, 2048, 2049, 8191, 8192, 8193, 20011))
def test_logits(V, dtype):
    Rows(V, [3, 1, 0, 5], V, dtype, pad=2, lead=1).check()


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
def test_logits_pitches_and_in_place(dtype):
    r = Rows(2, [2, 3], 4999, dtype, ldl=5003, ldo=5010, lda=160)
    a = r.check()
    b = r.check(in_place=True)
    assert torch.equal(a, b)
    r.ldl = r.ldo = 0
    assert torch.equal(a, r.check()) and torch.equal(a, r.check(in_place=True))


@pytest.mark.parametrize("without", [("draft",), ("history", "hist_len"), ("prompt_len",), ("repetition",), ("presence", "frequency"), ("bias_start",),
                                     ("allowed",), ("allowed_row",), ("repetition", "presence", "frequency"), ("hist_len", "draft"),
                                     ("repetition", "presence", "frequency", "bias_start", "allowed"), ("draft", "bias_start", "allowed"),
                                     ("bias_start", "history", "hist_len", "allowed", "allowed_row")], ids=str)
@pytest.mark.parametrize("dtype", ("bf16", "f32"))
def test_logits_without_some_rules(without, dtype):
    # hist_len without prompt_len: all of it is the answer
    Rows(len(without) + 5, [4, 2], 3001, dtype, without=without, states=7).check()


def test_logits_of_single_rows_without_starts():
    r = Rows(4, [1] * 70, 1500, "f32", max_new=1, pad=3)
    assert torch.equal(r.check(), r.check(start=False))
    r = Rows(4, [1] * 70, 1500, "bf16", max_new=0, without=("draft",))
    assert torch.equal(r.check(), r.check(start=False))


@pytest.mark.parametrize("rows, max_hist", [([256, 1, 100], 5), ([65, 64, 63], 3000), ([1] * 300, 9), ([0] * 70 + [2] * 5 + [0] * 200 + [1], 40), ([20], 20000)])
def test_logits_of_many_rows_and_long_histories(rows, max_hist):
    Rows(len(rows), rows, 700, "f32", max_hist=max_hist).check()


def test_logits_of_one_token_many_times():
    """Whole counts, whatever the order of their additions: 30000 of one token."""
    r = Rows(6, [2], 300, "f32", max_hist=30000, without=("bias_start", "allowed", "draft"))
    r.u["history"][:] = 17
    r.u["prompt_len"][:], r.u["hist_len"][:] = 0, 30000
    r.u["repetition"][:], r.u["frequency"][:], r.u["presence"][:] = 1.0, 2.0, 0.5
    out = r.run()
    assert (np.abs(f64(out)[:, 17] - (f64(r.l)[:, 17] - 60000.5)) <= 2.0 ** -7).all()
    out[:, 17] = r.l[:, 17]
    assert torch.equal(out, r.l)


def test_logits_that_are_not_numbers():
    """A grammar that allows nothing; infinities and NaN where they are allowed, and where not."""
    r = Rows(7, [3], 100, "f32", without=("draft", "bias_start"))
    r.u["allowed_row"][:] = [0, 1, 2]
    r.u["allowed"][0], r.u["allowed"][1], r.u["allowed"][2] = 0, 0xFFFFFFFF, 0x55555555
    r.l[:, 40] = math.nan
    r.l[:, 41] = math.inf
    r.l[:, 42] = -math.inf
    out = r.run()
    assert torch.isneginf(out[0]).all()
    assert torch.isnan(out[1, 40]) and out[1, 41] == math.inf and out[1, 42] == -math.inf and torch.isnan(out[1]).sum() == 1
    assert torch.isnan(out[2, 40]) and torch.isneginf(out[2, 41::2]).all() and torch.isnan(out[2]).sum() == 1


def test_logits_do_not_depend_on_the_run():
    r = Rows(8, [40, 33, 50], 50021, "bf16", max_hist=4000, n_bias=100)
    a = r.run()
    for _ in range(3):
        assert torch.equal(a, r.run())


def test_logits_with_long_lists_of_biases():
    """More entries than a workgroup has threads, most tokens named several times: the last counts."""
    Rows(9, [3, 2], 3001, "f32", n_bias=1500, without=("allowed",)).check()
    Rows(10, [1, 4], 50, "bf16", n_bias=700).check()


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
def test_large_logits_are_the_small_ones(dtype):
    """Many rows of a large vocabulary, several to a workgroup and past the caches: each
    request's rows have the bits that they get alone."""
    rows = [(7 * i) % 49 for i in range(60)]
    r = Rows(12, rows, 90001, dtype, max_hist=700, n_bias=40)
    out = r.run()
    whole, start = r.tensors(), r.start
    for q in (1, 20, 48, 59):
        lo, hi = start[q], start[q + 1]
        if lo == hi:
            continue
        u = {k: v for k, v in whole.items()}
        for k in ("history", "prompt_len", "hist_len", "repetition", "presence", "frequency"):
            u[k] = whole[k][q:q + 1].contiguous()
        u["bias_start"] = whole["bias_start"][q:q + 2].contiguous()
        for k in ("draft", "mask", "allowed_row"):
            u[k] = whole[k][lo:hi].contiguous()
        d = cola.logits_desc(hi - lo, r.V, 1, r.max_hist, r.max_new, dtype, len(r.u["bias"]), len(r.u["allowed"]))
        got = torch.empty((hi - lo, r.V), dtype=DT[dtype], device=DEV)
        cola.logits_adjust(d, cola.logits_rules(**u), r.l[lo:hi].contiguous(), i32([0, hi - lo]), got)
        assert torch.equal(torch.nan_to_num(out[lo:hi].float()), torch.nan_to_num(got.float()))


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
def test_logits_of_a_vocabulary_of_many_chunks(dtype):
    Rows(13, [48, 3], 90001, dtype, max_hist=300, n_bias=30, ldl=90013, ldo=90010).check()


def test_logits_past_4_gib():
    """Rows past 2^32 bytes: the bits that they get alone."""
    V, T = 1 << 20, 2050
    l = torch.zeros((T, V), dtype=torch.bfloat16, device=DEV)
    l[-2:] = rand(1, (2, V), "bf16")
    d = lambda T: cola.logits_desc(T, V, T, 8, 0, "bf16")
    u = dict(history=i32([[5, 6, V - 1, 5, 70000, 3, 2, 1]]), hist_len=i32([8]), repetition=torch.full((1,), 1.3, device=DEV),
             presence=torch.full((1,), 0.5, device=DEV))
    many = {k: v.repeat(T, *[1] * (v.dim() - 1)) for k, v in u.items()}
    want = torch.empty((1, V), dtype=torch.bfloat16, device=DEV)
    cola.logits_adjust(d(1), cola.logits_rules(**u), l[-1:].clone(), None, want)
    last = l[-2].clone()
    cola.logits_adjust(d(T), cola.logits_rules(**many), l, None, l)
    assert torch.equal(l[-1:], want) and not torch.equal(l[-2], last) and l[1000, 5] == -0.5 and l[1000, 9] == 0


# ---------------------------------------------------------------------------
# together
# ---------------------------------------------------------------------------

class Verifier:
    """A layer's cache, requests and their trees: tables, masks, append, attention and
    logits of a step that verifies drafted tokens, and the kept path's way to its place."""

    def __init__(self, n, hq, hk, hd, page, L, cap, max_new, V=500, seed=0):
        self.n, self.hq, self.hk, self.hd, self.page, self.L, self.cap, self.max_new, self.V = n, hq, hk, hd, page, L, cap, max_new, V
        self.rng = np.random.default_rng(seed)
        self.width = 8
        shared = -(-L // page)
        self.pages = shared + n * self.width
        ids = self.rng.permutation(self.pages)
        self.K = torch.full((self.pages, hk, page, hd), math.nan, dtype=torch.bfloat16, device=DEV)
        self.V_ = self.K.clone()
        self.ptab, self.free = i32(ids[:shared]), i32(ids[shared:])
        z = lambda *s, dt=torch.int32: torch.zeros(s, dtype=dt, device=DEV)
        self.kv, self.new, self.table, self.start = z(n), z(n), z(n, self.width) - 1, z(n + 1)
        self.slots, self.rows, self.pos, self.at, self.next = z(cap), z(cap), z(cap), z(1), z(1)
        self.parent, self.draft, self.kept = z(cap), z(cap), z(cap) - 1
        self.mask = z(cap, -(-max_new // 64), dt=torch.int64)
        self.x = z(cap, (hq + 2 * hk) * hd, dt=torch.bfloat16)
        self.qr, self.out, self.lse = z(cap, hq * hd, dt=torch.bfloat16), z(cap, hq * hd, dt=torch.bfloat16), z(hq, cap, dt=torch.float32)
        self.gq, self.gk = gain(seed + 1, hd, "bf16"), gain(seed + 2, hd, "bf16")
        self.l, self.chosen = z(cap, V, dt=torch.float32), z(cap, V, dt=torch.float32)
        self.c = cola.cache_desc(self.pages, page, hk, hd)
        ld = self.x.stride(0)
        self.rd = cola.rope_desc(cap, hq, hk, hd, ldq=ld, ldk=ld, ldv=ld)
        self.again = cola.rope_desc(cap, 0, hk, hd, ldk=ld, ldv=ld)
        self.md = cola.page_map_desc(n, cap, page, self.width, self.free.numel(), L)
        self.td = cola.tree_map_desc(n, cap, max_new, L)
        self.ad = cola.prefix_attn_desc(n, cap, hq, L, self.width * page, max_new)
        self.ws = torch.empty(max(1, cola.tree_attn_workspace_bytes(self.ad, self.c)), dtype=torch.uint8, device=DEV)
        self.history, self.hist_len = i32(self.rng.integers(0, V, (n, 300))), z(n)
        self.ld = cola.logits_desc(cap, V, n, 300, max_new)
        self.rules = cola.logits_rules(history=self.history, hist_len=self.hist_len, draft=self.draft, mask=self.mask,
                                       repetition=torch.full((n,), 1.2, device=DEV), presence=torch.full((n,), 0.3, device=DEV))
        self.past = [(np.zeros((0, hk * hd)), np.zeros((0, hk * hd)))] * n      # each request's normalised, turned keys, and values
        if L:
            k, v = rand(seed + 3, (L, hk * hd), "bf16"), rand(seed + 4, (L, hk * hd), "bf16")
            j = torch.arange(L, device=DEV)
            slots = (self.ptab.long()[j // page] * page + j % page).int()
            cola.norm_append(cola.rope_desc(L, 0, hk, hd), self.c, None, k, v, None, self.gk, None, slots, None, self.K, self.V_)
            self.past = [(self.key(f64(k), np.arange(L)), f64(v))] * n

    def part(self, name):
        a, b = self.hq * self.hd, (self.hq + self.hk) * self.hd
        return {"q": self.x[:, :a], "k": self.x[:, a:b], "v": self.x[:, b:]}[name]

    def key(self, k, pos):
        return W.norm_rope(k, f64(self.gk), self.hd, self.hd, pos, "bf16")[0]

    def feed(self, new, seed):
        """Trees of `new` nodes, their rows, and logits."""
        rng = np.random.default_rng(seed)
        self.new.copy_(i32(new))
        self.kv += self.new
        self.trees = [W.random_tree(rng, n) for n in new]
        parent = np.concatenate([np.asarray(t, int) for t in self.trees] + [np.full(self.cap - sum(new), 99)])
        self.parent.copy_(i32(parent))
        self.draft.copy_(i32(rng.integers(0, self.V, self.cap)))
        self.x.copy_(rand(seed, tuple(self.x.shape), "bf16"))
        self.l.copy_(rand(seed + 1, tuple(self.l.shape), "f32"))
        self.hist_len.copy_(i32(rng.integers(0, 300, self.n)))

    def step(self, stream=None):
        cola.page_map(self.md, self.kv, self.new, self.free, self.at, self.table, self.start, self.slots, self.rows, self.next, stream=stream)
        cola.tree_map(self.td, self.parent, self.kv, self.start, self.mask, self.pos, stream=stream)
        cola.norm_append(self.rd, self.c, self.part("q"), self.part("k"), self.part("v"), self.gq, self.gk, self.pos, self.slots, self.qr,
                         self.K, self.V_, stream=stream)
        cola.tree_attn(self.ad, self.c, self.qr, self.K, self.V_, self.ptab if self.L else None, self.table, self.kv, self.start, self.mask,
                       self.out, self.lse, self.ws, stream=stream)
        cola.logits_adjust(self.ld, self.rules, self.l, self.start, self.chosen, stream=stream)

    def keep(self, paths):
        """The path's j-th node into the slot of node j: rows' k and v once more."""
        slots, kept = self.slots.cpu().numpy(), np.full(self.cap, -1)
        row = 0
        for tree, path in zip(self.trees, paths):
            for j, i in enumerate(path):
                kept[row + i] = slots[row + j]
            row += len(tree)
        self.kept.copy_(i32(kept))
        cola.norm_append(self.again, self.c, None, self.part("k"), self.part("v"), None, self.gk, self.pos, self.kept, None, self.K, self.V_)
        self.kv += i32([len(p) for p in paths]) - self.new
        self.at.copy_(self.next)

    def path(self, r, i):
        """Node i of request r and its ancestors, the root first."""
        p = [i]
        while self.trees[r][p[0]] >= 0:
            p.insert(0, self.trees[r][p[0]])
        return p

    def check(self, paths):
        """Each row against its request's sequence as it would be after its path, in 64 bits."""
        torch.cuda.synchronize()
        q, k, v = (f64(self.part(x).contiguous()) for x in "qkv")
        row = 0
        for r, tree in enumerate(self.trees):
            ks, vs = self.past[r]
            p0 = len(ks)
            for i in range(len(tree)):
                path = self.path(r, i)
                pos = p0 + np.arange(len(path))
                assert int(self.pos[row + i]) == pos[-1]
                at = [row + j for j in path]
                kk, vv = np.concatenate([ks, self.key(k[at], pos)]), np.concatenate([vs, v[at]])
                qs = W.norm_rope(q[row + i:row + i + 1], f64(self.gq), self.hd, self.hd, pos[-1:], "bf16")[0][0]
                for h in range(self.hq):
                    x, y = slice(h * self.hd, (h + 1) * self.hd), h // (self.hq // self.hk)
                    y = slice(y * self.hd, (y + 1) * self.hd)
                    s = kk[:, y] @ qs[x] / math.sqrt(self.hd)
                    w = np.exp(s - s.max())
                    w /= w.sum()
                    # q and k rounded to bf16: scores to 2^-7 of |q||k|/sqrt(hd) a product, weights by e^that
                    ds = 2.0 ** -7 * (np.abs(kk[:, y]) @ np.abs(qs[x]) / math.sqrt(self.hd)).max()
                    tol = (2 * (math.exp(ds) - 1) + 2.0 ** -6) * (w @ np.abs(vv[:, y])) + 2.0 ** -8
                    assert (np.abs(f64(self.out[row + i, x]) - w @ vv[:, y]) <= tol).all(), (r, i, h)
            at = [row + j for j in paths[r]]
            self.past[r] = (np.concatenate([ks, self.key(k[at], p0 + np.arange(len(at)))]), np.concatenate([vs, v[at]]))
            row += len(tree)
        assert (self.out[row:] == 0).all() and (self.chosen[row:] == 0).all(), "idle rows are left"
        history, n = self.history.cpu().numpy(), self.hist_len.cpu().numpy()
        ref, bound, _ = W.logits(f64(self.l), self.start.cpu().tolist(), self.V, history=history, hist_len=n, draft=self.draft.cpu().numpy(),
                                 masks=[int(w[0]) & 2 ** 64 - 1 for w in self.mask.cpu().tolist()], repetition=np.full(self.n, np.float32(1.2)),
                                 presence=np.full(self.n, np.float32(0.3)))
        assert (np.abs(f64(self.chosen[:row]) - ref[:row]) <= bound[:row]).all()


@pytest.mark.parametrize("shape", [(5, 4, 2, 64, 16, 21, 60, 12), (3, 2, 2, 128, 32, 0, 40, 20), (2, 8, 2, 64, 16, 40, 120, 50)], ids=str)
def test_verifying_steps(shape):
    """Trees, a path kept of each, and on from there: five steps."""
    s = Verifier(*shape)
    rng = np.random.default_rng(shape[0])
    for i in range(5):
        new = rng.integers(1, shape[-1] + 1, s.n)
        if i == 2:
            new[-1] = 0
        if i == 3:
            new[:] = 1
        s.out.zero_(), s.chosen.zero_()
        s.feed(new, 100 + i)
        s.step()
        paths = [s.path(r, int(rng.integers(0, n))) if n else [] for r, n in enumerate(new)]
        s.check(paths)
        s.keep(paths)


def test_verifying_step_in_a_graph():
    """One captured step replayed: it follows lengths, trees, tables and histories; eager
    work and synchronisations between the replays."""
    s, e = (Verifier(4, 4, 2, 64, 16, 33, 64, 16) for _ in range(2))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for x in (s, e):
        x.feed([1, 2, 3, 4], 1)
    with torch.cuda.stream(side):
        s.step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        s.step()
    rng = np.random.default_rng(9)
    e.step()
    for i, new in enumerate(([16, 1, 7, 1], [1, 1, 1, 1], [0, 9, 16, 1], [5, 5, 5, 5])):
        paths = [x.path(r, int(rng.integers(0, len(t)))) if t else [] for r, t in enumerate(e.trees) for x in (e,)]
        for x in (s, e):
            x.keep(paths)
            x.out.zero_(), x.chosen.zero_()
            x.feed(new, 60 + i)
        g.replay()
        e.step()
        torch.cuda.synchronize()
        for a, b in ((s.out, e.out), (s.mask, e.mask), (s.pos, e.pos), (s.slots, e.slots), (s.chosen, e.chosen), (s.table, e.table)):
            assert torch.equal(a, b)
        assert torch.equal(torch.nan_to_num(s.K), torch.nan_to_num(e.K)) and torch.equal(torch.nan_to_num(s.V_), torch.nan_to_num(e.V_))


def test_norm_gradients_in_a_graph():
    """Captured with its two launches, replayed on other rows."""
    T, hq, hk, hd = 500, 6, 2, 64
    q, k, dq, dk = (rand(i, (T, h * hd), "bf16") for i, h in enumerate((hq, hk, hq, hk)))
    gq, gk = gain(5, hd, "bf16"), gain(6, hd, "bf16")
    d = cola.rope_desc(T, hq, hk, hd, seq_len=100)
    ws = workspace(d)
    o = [torch.empty_like(q), torch.empty_like(k), torch.empty(hd, device=DEV), torch.empty(hd, device=DEV)]
    e = [torch.empty_like(t) for t in o]
    cola.norm_rope_bwd(d, dq, dk, q, k, gq, gk, None, *o, ws)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        cola.norm_rope_bwd(d, dq, dk, q, k, gq, gk, None, *o, ws)
    for i in range(4):
        q.copy_(rand(20 + i, (T, hq * hd), "bf16"))
        for t in o:
            t.zero_()
        g.replay()
        torch.cuda.synchronize()
        cola.norm_rope_bwd(d, dq, dk, q, k, gq, gk, None, *e, workspace(d))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(o, e))


def test_two_graphs_of_trees_share_a_workspace():
    """Replayed one after the other, each leaves what it leaves alone."""
    made = []
    for seed, new, kv, hd in ((20, [5, 60], [200, 3000], 64), (21, [40, 35], [2500, 90], 64)):
        b = TreeBatch(seed, new, kv, 0, 4, 2, hd, 16)
        made.append((b, b.run()))
    n = max(cola.tree_attn_workspace_bytes(*b.desc()) for b, _ in made)
    assert n > 0
    ws = torch.empty(n, dtype=torch.uint8, device=DEV)
    graphs = []
    for b, _ in made:
        d, c = b.desc()
        t = [i32(x) for x in (b.tab, b.kv, b.start)] + [torch.from_numpy(W.words(b.masks, b.max_new)).to(DEV)]
        out, lse = torch.zeros_like(b.q), torch.zeros((b.hq, b.T), device=DEV)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            cola.tree_attn(d, c, b.q, b.K, b.V, None, *t, out, lse, ws)
        graphs.append((g, out, lse, t))
    for order in ((0, 1), (1, 0), (0, 0, 1, 1), (1, 0, 1, 0)):
        for g, out, lse, _ in graphs:
            out.zero_(), lse.zero_()
        for i in order:
            graphs[i][0].replay()
        torch.cuda.synchronize()
        for (_, out, lse, _), (b, (want, wl)) in zip(graphs, made):
            assert torch.equal(out, want) and torch.equal(lse, wl)


@pytest.mark.parametrize("L, hd", [(0, 64), (0, 128), (1300, 64), (1300, 128)])
def test_a_captured_tree_attention_follows_the_lengths(L, hd):
    """One captured call whose own keys are cut by the lengths, replayed on other lengths, starts, tables and masks in
    the same places: shorter and longer ones, empty requests, none at all.  The part's length, which the first launch
    leaves in the workspace for the second, is each replay's own; eager work and synchronisations between them."""
    from test_verify_abi import cut_by_lengths, tree_plan
    b = TreeBatch(50 + hd, [40, 130, 7, 60], [7000, 2000, 5000, 60], L, 16, 16, hd, 64, pad=3)
    d, c = b.desc()
    n = cola.tree_attn_workspace_bytes(d, c)
    plan = tree_plan(4, b.T, 16, 16, hd, L, b.max_kv, b.max_new, 64)
    words = lambda: torch.from_numpy(W.words(b.masks, b.max_new)).to(DEV)
    ptab, tab, kv, start, mask = i32(b.ptab) if L else None, i32(b.tab), i32(b.kv), i32(b.start), words()
    out, lse = torch.zeros_like(b.q), torch.zeros((b.hq, b.T), device=DEV)
    ws = torch.zeros(n, dtype=torch.uint8, device=DEV)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        cola.tree_attn(d, c, b.q, b.K, b.V, ptab, tab, kv, start, mask, out, lse, ws)
    whole, rng, lengths = b.tab.copy(), np.random.default_rng(hd), set()
    for new, old in (([40, 130, 7, 60], [7000, 2000, 5000, 60]), ([1, 2, 1, 3], [300, 64, 1, 3]), ([130, 0, 0, 100], [7000, 0, 0, 100]),
                     ([0, 0, 0, 0], [0, 0, 0, 0]), ([7, 60, 130, 40], [65, 1999, 4000, 40]), ([40, 130, 7, 60], [7000, 2000, 5000, 60])):
        b.new, b.kv = new, old
        b.start = [0] + np.cumsum(new).tolist()
        b.masks = [0] * b.T
        for r, k in enumerate(new):
            parent = W.random_tree(rng, k)
            for i in range(k):
                t = b.start[r] + i
                b.masks[t] = (b.masks[b.start[r] + parent[i]] if parent[i] >= 0 else 0) | 1 << i
        # pages that no token lies in are named by no one
        b.tab = np.where(np.arange(whole.shape[1]) < -(-np.asarray(old)[:, None] // 64), whole, -1)
        for to, x in ((tab, i32(b.tab)), (kv, i32(old)), (start, i32(b.start)), (mask, words())):
            to.copy_(x)
        out.fill_(7.0), lse.fill_(7.0)
        g.replay()
        torch.cuda.synchronize()
        lengths.add(int(ws[-64:-60].view(torch.int32)[0]))
        assert int(ws[-64:-60].view(torch.int32)[0]) == cut_by_lengths(plan, hd, 16, 1, L, b.max_new, b.max_kv, list(zip(new, old)))[0]
        # bits: of the hundred tokens of one request forty were never written, and give NaN
        want, wl = b.check() if old == [300, 64, 1, 3] else b.run()
        assert torch.equal(out.view(torch.int16), want.view(torch.int16)) and torch.equal(lse.view(torch.int32), wl.view(torch.int32)), old
        assert not torch.isnan(out[:b.start[3]].float()).any()
    assert len(lengths) > 1


def test_two_streams_verify_at_once():
    """Two programs on two streams, each with its own buffers: the serial results."""
    a, b = Verifier(6, 8, 2, 128, 16, 50, 100, 16), Verifier(6, 8, 2, 128, 16, 50, 100, 16, seed=5)
    want = []
    for s in (a, b):
        s.feed([16, 3, 9, 1, 12, 16], 7)
        s.step()
        torch.cuda.synchronize()
        want.append((s.out.clone(), s.chosen.clone()))
        s.out.zero_(), s.chosen.zero_()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(3):
        for s, st in zip((a, b), streams):
            s.step(stream=st)
    torch.cuda.synchronize()
    for s, (out, chosen) in zip((a, b), want):
        assert torch.equal(s.out, out) and torch.equal(s.chosen, chosen)


def test_timing_classes_count_the_launches_of_a_verifying_step():
    s = Verifier(2, 2, 2, 64, 16, 20, 16, 8)
    s.feed([5, 8], 3)
    d = cola.rope_desc(4, 2, 2, 64)
    x = [rand(i, (4, 128), "bf16") for i in range(6)]
    dg = [torch.empty(64, device=DEV) for _ in range(2)]
    cola.timing_enable(True)
    cola.timing_reset()
    try:
        s.step()
        cola.norm_rope_fwd(d, x[0], x[1], None, None, None, x[2], x[3])
        cola.norm_rope_bwd(d, x[2], x[3], x[0], x[1], None, None, None, x[4], x[5], *dg, workspace(d))
        n = {k: cola.timing_read(i)[0] for i, k in enumerate(cola.KERNEL_CLASSES)}
    finally:
        cola.timing_enable(False)
        cola.timing_reset()
    assert n["pointwise"] == 3 and n["attn_fwd"] == 1 and n["norm"] == 2 and n["norm_bwd"] == 2 and sum(n.values()) == 8
