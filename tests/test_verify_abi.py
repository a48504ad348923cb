"""Head norms, drafted trees and rules on logits on the CPU: what must be refused before
anything is enqueued, workspace sizes, the Python checks, and the plain references
against closed forms and differences."""
import ctypes
import math

import numpy as np
import pytest
import torch

import serve_ref as R
import verify_ref as W
from paper_2502_10940_amd import cola
from test_serve_abi import BF, FAKE, I32, KINDS, Plan, Shape, attn_args, refused


# ---- norms ----

def fwd(d, q=FAKE, k=FAKE, gq=FAKE, gk=FAKE, pos=None, qo=FAKE, ko=FAKE, eps=1e-6):
    cola.norm_rope_fwd(d, q, k, gq, gk, pos, qo, ko, eps, 0)


def bwd(d, dqo=FAKE, dko=FAKE, q=FAKE, k=FAKE, gq=FAKE, gk=FAKE, pos=None, dq=FAKE, dk=FAKE, dgq=FAKE, dgk=FAKE + 4096, ws=FAKE,
        n=1 << 40, eps=1e-6):
    cola.norm_rope_bwd(d, dqo, dko, q, k, gq, gk, pos, dq, dk, dgq, dgk, ws, n, eps, 0)


@pytest.mark.parametrize("fn", (fwd, bwd))
def test_norm_refusals(fn):
    D = cola.rope_desc
    for d in (D(4, 0, 0, 64), D(-1, 2, 2, 64), D(4, 2, 2, 0), D(4, 2, 2, 513), D(4, 2, 2, 64, 63), D(4, 2, 2, 64, ldq=127),
              D(4, 2, 2, 64, ldko=127), D(1 << 31, 2, 2, 64)):
        refused(cola.ERR_BAD_SHAPE, fn, d)
        assert cola.norm_rope_workspace_bytes(d) == 0
    refused(cola.ERR_INVALID_ARG, fn, D(4, 2, 2, 64, dtype=7))
    d = D(4, 2, 2, 64)
    for eps in (0.0, -1.0, math.nan, math.inf, 1e300, 1e-60, 1e-45, 1.1e-38):
        refused(cola.ERR_INVALID_ARG, lambda: fn(d, eps=eps))
    for key in ("q", "k"):
        refused(cola.ERR_INVALID_ARG, lambda: fn(d, **{key: None}))
    for key, p in (("q", FAKE + 1), ("gq", FAKE + 1), ("gk", FAKE + 1), ("pos", FAKE + 2)):
        refused(cola.ERR_INVALID_ARG, lambda: fn(d, **{key: p}))
    refused(cola.ERR_INVALID_ARG, lambda: fn(D(4, 2, 2, 64, dtype="f32"), gq=FAKE + 2))


def test_norm_refusals_of_each_direction():
    D = cola.rope_desc
    for key in ("qo", "ko"):
        refused(cola.ERR_INVALID_ARG, lambda: fwd(D(4, 2, 2, 64), **{key: None}))
    refused(cola.ERR_INVALID_ARG, lambda: fwd(D(4, 2, 2, 64, ldqo=256)))               # in place at another pitch
    refused(cola.ERR_INVALID_ARG, lambda: bwd(D(4, 2, 2, 64, ldqo=256)))
    fwd(D(0, 2, 2, 64), None, None, None, None, None, None, None)                      # an empty batch enqueues nothing
    d = D(4, 2, 2, 64)
    for key in ("dqo", "dko", "dq", "dk"):
        refused(cola.ERR_INVALID_ARG, lambda: bwd(d, **{key: None}))
    for key in ("dgq", "dgk", "ws"):
        refused(cola.ERR_INVALID_ARG, lambda: bwd(d, **{key: FAKE + 2}))
    refused(cola.ERR_INVALID_ARG, lambda: bwd(d, dgk=FAKE))                            # both gains' gradients in one place
    refused(cola.ERR_INVALID_ARG, lambda: bwd(D(4, 2, 0, 64), dko=None, k=None, dk=None))
    need = cola.norm_rope_workspace_bytes(d)
    assert need > 0 and need % (2 * 64 * 4) == 0
    refused(cola.ERR_WORKSPACE, lambda: bwd(d, n=need - 1))
    refused(cola.ERR_WORKSPACE, lambda: bwd(d, ws=None))
    assert cola.norm_rope_workspace_bytes(D(0, 2, 2, 64)) == 0
    # at most 1024 workgroups' sums, however many rows
    assert cola.norm_rope_workspace_bytes(D(1 << 20, 32, 32, 128)) <= 1024 * 2 * 128 * 4


def test_norm_append_refusals():
    D, C = cola.rope_desc, cola.cache_desc

    def call(d, c, q=FAKE, k=FAKE, v=FAKE, gq=FAKE, gk=FAKE, pos=None, slots=FAKE, qo=FAKE, K=FAKE, V=FAKE + 4096, eps=1e-6):
        cola.norm_append(d, c, q, k, v, gq, gk, pos, slots, qo, K, V, eps, 0)

    d, c = D(4, 4, 2, 64), C(8, 16, 2, 64)
    for bad in (C(8, 16, 3, 64), C(8, 16, 2, 128), C(8, 24, 2, 64)):
        refused(cola.ERR_BAD_SHAPE, call, d, bad)
    refused(cola.ERR_INVALID_ARG, call, d, C(8, 16, 2, 64, "f32"))
    refused(cola.ERR_INVALID_ARG, lambda: call(d, c, eps=0.0))
    for key in ("q", "k", "v", "slots", "qo", "K", "V"):
        refused(cola.ERR_INVALID_ARG, lambda: call(d, c, **{key: None}))
    for key, p in (("K", FAKE + 8), ("V", FAKE), ("slots", FAKE + 2), ("gk", FAKE + 1)):
        refused(cola.ERR_INVALID_ARG, lambda: call(d, c, **{key: p}))
    call(D(0, 4, 2, 64), c, *[None] * 10)


@pytest.mark.parametrize("layout", ("half", "interleaved"))
def test_reference_norm_gradients_against_differences(layout):
    """The 64-bit backward against central differences of the 64-bit forward: 2^-14 steps
    leave 2^-28 of the third derivative (of order one) and 2^-52 / 2^-14 of rounding."""
    rng = np.random.default_rng(3)
    T, h, hd, rot = 3, 2, 12, 8
    x, g, dy = rng.standard_normal((T, h * hd)), 1 + 0.3 * rng.standard_normal(hd), rng.standard_normal((T, h * hd))
    pos = [0, 7, 100]
    f = lambda x, g: (W.norm_rope(x, g, hd, rot, pos, "f32", layout, mscale=1.3)[0] * dy).sum()
    (dx, _), (dg, _) = W.norm_rope_bwd(dy, x, g, hd, rot, pos, "f32", layout, mscale=1.3)
    s = 2.0 ** -14
    for at in ((0, 0), (1, 9), (2, 23), (1, 13)):
        e = np.zeros_like(x)
        e[at] = s
        assert abs((f(x + e, g) - f(x - e, g)) / (2 * s) - dx[at]) < 1e-6
    for at in (0, 3, 11):
        e = np.zeros_like(g)
        e[at] = s
        assert abs((f(x, g + e) - f(x, g - e)) / (2 * s) - dg[at]) < 1e-6


# ---- trees ----

def test_tree_map_refusals():
    D = cola.tree_map_desc

    def call(d, parent=FAKE, kv=FAKE, start=FAKE, mask=FAKE + 4096, pos=FAKE + 8192):
        cola.tree_map(d, parent, kv, start, mask, pos, 0)

    for bad in (D(-1, 4, 8), D(65536, 4, 8), D(2, -1, 8), D(2, 1 << 31, 8), D(2, 4, 0), D(2, 4, 257), D(2, 4, 8, -1),
                D(2, 4, 8, 1 << 31)):
        refused(cola.ERR_BAD_SHAPE, call, bad)
    d = D(2, 4, 8)
    for key in ("parent", "kv", "mask", "pos"):
        refused(cola.ERR_INVALID_ARG, lambda: call(d, **{key: None}))
    for key, p in (("parent", FAKE + 2), ("kv", FAKE + 1), ("start", FAKE + 2), ("pos", FAKE + 2), ("mask", FAKE + 4),
                   ("pos", FAKE), ("mask", FAKE), ("mask", FAKE + 8192)):
        refused(cola.ERR_INVALID_ARG, lambda: call(d, **{key: p}))
    call(D(2, 0, 8), None, None, None, None, None)


def test_tree_attention_refusals():
    D, C = cola.prefix_attn_desc, cola.cache_desc

    def call(d, c, mask=FAKE, **kw):
        a = attn_args(**kw)
        cola.tree_attn(d, c, *a[:7], mask, *a[7:], 0)

    c, d = C(8, 16, 2, 64), D(3, 5, 4, 40, 30, 2)
    refused(cola.ERR_UNSUPPORTED, call, d, C(8, 16, 2, 64, "f32"))
    for bad in (D(-1, 5, 4, 40, 30), D(3, 5, 3, 40, 30), D(3, 5, 4, 40, 30, 0), D(3, 5, 4, 40, 30, 257), D(3, 5, 4, 40, 30, max_pages=1)):
        refused(cola.ERR_BAD_SHAPE, call, bad, c)
        assert cola.tree_attn_workspace_bytes(bad, c) == 0
    for key in ("q", "K", "V", "ptab", "tab", "kv", "out", "mask"):
        refused(cola.ERR_INVALID_ARG, lambda: call(d, c, **{key: None}))
    for key, p in (("mask", FAKE + 4), ("q", FAKE + 8), ("kv", FAKE + 2), ("out", FAKE)):
        refused(cola.ERR_INVALID_ARG, lambda: call(d, c, **{key: p}))
    far = D(3, 5, 4, 4000, 30, 2)
    need = cola.tree_attn_workspace_bytes(far, c)
    assert need > 0
    refused(cola.ERR_WORKSPACE, lambda: call(far, c, n=need - 1))
    for e in (D(0, 5, 4, 40, 30), D(3, 0, 4, 40, 30)):
        cola.tree_attn(e, c, *[None] * 11, 0, 0)


def test_reference_masks_and_attention():
    """A chain's masks make the rows causal."""
    rng = np.random.default_rng(1)
    start, kv = [0, 4, 9], [6, 5]
    masks, pos = W.tree_map([-1, 0, 1, 2, -1, 0, 1, 2, 3], kv, start, 9, 64, 10)
    assert masks == [1, 3, 7, 15, 1, 3, 7, 15, 31] and pos == [12, 13, 14, 15, 10, 11, 12, 13, 14]
    masks2, pos2 = W.tree_map([-1, 0, 0, 1, -1, -1, 9, 1, 0], kv, start, 9, 4, 0)
    assert masks2 == [1, 3, 5, 11, 1, 2, 4, 10, 0] and pos2 == [2, 3, 3, 4, 0, 0, 0, 1, 0]
    K, V = rng.standard_normal((3, 1, 16, 8)), rng.standard_normal((3, 1, 16, 8))
    q = rng.standard_normal((9, 16))
    a = W.attention(q, K, V, 2, [2], 3, [[0], [1]], kv, start, 16, masks)
    b = R.attention(q, K, V, 2, [2], 3, [[0], [1]], kv, start, 16)
    for x, y in zip(a, b):
        assert np.allclose(x, y, rtol=0, atol=1e-14)
    assert W.words([1 << 70 | 5], 100).tolist() == [[5, 64]]


def tree_plan(n_req, T, hq, hk, hd, prefix, max_kv, max_new, page=16):
    f = cola.lib()._ZN4cola14plan_tree_attnERKNS_15PrefixAttnShapeE
    f.restype, f.argtypes = Plan, [ctypes.POINTER(Shape)]
    p = f(ctypes.byref(Shape(n_req, T, max_new, prefix, max_kv, -(-max_kv // page), 1 << 20, page, hq, hk, hd, hq * hd, hq * hd, hd ** -0.5)))
    d, c = cola.prefix_attn_desc(n_req, T, hq, prefix, max_kv, max_new), cola.cache_desc(1 << 20, page, hk, hd)
    assert p.rows == T * hq and p.ws_bytes == cola.tree_attn_workspace_bytes(d, c)
    return p


@pytest.mark.parametrize("hd", (64, 128))
def test_gpu_tests_of_trees_run_every_kernel(hd):
    """The plans of the GPU tests' batches: every pair of kinds that there is a kernel for,
    the parts cut by the lengths among them."""
    from test_gpu_verify import CUT, TREES
    seen = set()
    cases = [(len(new), sum(new) + 2, hq, hk, L, max(kv), max(new)) for new, kv, L, hq, hk in TREES.values()]
    cases += [(len(new), sum(new) + 3, hq, hk, L, max_kv or max(kv), max(new)) for new, kv, L, hq, hk, max_kv in CUT.values()]
    for n, T, hq, hk, L, max_kv, max_new in cases:
        p = tree_plan(n, T, hq, hk, hd, L, max_kv, max_new, 16 if hd == 64 else 64)
        full = 512 if hd == 128 else 1024
        counted = p.kind_s == 8 and p.splits_s > 1 and n <= 256 and n * p.tiles_s * hk < full // 2
        seen.add((p.kind_p, p.kind_s, counted))
    k = dict(KINDS, four=6)
    every = [("along", "one"), ("along", "two"), ("along", "wide"), ("one", "one"), ("two", "one"), ("two", "two"), ("wide", "one"), ("wide", "two"),
             ("wide", "wide"), ("wide", "wide", True)]
    if hd == 64:
        every += [("along", "four"), ("four", "four")]
    every = {(k[x[0]], k[x[1]], len(x) > 2) for x in every}
    assert seen == every, (sorted(every - seen), sorted(seen - every))


def cut_by_lengths(p, hd, hk, g, prefix, max_new, max_kv, lens):
    """What the kernels make of lengths (rows, own tokens) on the GPU where they cut the own keys by them, step for step:
    (the part's length, the item of each turn behind the prefix's or None)."""
    stage, slots = 64, 512 if hd == 128 else 1024
    tiles = [-(-min(n, max_new) * g // 128) for n, _ in lens]
    ends = [min(kv, max_kv) for _, kv in lens]
    parts = max(slots - sum(tiles) * hk // 2, slots // 2)
    work = sum(t * -(-e // stage) for t, e in zip(tiles, ends)) * hk
    if p.splits_p:
        work += hk * p.tiles_p * -(-prefix // stage)
    longest = max([e for t, e in zip(tiles, ends) if t] + [0])
    up = lambda x, n: -(-x // n)
    least = max(up(up(longest, p.splits_s), stage) * stage, min(p.chunk_s, 256))
    chunk = min(max(-(-work // parts) * stage, least), 1 << 30)
    items = []
    for r, (t, e) in enumerate(zip(tiles, ends)):
        units = min(-(-e // chunk), p.splits_s) * hk if t else 0
        for j in range(units if t == 1 else -(-units // 8) * 8 * t):
            unit, tile = (j, 0) if t == 1 else ((j >> 3) // t * 8 + (j & 7), (j >> 3) % t)
            items.append((r, unit % hk, unit // hk, tile) if unit < units else None)
    return chunk, items


def test_trees_cut_by_their_lengths_fit_the_launch_and_the_workspace():
    """Whatever the lengths: every item that the join reads has a turn of the launch, once, and its
    part a place in the workspace.  Bounds near the lengths and far above them, launches of just under
    half of the chip, several tiles to a request, empty requests and such that see nothing."""
    rng = np.random.default_rng(5)
    cut, most = 0, 0.0
    for i in range(1500):
        hd = int(rng.choice([64, 128]))
        hk, g = int(rng.choice([1, 2, 4, 8, 16])), int(rng.choice([1, 2, 4, 8]))
        full = 512 if hd == 128 else 1024
        max_new = int(rng.integers(1, 257))
        t_s = -(-max_new * g // 128)
        n = int(min(256, max(1, (full // 2 - 1) // (t_s * hk)))) if i % 2 else int(rng.integers(1, 33))
        longest = int(2 ** rng.uniform(8, 15))
        max_kv = longest if i % 3 else int(min(1 << 20, longest * 2 ** rng.uniform(0, 8)))
        prefix = int(rng.choice([0, 0, 1, 700, 5000]))
        T = n * max_new + int(rng.integers(0, 5))
        p = tree_plan(n, T, hk * g, hk, hd, prefix, max_kv, max_new)
        if not (p.kind_s == 8 and p.splits_s > 1 and n * p.tiles_s * hk < full // 2):
            continue
        cut += 1
        turns = full + n * p.tiles_s * hk + (8 * n * p.tiles_s if p.tiles_s > 1 else 0)       # the launch, without the prefix's
        for spread in range(3):
            rows = rng.integers(0, max_new + 9, n) if spread else np.full(n, max_new)
            kv = (longest * rng.random(n) ** spread).astype(int) + 1
            chunk, items = cut_by_lengths(p, hd, hk, g, prefix, max_new, max_kv, list(zip(rows.tolist(), kv.tolist())))
            assert chunk % 64 == 0 and len(items) <= turns
            most = max(most, len(items) / turns)
            there = [x for x in items if x is not None]
            want = {(r, h, s, t) for r in range(n) for h in range(hk) for s in range(-(-min(int(kv[r]), max_kv) // chunk))
                    for t in range(-(-min(int(rows[r]), max_new) * g // 128))}
            assert len(there) == len(set(there)) and set(there) == want and all(x[2] < p.splits_s for x in there)
    assert cut > 300 and most > 0.9


# ---- logits ----

def test_logits_refusals():
    D = cola.logits_desc

    def call(d, logits=FAKE, start=None, out=FAKE + 4096, rules=None, **u):
        cola.logits_adjust(d, cola.logits_rules(**u) if rules is None else rules, logits, start, out, 0)

    for bad in (D(-1, 8, 1), D(4, 0, 1), D(4, (1 << 22) + 1, 1), D(4, 8, -1), D(4, 8, 65536), D(4, 8, 1, -1), D(4, 8, 1, 1 << 30),
                D(4, 8, 1, 4, -1), D(4, 8, 1, 4, 257), D(4, 8, 1, n_bias=-1), D(4, 8, 1, n_bias=1 << 30), D(4, 8, 1, n_allowed=-1), D(4, 8, 1, ldl=7),
                D(4, 8, 1, ldo=7), D(4, 64, 1, lda=1), D(1 << 31, 8, 1), D(4, 8, 1, ldl=(1 << 22) + 1)):
        refused(cola.ERR_BAD_SHAPE, call, bad)
    refused(cola.ERR_INVALID_ARG, call, D(4, 8, 1, dtype=9))
    d = D(4, 40, 2, 6, 3, n_bias=5, n_allowed=4)
    d.reserved = 1
    refused(cola.ERR_INVALID_ARG, call, d)
    d.reserved = 0
    for kw in (dict(logits=None), dict(out=None), dict(logits=FAKE + 2), dict(start=FAKE + 1), dict(hist_len=FAKE), dict(draft=FAKE),
               dict(draft=FAKE, mask=FAKE + 4), dict(bias_start=FAKE), dict(bias_start=FAKE, bias=FAKE), dict(presence=FAKE + 2),
               dict(allowed=FAKE + 1), dict(allowed_row=FAKE + 2), dict(history=FAKE + 2, hist_len=FAKE)):
        refused(cola.ERR_INVALID_ARG, lambda: call(d, **kw))
    refused(cola.ERR_INVALID_ARG, lambda: call(D(4, 40, 2, 6, 0), draft=FAKE, mask=FAKE))
    refused(cola.ERR_INVALID_ARG, lambda: call(D(4, 40, 2, ldo=48), out=FAKE))          # in place at another pitch
    call(D(0, 8, 1), None, None, None)
    call(D(4, 8, 0), None, None, None)
    with pytest.raises(ValueError, match="no such rule"):
        cola.logits_rules(temperature=1)
    assert ctypes.sizeof(cola.LogitsRules) == 13 * ctypes.sizeof(ctypes.c_void_p)


def test_reference_logits():
    """By hand: a vocabulary of 5, one prompt token, an answer with a repetition, a bias given twice."""
    l = np.array([[1.0, -2.0, 0.5, 3.0, 0.0]])
    y, err, touched = W.logits(l, [0, 1], 5, np.array([[0, 1, 1, 7]]), [1], [4], repetition=[2.0], presence=[0.25], frequency=[0.5],
                               bias_start=[0, 3], bias_token=[2, 3, 2], bias=[9.0, 1.0, -0.5], allowed=[[0b01111]])
    assert np.array_equal(y[0], [0.5, -4.0 - 1.0 - 0.25, 0.0, 4.0, -np.inf])
    assert np.array_equal(touched[0], [True, True, True, True, True])


def test_python_checks():
    z = lambda *s, dt=BF: torch.zeros(s, dtype=dt)
    i = lambda *s: torch.zeros(s, dtype=I32)
    f = lambda *s: torch.zeros(s)
    d = cola.rope_desc(4, 2, 1, 64)
    ok = [z(4, 128), z(4, 64), z(64), z(64), i(4), z(4, 128), z(4, 64)]
    for j, t in ((0, f(4, 128)), (0, z(3, 128)), (2, z(63)), (3, f(64)), (2, z(2, 64)), (4, i(3)), (6, z(4, 63)), (2, z(128)[::2])):
        a = list(ok)
        a[j] = t
        with pytest.raises(ValueError):
            cola.norm_rope_fwd(d, *a)
    with pytest.raises(ValueError, match="GPU"):
        cola.norm_rope_fwd(d, *ok)
    ok = [z(4, 128), z(4, 64), z(4, 128), z(4, 64), z(64), z(64), i(4), z(4, 128), z(4, 64), f(64), f(64)]
    for j, t in ((0, f(4, 128)), (7, z(4, 127)), (8, f(4, 64)), (9, z(64)), (10, f(63))):
        a = list(ok)
        a[j] = t
        with pytest.raises(ValueError):
            cola.norm_rope_bwd(d, *a)
    c, K = cola.cache_desc(3, 16, 1, 64), z(3, 1, 16, 64)
    with pytest.raises(ValueError):
        cola.norm_append(d, c, z(4, 128), z(4, 64), z(4, 64), z(64), z(63), None, i(4), z(4, 128), K, K)
    with pytest.raises(ValueError):
        cola.norm_append(d, c, z(4, 128), z(4, 64), z(4, 63), z(64), z(64), None, i(4), z(4, 128), K, K)
    m = cola.tree_map_desc(2, 4, 70)
    good = [i(4), i(2), i(3), torch.zeros((4, 2), dtype=torch.int64), i(4)]
    for j, t in ((0, i(3)), (1, i(1)), (2, i(2)), (3, good[3][:, :1]), (3, i(4, 2)), (4, i(4).long())):
        a = list(good)
        a[j] = t
        with pytest.raises(ValueError):
            cola.tree_map(m, *a)
    ad = cola.prefix_attn_desc(2, 3, 2, 20, 40, 65)
    good = [z(3, 128), K, K, i(2), i(2, 3), i(2), i(3), torch.zeros((3, 2), dtype=torch.int64), z(3, 128), f(2, 3)]
    for j, t in ((7, torch.zeros((3, 1), dtype=torch.int64)), (7, i(3, 2)), (7, torch.zeros((2, 2), dtype=torch.int64)), (0, z(3, 127))):
        a = list(good)
        a[j] = t
        with pytest.raises(ValueError):
            cola.tree_attn(ad, c, *a)
    d = cola.logits_desc(4, 40, 2, 6, 3, n_bias=5, n_allowed=4)
    good = dict(history=i(2, 6), prompt_len=i(2), hist_len=i(2), draft=i(4), mask=torch.zeros((4, 1), dtype=torch.int64), repetition=f(2),
                presence=f(2), frequency=f(2), bias_start=i(3), bias_token=i(5), bias=f(5), allowed=i(4, 2), allowed_row=i(4))
    for key, t in dict(history=i(2, 5), prompt_len=i(1), draft=i(3), mask=i(4, 1), repetition=i(2), bias_start=i(2), bias=f(4),
                       allowed=i(4, 3), allowed_row=i(4).long()).items():
        with pytest.raises(ValueError, match=key):
            cola.logits_adjust(d, cola.logits_rules(**{**good, key: t}), f(4, 40), i(3), f(4, 40))
    with pytest.raises(ValueError, match="GPU"):
        cola.logits_adjust(d, cola.logits_rules(**good), f(4, 40), i(3), f(4, 40))
    for bad in (z(4, 40), f(4, 39), f(3, 40)):
        with pytest.raises(ValueError):
            cola.logits_adjust(d, cola.logits_rules(**good), f(4, 40), i(3), bad)
    with pytest.raises(ValueError, match="rules"):
        cola.logits_adjust(d, (), f(4, 40), i(3), f(4, 40))
