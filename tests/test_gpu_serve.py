"""The serving operators on the GPU against their definitions in 64 bits
(tests/serve_ref.py), element by element within the bounds derived there: odd and
smallest sizes, layouts and scalings, far positions, strides and alignments,
padded batches, missing pages, lengths of zero and one, masked infinities and
NaN; gradients against the formula and against differences; streams, graphs,
workspace contents; and a run of them together as a program uses them."""
import math

import numpy as np
import pytest
import torch

import serve_ref as R
from paper_2502_10940_amd import cola

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module", autouse=True)
def _device():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    cola.lib()
    yield


def rand(seed, shape, dtype, std=1.0):
    x = np.random.default_rng(seed).standard_normal(shape).astype(np.float32) * std
    return torch.from_numpy(x).to(DT[dtype]).to(DEV)


def f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


def pitched(x, ld, offset=0, fill=float("nan")):
    """x's rows at a pitch of ld, `offset` elements into a buffer of `fill`."""
    T, w = x.shape
    buf = torch.full((T * ld + offset + 64,), fill, dtype=x.dtype, device=DEV)
    v = buf.as_strided((T, w), (ld, 1), offset)
    v.copy_(x)
    return v, buf


# ---------------------------------------------------------------------------
# rotation
# ---------------------------------------------------------------------------

SCALINGS = {"none": {}, "linear": dict(factor=3.0), "base": dict(factor=4.0),
            "yarn": dict(factor=8.0, orig_len=512, low=1.0, high=32.0),
            "wavelength": dict(factor=8.0, orig_len=8192, low=1.0, high=4.0)}

# (T, heads_q, heads_k, head_dim, rot_dim)
ROPE = [(1, 1, 1, 2, 2), (1, 32, 8, 128, 128), (3, 2, 1, 64, 32), (5, 3, 3, 80, 40), (17, 5, 2, 96, 96), (2, 1, 0, 33, 10),
        (4, 0, 2, 7, 0), (300, 8, 8, 64, 64), (9, 12, 4, 256, 64), (2, 2, 2, 512, 512), (1031, 16, 2, 128, 64),
        (7, 1, 1, 20, 12)]


@pytest.mark.parametrize("layout", ("half", "interleaved"))
@pytest.mark.parametrize("dtype", ("bf16", "f32"))
@pytest.mark.parametrize("case", range(len(ROPE)), ids=["%dx%d+%dx%d-%d" % c for c in ROPE])
def test_rope(case, dtype, layout):
    T, hq, hk, hd, rot = ROPE[case]
    name = sorted(SCALINGS)[case % len(SCALINGS)]
    if name == "base" and rot <= 2:
        name = "linear"
    sc = dict(SCALINGS[name], base=500000.0 if case % 2 else 10000.0)
    rng = np.random.default_rng(100 + case)
    pos = rng.integers(0, 1 << 20, T)
    pos[0] = (2 ** 31 - 1) if case % 2 else -5
    m = 1.25 if case % 3 == 0 else 0.0
    q, k = rand(case, (T, max(hq, 1) * hd), dtype), rand(case + 50, (T, max(hk, 1) * hd), dtype)
    d = cola.rope_desc(T, hq, hk, hd, rot, dtype, layout, name, mscale=m, **sc)
    for fn, back in ((cola.rope_fwd, False), (cola.rope_bwd, True)):
        qo, ko = torch.full_like(q, math.nan), torch.full_like(k, math.nan)
        fn(d, q if hq else None, k if hk else None, i32(pos), qo if hq else None, ko if hk else None)
        torch.cuda.synchronize()
        scale = m or R.frequencies(max(rot, 4), name, **sc)[1]
        for h, x, got in ((hq, q, qo), (hk, k, ko)):
            if h == 0:
                assert torch.isnan(got).all()
                continue
            ref = R.rope(f64(x), h, hd, rot, pos, layout, back, m, scaling=name, **sc)
            err = np.abs(f64(got) - ref)
            assert (err <= R.rope_bound(f64(x), h, hd, rot, ref, dtype, layout, scale)).all(), (fn.__name__, err.max())


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
def test_rope_pitches_alignment_and_in_place(dtype):
    """Slices of one buffer at an odd pitch and an odd start: the same bits as tight
    rows, nothing else touched; in place too; positions by sequence."""
    T, hq, hk, hd, seq = 37, 4, 2, 64, 10
    q, k = rand(1, (T, hq * hd), dtype), rand(2, (T, hk * hd), dtype)
    want = [torch.empty_like(q), torch.empty_like(k)]
    cola.rope_fwd(cola.rope_desc(T, hq, hk, hd, dtype=dtype, seq_len=seq), q, k, None, *want)
    pos = np.arange(T) % seq
    for x, h, w in ((q, hq, want[0]), (k, hk, want[1])):
        ref = R.rope(f64(x), h, hd, hd, pos)
        assert (np.abs(f64(w) - ref) <= R.rope_bound(f64(x), h, hd, hd, ref, dtype)).all()
    for ld_q, ld_k, off in ((hq * hd + hk * hd, hq * hd + hk * hd, 8), (hq * hd + 3, hk * hd + 1, 1), (hq * hd + 37, hk * hd, 5)):
        (pq, bq), (pk, bk) = pitched(q, ld_q, off), pitched(k, ld_k, off)
        before = [bq.clone(), bk.clone()]
        oq, ob = pitched(torch.zeros_like(q), hq * hd + 5, 3)
        ok, okb = pitched(torch.zeros_like(k), hk * hd + 7, 1)
        d = cola.rope_desc(T, hq, hk, hd, dtype=dtype, seq_len=seq, ldq=ld_q, ldk=ld_k, ldqo=hq * hd + 5, ldko=hk * hd + 7)
        cola.rope_fwd(d, pq, pk, None, oq, ok)
        assert torch.equal(oq, want[0]) and torch.equal(ok, want[1])
        for b, x, n in ((ob, oq, q), (okb, ok, k)):
            assert torch.isnan(b).sum() == b.numel() - n.numel()         # the padding stayed
        assert all(torch.equal(torch.nan_to_num(a), torch.nan_to_num(b)) for a, b in zip(before, (bq, bk)))
        d = cola.rope_desc(T, hq, hk, hd, dtype=dtype, seq_len=seq, ldq=ld_q, ldk=ld_k, ldqo=ld_q, ldko=ld_k)
        cola.rope_fwd(d, pq, pk, None, pq, pk)
        assert torch.equal(pq, want[0]) and torch.equal(pk, want[1])


@pytest.mark.parametrize("layout", ("half", "interleaved"))
def test_rope_gradient_against_differences(layout):
    """<dq, e> against the change of <y, g> for a change e of the input: the map is
    linear, so a step of one unit has no truncation error."""
    T, h, hd, rot = 6, 2, 32, 24
    x, e, g = (rand(s, (T, h * hd), "f32") for s in (1, 2, 3))
    pos = i32([0, 1, 5, 100, 70000, 3])
    d = cola.rope_desc(T, h, 0, hd, rot, "f32", layout, "yarn", **SCALINGS["yarn"])
    y = [torch.empty_like(x) for _ in range(3)]
    cola.rope_fwd(d, x, None, pos, y[0], None)
    cola.rope_fwd(d, x + e, None, pos, y[1], None)
    cola.rope_bwd(d, g, None, pos, y[2], None)
    change = ((f64(y[1]) - f64(y[0])) * f64(g)).sum()
    grad = (f64(y[2]) * f64(e)).sum()
    # fp32 rounding of x + e (2^-24 |x + e|), of y (2^-21 of a pair's magnitude): the sum over all elements of |g|
    bound = 2.0 ** -20 * 1.3 * (2 * np.abs(f64(x)) + 2 * np.abs(f64(e))).max() * 2 * np.abs(f64(g)).sum()
    assert abs(change - grad) <= bound
    # and there and back: the rotation times its scale squared
    back = torch.empty_like(x)
    cola.rope_bwd(d, y[0], None, pos, back, None)
    m = R.frequencies(rot, "yarn", **SCALINGS["yarn"])[1]
    want = f64(x).reshape(T, h, hd).copy()
    want[..., :rot] *= m * m
    assert np.abs(f64(back).reshape(T, h, hd) - want).max() <= 2.0 ** -19 * 2 * m * m * 5


# ---------------------------------------------------------------------------
# into the cache
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ("bf16", "f32"))
@pytest.mark.parametrize("case", [(1, 1, 1, 64, 64, 16), (19, 8, 2, 128, 128, 32), (33, 5, 5, 80, 40, 16), (7, 0, 3, 33, 0, 64),
                                  (400, 4, 4, 64, 64, 128)], ids=str)
def test_append(case, dtype):
    T, hq, hk, hd, rot, page = case
    rng = np.random.default_rng(T)
    pages = -(-T // page) + 2
    slots = rng.permutation(pages * page)[:T].astype(np.int64)
    if T > 4:
        slots[1], slots[2], slots[3] = -1, pages * page, 2 ** 31 - 1      # rows that are not stored
    pos = rng.integers(0, 5000, T)
    q, k, v = (rand(s, (T, max(h, 1) * hd), dtype) for s, h in ((1, hq), (2, hk), (3, hk)))
    K, V = rand(4, (pages, hk, page, hd), dtype), rand(5, (pages, hk, page, hd), dtype)
    K0, V0 = K.clone(), V.clone()
    qo = torch.empty_like(q)
    d, c = cola.rope_desc(T, hq, hk, hd, rot, dtype), cola.cache_desc(pages, page, hk, hd, dtype)
    cola.cache_append(d, c, q if hq else None, k, v, i32(pos), i32(slots), qo if hq else None, K, V)
    # the rotation is rope_fwd's, bit for bit
    want_q, want_k = torch.empty_like(q), torch.empty_like(k)
    cola.rope_fwd(d, q if hq else None, k, i32(pos), want_q if hq else None, want_k)
    assert hq == 0 or torch.equal(qo, want_q)
    for t in range(T):
        if 0 <= slots[t] < pages * page:
            p, o = divmod(int(slots[t]), page)
            K0[p, :, o], V0[p, :, o] = want_k[t].view(hk, hd), v[t].view(hk, hd)
    assert torch.equal(K, K0) and torch.equal(V, V0)


@pytest.mark.parametrize("layout", ("half", "interleaved"))
def test_large_results_are_the_small_ones(layout):
    """Results of more than 48 MB leave by other stores: the bits of the same rows in parts."""
    T, hq, hk, hd, page = 6300, 32, 8, 128, 16
    q, k, v = (rand(s, (T, h * hd), "bf16") for s, h in ((1, hq), (2, hk), (3, hk)))
    pos = torch.arange(T, dtype=torch.int32, device=DEV) * 7
    slots = torch.randperm(T, device=DEV).int()
    pages = -(-T // page)
    c = cola.cache_desc(pages, page, hk, hd)
    got, want = ([torch.zeros_like(q), torch.zeros_like(k)] + [torch.zeros((pages, hk, page, hd), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
                 for _ in range(2))
    for res, step in ((got, T), (want, 1575)):
        for at in range(0, T, step):
            n = slice(at, at + step)
            d = cola.rope_desc(step, hq, hk, hd, 64, layout=layout)
            cola.rope_bwd(d, q[n], k[n], pos[n], res[0][n], res[1][n])
            cola.cache_append(d, c, q[n], k[n], v[n], pos[n], slots[n], torch.empty_like(q[n]), res[2], res[3])
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    qo = torch.empty_like(q)
    cola.cache_append(cola.rope_desc(T, hq, hk, hd, 64, layout=layout), c, q, k, v, pos, slots, qo, got[2], got[3])
    back = torch.empty_like(q)
    cola.rope_fwd(cola.rope_desc(T, hq, 0, hd, 64, layout=layout), q, None, pos, back, None)
    assert torch.equal(qo, back)


def test_append_past_4_gib():
    """Slots whose bytes lie past 2^32 of the cache."""
    hk, hd, page = 8, 128, 64
    pages = (9 << 29) // (hk * hd * page)            # 4.5 Gi elements of 2 bytes
    K = torch.zeros((pages, hk, page, hd), dtype=torch.bfloat16, device=DEV)
    V = torch.zeros_like(K)
    slots = [0, pages * page // 2 + 3, pages * page - 1]
    k, v = rand(1, (3, hk * hd), "bf16"), rand(2, (3, hk * hd), "bf16")
    d, c = cola.rope_desc(3, 0, hk, hd, 0), cola.cache_desc(pages, page, hk, hd)
    cola.cache_append(d, c, None, k, v, None, i32(slots), None, K, V)
    for t, s in enumerate(slots):
        p, o = divmod(s, page)
        assert torch.equal(K[p, :, o].reshape(-1), k[t]) and torch.equal(V[p, :, o].reshape(-1), v[t])
    assert int((K != 0).sum()) == int((k != 0).sum())
    # and attention reads them there: one request whose only page is the last
    q = rand(3, (1, hk * hd), "bf16")
    out = torch.empty_like(q)
    ad = cola.prefix_attn_desc(1, 1, hk, 0, page, 1)
    ws = torch.empty(max(1, cola.prefix_attn_workspace_bytes(ad, c)), dtype=torch.uint8, device=DEV)
    cola.prefix_attn(ad, c, q, K, V, None, i32([[pages - 1]]), i32([page]), None, out, None, ws)
    ref, _, w = R.attention(f64(q), f64(K[-1:]), f64(V[-1:]), hk, [], 0, [[0]], [page], [0, 1], page)
    assert (np.abs(f64(out) - ref) <= R.attention_bound(ref, w, page)).all()


@pytest.mark.parametrize("rows", (1, 20, 64))
def test_attention_past_4_gib(rows):
    """Every kind of tile reads pages whose bytes lie past 2^32 of the cache."""
    hk, hd, page = 2, 64, 64
    pages = (5 << 29) // (hk * hd * page)            # 2.5 Gi elements of 2 bytes
    K = torch.empty((pages, hk, page, hd), dtype=torch.bfloat16, device=DEV)
    V = torch.empty_like(K)
    last = [pages - 1, pages // 2, 0]                # in the small cache: 0, 1, 2
    for x, seed in ((K, 1), (V, 2)):
        for p in last:
            x[p] = rand(seed + p % 7, (hk, page, hd), "bf16")
    small = [f64(torch.stack([x[p] for p in last])) for x in (K, V)]
    hq, kv, L = 4, 2 * page - 5, 60
    q = rand(3, (rows, hq * hd), "bf16")
    out, lse = torch.empty_like(q), torch.empty((hq, rows), device=DEV)
    d, c = cola.prefix_attn_desc(1, rows, hq, L, kv, rows), cola.cache_desc(pages, page, hk, hd)
    ws = torch.empty(max(1, cola.prefix_attn_workspace_bytes(d, c)), dtype=torch.uint8, device=DEV)
    cola.prefix_attn(d, c, q, K, V, i32([last[0]]), i32([last[1:]]), i32([kv]), i32([0, rows]), out, lse, ws)
    ref, rl, w = R.attention(f64(q), *small, hq, [0], L, [[1, 2]], [kv], [0, rows], page)
    assert (np.abs(f64(out) - ref) <= R.attention_bound(ref, w, L + kv)).all()
    assert (np.abs(f64(lse) - rl) <= R.lse_bound(rl, L + kv)).all()


# ---------------------------------------------------------------------------
# tables
# ---------------------------------------------------------------------------

def run_map(kv, n, free, at, table, page, T, pos0):
    d = cola.page_map_desc(len(kv), T, page, table.shape[1], len(free), pos0)
    t = i32(table) if table.size else torch.empty(table.shape, dtype=torch.int32, device=DEV)
    start, slots, pos = (torch.full((m,), -77, dtype=torch.int32, device=DEV) for m in (len(kv) + 1, T, T))
    nxt = i32([-77])
    cola.page_map(d, i32(kv), i32(n), i32(free), None if at is None else i32([at]), t, start, slots, pos, nxt)
    torch.cuda.synchronize()
    return t.cpu().numpy(), start.tolist(), slots.tolist(), pos.tolist(), int(nxt[0])


def check_map(kv, n, free, at, table, page, T, pos0):
    got = run_map(kv, n, free, at, table, page, T, pos0)
    want = R.page_map(kv, n, free, at or 0, table, page, T, pos0)
    assert (got[0] == want[0]).all()
    assert got[1:] == (want[1], want[2], want[3], want[4])


@pytest.mark.parametrize("n_req", (1, 2, 63, 64, 65, 255, 256, 257, 1000, 4096))
@pytest.mark.parametrize("page", (1, 16, 128))
def test_page_map(n_req, page):
    rng = np.random.default_rng(n_req + page)
    n = rng.integers(0, 40 if n_req < 300 else 6, n_req)
    kv = n + rng.integers(0, 60, n_req)
    width = int(-(-kv.max() // page)) + 1
    table = rng.integers(0, 10 ** 5, (n_req, width))
    free = rng.permutation(10 ** 6)[: 64 * n_req + 10]
    check_map(kv, n, free, 3, table, page, int(n.sum()) + 13, 100)


def test_page_map_edges():
    t = np.arange(12).reshape(3, 4) + 100
    free = np.arange(50, 70)
    check_map([0, 0, 0], [0, 0, 0], free, None, t, 16, 5, 0)                   # nothing to do
    check_map([1, 16, 17], [1, 16, 17], free, None, t, 16, 34, 7)              # fresh requests: one, a page, a page and one
    check_map([16, 17, 32], [1, 1, 1], free, 2, t, 16, 3, 0)                   # the last of a page, the first of the next
    check_map([-5, 10, 10], [3, -2, 99], free, 0, t, 16, 20, 0)                # lengths outside their range
    check_map([40, 40, 40], [40, 40, 40], free[:5], 0, t, 16, 120, 0)          # the list ends too early
    check_map([40, 40, 40], [9, 9, 9], free, 18, t, 16, 27, 0)                 # ... from its middle
    check_map([100, 3, 100], [60, 3, 5], free, 0, t, 16, 70, 0)                # tokens past the table's row
    check_map([40, 40, 40], [40, 40, 40], free, 0, t, 16, 50, 0)               # more tokens than rows
    check_map([5, 6, 7], [5, 6, 7], free, 0, t, 16, 0, 0)                      # no rows
    check_map([], [], free, 4, np.zeros((0, 3), np.int64), 16, 3, 0)           # no requests
    check_map([5], [5], free, -3, np.zeros((1, 2), np.int64), 1, 6, 0)         # a place before the list, a narrow table
    big = 2 ** 31 - 1
    got = run_map([big, big], [big, big], free, 0, np.zeros((2, 1), np.int64), 4096, 4, 5)
    assert got[1] == [0, big, big] and got[2] == [50 * 4096 + i for i in range(4)] and got[3] == [5, 6, 7, 8]


def test_page_map_twice_writes_the_same():
    rng = np.random.default_rng(0)
    n, kv = rng.integers(1, 5, 300), rng.integers(5, 100, 300)
    t = i32(rng.integers(0, 1000, (300, 8)))
    d = cola.page_map_desc(300, 2000, 16, 8, 3000, 0)
    bufs = [i32(kv), i32(n), i32(rng.permutation(3000)), i32([5]), t] + [torch.zeros(m, dtype=torch.int32, device=DEV) for m in (301, 2000, 2000, 1)]
    cola.page_map(d, *bufs)
    first = [b.clone() for b in bufs]
    cola.page_map(d, *bufs)
    assert all(torch.equal(a, b) for a, b in zip(first, bufs))


# ---------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------

class Batch:
    """A cache with its pages in random order, requests' lengths, and q."""

    def __init__(self, seed, new, kv, L, hq, hk, hd, page, pad=0, lead=0, spare=2, ldq=0, ldo=0, scale=0.0, max_kv=None,
                 max_new=None, junk=float("nan")):
        rng = np.random.default_rng(seed)
        self.new, self.kv, self.L, self.hq, self.hk, self.hd, self.page = list(new), list(kv), L, hq, hk, hd, page
        self.start = [lead]
        for x in new:
            self.start.append(self.start[-1] + x)
        T = self.T = self.start[-1] + pad
        pages = [-(-x // page) for x in kv]
        shared = -(-L // page)
        total = sum(pages) + shared + spare
        ids = rng.permutation(total)
        self.ptab = ids[:shared]
        self.max_kv = max([0] + self.kv) if max_kv is None else max_kv
        self.max_new = max([1] + self.new) if max_new is None else max_new
        width = max(1, -(-self.max_kv // page))
        self.tab = np.full((len(new), width), -1)
        at = shared
        for r, n in enumerate(pages):
            self.tab[r, :n] = ids[at:at + n]
            at += n
        # what no token has been written to holds `junk`
        held = np.zeros((total, page), bool)
        for j in range(L):
            held[self.ptab[j // page], j % page] = True
        for r, n in enumerate(kv):
            for j in range(n):
                held[self.tab[r, j // page], j % page] = True
        held = torch.from_numpy(held).to(DEV)[:, None, :, None]
        self.K, self.V = (torch.where(held, rand(seed + i, (total, hk, page, hd), "bf16"), torch.tensor(junk, dtype=torch.bfloat16, device=DEV))
                          for i in (1, 2))
        self.q = rand(seed + 3, (T, hq * hd), "bf16", 1.5)
        self.ldq, self.ldo, self.scale = ldq, ldo, scale

    def desc(self):
        return (cola.prefix_attn_desc(len(self.new), self.T, self.hq, self.L, self.max_kv, self.max_new, 0, self.ldq, self.ldo, self.scale),
                cola.cache_desc(self.K.shape[0], self.page, self.hk, self.hd))

    def run(self, ws_fill=0xFF, lse=True, start=True, stream=None):
        d, c = self.desc()
        q = self.q if not self.ldq else pitched(self.q, self.ldq, 8)[0]
        out = torch.full((self.T, self.ldo or self.hq * self.hd), 7.0, dtype=torch.bfloat16, device=DEV)
        ls = torch.full((self.hq, self.T), 7.0, device=DEV) if lse else None
        n = cola.prefix_attn_workspace_bytes(d, c)
        ws = torch.full((n,), ws_fill, dtype=torch.uint8, device=DEV) if n else None
        cola.prefix_attn(d, c, q, self.K, self.V, i32(self.ptab) if self.L else None, i32(self.tab) if self.max_kv else None,
                         i32(self.kv) if self.max_kv else None, i32(self.start) if start else None, out, ls, ws, stream=stream)
        torch.cuda.synchronize()
        return out, ls

    def reference(self):
        return R.attention(f64(self.q), f64(self.K), f64(self.V), self.hq, self.ptab, self.L, self.tab, self.kv, self.start, self.page,
                           self.scale or None)

    def check(self, **kw):
        out, lse = self.run(**kw)
        ref, rl, w = self.reference()
        lo, hi, W = self.start[0], self.start[-1], self.hq * self.hd
        o = f64(out)
        assert (o[:lo] == 7).all() and (o[hi:] == 7).all() and (o[:, W:] == 7).all(), "rows of no request are left"
        keys = self.L + max([0] + self.kv)
        err = np.abs(o[lo:hi, :W] - ref[lo:hi])
        assert np.isfinite(o[lo:hi, :W]).all()
        assert (err <= R.attention_bound(ref, w, keys)[lo:hi]).all(), err.max()
        if lse is not None:
            g = f64(lse)
            assert (g[:, :lo] == 7).all() and (g[:, hi:] == 7).all()
            g, e = g[:, lo:hi], rl[:, lo:hi]
            assert (np.isneginf(g) == np.isneginf(e)).all()
            fin = np.isfinite(e)
            assert (np.abs(g[fin] - e[fin]) <= R.lse_bound(e[fin], keys)).all()
        return out, lse


ATTN = {
    # decode: one token each
    "one": dict(new=[1], kv=[1], L=0, hq=1, hk=1, hd=64, page=16),
    "one-key-prefix": dict(new=[1], kv=[1], L=1, hq=2, hk=1, hd=128, page=16),
    "page-ends": dict(new=[1] * 6, kv=[15, 16, 17, 31, 32, 33], L=33, hq=4, hk=2, hd=64, page=16),
    "blocks": dict(new=[1] * 5, kv=[127, 128, 129, 255, 257], L=128, hq=8, hk=8, hd=128, page=32, pad=3),
    "group-of-3": dict(new=[1] * 7, kv=[5, 90, 1, 300, 64, 2, 40], L=70, hq=6, hk=2, hd=64, page=64),
    "group-of-20": dict(new=[1] * 3, kv=[50, 7, 200], L=45, hq=20, hk=1, hd=128, page=16),
    "no-prefix": dict(new=[1] * 4, kv=[3, 700, 31, 260], L=0, hq=4, hk=4, hd=64, page=16),
    "no-own": dict(new=[1] * 5, kv=[0] * 5, L=77, hq=4, hk=2, hd=128, page=16, pad=2, lead=1),
    "nothing": dict(new=[1, 2], kv=[0, 0], L=0, hq=2, hk=2, hd=64, page=16, pad=1),
    "some-empty": dict(new=[1, 1, 0, 1], kv=[0, 5, 9, 0], L=0, hq=2, hk=2, hd=64, page=16),
    "long-prefix": dict(new=[1] * 3, kv=[2, 40, 9], L=9001, hq=2, hk=1, hd=64, page=256),
    "many-requests": dict(new=[1] * 70, kv=[(37 * i) % 90 for i in range(70)], L=50, hq=4, hk=4, hd=64, page=16),
    # several tokens each
    "chunk": dict(new=[5, 1, 17, 0, 2], kv=[5, 30, 40, 12, 2], L=35, hq=4, hk=2, hd=64, page=16, pad=4, lead=2),
    "chunk-group": dict(new=[33, 16, 1], kv=[100, 16, 9], L=20, hq=8, hk=2, hd=128, page=16),
    "fresh": dict(new=[64, 65, 1], kv=[64, 65, 1], L=0, hq=2, hk=2, hd=128, page=32),
    "older-than-rows": dict(new=[9, 4], kv=[3, 0], L=0, hq=2, hk=2, hd=64, page=16),
    "older-than-rows-prefix": dict(new=[9, 40], kv=[3, 7], L=18, hq=2, hk=2, hd=64, page=16),
    "wide": dict(new=[130, 70], kv=[200, 131], L=100, hq=2, hk=1, hd=64, page=64),
    "wide-128": dict(new=[150, 20, 131], kv=[290, 20, 140], L=161, hq=4, hk=1, hd=128, page=16, pad=1),
}


# Each kernel of the launch plan: how the prefix's rows are tiled (along with the
# requests, 16, 32 or 128 to a tile), and a request's own (one token: four waves or
# one to a tile; 16, 32 or 128 rows).  (new, kv, L, hq, hk)
KERNELS = {
    "along-flat": ([1, 1], [30, 70], 90, 2, 1), "along-one": ([5, 2], [30, 70], 90, 2, 1), "along-two": ([12, 3], [30, 70], 90, 2, 1),
    "along-wide": ([50, 5], [70, 20], 90, 2, 1), "along-wide-tiles": ([150, 1, 90], [300, 40, 90], 333, 4, 2),
    "along-wide-no-own": ([70, 130], [0, 0], 90, 2, 1),
    "along-no-own": ([1, 1, 1], [0, 0, 0], 90, 2, 1),
    "one-one": ([3, 2], [50, 9], 700, 2, 1), "one-flat": ([1, 1], [50, 9], 700, 4, 2),
    "one-solo": ([1] * 514, [(7 * i) % 50 for i in range(514)], 0, 8, 8),
    "two-one": ([4] * 6, [4, 10, 33, 50, 7, 64], 700, 2, 2), "two-flat": ([1] * 12, [5 * i for i in range(12)], 700, 4, 2),
    "two-two": ([20, 5], [30, 100], 700, 2, 2), "two-no-prefix": ([20, 5], [30, 100], 0, 2, 2),
    "wide-one": ([3] * 20, [3 + 9 * i for i in range(20)], 700, 2, 2), "wide-flat": ([1] * 40, [7 * i for i in range(40)], 700, 4, 2),
    "wide-solo": ([1] * 513, [(5 * i) % 40 for i in range(513)], 650, 8, 8),
    "wide-two": ([20] * 3, [20, 50, 131], 700, 2, 2), "wide-wide": ([50, 40], [50, 333], 700, 2, 2),
    # many parts of the keys, of the requests' own and of the prefix
    "parts": ([1, 1], [5000, 3], 3000, 2, 1), "parts-own": ([40], [3000], 0, 2, 2), "prompt": ([300], [300], 0, 6, 3), "prompt-parts": ([1000], [1100], 0, 2, 1),
    "prompt-behind": ([500], [530], 1200, 2, 2), "parts-wide": ([70, 40, 1, 50, 200], [5000, 200, 4100, 3, 1700], 0, 4, 2),
    "parts-chunk": ([9, 30], [2000, 30], 2500, 2, 1),
}


@pytest.mark.parametrize("hd", (64, 128))
@pytest.mark.parametrize("name", sorted(KERNELS))
def test_attention_kernels(name, hd):
    new, kv, L, hq, hk = KERNELS[name]
    print("kernels", name, hd, flush=True)
    Batch(len(name) + hd, new, kv, L, hq, hk, hd, 16 if hd == 64 else 64, pad=2).check()


@pytest.mark.parametrize("name", sorted(ATTN))
def test_attention(name):
    print("attention", name, ATTN[name], flush=True)
    Batch(len(name), **ATTN[name]).check()


def test_attention_without_starts_pitches_and_scale():
    b = Batch(1, [1] * 9, [4, 0, 17, 60, 33, 1, 16, 100, 12], 40, 4, 2, 64, 16, pad=3, ldq=4 * 64 + 24, ldo=4 * 64 + 8, scale=0.3)
    a, la = b.check()
    c, lc = b.check(start=False)
    assert torch.equal(a, c) and torch.equal(la, lc)
    d, _ = b.run(lse=False)
    assert torch.equal(a, d)


def test_attention_bounds_above_the_lengths():
    """Descriptors sized for more than the batch holds give the same values."""
    kw = dict(new=[1, 3, 2], kv=[20, 65, 2], L=50, hq=4, hk=2, hd=64, page=16)
    for extra in (dict(max_kv=3000), dict(max_new=200), dict(max_kv=1000, max_new=40)):
        Batch(7, **kw, **extra).check()


def test_attention_bounds_below_the_lengths():
    """Tokens past max_kv are not seen, rows past max_new are left."""
    b = Batch(3, [1, 1], [50, 20], 0, 2, 2, 64, 16)
    ref, _, w = R.attention(f64(b.q), f64(b.K), f64(b.V), 2, [], 0, b.tab, [30, 20], b.start, 16)
    b.max_kv, tab = 30, b.tab
    b.tab = np.ascontiguousarray(tab[:, :2])
    out, _ = b.run()
    assert (np.abs(f64(out) - ref) <= R.attention_bound(ref, w, 30)).all()
    b = Batch(4, [5, 2], [9, 20], 11, 2, 2, 64, 16)
    full, _ = b.run()
    b.max_new = 3
    out, lse = b.run()
    assert (out[3:5] == 7).all() and (lse[:, 3:5] == 7).all()
    keep = [0, 1, 2, 5, 6]
    ref, _, w = b.reference()
    assert (np.abs(f64(out) - ref) <= R.attention_bound(ref, w, 31))[keep].all()


@pytest.mark.parametrize("bad", (-1, 10 ** 6, 2 ** 31 - 1, -2 ** 31))
def test_attention_missing_pages(bad):
    """Keys in pages outside the cache are not seen: of the prefix, of a request,
    all of a row's."""
    b = Batch(5, [1, 2, 1, 1], [70, 33, 10, 40], 64, 4, 2, 64, 16)
    b.ptab = b.ptab.copy()
    b.ptab[1] = bad
    b.tab[0, 1] = b.tab[1, 0] = b.tab[2, 0] = bad
    b.check()
    b.ptab[:] = bad
    b.tab[3, :] = bad
    b.check()


@pytest.mark.parametrize("hd, page, L", [(64, 16, 64), (64, 64, 1100), (128, 16, 1100), (128, 128, 200)])
def test_attention_missing_pages_under_wide_tiles(hd, page, L):
    """The same for tiles of 128 rows, whose stages take several pages or lie in one."""
    b = Batch(18, [70, 40, 130], [300, 40, 333], L, 4, 2, hd, page, pad=1)
    b.check()
    b.ptab = b.ptab.copy()
    b.ptab[0] = -1
    b.tab[0, 1] = 10 ** 6
    b.tab[2, -1] = -2 ** 31
    b.check()
    b.ptab[:] = -1
    b.tab[1, :] = 2 ** 31 - 1
    b.check()


def test_attention_of_pages_that_several_requests_name():
    """A page twice in a table, in two requests' tables and in the prefix's: keys are
    read where the tables say, as often as they say."""
    for new in ([1, 1, 1], [3, 9, 2], [60, 50, 33]):
        for L in (70, 1300):
            b = Batch(19, new, [90, 90, 64], L, 4, 2, 64, 16, pad=1)
            b.ptab = b.ptab.copy()
            b.ptab[2] = b.ptab[1]
            b.tab[1, :3] = b.tab[0, :3]
            b.tab[2, 1] = b.tab[2, 0]
            b.tab[0, 4] = b.ptab[0]
            b.check()


@pytest.mark.parametrize("value", (math.inf, -math.inf, math.nan))
def test_attention_masked_values_do_not_reach_a_row(value):
    """A later token whose key or value is not finite changes the rows that see it
    and no other."""
    kw = dict(new=[12, 1], kv=[40, 20], L=20, hq=4, hk=2, hd=64, page=16)
    for seed, kw in ((11, kw), (12, dict(kw, hd=128)), (13, dict(kw, new=[40, 1], L=0)), (14, dict(kw, new=[40, 1], hd=128, L=700)),
                     (15, dict(kw, new=[5, 1])), (17, dict(kw, new=[40, 1], L=1100)),
                     (16, dict(kw, new=[3, 1], hd=128, L=900))):
        b = Batch(seed, **kw)
        clean, cl = b.run()
        n = kw["new"][0]
        for key in (37, 39):
            for cache in (b.K, b.V):
                p, o = int(b.tab[0, key // 16]), key % 16
                keep = cache[p, :, o].clone()
                cache[p, :, o] = value
                out, lse = b.run()
                first = key - (40 - n)                  # the row that is this token
                assert torch.equal(out[:first], clean[:first]) and torch.equal(out[n:], clean[n:])
                assert torch.equal(lse[:, :first], cl[:, :first])
                bad = ~torch.isfinite(out[first:n].float())
                # an infinite key gives scores of either sign: a row may give it no weight
                assert bad.any() if cache is b.K else bad.all()
                if cache is b.V:
                    want = torch.full_like(out[first:n], value)
                    assert torch.equal(torch.nan_to_num(out[first:n].float(), 5.0, 9.0, -9.0), torch.nan_to_num(want.float(), 5.0, 9.0, -9.0))
                cache[p, :, o] = keep


def test_attention_unwritten_slots_hold_anything():
    for junk in (math.nan, math.inf, -3.0e38):
        Batch(6, [1, 4, 1], [17, 40, 3], 21, 4, 2, 64, 32, junk=junk).check()


def test_attention_large_scores():
    """Scores of thousands: the running maximum moves by more than any slack."""
    b = Batch(8, [1, 3], [100, 300], 90, 2, 1, 64, 16, scale=30.0)
    out, lse = b.run()
    ref, rl, _ = b.reference()
    # scores up to 2^12 in fp32 are good to 2^-12: a probability to e^(2^-11) - 1 and its rounding
    assert np.abs(f64(out) - ref).max() <= (2.0 ** -10 + 2.0 ** -7) * 4.5
    assert (np.abs(f64(lse) - rl) <= 2.0 ** -10 + 2.0 ** -22 * np.abs(rl)).all()


def test_attention_does_not_depend_on_the_workspace_s_contents_or_the_run():
    b = Batch(9, [3, 1, 20], [50, 600, 20], 700, 8, 2, 128, 16, pad=5)
    a = b.run(ws_fill=0)
    for fill in (0xFF, 0x7F, 0):
        c = b.run(ws_fill=fill)
        assert torch.equal(a[0], c[0]) and torch.equal(a[1], c[1])


def test_attention_of_one_row_does_not_depend_on_its_place():
    """The same request at another place of the batch: the same bits."""
    b = Batch(10, [1] * 6, [40] * 6, 100, 4, 4, 64, 16)
    b.q[3] = b.q[0]
    for c in (b.K, b.V):
        for j in range(b.tab.shape[1]):
            c[int(b.tab[3, j])] = c[int(b.tab[0, j])]
    out, lse = b.run()
    assert torch.equal(out[0], out[3]) and torch.equal(lse[:, 0], lse[:, 3])


# ---------------------------------------------------------------------------
# together
# ---------------------------------------------------------------------------

class Server:
    """A layer's cache, requests and buffers: append, attend, step by step."""

    def __init__(self, n, hq, hk, hd, page, L, cap, layout="half", seed=0):
        self.n, self.hq, self.hk, self.hd, self.page, self.L, self.cap = n, hq, hk, hd, page, L, cap
        self.rng = np.random.default_rng(seed)
        self.width = 8
        shared = -(-L // page)
        self.pages = shared + n * self.width
        ids = self.rng.permutation(self.pages)
        self.K = torch.full((self.pages, hk, page, hd), math.nan, dtype=torch.bfloat16, device=DEV)
        self.V = self.K.clone()
        self.ptab, self.free = i32(ids[:shared]), i32(ids[shared:])
        z = lambda *s: torch.zeros(s, dtype=torch.int32, device=DEV)
        self.kv, self.new, self.table, self.start = z(n), z(n), z(n, self.width) - 1, z(n + 1)
        self.slots, self.pos, self.at, self.next = z(cap), z(cap), z(1), z(1)
        self.q = torch.zeros((cap, (hq + 2 * hk) * hd), dtype=torch.bfloat16, device=DEV)
        self.qr = torch.zeros((cap, hq * hd), dtype=torch.bfloat16, device=DEV)
        self.out = torch.zeros_like(self.qr)
        self.lse = torch.zeros((hq, cap), device=DEV)
        self.c = cola.cache_desc(self.pages, page, hk, hd)
        ld = self.q.stride(0)
        self.rd = cola.rope_desc(cap, hq, hk, hd, layout=layout, ldq=ld, ldk=ld, ldv=ld)
        self.md = cola.page_map_desc(n, cap, page, self.width, self.free.numel(), L)
        self.ad = cola.prefix_attn_desc(n, cap, hq, L, self.width * page, cap)
        self.ws = torch.empty(max(1, cola.prefix_attn_workspace_bytes(self.ad, self.c)), dtype=torch.uint8, device=DEV)
        # the prompt that all share
        if L:
            k, v = rand(seed + 1, (L, hk * hd), "bf16"), rand(seed + 2, (L, hk * hd), "bf16")
            j = torch.arange(L, device=DEV)
            slots = (self.ptab.long()[j // page] * page + j % page).int()
            cola.cache_append(cola.rope_desc(L, 0, hk, hd, layout=layout), self.c, None, k, v, None, slots, None, self.K, self.V)
            self.history = [(R.rope(f64(k), hk, hd, hd, np.arange(L), layout), f64(v))] * n
        else:
            self.history = [(np.zeros((0, hk * hd)), np.zeros((0, hk * hd)))] * n
        self.layout = layout

    def part(self, name):
        a, b = self.hq * self.hd, (self.hq + self.hk) * self.hd
        return {"q": self.q[:, :a], "k": self.q[:, a:b], "v": self.q[:, b:]}[name]

    def step(self, stream=None):
        cola.page_map(self.md, self.kv, self.new, self.free, self.at, self.table, self.start, self.slots, self.pos, self.next, stream=stream)
        cola.cache_append(self.rd, self.c, self.part("q"), self.part("k"), self.part("v"), self.pos, self.slots, self.qr, self.K, self.V, stream=stream)
        cola.prefix_attn(self.ad, self.c, self.qr, self.K, self.V, self.ptab if self.L else None, self.table, self.kv, self.start, self.out,
                         self.lse, self.ws, stream=stream)

    def feed(self, new, seed):
        self.new.copy_(i32(new))
        self.kv += self.new
        self.q.copy_(rand(seed, tuple(self.q.shape), "bf16"))

    def check(self, new):
        """Against every request as one sequence of its own, in 64 bits."""
        torch.cuda.synchronize()
        q, k, v = (f64(self.part(x).contiguous()) for x in "qkv")
        row = 0
        for r, n in enumerate(new):
            ks, vs = self.history[r]
            p0 = len(ks)
            pos = p0 + np.arange(n)
            ks = np.concatenate([ks, R.rope(k[row:row + n], self.hk, self.hd, self.hd, pos, self.layout)])
            vs = np.concatenate([vs, v[row:row + n]])
            self.history[r] = (ks, vs)
            qs = R.rope(q[row:row + n], self.hq, self.hd, self.hd, pos, self.layout)
            for i in range(n):
                for h in range(self.hq):
                    x, y = slice(h * self.hd, (h + 1) * self.hd), h // (self.hq // self.hk)
                    y = slice(y * self.hd, (y + 1) * self.hd)
                    s = ks[:p0 + i + 1, y] @ qs[i, x] / math.sqrt(self.hd)
                    w = np.exp(s - s.max())
                    w /= w.sum()
                    # q and k rounded to bf16 after turning: scores to 2^-7 of |q||k|/sqrt(hd) a product, weights by e^that
                    ds = 2.0 ** -7 * (np.abs(ks[:p0 + i + 1, y]) @ np.abs(qs[i, x]) / math.sqrt(self.hd)).max()
                    tol = (2 * (math.exp(ds) - 1) + 2.0 ** -6) * (w @ np.abs(vs[:p0 + i + 1, y])) + 2.0 ** -8
                    assert (np.abs(f64(self.out[row + i, x]) - w @ vs[:p0 + i + 1, y]) <= tol).all(), (r, i, h)
            row += n
        assert (self.out[row:] == 0).all(), "idle rows are left"
        self.at.copy_(self.next)


@pytest.mark.parametrize("shape", [(5, 4, 2, 64, 16, 21, 40, "half"), (3, 2, 2, 128, 32, 0, 30, "interleaved")], ids=str)
def test_serving_steps(shape):
    n, hq, hk, hd, page, L, cap, layout = shape
    s = Server(n, hq, hk, hd, page, L, cap, layout)
    rng = np.random.default_rng(n)
    for i in range(6):
        new = rng.integers(1, 7, n) if i % 3 == 0 else np.ones(n, int)
        if i == 4:
            new[1] = 0
        s.out.zero_()
        s.feed(new, 100 + i)
        s.step()
        s.check(new)


def test_serving_step_in_a_graph():
    """One captured step replayed: it follows the lengths and the free list."""
    s, e = (Server(4, 4, 2, 64, 16, 33, 12) for _ in range(2))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        s.feed([1, 1, 1, 1], 1)
        s.step()
    torch.cuda.current_stream().wait_stream(side)
    e.feed([1, 1, 1, 1], 1)
    e.step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        s.step()
    for i, new in enumerate(([3, 1, 2, 1], [1, 1, 1, 1], [0, 9, 1, 1], [1, 1, 0, 2])):
        for x in (s, e):
            x.at.copy_(x.next)
            x.out.zero_()
            x.feed(new, 50 + i)
        g.replay()
        e.step()
        torch.cuda.synchronize()
        for a, b in ((s.out, e.out), (s.table, e.table), (s.slots, e.slots), (s.next, e.next)):
            assert torch.equal(a, b)
        assert torch.equal(torch.nan_to_num(s.K), torch.nan_to_num(e.K))
        live = int(s.start[-1])
        assert torch.equal(s.lse[:, :live], e.lse[:, :live])


@pytest.mark.parametrize("shape", [(3, 45, 128, 2), (2, 130, 256, 2)], ids=("hd64", "hd128"))
def test_the_block_s_attention_through_the_cache(shape):
    """The decoder block's q, k and v, appended as three prompts and attended, give
    the block's attention (the layer's contract for bf16, 1e-2)."""
    from paper_2502_10940_amd import inputs as I
    from block_runner import BlockRun
    n_seq, L, d, heads = shape
    T, hd, page = n_seq * L, d // heads, 16
    run = BlockRun(I.block_inputs(77, n_seq, L, d, 96, 32), n_seq, L, d, 96, heads, 32)
    run.forward()
    q, k, v, att = (run.slot(n, d) for n in ("q", "k", "v", "att"))
    pages = -(-L // page)
    table = torch.randperm(n_seq * pages, device=DEV).int().view(n_seq, pages)
    t = torch.arange(T, device=DEV)
    slots = (table.long()[t // L, t % L // page] * page + t % L % page).int()
    c = cola.cache_desc(n_seq * pages, page, heads, hd)
    K, V = (torch.zeros((n_seq * pages, heads, page, hd), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    qr, out = torch.empty_like(q), torch.empty_like(q)
    ld = q.stride(0)
    cola.cache_append(cola.rope_desc(T, heads, heads, hd, seq_len=L, ldq=ld, ldk=k.stride(0), ldv=v.stride(0), ldqo=qr.stride(0)), c, q, k, v, None, slots,
                      qr, K, V)
    ad = cola.prefix_attn_desc(n_seq, T, heads, 0, L, L, ldq=qr.stride(0), ldo=out.stride(0))
    ws = torch.empty(max(1, cola.prefix_attn_workspace_bytes(ad, c)), dtype=torch.uint8, device=DEV)
    cola.prefix_attn(ad, c, qr, K, V, None, table, i32([L] * n_seq), i32(np.arange(n_seq + 1) * L), out, None, ws)
    torch.cuda.synchronize()
    assert np.linalg.norm(f64(out) - f64(att)) <= 1e-2 * np.linalg.norm(f64(att))


def test_two_graphs_share_a_workspace():
    """Replayed one after the other, each leaves what it leaves alone."""
    made = []
    for seed, new, kv in ((20, [1] * 9, [9 * i for i in range(9)]), (21, [30, 5], [200, 90])):
        b = Batch(seed, new, kv, 1500, 4, 2, 64, 16)
        made.append((b, b.run()))
    n = max(cola.prefix_attn_workspace_bytes(*b.desc()) for b, _ in made)
    assert n > 0
    ws = torch.empty(n, dtype=torch.uint8, device=DEV)
    graphs = []
    for b, _ in made:
        d, c = b.desc()
        t = [i32(x) for x in (b.ptab, b.tab, b.kv, b.start)]
        out, lse = torch.zeros_like(b.q), torch.zeros((b.hq, b.T), device=DEV)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            cola.prefix_attn(d, c, b.q, b.K, b.V, *t, out, lse, ws)
        graphs.append((g, out, lse, t))
    for order in ((0, 1), (1, 0), (0, 0, 1, 1), (1, 0, 1, 0)):
        for g, out, lse, _ in graphs:
            out.zero_()
            lse.zero_()
        for i in order:
            graphs[i][0].replay()
        torch.cuda.synchronize()
        for (_, out, lse, _), (b, (want, wl)) in zip(graphs, made):
            assert torch.equal(out, want) and torch.equal(lse, wl)


def test_two_streams_at_once():
    """Two servers on two streams, each with its own buffers: the serial results."""
    a, b = Server(6, 8, 2, 128, 16, 500, 20), Server(6, 8, 2, 128, 16, 500, 20, seed=5)
    want = []
    for s in (a, b):
        s.feed([2] * 6, 7)
        s.step()
        torch.cuda.synchronize()
        want.append(s.out.clone())
        s.out.zero_()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(3):
        for s, st in zip((a, b), streams):
            s.step(stream=st)
    torch.cuda.synchronize()
    assert torch.equal(a.out, want[0]) and torch.equal(b.out, want[1])


@pytest.mark.parametrize("L, launches", [(20, 1), (1000, 2)])
def test_timing_classes_count_the_launches(L, launches):
    """A short prefix goes along with the requests' own keys; a long one has parts to join."""
    s = Server(2, 2, 2, 64, 16, L, 4)
    s.feed([1, 1], 3)
    cola.timing_enable(True)
    cola.timing_reset()
    try:
        s.step()
        cola.rope_fwd(cola.rope_desc(4, 2, 0, 64), s.qr, None, None, s.out, None)
        n = {k: cola.timing_read(i)[0] for i, k in enumerate(cola.KERNEL_CLASSES)}
    finally:
        cola.timing_enable(False)
        cola.timing_reset()
    assert n["pointwise"] == 3 and n["attn_fwd"] == launches and sum(n.values()) == 3 + launches


# ---------------------------------------------------------------------------
# batches with fewer rows than their requests have tokens
# ---------------------------------------------------------------------------

# (new, kv, L, hq, hk, rows): tiles of 16, 32 and 128 rows, the prefix along and apart
CUT = {"one": ([2, 3], [9, 40], 0, 2, 2, 3), "one-along": ([2, 5], [9, 40], 30, 2, 1, 4), "one-prefix": ([2, 5], [9, 40], 1300, 2, 1, 5),
       "two": ([5, 20], [9, 40], 0, 2, 2, 12), "two-prefix": ([5, 20], [9, 40], 1300, 2, 2, 9),
       "wide": ([30, 90], [60, 300], 0, 4, 2, 75), "wide-along": ([30, 90], [60, 300], 50, 4, 2, 31), "wide-prefix": ([30, 90], [60, 300], 1300, 4, 2, 75),
       "a-request-past-the-end": ([4, 9, 2], [4, 20, 2], 20, 2, 2, 4)}


@pytest.mark.parametrize("hd", (64, 128))
@pytest.mark.parametrize("name", sorted(CUT))
def test_attention_of_a_batch_cut_at_its_rows(name, hd):
    """A request whose last tokens have no row (page_map: "tokens past T have no row"):
    the rows that are there see what they see in the whole batch, and not the later
    tokens, which nothing has written to the cache."""
    new, kv, L, hq, hk, rows = CUT[name]
    b = Batch(30 + hd, new, kv, L, hq, hk, hd, 16)
    for r, n in enumerate(new):
        for i in range(n):
            if b.start[r] + i >= rows:
                j = kv[r] - n + i
                for c in (b.K, b.V):
                    c[int(b.tab[r, j // 16]), :, j % 16] = math.nan
    ref, rl, w = b.reference()
    b.T, b.q = rows, b.q[:rows].contiguous()
    out, lse = b.run()
    keys = L + max(kv)
    assert (np.abs(f64(out) - ref[:rows]) <= R.attention_bound(ref, w, keys)[:rows]).all()
    assert (np.abs(f64(lse) - rl[:, :rows]) <= R.lse_bound(rl[:, :rows], keys)).all()


# ---------------------------------------------------------------------------
# yarn's ramp where its end lies past the slowest pair
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("rot, orig_len, base", [(128, 65536, 10000.0), (64, 131072, 10000.0), (64, 1 << 40, 10000.0), (32, 4, 500000.0)])
def test_yarn_ramp_past_the_slowest_pair(rot, orig_len, base):
    """The ramp ends at the index, rounded up, at which a pair makes `low` turns.  It may
    lie past the last pair, up to rot_dim - 1, and the ramp keeps its slope.  An
    original length in which every pair makes `high` turns leaves them all as they
    are; one in which none makes a turn divides all but the first."""
    hd, T, low, high, factor = rot, 9, 1.0, 32.0, 8.0
    pos = np.array([0, 1, 2, 3, 77, 1000, 4095, 65535, 500000])
    turns_at = lambda t: rot * math.log(orig_len / (2 * math.pi * t)) / (2 * math.log(base))
    lo, hi = (min(max(x, 0), rot - 1) for x in (math.floor(turns_at(high)), math.ceil(turns_at(low))))
    if orig_len == 65536:
        assert (lo, hi) == (40, 65)
    f = []
    for i in range(rot // 2):
        x = min(max((i - lo) / max(hi - lo, 0.001), 0.0), 1.0)
        f.append((1 - x) * base ** (-2 * i / rot) + x * base ** (-2 * i / rot) / factor)
    m = 1 + 0.1 * math.log(factor)
    q = rand(5, (T, hd), "f32")
    out = torch.empty_like(q)
    d = cola.rope_desc(T, 1, 0, hd, rot, "f32", "half", "yarn", base=base, factor=factor, orig_len=orig_len, low=low, high=high)
    cola.rope_fwd(d, q, None, i32(pos), out, None)
    x = f64(q)
    a = pos[:, None] * np.array(f)
    c, s = m * np.cos(a), m * np.sin(a)
    u, v = x[:, :rot // 2], x[:, rot // 2:]
    want = np.concatenate([u * c - v * s, v * c + u * s], 1)
    assert (np.abs(f64(out) - want) <= R.rope_bound(x, 1, hd, rot, want, "f32", "half", m)).all()


# ---------------------------------------------------------------------------
# joins of many parts
# ---------------------------------------------------------------------------

# Rows that fill the chip with a thread for four elements, and fewer: (new, kv, L, hq, hk, max_kv)
JOINS = {"many-rows": ([1] * 130, [(11 * i) % 70 for i in range(130)], 2600, 32, 1, None),
         "many-rows-loose-bound": ([33] * 4, [33, 50, 300, 1600], 0, 32, 1, 40000),
         "few-rows-loose-bound": ([33] * 4, [33, 50, 300, 1600], 0, 4, 1, 40000)}


@pytest.mark.parametrize("hd", (64, 128))
@pytest.mark.parametrize("name", sorted(JOINS))
def test_attention_joins_of_more_than_eight_parts(name, hd):
    new, kv, L, hq, hk, max_kv = JOINS[name]
    b = Batch(40 + hd, new, kv, L, hq * 128 // hd if name.startswith("many") else hq, hk, hd, 64, pad=2, max_kv=max_kv)
    d, c = b.desc()
    assert cola.prefix_attn_workspace_bytes(d, c) > 8 * b.T * b.hq * (hd + 2) * 4
    assert name.startswith("few") == (b.T * b.hq * hd // 4 < 1 << 17)
    b.check()


@pytest.mark.parametrize("L", (0, 700))
def test_attention_of_more_turns_than_a_grid(L):
    """More than 2^23 workgroups go out in several launches: rows of the first request, of
    one in the middle and of the last, whose turns are past the first launch."""
    n, heads = 65535, 129
    new, kv = [0] * n, [0] * n
    for r, (x, y) in {0: (2, 20), 40000: (1, 5), n - 1: (2, 33)}.items():
        new[r], kv[r] = x, y
    assert (n - 1) * heads > 1 << 23
    Batch(50, new, kv, L, heads, heads, 64, 16).check()


# ---------------------------------------------------------------------------
# paths that only large calls take
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("n_req, mean, page, idle, listed", [(1024, 90, 16, 3, None), (300, 310, 128, 1, None), (2, 40000, 64, 0, None),
                                                             (4096, 23, 1, 2, 50000), (1, 65550, 4096, 0, 7)])
def test_page_map_of_many_rows(n_req, mean, page, idle, listed):
    """More than 65536 rows, four to a thread: requests without tokens among the others,
    rows that no four divide, a free list that ends too early."""
    rng = np.random.default_rng(n_req)
    n = rng.integers(0, 2 * mean, n_req) if n_req > 2 else np.full(n_req, mean)
    n[::7] = 0 if n_req > 2 else mean
    kv = n + rng.integers(0, 300, n_req)
    width = int(-(-kv.max() // page)) + 1
    table = rng.integers(0, 10 ** 5, (n_req, width))
    free = rng.permutation(4 * 10 ** 5)[:listed]
    T = int(n.sum()) + idle
    assert T > 1 << 16
    for rows in (T, T - 5):
        check_map(kv, n, free, 2, table, page, rows, 1000)


def test_page_map_of_many_rows_at_any_alignment():
    """Slots and positions that begin at any element."""
    n_req, each, page = 70, 1000, 32
    T, width = n_req * each + 2, -(-each // page)
    kv, free = i32([each] * n_req), torch.randperm(n_req * width, device=DEV).int()
    d = cola.page_map_desc(n_req, T, page, width, free.numel(), 9)
    want = None
    for off in (0, 1, 2, 3):
        table = torch.full((n_req, width), -1, dtype=torch.int32, device=DEV)
        start, nxt = torch.zeros(n_req + 1, dtype=torch.int32, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
        slots, pos = (torch.full((T + 8,), -77, dtype=torch.int32, device=DEV) for _ in range(2))
        cola.page_map(d, kv, kv, free, None, table, start, slots[off:off + T], pos[off:off + T], nxt)
        for b in (slots, pos):
            assert (b[:off] == -77).all() and (b[off + T:] == -77).all()
        got = [table, start, slots[off:off + T].clone(), pos[off:off + T].clone(), nxt]
        want = want or got
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    ref = R.page_map([each] * n_req, [each] * n_req, free.tolist(), 0, np.full((n_req, width), -1), page, T, 9)
    assert (want[0].cpu().numpy() == ref[0]).all() and want[2].tolist() == ref[2] and want[3].tolist() == ref[3]


def test_page_map_past_32_bits():
    """Slots and positions that an int32 does not hold."""
    big = 2 ** 31 - 1
    free = np.array([2 ** 19 - 1, 2 ** 19, 2 ** 30])
    got = run_map([1, 1, 1], [1, 1, 1], free, 0, np.zeros((3, 1), np.int64), 4096, 3, big)
    assert got[2] == [(2 ** 19 - 1) * 4096, -1, -1] and got[3] == [big] * 3
    got = run_map([20], [20], free, 0, np.zeros((1, 1), np.int64), 4096, 20, big - 5)
    assert got[3] == [min(big - 5 + i, big) for i in range(20)]


@pytest.mark.parametrize("layout", ("half", "interleaved"))
def test_large_fp32_results_are_the_small_ones(layout):
    """fp32 results of more than 48 MB leave by other stores: the bits of the same rows in
    parts; and so do rows of the cache."""
    T, hq, hk, hd, page = 3200, 32, 8, 128, 16
    q, k, v = (rand(s, (T, h * hd), "f32") for s, h in ((1, hq), (2, hk), (3, hk)))
    pos = torch.arange(T, dtype=torch.int32, device=DEV) * 7
    slots = torch.randperm(T, device=DEV).int()
    c = cola.cache_desc(T // page, page, hk, hd, "f32")
    assert 4 * T * (hq + hk) * hd > 48e6 > 4 * T // 4 * (hq + 2 * hk) * hd
    res = []
    for step in (T, T // 4):
        r = [torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(q)] + [torch.zeros((T // page, hk, page, hd), device=DEV) for _ in range(2)]
        for at in range(0, T, step):
            n = slice(at, at + step)
            d = cola.rope_desc(step, hq, hk, hd, 96, "f32", layout)
            cola.rope_fwd(d, q[n], k[n], pos[n], r[0][n], r[1][n])
            cola.cache_append(d, c, q[n], k[n], v[n], pos[n], slots[n], r[2][n], r[3], r[4])
        res.append(r)
    assert all(torch.equal(a, b) for a, b in zip(*res))
    ref = R.rope(f64(q[-3:]), hq, hd, 96, f64(pos[-3:]), layout)
    assert (np.abs(f64(res[0][0][-3:]) - ref) <= R.rope_bound(f64(q[-3:]), hq, hd, 96, ref, "f32", layout)).all()
    assert torch.equal(res[0][0], res[0][2])


@pytest.mark.parametrize("hd, hq, new", [(64, 2, 1), (128, 4, 1), (64, 2, 3)])
def test_attention_joins_of_more_than_64_parts(hd, hq, new):
    """The wave that joins a row has the statistics of two parts to a lane."""
    b = Batch(60 + hd, [new], [2300], 20000, hq, 1, hd, 64)
    d, c = b.desc()
    assert cola.prefix_attn_workspace_bytes(d, c) > 64 * b.T * b.hq * (hd + 2) * 4
    b.check()


@pytest.mark.parametrize("name", ["one-one", "one-flat", "one-solo", "two-one", "two-flat", "two-two", "wide-one", "wide-flat", "wide-solo", "wide-two",
                                  "wide-wide", "along-one", "along-two", "along-wide"])
def test_attention_kernels_past_4_gib(name):
    """Each kernel on pages whose bytes lie past 2^32 of the cache: the bits that it
    gives where they lie at its beginning."""
    new, kv, L, hq, hk = KERNELS[name]
    hd, page = 64, 16
    b = Batch(70, new, kv, L, hq, hk, hd, page, pad=1, junk=0.0)
    want = b.run()
    n, pages = b.K.shape[0], (5 << 29) // (hk * hd * page)      # 2.5 Gi elements of 2 bytes
    rng = np.random.default_rng(1)
    at = pages - 1 - rng.permutation(pages // 8)[:n - 1]         # the last eighth: past 0.8 of the cache
    at = np.concatenate([[0], at])
    assert 2 * int(at[1:].min()) * hk * hd * page > 1 << 32
    K, V = (torch.empty((pages, hk, page, hd), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    for x, y in ((K, b.K), (V, b.V)):
        x[torch.from_numpy(at).to(DEV)] = y
    b.K, b.V = K, V
    b.ptab, b.tab = at[b.ptab], np.where(b.tab >= 0, at[np.maximum(b.tab, 0)], -1)
    got = b.run()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("new, L", [([1, 1], 40), ([1, 1], 2000), ([3, 2], 40), ([20, 5], 2000), ([90, 2], 40), ([90, 2], 2000)])
def test_attention_of_a_cache_without_pages(new, L):
    """No page is in the cache: every row sees nothing."""
    T, hq = sum(new) + 1, 2
    d, c = cola.prefix_attn_desc(len(new), T, hq, L, 64, max(new)), cola.cache_desc(0, 16, 2, 64)
    q = rand(1, (T, hq * 64), "bf16")
    out, lse = torch.full_like(q, 7.0), torch.full((hq, T), 7.0, device=DEV)
    K = torch.empty((0, 2, 16, 64), dtype=torch.bfloat16, device=DEV)
    n = cola.prefix_attn_workspace_bytes(d, c)
    ws = torch.full((n,), 0xFF, dtype=torch.uint8, device=DEV) if n else None
    cola.prefix_attn(d, c, q, K, K, torch.zeros(-(-L // 16), dtype=torch.int32, device=DEV), torch.zeros((len(new), 4), dtype=torch.int32, device=DEV),
                     i32([64] * len(new)), i32(np.cumsum([0] + new)), out, lse, ws)
    assert (out[:-1] == 0).all() and torch.isneginf(lse[:, :-1]).all() and (out[-1] == 7).all() and (lse[:, -1] == 7).all()
